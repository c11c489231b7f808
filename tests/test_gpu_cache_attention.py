"""Attention over the paged 8-bit cache against a 64-bit implementation: both
kernels, split and whole keys, ragged and empty sequences, windows with sinks,
missing pages, whatever lies behind the last token."""
import pytest
import torch

import helpers_cache as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
# P's rounding: two bf16 terms leave 2^-16 (the second is rounded to 2^-8 of the first's 2^-8), one leaves 2^-8
P_ROWS, P_TILE = 2.0 ** -16, 2.0 ** -8


def _run(seed, lens, new, Hq, Hkv, D, page, window=0, sinks=0, max_q=None, max_len=None, poison=True, layer=1, q_scale=0.05,
         break_table=None, spare=0):
    pages = sum(-(-n // page) for n in lens) + 3
    pool = H.Pool(seed, 2, pages, Hkv, page, D)
    table = pool.tables(lens, spare=spare)
    if break_table:
        break_table(table, pages)
    q = (torch.randn((sum(new), Hq, D), generator=pool.g) * q_scale * 8).to(torch.bfloat16)
    dev_pool = H.Pool(seed, 2, pages, Hkv, page, D)
    for a, b in zip(dev_pool.arrays(), pool.arrays()):
        a.copy_(b)
    if poison:                                        # NaN codes on every position that holds no token
        held = torch.zeros((pages, page), dtype=torch.bool)
        for b, n in enumerate(lens):
            for j in range(min(-(-n // page), table.shape[1])):
                at = int(table[b, j])
                if 0 <= at < pages:
                    held[at, :min(page, n - j * page)] = True
        dev_pool.k[:] = torch.where(held[None, :, None, :, None], dev_pool.k, 0x7F)
        hv = held.view(pages, page // 16, 1, 16)
        dev_pool.v[:] = torch.where(hv[None, :, None], dev_pool.v, 0xFF)
    cache = dev_pool.to(DEV)
    cu = H.cumulative(new, DEV)
    o, lse = cache.attention(layer, q.to(DEV), cu, H.ints(lens, DEV), table.to(DEV), max_q or max(new), max_len or max(lens),
                             window, sinks)
    torch.cuda.synchronize()
    refs = []
    for b, n in enumerate(lens):
        k, v, ok = H.sequence_kv(pool, layer, table[b], n)
        r0 = sum(new[:b])
        k, v = torch.where(ok[None, :, None], k, 0), torch.where(ok[None, :, None], v, 0)
        refs.append(H.attend(q[r0:r0 + new[b]], k, v, range(n - new[b], n), window, sinks, ok))
    ref = [torch.cat(x) for x in zip(*refs)]
    few = (max_q or max(new)) * (Hq // Hkv) <= 64
    H.check(o, lse, ref, max(max(lens), 1), D, P_ROWS if few else P_TILE, f"{lens} {new} {Hq}/{Hkv} {D} {page} {window} {sinks}")
    return o, lse


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (100, 4), (64, 70), (257, 1)])
def test_decode(page, D, window, sinks):
    _run(page + D, [1, 15, 64, 65, 333, 700], [1] * 6, 8, 2, D, page, window, sinks)


@pytest.mark.parametrize("heads", [(1, 1), (3, 1), (5, 5), (16, 1), (14, 2), (40, 8)])
def test_decode_heads(heads):
    _run(3, [130, 1, 77], [1, 1, 1], *heads, 128, 32, 50, 2)


@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5)])
def test_decode_split_keys(window, sinks):
    """Few sequences, long: the keys are split over workgroups."""
    _run(5, [5000, 37], [1, 1], 4, 1, 128, 64, window, sinks)
    _run(6, [2111], [1], 4, 1, 64, 16, window, sinks)


@pytest.mark.parametrize("window,sinks", [(0, 0), (40, 3)])
def test_few_rows(window, sinks):
    """Several new tokens per sequence, some with none; more than one tile of rows."""
    _run(7, [9, 0, 200, 3, 130], [9, 0, 8, 1, 5], 8, 2, 128, 16, window, sinks)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (50, 0), (130, 70)])
def test_chunk(page, D, window, sinks):
    _run(11 + page, [300, 100, 65, 0, 7], [70, 100, 1, 0, 7], 4, 2, D, page, window, sinks)


@pytest.mark.parametrize("page", [16, 32, 64, 128])
@pytest.mark.parametrize("window,sinks", [(0, 0), (2000, 30)])
def test_chunk_of_long_calls(page, window, sinks):
    """The wider tile of calls that announce long keys, whatever their sequences have."""
    _run(33, [300, 100, 65, 0, 7], [70, 100, 1, 0, 7], 4, 2, 128, page, window, sinks, max_len=9000)
    _run(34, [2300, 513], [101, 513], 3, 1, 128, page, window, sinks)


@pytest.mark.parametrize("G", [1, 3, 8])
def test_chunk_heads(G):
    _run(13, [410, 90], [100, 90], 2 * G, 2, 128, 64)


def test_chunk_split_keys():
    _run(14, [4000, 130], [40, 33], 2, 1, 128, 64)
    _run(15, [3001], [65], 1, 1, 64, 32, 900, 4)


@pytest.mark.parametrize("new", [1, 80])
def test_missing_pages(new):
    """Entries that are no page hide their tokens; a row that has none left is empty."""
    def cut(table, pages):
        table[0, 1] = -1
        table[0, 3] = pages
        table[1, :] = -7
        table[2, 0] = 1 << 30
    _run(17, [new + 300, new + 20, new + 64, new + 90], [new] * 4, 4, 2, 128, 64, break_table=cut)
    _run(18, [new + 300, new + 20, new + 64, new + 90], [new] * 4, 4, 2, 64, 16, 70, 3, break_table=cut)


def test_longer_than_the_table():
    """Lengths past the table's width: only what it holds is seen, positions stay."""
    pool = H.Pool(19, 1, 8, 1, 16, 64)
    table = torch.tensor([[3, 5]], dtype=torch.int32)
    q = torch.randn((1, 1, 64), generator=pool.g).to(torch.bfloat16)
    cache = pool.to(DEV)
    o, lse = cache.attention(0, q.to(DEV), H.ints([0, 1], DEV), H.ints([50], DEV), table.to(DEV), 1, 50, 40, 0)
    k, v, ok = H.sequence_kv(pool, 0, [3, 5], 32)
    ref = H.attend(q, k, v, [49], 40, 0)              # positions 10 .. 31 of it
    H.check(o, lse, ref, 32, 64, P_ROWS)


@pytest.mark.parametrize("new", [1, 9, 80, 300])
def test_windows_that_end_behind_the_table(new):
    """.. whatever the place of the table's end and of the window in a block of keys."""
    for D, page, width, n in ((64, 16, 5, 200), (128, 16, 9, 150), (128, 64, 2, 190), (64, 128, 1, 1000)):
        pool = H.Pool(30, 1, 20, 2, page, D)
        table = pool.tables([width * page, width * page])
        q = (torch.randn((2 * new, 4, D), generator=pool.g) * 0.4).to(torch.bfloat16)
        cache = pool.to(DEV)
        for window, sinks in ((0, 0), (n - 70, 0), (n - 33, 20), (n, 0)):
            o, lse = cache.attention(0, q.to(DEV), H.ints([0, new, 2 * new], DEV), H.ints([n, n + 13], DEV), table.to(DEV), new,
                                     n + 13, window, sinks)
            refs = []
            for b, m in enumerate((n, n + 13)):
                k, v, ok = H.sequence_kv(pool, 0, table[b], width * page)
                refs.append(H.attend(q[b * new:(b + 1) * new], k, v, range(m - new, m), window, sinks))
            H.check(o, lse, [torch.cat(x) for x in zip(*refs)], n + 13, D, P_ROWS if new * 2 <= 64 else P_TILE,
                    f"{D} {page} {window} {sinks}")


def test_rows_of_nobody_are_left_alone():
    import paper_2602_02071_amd as baps
    for new, fill in (([2, 0, 3], 7.0), ([70, 0, 90], 5.0)):
        lens = [n + 30 for n in new]
        pool = H.Pool(20, 1, 40, 2, 16, 128)
        table = pool.tables(lens)
        cache = pool.to(DEV)
        T = sum(new) + 9
        q = torch.randn((T, 4, 128), generator=pool.g).to(torch.bfloat16).to(DEV)
        o = torch.full((T, 4, 128), fill, dtype=torch.bfloat16, device=DEV)
        lse = torch.full((T, 4), fill, device=DEV)
        cu = H.ints([4 + sum(new[:i]) for i in range(4)], DEV)
        for max_len in (max(lens), 100000):           # without and with split keys
            n = baps.baps_cache_attention_workspace(cache.c, 3, 4, T, max(new), max_len)
            ws = torch.empty(max(n, 1), dtype=torch.uint8, device=DEV)
            assert (n > 0) == (max_len > 1000)
            baps.baps_cache_attention(cache.c, 0, q, 512, o, lse, cu, H.ints(lens, DEV), table.to(DEV), table.shape[1], 3, 4, T,
                                      max(new), max_len, workspace=ws, workspace_bytes=n)
            torch.cuda.synchronize()
            own = torch.zeros(T, dtype=torch.bool, device=DEV)
            own[4:4 + sum(new)] = True
            assert bool((o[~own] == fill).all()) and bool((lse[~own] == fill).all())
            assert not bool((lse[own] == fill).any())


def test_offsets_that_make_no_sense():
    """Sequences whose rows lie outside the call, or with more new tokens than they are long, do no harm."""
    pool = H.Pool(21, 1, 20, 1, 16, 64)
    cache = pool.to(DEV)
    table = pool.tables([40, 40, 40, 40]).to(DEV)
    q = torch.randn((6, 2, 64), generator=pool.g).to(torch.bfloat16).to(DEV)
    lens = H.ints([40, 1, 40, -5], DEV)
    o, lse = cache.attention(0, q, H.ints([0, 2, 5, 9, 6], DEV), lens, table, 4, 40)
    torch.cuda.synchronize()
    k, v, ok = H.sequence_kv(pool, 0, table[0].cpu(), 40)
    H.check(o[:2], lse[:2], H.attend(q[:2].cpu(), k, v, [38, 39], 0, 0), 40, 64, P_ROWS)
    # three new tokens of a sequence of one: the first two have no position
    k, v, ok = H.sequence_kv(pool, 0, table[1].cpu(), 1)
    H.check(o[2:5], lse[2:5], H.attend(q[2:5].cpu(), k, v, [-2, -1, 0], 0, 0), 40, 64, P_ROWS)


@pytest.mark.parametrize("new,n", [(7, 3), (100, 30), (100, 99)])
def test_rows_in_front_of_position_zero(new, n):
    """More new tokens than the sequence is long: the first rows see nothing, whatever the window."""
    for window in (0, 1, 50, 2 ** 31 - 1):
        _run(26, [n, 200], [new, 1], 4, 2, 128, 16, window, 0 if not window else 2 ** 31 - 1 - new)


@pytest.mark.parametrize("max_q", [3, 100])
def test_numbers_near_the_end_of_their_type(max_q):
    """Offsets, lengths, window and sinks at the ends of int32."""
    import paper_2602_02071_amd as baps
    top = 2 ** 31 - 1
    pool = H.Pool(27, 1, 20, 1, 16, 64)
    cache = pool.to(DEV)
    table = pool.tables([40, 40, 40]).to(DEV)
    q = torch.randn((6, 2, 64), generator=pool.g).to(torch.bfloat16).to(DEV)
    o = torch.full((6, 2, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    for cu, lens in (([0, 2, -top - 1, 6], [40, top, top]), ([0, 2, top, 0], [40, -top - 1, top])):
        baps.baps_cache_attention(cache.c, 0, q, 128, o, None, H.ints(cu, DEV), H.ints(lens, DEV), table, table.shape[1], 3, 2, 6,
                                  max_q, 40, top, top)
        torch.cuda.synchronize()
        k, v, ok = H.sequence_kv(pool, 0, table[0].cpu(), 40)
        ref = H.attend(q[:2].cpu(), k, v, [38, 39], 0, 0)
        assert (o[:2].cpu().double() - ref[0]).abs().max() < 0.05 * ref[3].max()
        assert bool((o[2:] == 3.0).all())
    # a length of 2^31 - 1 counts as 2^30: its row sees all that the table holds
    o, lse = cache.attention(0, q[:1], H.ints([0, 1], DEV), H.ints([top], DEV), table[:1].contiguous(), max_q, 40, top, top)
    n = 16 * table.shape[1]
    k, v, ok = H.sequence_kv(pool, 0, table[0].cpu(), n)
    H.check(o, lse, H.attend(q[:1].cpu(), k, v, [n - 1], 0, 0, ok), n, 64, P_TILE)


@pytest.mark.parametrize("B", [65, 150])
def test_many_sequences(B):
    """Chunks of more sequences than a wave has lanes, some of one length, some with nothing."""
    lens = [(37 * b) % 50 + 1 if b % 7 else 0 for b in range(B)]
    lens[3] = lens[B - 1] = 170
    new = [min(n, 5 + 13 * (b % 3)) for b, n in enumerate(lens)]
    new[3] = new[B - 1] = 90
    _run(28, lens, new, 4, 2, 64, 16)
    _run(29, lens, new, 4, 2, 128, 16, 20, 3)


@pytest.mark.parametrize("B,D,window", [(40, 128, 0), (64, 64, 0), (33, 128, 1200), (63, 128, 0)])
def test_large_ragged_decode(B, D, window):
    """More workgroups than CUs: sequences taken in another order than the batch's, keys split or not."""
    lens = [(211 * b) % 700 + 1 for b in range(B)]
    lens[5], lens[6], lens[B - 1], lens[7], lens[8] = 2300, 0, 2300, 640, 640
    new = [min(n, 1) for n in lens]
    _run(31, lens, new, 8, 8, D, 64, window, 5 if window else 0)
    _run(32, lens, [min(n, 1 + b % 3) for b, n in enumerate(lens)], 16, 8, D, 64, window, 0, max_len=5000)


def test_strided_rows_and_scale():
    """q as a slice of a wider projection; a score scale of the caller's."""
    pool = H.Pool(22, 1, 12, 2, 32, 128)
    cache = pool.to(DEV)
    lens, new = [70, 33], [3, 33]
    table = pool.tables(lens)
    wide = torch.randn((36, 6, 128), generator=pool.g).to(torch.bfloat16)
    for s in (1, 2):
        part = wide[:, s:s + 4]
        o, lse = cache.attention(0, wide.to(DEV)[:, s:s + 4], H.cumulative(new, DEV), H.ints(lens, DEV), table.to(DEV), 33, 70,
                                 scale_log2=0.01)
        refs = []
        for b in range(2):
            k, v, ok = H.sequence_kv(pool, 0, table[b], lens[b])
            refs.append(H.attend(part[sum(new[:b]):sum(new[:b + 1])], k, v, range(lens[b] - new[b], lens[b]), 0, 0,
                                 scale=0.01 * 0.6931471805599453))
        H.check(o, lse, [torch.cat(x) for x in zip(*refs)], 70, 128, P_TILE)


def test_large_scores():
    """Scores in the hundreds: one key takes all the weight, the others vanish without a NaN."""
    _run(23, [200, 90], [1, 1], 4, 2, 128, 64, q_scale=20.0)
    _run(24, [200, 90], [60, 90], 4, 2, 64, 64, q_scale=20.0)


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes of K: the last page's address."""
    import paper_2602_02071_amd as baps
    page, Hkv, D = 128, 8, 128
    pages = (1 << 32) // (page * Hkv * D) + 5
    small = H.Pool(25, 1, 2, Hkv, page, D)
    cache = baps.PagedCache(*(torch.zeros((1, pages) + tuple(x.shape[2:]), dtype=torch.uint8, device=DEV)
                              for x in small.arrays()))
    for dst, src in zip((cache.k, cache.v, cache.k_exp, cache.v_exp), small.arrays()):
        dst[0, pages - 2:] = src[0].to(DEV)
    for new in (1, 40):
        q = (torch.randn((new, 16, D), generator=small.g) * 0.4).to(torch.bfloat16)
        table = torch.tensor([[pages - 1, pages - 2]], dtype=torch.int32)
        o, lse = cache.attention(0, q.to(DEV), H.ints([0, new], DEV), H.ints([200], DEV), table.to(DEV), new, 200)
        k, v, ok = H.sequence_kv(small, 0, [1, 0], 200)
        H.check(o, lse, H.attend(q, k, v, range(200 - new, 200), 0, 0), 200, D, P_ROWS if new == 1 else P_TILE)
