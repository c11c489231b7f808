"""New tokens into the paged 8-bit cache: codes and exponents equal those of a
page-by-page implementation, everything else stays as it was."""
import math

import pytest
import torch

import helpers_cache as H

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _new(g, T, Hkv, D, spread=1.0):
    x = torch.randn((T, Hkv, D), generator=g)
    x *= torch.exp2(torch.randint(-3, 4, (T, 1, 1), generator=g).float()) * spread
    return x.to(torch.bfloat16)


def _same(cache, pool, label=""):
    torch.cuda.synchronize()
    for name, got, want in zip(("k", "v", "k_exp", "v_exp"), (cache.k, cache.v, cache.k_exp, cache.v_exp), pool.arrays()):
        got = got.cpu()
        if name in "kv":                              # codes as values: the sign of a zero apart, NaN as NaN
            got, want = got.view(H.F8).float(), want.view(H.F8).float()
            assert torch.equal(got.isnan(), want.isnan()), f"{label} {name}"
            got, want = got.nan_to_num(), want.nan_to_num()
        bad = (got != want).nonzero()
        assert not len(bad), f"{label} {name}: {len(bad)} differ, first at {bad[:3].tolist()}"


def _append(pool, cache, layer, k, v, cu, lens, table, max_new):
    H.append(pool, layer, k, v, cu, lens, table)
    cache.append(layer, k.to(DEV), v.to(DEV), H.ints(cu, DEV), H.ints(lens, DEV), table.to(DEV), max_new)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_append(page, D):
    """Prompts, then a few tokens, then one by one, into two layers."""
    pool = H.Pool(page + D, 2, 24, 2, page, D)
    cache = pool.to(DEV)
    final = [3 * page + 5, page, 1, 2 * page - 1, 40]
    table = pool.tables(final, spare=1)
    lens = [0] * 5
    for step, new in enumerate(([2 * page + 3, page, 0, 1, 17], [7, 0, 0, 5, 1], [1, 0, 1, 1, 1], [1, 0, 0, 1, 1])):
        lens = [a + b for a, b in zip(lens, new)]
        cu = [sum(new[:i]) for i in range(6)]
        k, v = _new(pool.g, sum(new), 2, D, 2.0 ** step), _new(pool.g, sum(new), 2, D)
        _append(pool, cache, step % 2, k, v, cu, lens, table, max(new))
        _same(cache, pool, f"step {step}")


def test_growing_range_moves_the_page():
    """A page's scale rises with its tokens; the older codes move, by one and by many binades."""
    pool = H.Pool(1, 1, 6, 3, 16, 64)
    cache = pool.to(DEV)
    table = torch.tensor([[4, 2]], dtype=torch.int32)
    n = 0
    for spread in (1.0, 1.9, 2.0, 0.01, 300.0, 1e-20, 1e30, 1e38):
        k, v = _new(pool.g, 3, 3, 64, spread), _new(pool.g, 3, 3, 64, spread)
        n += 3
        _append(pool, cache, 0, k, v, [0, 3], [n], table, 3)
        _same(cache, pool, f"{spread}")


def test_scale_borders():
    """amax at and next to 448 * 2^e; zeros; the least and the largest bf16 numbers."""
    vals = [448.0, 450.0, 446.0, 1.75, 1.7578125, 0.875, 0.0, 2.0 ** -126, 2.0 ** -133, 3.3895e38, 1.0, 2.0 ** -100 * 448,
            2.0 ** -100 * 450, 1.75 * 2.0 ** 127, 2.0 ** 127 * 1.7578125]
    pool = H.Pool(2, 1, len(vals), 1, 16, 64)
    cache = pool.to(DEV)
    table = torch.arange(len(vals), dtype=torch.int32).reshape(-1, 1)
    x = torch.zeros((len(vals), 1, 64))
    for i, a in enumerate(vals):
        x[i, 0, :8] = torch.tensor([a, -a, a / 3, a / 448, -a / 7, a / 1000, a / 300000, 0.0])
    x = x.to(torch.bfloat16)
    _append(pool, cache, 0, x, x, list(range(len(vals) + 1)), [1] * len(vals), table, 1)
    _same(cache, pool)


def test_every_rounding():
    """All bf16 numbers of eleven binades below the scale: ties go to the even code, the smallest to zero."""
    bits = torch.arange(0x3F80 - 11 * 128, 0x3F80 + 1, dtype=torch.int32)
    x = (bits << 16).view(torch.float32)
    x = torch.cat((x, -x, torch.zeros(-2 * len(x) % 1024)))
    x = x.reshape(-1, 1024) * 256
    x[:, 0] = 448.0                                   # fixes the scale at one
    x = x.reshape(-1, 1, 128).to(torch.bfloat16)
    pool = H.Pool(3, 1, 64, 1, 16, 128)
    cache = pool.to(DEV)
    n = x.shape[0]
    table = torch.arange(-(-n // 16), dtype=torch.int32).reshape(1, -1)
    _append(pool, cache, 0, x, x, [0, n], [n], table, n)
    _same(cache, pool)


def test_inf_and_nan():
    """An infinity saturates and sets the largest scale, a NaN stays one and sets none; other heads and pages do not notice."""
    pool = H.Pool(4, 1, 4, 2, 32, 128)
    cache = pool.to(DEV)
    table = torch.tensor([[3, 1], [0, 2]], dtype=torch.int32)
    k, v = _new(pool.g, 50, 2, 128), _new(pool.g, 50, 2, 128)
    k[3, 0, 5], k[40, 1, 127], v[7, 1, 0], v[8, 0, 64] = math.nan, math.inf, -math.inf, -math.nan
    k[45] = math.nan                                  # a token of nothing else
    _append(pool, cache, 0, k, v, [0, 30, 50], [40, 20], table, 30)
    _same(cache, pool)


def test_bad_pages_and_rows():
    """Entries that are no page, rows outside the call, more tokens than the sequence is long: skipped."""
    pool = H.Pool(5, 1, 5, 1, 16, 64)
    cache = pool.to(DEV)
    table = torch.tensor([[0, -1, 9], [5, 1 << 30, 2], [1, 3, 4], [-9, -9, -9], [-1, -1, -1]], dtype=torch.int32)
    k, v = _new(pool.g, 100, 1, 64), _new(pool.g, 100, 1, 64)
    _append(pool, cache, 0, k, v, [0, 40, 80, 90, 120, 100], [40, 44, 9, 60, 7], table, 40)
    _same(cache, pool)
    _append(pool, cache, 0, k, v, [0, 40, 40, 40, 40, 40], [70, 0, 0, 0, 0], table, 40)       # past the table's width
    _same(cache, pool)
    _append(pool, cache, 0, k, v, [-3, 5, 5, 5, 5, 4], [20, 0, 0, 0, -4], table, 40)
    _same(cache, pool)


def test_numbers_near_the_end_of_their_type():
    pool = H.Pool(8, 1, 5, 1, 16, 64)
    cache = pool.to(DEV)
    table = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32)
    k, v = _new(pool.g, 60, 1, 64), _new(pool.g, 60, 1, 64)
    top = 2 ** 31 - 1
    for cu, lens in (([0, 5, 40], [top, 20]), ([0, 40, -top - 1], [20, top]), ([5, -top - 1, 40], [top, 20]), ([top, 5, 9], [top, -top - 1])):
        _append(pool, cache, 0, k, v, cu, lens, table, 40)
        _same(cache, pool, f"{cu} {lens}")


def test_strided_rows():
    """k and v as slices of one wide projection."""
    pool = H.Pool(6, 1, 8, 2, 16, 64)
    cache = pool.to(DEV)
    wide = torch.randn((33, 3 * 2 * 64 + 16), generator=pool.g).to(torch.bfloat16)
    k, v = (wide[:, a:a + 128].unflatten(1, (2, 64)) for a in (8, 144))
    table = pool.tables([50, 20])
    H.append(pool, 0, k, v, [0, 20, 33], [50, 20], table)
    d = wide.to(DEV)
    cache.append(0, d[:, 8:136].unflatten(1, (2, 64)), d[:, 144:272].unflatten(1, (2, 64)), H.ints([0, 20, 33], DEV),
                 H.ints([50, 20], DEV), table.to(DEV), 20)
    _same(cache, pool)


def test_same_bits_again():
    """The same tokens once more change nothing."""
    pool = H.Pool(7, 1, 9, 2, 32, 128)
    cache = pool.to(DEV)
    table = pool.tables([70, 33])
    k, v = _new(pool.g, 63, 2, 128), _new(pool.g, 63, 2, 128)
    for _ in range(2):
        _append(pool, cache, 0, k, v, [0, 40, 63], [70, 33], table, 40)
        _same(cache, pool)
