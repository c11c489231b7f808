"""Plain 64-bit implementations of the cache operators for the tests, and the
inputs they share.  Nothing here calls the library."""
import math

import torch

F8 = torch.float8_e4m3fn
EPS32 = 2.0 ** -24                     # half a step of fp32, relative
EPS16 = 2.0 ** -8                      # of bf16


def ints(v, dev):
    return torch.tensor(v, dtype=torch.int32, device=dev)


def cumulative(n, dev):
    return ints([sum(n[:i]) for i in range(len(n) + 1)], dev)


def random_codes(g, *shape):
    """E4M3 codes without NaN."""
    x = torch.randint(0, 256, shape, generator=g, dtype=torch.uint8)
    return torch.where((x & 0x7F) == 0x7F, x - 1, x)


class Pool:
    """A pool on the CPU: random codes of moderate size, exponents around one."""

    def __init__(self, seed, layers, pages, Hkv, page, D):
        g = torch.Generator().manual_seed(seed)
        self.g, self.shape = g, (layers, pages, Hkv, page, D)
        x = torch.randn((layers, pages, Hkv, page, D), generator=g) * 40
        self.k = x.to(F8).view(torch.uint8)
        x = torch.randn((layers, pages, Hkv, page // 16, D, 16), generator=g) * 40
        self.v = x.to(F8).view(torch.uint8)
        self.ke = torch.randint(119, 124, (layers, pages, Hkv), generator=g, dtype=torch.uint8)
        self.ve = torch.randint(119, 124, (layers, pages, Hkv), generator=g, dtype=torch.uint8)

    def arrays(self):
        return self.k, self.v, self.ke, self.ve

    def to(self, dev):
        import paper_2602_02071_amd as baps
        return baps.PagedCache(*(x.clone().to(dev) for x in self.arrays()))

    def tables(self, lens, width=None, spare=0):
        """Distinct random pages for every row, -1 behind them."""
        layers, pages, Hkv, page, D = self.shape
        n = [-(-x // page) for x in lens]
        width = width or max(max(n), 1) + spare
        perm = torch.randperm(pages, generator=self.g).tolist()
        assert sum(n) <= pages
        rows, at = [], 0
        for x in n:
            rows.append(perm[at:at + x] + [-1] * (width - x))
            at += x
        return torch.tensor(rows, dtype=torch.int32).reshape(len(lens), width)


def values_k(k, ke):
    """[.., page, D] codes and [..] exponents -> 64-bit values."""
    return k.view(F8).double() * torch.exp2(ke.double() - 127)[..., None, None]


def values_v(v, ve):
    """[.., page/16, D, 16] -> [.., page, D]."""
    return values_k(v.transpose(-1, -2).flatten(-3, -2).contiguous(), ve)


def sequence_kv(pool, layer, row, n):
    """K and V [Hkv, n, D] of a sequence in 64 bits; a missing page gives NaN and False in ok [n]."""
    layers, pages, Hkv, page, D = pool.shape
    k, v, ok = [], [], []
    for j in range(-(-n // page)):
        at = int(row[j])
        good = 0 <= at < pages
        k.append(values_k(pool.k[layer, at], pool.ke[layer, at]) if good else torch.full((Hkv, page, D), math.nan, dtype=torch.float64))
        v.append(values_v(pool.v[layer, at], pool.ve[layer, at]) if good else torch.full((Hkv, page, D), math.nan, dtype=torch.float64))
        ok += [good] * page
    if not k:
        z = torch.zeros((Hkv, 0, D), dtype=torch.float64)
        return z, z, torch.zeros(0, dtype=torch.bool)
    return torch.cat(k, 1)[:, :n], torch.cat(v, 1)[:, :n], torch.tensor(ok[:n])


def attend(q, k, v, pos, window, sinks, ok=None, scale=None):
    """q [n, Hq, D] at positions pos [n], k, v [Hkv, len, D]: o [n, Hq, D], lse [n, Hq], and per row the largest
    sum of |q_d k_d| scale over its keys and the weighted mean of |v| (what rounding errors go by)."""
    n, Hq, D = q.shape
    G = Hq // k.shape[0]
    scale = scale or 1.0 / math.sqrt(D)
    o = torch.zeros((n, Hq, D), dtype=torch.float64)
    lse = torch.full((n, Hq), -math.inf, dtype=torch.float64)
    size = torch.zeros((n, Hq), dtype=torch.float64)
    mean = torch.zeros((n, Hq, D), dtype=torch.float64)
    c, t = torch.arange(k.shape[1]), torch.as_tensor(list(pos), dtype=torch.int64)[:, None]
    seen = c <= t
    if window:
        seen &= (c > t - window) | (c < sinks)
    if ok is not None:
        seen &= ok
    if not n or not len(c):
        return o, lse, size, mean
    q = q.double()
    for h in range(Hq):
        kk, vv = k[h // G], v[h // G]
        s = torch.where(seen, q[:, h] @ kk.t() * scale, -math.inf)
        size[:, h] = torch.where(seen, q[:, h].abs() @ kk.abs().t() * scale, 0).amax(1)
        lse[:, h] = torch.logsumexp(s, 1)
        w = torch.exp(s - lse[:, h].where(seen.any(1), torch.zeros(()).double())[:, None])
        o[:, h] = w @ vv
        mean[:, h] = w @ vv.abs()
    return o, lse, size, mean


def bounds(o, lse, size, mean, keys, D, p_error, out_error=EPS16):
    """How far a kernel that rounds as documented may be off: o's own rounding
    (half a step of its type); P's own rounding p_error and the error of the scores
    (fp32 sums of D products: D 2^-24 of the sum of magnitudes, and the
    product with the scale, in numerator and denominator), weighted with |v|;
    the fp32 sums over the keys and exp2 / log2 within four units of 2^-23."""
    ds = (D + 4) * EPS32 * size + 8 * EPS32
    acc = (2 * keys + 8) * EPS32
    o_tol = out_error * o.abs() + (1 + EPS16) * (p_error + 2 * ds[..., None] + acc) * mean + 1e-30
    lse_tol = ds + acc + 4 * EPS32 * lse.abs().nan_to_num(0, 0, 0)
    return o_tol, lse_tol


def check(o, lse, ref, keys, D, p_error, label="", out_error=EPS16):
    o, lse = o.double().cpu(), lse.double().cpu()
    ro, rl = ref[0], ref[1]
    o_tol, lse_tol = bounds(*ref, keys, D, p_error, out_error)
    fin = torch.isfinite(rl)
    assert torch.equal(fin, torch.isfinite(lse)), f"{label}: rows without a key differ"
    assert bool((lse[~fin] == -math.inf).all()) and bool((o[~fin] == 0).all()), label
    bad = ((lse - rl).abs() > lse_tol) & fin
    assert not bool(bad.any()), f"{label}: lse at {bad.nonzero()[:4].tolist()}: {lse[bad][:4].tolist()} {rl[bad][:4].tolist()}"
    bad = (o - ro).abs() > o_tol
    assert not bool(bad.any()), (f"{label}: o at {bad.nonzero()[:4].tolist()}: {o[bad][:4].tolist()} {ro[bad][:4].tolist()} "
                                 f"bound {o_tol[bad][:4].tolist()}")


def e4m3(x):
    """The nearest E4M3 value, ties to even, saturating at 448; NaN stays."""
    a = x.abs().clamp(max=448.0)
    step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -9))).clamp(min=-6.0) - 3)
    return torch.copysign(torch.round(a / step) * step, x).where(~x.isnan(), x)


def page_exponent(amax):
    """Least e in [27, 246] with amax <= 448 2^(e-127)."""
    e = 27
    while e < 246 and not amax <= 448.0 * 2.0 ** (e - 127):
        e += 1
    return e


def append(pool, layer, k_new, v_new, cu, lens, table):
    """The append of new tokens on a Pool, page by page."""
    layers, pages, Hkv, page, D = pool.shape
    for b in range(len(lens)):
        n = int(cu[b + 1]) - int(cu[b])
        length = min(int(lens[b]), table.shape[1] * page)
        start = int(lens[b]) - n
        if n <= 0 or start < 0 or cu[b] < 0 or cu[b + 1] > k_new.shape[0]:
            continue
        for j in range(start // page, -(-length // page)):
            at = int(table[b, j])
            if not 0 <= at < pages:
                continue
            lo, hi = max(start, j * page) - j * page, min(length, (j + 1) * page) - j * page
            rows = slice(int(cu[b]) + j * page + lo - start, int(cu[b]) + j * page + hi - start)
            for new, codes, exps in ((k_new, pool.k, pool.ke), (v_new, pool.v, pool.ve)):
                for h in range(Hkv):
                    c = codes[layer, at, h]
                    old = c if codes is pool.k else c.transpose(-1, -2).reshape(page, D)
                    out = old.clone()
                    x = new[rows, h].double()
                    fin = x.nan_to_num(0.0, float("inf"), float("-inf")).abs()
                    e = page_exponent(float(fin.max()))
                    if lo > 0:
                        e0 = min(int(exps[layer, at, h]), 246)
                        if e > e0:
                            out[:lo] = e4m3(old[:lo].view(F8).double() * 2.0 ** (e0 - e)).float().to(F8).view(torch.uint8)
                        e = max(e, e0)
                    out[lo:hi] = e4m3((x * 2.0 ** (127 - e))).float().to(F8).view(torch.uint8)
                    exps[layer, at, h] = e
                    codes[layer, at, h] = out if codes is pool.k else out.reshape(page // 16, 16, D).transpose(-1, -2)


def fork(page, pages, table, lens, refs, parent, grow):
    """(table, lens, refs, missing, copies [(src, dst)])."""
    B, width = table.shape
    refs, held = refs.tolist(), refs.tolist()
    out, out_lens, need, missing = [], [], [], 0
    parent = parent.tolist()
    for row in table.tolist():
        for at in row:
            if 0 <= at < pages:
                refs[at] -= 1
    for i, p in enumerate(parent):
        row, n, tail, full = [-1] * width, 0, None, 0
        if 0 <= p < B:
            n = min(max(int(lens[p]), 0), width * page)
            full = -(-n // page)
            row[:full] = table[p, :full].tolist()
            if n % page:
                at = row[full - 1]
                if 0 <= at < pages and not (p not in parent[:i] and held[at] == 1):
                    tail = at
                    row[full - 1] = -1
            for c in range(full):
                if 0 <= row[c] < pages:
                    refs[row[c]] += 1
                else:
                    row[c] = -1
        want = -(-(n + (max(int(grow[i]), 0) if grow is not None else 0)) // page)
        more = max(min(want, width) - full, 0)
        missing += max(want - width, 0)
        out.append(row)
        out_lens.append(n)
        need.append((tail, full, more))
    free = [at for at in range(pages) if refs[at] == 0 and at not in {tail for tail, _, _ in need}]
    copies = []
    for i, (tail, full, more) in enumerate(need):
        for c in ([full - 1] if tail is not None else []) + list(range(full, full + more)):
            if not free:
                missing += 1
                continue
            at = free.pop(0)
            out[i][c] = at
            refs[at] = 1
            if tail is not None and c == full - 1:
                copies.append((tail, at))
    as_int = lambda v, *s: torch.tensor(v, dtype=torch.int32).reshape(*s)  # noqa: E731
    return as_int(out, len(parent), width), as_int(out_lens, -1), as_int(refs, -1), missing, copies


def compact(pages, table, refs):
    refs = refs.tolist()
    n = sum(r > 0 for r in refs)
    moves = list(zip([i for i in range(n, pages) if refs[i] > 0], [i for i in range(n) if refs[i] <= 0]))
    remap = [i if r > 0 else -1 for i, r in enumerate(refs)]
    out = refs[:n] + [0] * (pages - n)
    for src, dst in moves:
        remap[src], out[dst] = dst, refs[src]
    t = torch.tensor([[remap[x] if 0 <= x < pages else -1 for x in row] for row in table.tolist()], dtype=torch.int32)
    return t.reshape(table.shape), torch.tensor(out, dtype=torch.int32), torch.tensor(remap, dtype=torch.int32), n, moves


def moved(pool, moves):
    for src, dst in moves:
        for x in pool.arrays():
            x[:, dst] = x[:, src]
