"""The serving operators of the BAPS library: windowed attention with sink
tokens, the paged 8-bit key/value cache (append, attention) and the operators
on its pages (fork, compact).

listed() holds twelve cases and draw() gives more of the same ranges.  With
own = False a case runs in its plain form, elementary torch operations in 32
bits; with own = True it makes the library's calls.  exact() computes the
same in 64 bits, written apart from the plain form.

Sizes follow the library's workloads (GQA 32/8 at head dimension 128, 16 heads
at head dimension 64) with short, odd and ragged lengths beside them.

The cache holds FP8 E4M3 codes in pages of `page` tokens; every (page, head)
has one power-of-two scale for K and one for V, kept as its biased exponent e
(the value is code * 2^(e - 127)):
  k [layers, pages, Hkv, page, D],  v [layers, pages, Hkv, page / 16, D, 16],
  k_exp, v_exp [layers, pages, Hkv].
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
NINF = float("-inf")
# the scale's exponent: the least e with amax <= 448 * 2^e, within these bounds
EXP_LO, EXP_HI = 27, 246


# ------------------------------------------------------------------ the cases
def _window(name=None, B=1, Hq=32, Hkv=8, Sq=1, Sk=1, D=128, window=1024, sinks=4):
    c = dict(op="window", B=B, Hq=Hq, Hkv=Hkv, Sq=Sq, Sk=Sk, D=D, window=window, sinks=sinks)
    return dict(c, name=name) if name else c


def _cache(op, name=None, B=1, Hq=32, Hkv=8, D=128, page=64, lo=1, hi=1, new_lo=1, new_hi=1, window=0, sinks=0):
    """Lengths after the new tokens are spread over [lo, hi], new tokens over [new_lo, new_hi]."""
    c = dict(op=op, B=B, Hq=Hq, Hkv=Hkv, D=D, page=page, lo=lo, hi=hi, new_lo=new_lo, new_hi=new_hi, window=window,
             sinks=sinks)
    return dict(c, name=name) if name else c


def _fork(name=None, B=4, B_out=4, keep=3, layers=2, Hkv=8, D=128, page=16, lo=1, hi=64, grow=1):
    """B_out sequences that go on from the first `keep` of B."""
    c = dict(op="fork", B=B, B_out=B_out, keep=keep, layers=layers, Hkv=Hkv, D=D, page=page, lo=lo, hi=hi, grow=grow)
    return dict(c, name=name) if name else c


def _compact(name=None, layers=2, pages=256, live=0.5, rows=8, Hkv=8, D=128, page=16):
    c = dict(op="compact", layers=layers, pages=pages, live=live, rows=rows, Hkv=Hkv, D=D, page=page)
    return dict(c, name=name) if name else c


def listed():
    return [
        # one decode step of a few chats with a sliding window: latency, and few workgroups without a split
        _window("window_decode_b3_5001", B=3, Sk=5001, window=1024),
        # prompts of odd length through an encoder-sized layer with a short window
        _window("window_prompt_1501_d64", B=2, Hq=16, Hkv=16, Sq=1501, Sk=1501, D=64, window=300, sinks=0),
        # a long document in one call: the largest matrix work of the windowed layers
        _window("window_prefill_16384", Sq=16384, Sk=16384, window=4096, sinks=4),
        # one decode step of a small ragged batch, small pages, a window with sinks
        _cache("attention", "cache_decode_b5_window", B=5, page=16, lo=700, hi=4003, window=2048, sinks=4),
        # batched decode of a serving loop: streams the cache
        _cache("attention", "cache_decode_b64_8192", B=64, lo=5000, hi=8192),
        # chunked prefill: the next tokens of three prompts against what is cached
        _cache("attention", "cache_chunk_b3_9001", B=3, lo=2500, hi=9001, new_lo=777, new_hi=2048),
        # a decode step's new tokens into the cache
        _cache("append", "append_decode_b48", B=48, lo=100, hi=4000),
        # the prompts of a batch into the cache, head dimension 128, odd lengths
        _cache("append", "append_prompts_b8", B=8, lo=2100, hi=6500, new_lo=2100, new_hi=6500),
        # beam search or sampled continuations: eight beams go on from five, all layers of a small model
        _fork("fork_beams_b8", B=8, B_out=8, keep=5, layers=4, page=16, lo=60, hi=400),
        # a serving batch: finished requests leave, prompts fan out, every row gets its next pages
        _fork("fork_batch_b192", B=160, B_out=192, keep=120, layers=4, page=64, lo=40, hi=2000, grow=64),
        # closing the holes of a small pool
        _compact("compact_512", layers=2, pages=512, live=0.4, rows=16, page=16),
        # a large pool after a burst of requests, before it is given back
        _compact("compact_3000", layers=4, pages=3000, live=0.55, rows=64, page=64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "window", "attention", "attention", "append", "fork", "compact"])
    D = rng.choice([64, 128, 128])
    Hkv = rng.choice([1, 2, 4, 8, 8])
    Hq = Hkv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8])
    page = rng.choice([16, 32, 64, 64, 128])
    if op == "window":
        window, sinks = _log(rng, 16, 4096), rng.choice([0, 1, 4, 4, 16, 130])
        if rng.random() < 0.4:                                   # decode, or a few drafted tokens
            return _window(None, rng.randint(1, 16), Hq, Hkv, rng.choice([1, 1, 2, 5]), _log(rng, 40, 20000), D, window,
                           sinks)
        Sq = _log(rng, 33, 8000)
        return _window(None, rng.choice([1, 1, 2]), min(Hq, 32), min(Hkv, 8), Sq, Sq + rng.choice([0, 0, 500, 3001]), D,
                       window, sinks)
    if op == "attention":
        window, sinks = rng.choice([(0, 0), (0, 0), (_log(rng, 64, 4096), rng.choice([0, 1, 4, 20]))])
        if rng.random() < 0.55:
            B = _log(rng, 1, 64)
            hi = _log(rng, 30, min(60000, 500000 // B))
            return _cache(op, None, B, min(Hq, 40), Hkv, D, page, _log(rng, 1, hi), hi, 1, rng.choice([1, 1, 1, 4]), window,
                          sinks)
        hi = _log(rng, 40, 12000)
        return _cache(op, None, rng.randint(1, 4), min(Hq, 32), Hkv, D, page, _log(rng, 20, hi), hi, _log(rng, 9, 500),
                      _log(rng, 500, 2000), window, sinks)
    if op == "append":
        if rng.random() < 0.5:
            return _cache(op, None, _log(rng, 1, 256), Hkv, Hkv, D, page, 1, _log(rng, 20, 4000), 1, rng.choice([1, 1, 5]))
        hi = _log(rng, 100, 6500)
        return _cache(op, None, rng.randint(1, 8), Hkv, Hkv, D, page, _log(rng, 20, hi), hi, _log(rng, 10, 100), hi)
    if op == "fork":
        B = _log(rng, 2, 128)
        return _fork(None, B, _log(rng, 2, 160), rng.randint(1, B), rng.choice([1, 2, 4]), Hkv, D, page, _log(rng, 1, 60),
                     _log(rng, 60, 1500), rng.choice([0, 1, 30]))
    return _compact(None, rng.choice([1, 2, 4]), _log(rng, 64, min(6000, 190000 // page)), round(rng.uniform(0.1, 0.95), 3), rng.randint(1, 64),
                    Hkv, D, page)


def _spread(n, lo, hi, phase=0.618034):
    """n whole numbers over [lo, hi], the same for every seed (work() goes by them)."""
    lo = min(lo, hi)
    return [lo + int((hi - lo + 1) * ((i + 1) * phase % 1.0)) for i in range(n)]


def _lengths(c):
    lens = _spread(c["B"], c["lo"], c["hi"])
    lens[-1] = c["hi"]
    new = [min(n, m) for n, m in zip(lens, _spread(c["B"], c["new_lo"], c["new_hi"], 0.7548777))]
    new[-1] = min(c["hi"], c["new_hi"])
    return lens, new


def _parents(c):
    """What the B_out sequences go on from: every kept one once, then some of them again."""
    return [i if i < c["keep"] else int(c["keep"] * (i * 0.618034 % 1.0)) for i in range(c["B_out"])]


# ------------------------------------------------------------------ inputs
def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(int(seed))


def _normal(g, *shape, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(torch.bfloat16)


def _keys(g, *shape):
    """Keys as a model has them: each token with a norm of its own (log-normal),
    a hundredth of the channels several times the others."""
    x = torch.randn(shape, generator=g, device=DEV)
    x *= torch.exp(0.5 * torch.randn(shape[:-1], generator=g, device=DEV))[..., None]
    x[..., :: 97] *= 6.0
    return x.to(torch.bfloat16)


def _up(n, m):
    return -(-n // m)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _tables(g, counts, pages, width):
    """Page tables: row i holds counts[i] pages of its own, in a random order over the pool; -1 behind them."""
    perm = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    cols = torch.arange(width, device=DEV)
    n = torch.tensor(counts, device=DEV)
    at = (torch.cumsum(n, 0) - n)[:, None] + cols
    return torch.where(cols < n[:, None], perm[at.clamp(max=pages - 1)], -1).to(torch.int32).contiguous()


def _codes(g, *shape):
    x = torch.randint(0, 256, shape, generator=g, device=DEV, dtype=torch.uint8)
    return x - ((x & 0x7F) == 0x7F).to(torch.uint8)              # (no NaN codes)


def _prepare_cache(c, seed):
    g = _gen(seed)
    lens, new = _lengths(c)
    B, Hkv, D, page = c["B"], c["Hkv"], c["D"], c["page"]
    counts = [_up(n, page) for n in lens]
    pages, width = sum(counts) + 8, max(counts)
    st = dict(op=c["op"], page=page, max_len=max(lens), max_new=max(new), window=c["window"], sinks=c["sinks"])
    st["table"] = _tables(g, counts, pages, width)
    st["lens"] = _ints(lens)
    st["cu"] = _ints([sum(new[:i]) for i in range(B + 1)])
    if c["op"] == "attention":
        # a pool that an earlier call has filled: quantised keys and values
        k, ke, v, ve = [], [], [], []
        for n in torch.arange(pages).split(1024):
            x, e = _quantise(_keys(g, len(n), Hkv, page, D).float())
            k.append(x)
            ke.append(e)
            x, e = _quantise(torch.randn((len(n), Hkv, page, D), generator=g, device=DEV))
            v.append(_v_to_pool(x))
            ve.append(e)
        st["k"], st["k_exp"], st["v"], st["v_exp"] = (torch.cat(x)[None].contiguous() for x in (k, ke, v, ve))
        st["q"] = _normal(g, sum(new), c["Hq"], D, scale=1.0)
    else:
        st["k"], st["v"] = _codes(g, 1, pages, Hkv, page, D), _codes(g, 1, pages, Hkv, page // 16, D, 16)
        st["k_exp"], st["v_exp"] = (torch.randint(115, 122, (1, pages, Hkv), generator=g, device=DEV, dtype=torch.uint8)
                                    for _ in range(2))
        st["k_new"], st["v_new"] = _keys(g, sum(new), Hkv, D), _normal(g, sum(new), Hkv, D)
    return st


def _prepare_pool(g, c, pages):
    Hkv, D, page, layers = c["Hkv"], c["D"], c["page"], c["layers"]
    st = dict(op=c["op"], page=page)
    st["k"], st["v"] = _codes(g, layers, pages, Hkv, page, D), _codes(g, layers, pages, Hkv, page // 16, D, 16)
    st["k_exp"], st["v_exp"] = (torch.randint(110, 130, (layers, pages, Hkv), generator=g, device=DEV, dtype=torch.uint8)
                                for _ in range(2))
    return st


def _prepare_fork(c, seed):
    g = _gen(seed)
    lens = _spread(c["B"], c["lo"], c["hi"])
    counts = [_up(n, c["page"]) for n in lens]
    width = max(counts) + _up(c["grow"], c["page"])
    pages = sum(counts) + c["B_out"] * (1 + _up(c["grow"], c["page"])) + 5
    st = _prepare_pool(g, c, pages)
    st["table"] = _tables(g, counts, pages, width)
    st["refs"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
    st["refs"][st["table"][st["table"] >= 0].long()] = 1
    st["lens"], st["parent"] = _ints(lens), _ints(_parents(c))
    st["grow"] = _ints([c["grow"]] * c["B_out"])
    return st


def _live(c):
    return [i for i in range(c["pages"]) if (i + 1) * 0.618034 % 1.0 < c["live"]]


def _prepare_compact(c, seed):
    g = _gen(seed)
    st = _prepare_pool(g, c, c["pages"])
    live = torch.tensor(_live(c), device=DEV)
    st["refs"] = torch.zeros(c["pages"], dtype=torch.int32, device=DEV)
    st["refs"][live] = 1
    width = _up(len(live), c["rows"]) + 2
    own_pages = live[torch.randperm(len(live), generator=g, device=DEV)]
    table = torch.full((c["rows"], width), -1, dtype=torch.int32, device=DEV)
    at = torch.arange(len(live), device=DEV)
    table[at % c["rows"], at // c["rows"] + 1] = own_pages.to(torch.int32)
    shared = live[:1].to(torch.int32)                            # a prefix page that every row holds
    table[:, 0] = shared
    st["refs"][live[:1]] += c["rows"]
    st["table"] = table
    return st


def prepare(case, seed):
    c = case
    if c["op"] == "window":
        g = _gen(seed)
        return dict(op="window", window=c["window"], sinks=c["sinks"], q=_normal(g, c["B"], c["Hq"], c["Sq"], c["D"]),
                    k=_keys(g, c["B"], c["Hkv"], c["Sk"], c["D"]), v=_normal(g, c["B"], c["Hkv"], c["Sk"], c["D"]))
    st = {"attention": _prepare_cache, "append": _prepare_cache, "fork": _prepare_fork, "compact": _prepare_compact}[
        c["op"]](c, seed)
    if own:
        # the handle that a program keeps for its cache
        import paper_2602_02071_amd as baps
        st["cache"] = baps.PagedCache(st["k"], st["v"], st["k_exp"], st["v_exp"])
    return st


# ------------------------------------------------------------------ the plain forms
def _quantise(x):
    """fp32 [.., Hkv, page, D] -> (E4M3 codes, exponents [.., Hkv])."""
    e = _exponents(x.abs().amax((-1, -2)))
    return _encode(x, e[..., None, None]), e.to(torch.uint8)


def _exponents(amax):
    m, x = torch.frexp(amax)                                     # amax = m 2^x, m in [0.5, 1): 448 = 0.875 2^9
    e = x - 9 + (m > 0.875).int() + 127
    return torch.where(amax > 0, e, EXP_LO).clamp(EXP_LO, EXP_HI)


def _encode(x, e):
    return (torch.ldexp(x, 127 - e).clamp(-448, 448)).to(torch.float8_e4m3fn).view(torch.uint8)


def _values(codes, e):
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float(), e.int() - 127)


def _v_to_pool(x):
    """[.., page, D] -> [.., page / 16, D, 16]."""
    return x.unflatten(-2, (-1, 16)).transpose(-1, -2).contiguous()


def _v_from_pool(x):
    return x.transpose(-1, -2).flatten(-3, -2)


def _softmax_rows(s, v):
    """s [n, rows, keys] scores with -inf where masked, v [n, keys, D]: (o, lse); a row with no key gives 0, -inf."""
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == NINF, 0.0, m)
    p = torch.exp(s.sub_(m))
    d = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(d > 0, d, 1.0), (m + torch.log(d)).squeeze(-1)


def _visible(pos, key, window, sinks):
    """Whether the query at position pos sees the key: causal, within the window or a sink."""
    seen = key <= pos
    return seen & ((key > pos - window) | (key < sinks)) if window else seen


def _plain_window(st):
    q, k, v = (st[x].float() for x in "qkv")
    B, Hq, Sq, D = q.shape
    Hkv, Sk = k.shape[1], k.shape[2]
    G = Hq // Hkv
    q = (q / math.sqrt(D)).view(B * Hkv, G, Sq, D)
    k, v = k.reshape(B * Hkv, Sk, D), v.reshape(B * Hkv, Sk, D)
    kt = k.transpose(1, 2).contiguous()
    key = torch.arange(Sk, device=q.device)
    o, lse = [], []
    for r0 in range(0, Sq, 1024):                                # (queries in parts: all scores at once would not fit)
        n = min(1024, Sq - r0)
        pos = torch.arange(r0, r0 + n, device=q.device) + (Sk - Sq)
        lo, hi = max(0, r0 + Sk - Sq - st["window"] + 1), r0 + n + Sk - Sq
        ns = min(st["sinks"], lo)                                # sinks in front of the part's window
        cut = lambda x, d: torch.cat((x.narrow(d, 0, ns), x.narrow(d, lo, hi - lo)), d)  # noqa: E731
        s = torch.matmul(q[:, :, r0:r0 + n].reshape(B * Hkv, G * n, D), cut(kt, 2))
        seen = _visible(pos[:, None], cut(key, 0)[None, :], st["window"], st["sinks"])
        s.masked_fill_(~seen.repeat(G, 1), NINF)
        x, y = _softmax_rows(s, cut(v, 1))
        o.append(x.view(B, Hq, n, D))
        lse.append(y.view(B, Hq, n))
    return dict(o=torch.cat(o, 2).to(torch.bfloat16), lse=torch.cat(lse, 2))


def _plain_attention(st):
    page, B = st["page"], st["lens"].numel()
    at = st["table"].clamp(min=0).long()
    k = _values(st["k"][0][at], st["k_exp"][0][at][..., None, None])          # [B, n, Hkv, page, D]
    v = _values(_v_from_pool(st["v"][0][at]), st["v_exp"][0][at][..., None, None])
    Hkv, D = k.shape[2], k.shape[4]
    k = k.permute(0, 2, 4, 1, 3).reshape(B * Hkv, D, -1)                       # K^T
    v = v.transpose(1, 2).reshape(B * Hkv, -1, D)
    q = st["q"].float() / math.sqrt(D)
    Hq = q.shape[1]
    G, mq = Hq // Hkv, st["max_new"]
    lens, cu = st["lens"].long(), st["cu"].long()
    n = cu[1:] - cu[:-1]
    i = torch.arange(mq, device=q.device)
    rows = (cu[:-1, None] + i).clamp(max=q.shape[0] - 1)                       # [B, mq] packed rows
    qp = q[rows].view(B, mq, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * mq, D)
    pos = (lens - n)[:, None] + i                                              # [B, mq]
    key = torch.arange(k.shape[2], device=q.device)
    seen = _visible(pos[:, :, None], key, st["window"], st["sinks"])
    s = torch.matmul(qp, k).view(B, Hkv, G, mq, -1)
    s.masked_fill_(~seen[:, None, None], NINF)
    o, lse = _softmax_rows(s.view(B * Hkv, G * mq, -1), v)
    o = o.view(B, Hkv, G, mq, D).permute(0, 3, 1, 2, 4).reshape(B, mq, Hq, D)
    lse = lse.view(B, Hkv, G, mq).permute(0, 3, 1, 2).reshape(B, mq, Hq)
    held = i < n[:, None]
    return dict(o=o[held].to(torch.bfloat16), lse=lse[held])


def _pool_out(st, **more):
    """The cache as values: codes as the 8-bit floats that they are, scales as their exponents."""
    f8 = torch.float8_e4m3fn
    return dict(k=st["k"].view(f8), v=st["v"].view(f8), k_exp=st["k_exp"], v_exp=st["v_exp"], **more)


def _plain_append(st):
    page, B = st["page"], st["lens"].numel()
    lens, cu = st["lens"].long(), st["cu"].long()
    start = lens - (cu[1:] - cu[:-1])
    first = start // page
    T = _up(st["max_new"] + page - 1, page)                                    # pages that a row may touch
    slot = first[:, None] + torch.arange(T, device=lens.device)                # [B, T]
    valid = (slot * page < lens[:, None]) & (slot < st["table"].shape[1])
    at = st["table"].long().gather(1, slot.clamp(max=st["table"].shape[1] - 1))
    pos = slot[..., None] * page + torch.arange(page, device=lens.device)      # [B, T, page]
    fresh = (pos >= start[:, None, None]) & (pos < lens[:, None, None])
    held = pos < start[:, None, None]
    row = (cu[:-1, None, None] + pos - start[:, None, None]).clamp(0, st["k_new"].shape[0] - 1)
    keep = valid.nonzero(as_tuple=True)
    at, row, fresh, held = at[keep], row[keep], fresh[keep], held[keep]
    for name in "kv":
        x = st[name + "_new"][row].float().transpose(1, 2)                     # [n, Hkv, page, D]
        pool, exps = st[name][0], st[name + "_exp"][0]
        old = pool[at] if name == "k" else _v_from_pool(pool[at])
        new, before = fresh[:, None, :, None], held[:, None, :, None]
        e0 = torch.where(held.any(-1)[:, None], exps[at].int(), 0)
        e = torch.maximum(_exponents(torch.where(new, x, 0).abs().amax((-1, -2))), e0)
        moved = _encode(_values(old, e0[..., None, None]), e[..., None, None])
        out = torch.where(new, _encode(x, e[..., None, None]), torch.where(before & (e > e0)[..., None, None], moved, old))
        pool[at] = out if name == "k" else _v_to_pool(out)
        exps[at] = e.to(torch.uint8)
    return _pool_out(st)


def _plain_fork(st):
    page, table, refs = st["page"], st["table"].long(), st["refs"]
    parent, lens = st["parent"].long(), st["lens"].long()
    P, width = refs.numel(), table.shape[1]
    L = lens[parent]
    full = _up(L, page)
    wanted = _up(L + st["grow"], page)
    twin = parent[:, None] == parent[None, :]
    first = ~(twin & torch.ones_like(twin).tril(-1)).any(1)                    # the first that goes on from its parent
    tail = table[parent].gather(1, (full - 1).clamp(min=0)[:, None])[:, 0]
    copied = (L % page != 0) & ~(first & (refs[tail.clamp(min=0)] == 1))
    col = torch.arange(width, device=table.device)
    taken = (col < full[:, None]) & ~(copied[:, None] & (col == full[:, None] - 1))
    fresh = (copied[:, None] & (col == full[:, None] - 1)) | ((col >= full[:, None]) & (col < wanted[:, None]))
    out = torch.where(taken, table[parent], -1)
    count = lambda x: torch.bincount(x[x >= 0], minlength=P).int()  # noqa: E731
    refs = refs - count(table) + count(out)
    free = (refs == 0).nonzero()[:, 0]
    rank = (fresh.flatten().cumsum(0) - 1).view_as(fresh)
    out = torch.where(fresh, free[rank.clamp(0, free.numel() - 1)], out)
    refs[out[fresh]] = 1
    src, dst = tail[copied], out.gather(1, (full - 1).clamp(min=0)[:, None])[:, 0][copied]
    for name in ("k", "v", "k_exp", "v_exp"):
        st[name][:, dst] = st[name][:, src]
    short = torch.zeros(1, dtype=torch.int32, device=table.device)
    return _pool_out(st, table=out.int(), lens=L.int(), refs=refs, short=short)


def _plain_compact(st):
    refs = st["refs"]
    held = refs > 0
    n = held.sum()
    index = torch.arange(refs.numel(), device=refs.device)
    to, frm = (~held & (index < n)).nonzero()[:, 0], (held & (index >= n)).nonzero()[:, 0]
    remap = torch.where(held, index, -1)
    remap[frm] = to
    out = torch.zeros_like(refs)
    out[remap[held]] = refs[held]
    for name in ("k", "v", "k_exp", "v_exp"):
        st[name][:, to] = st[name][:, frm]
    table = torch.where(st["table"] >= 0, remap[st["table"].clamp(min=0).long()], -1)
    return _pool_out(st, table=table.int(), refs=out, remap=remap.int(), live=n.int().view(1))


# ------------------------------------------------------------------ the library's calls
def _own(st):
    import paper_2602_02071_amd as baps
    op = st["op"]
    if op == "window":
        o, lse = baps.attention_window(st["q"], st["k"], st["v"], st["window"], st["sinks"], mode=baps.BAPS_MODE_DEFAULT,
                                       out_bf16=True)
        return dict(o=o, lse=lse)
    cache = st["cache"]
    if op == "attention":
        o, lse = cache.attention(0, st["q"], st["cu"], st["lens"], st["table"], st["max_new"], st["max_len"], st["window"],
                                 st["sinks"])
        return dict(o=o, lse=lse)
    if op == "append":
        cache.append(0, st["k_new"], st["v_new"], st["cu"], st["lens"], st["table"], st["max_new"])
        return _pool_out(st)
    if op == "fork":
        table, lens, refs, short = cache.fork(st["table"], st["lens"], st["refs"], st["parent"], st["grow"])
        return _pool_out(st, table=table, lens=lens, refs=refs, short=short)
    table, refs, remap, live = cache.compact(st["table"], st["refs"])
    return _pool_out(st, table=table, refs=refs, remap=remap, live=live)


PLAIN = dict(window=_plain_window, attention=_plain_attention, append=_plain_append, fork=_plain_fork, compact=_plain_compact)


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["op"]](state)


# ------------------------------------------------------------------ least bytes and operations
def _pairs(first, n, window, sinks):
    """Keys that the n queries at positions first, first + 1, .. see, all together."""
    total = 0
    for t in range(first, first + n):
        if t >= 0:
            total += t + 1 if not window else min(t + 1, window) + max(0, min(sinks, t + 1 - window))
    return total


def _reach(first, n, window, sinks):
    """Keys that any of them sees."""
    last = first + n
    if last <= 0 or n <= 0:
        return 0
    lo = max(0, first - window + 1) if window else 0
    return last - lo + min(lo, sinks)


def work(case):
    c = case
    if c["op"] == "window":
        first = c["Sk"] - c["Sq"]
        pairs, reach = _pairs(first, c["Sq"], c["window"], c["sinks"]), _reach(first, c["Sq"], c["window"], c["sinks"])
        q = c["B"] * c["Hq"] * c["Sq"]
        return dict(bytes=q * (4 * c["D"] + 4) + 4 * c["B"] * c["Hkv"] * reach * c["D"],
                    flops=4.0 * c["D"] * c["B"] * c["Hq"] * pairs)
    if c["op"] == "compact":
        live = _live(c)
        moved = sum(i >= len(live) for i in live)
        per = c["layers"] * c["Hkv"] * 2 * (c["page"] * c["D"] + 1)
        return dict(bytes=2 * moved * per + 12 * c["pages"] + 8 * len(live), flops=0)
    if c["op"] == "fork":
        lens, parents = _spread(c["B"], c["lo"], c["hi"]), _parents(c)
        copies = sum(lens[p] % c["page"] != 0 and p in parents[:i] for i, p in enumerate(parents))
        width = _up(max(lens), c["page"]) + _up(c["grow"], c["page"])
        pages = sum(_up(n, c["page"]) for n in lens) + c["B_out"] * (1 + _up(c["grow"], c["page"])) + 5
        per = c["layers"] * c["Hkv"] * 2 * (c["page"] * c["D"] + 1)
        return dict(bytes=2 * copies * per + 8 * pages + 4 * width * (c["B"] + c["B_out"]) + 16 * c["B_out"], flops=0)
    lens, new = _lengths(c)
    if c["op"] == "append":
        # each new K and V element read in 16 bits and written in 8
        return dict(bytes=2 * 3 * sum(new) * c["Hkv"] * c["D"] + 8 * c["B"] * c["Hkv"], flops=0)
    pairs = sum(_pairs(n - m, m, c["window"], c["sinks"]) for n, m in zip(lens, new))
    reach = sum(_reach(n - m, m, c["window"], c["sinks"]) for n, m in zip(lens, new))
    return dict(bytes=2 * c["Hkv"] * reach * c["D"] + sum(new) * c["Hq"] * (4 * c["D"] + 4),
                flops=4.0 * c["D"] * c["Hq"] * pairs)


# ------------------------------------------------------------------ the definition in 64 bits
def _exact_rows(q, k, v, pos, window, sinks):
    """One key/value head: q [n, D] at positions pos, keys 0.. of k and v [len, D], all in 64 bits."""
    s = (q @ k.t()) / math.sqrt(q.shape[1])
    c = torch.arange(k.shape[0], device=q.device).expand_as(s)
    t = pos[:, None]
    hidden = c > t
    if window:
        hidden |= (c <= t - window) & (c >= sinks)
    s[hidden] = NINF
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - torch.where(lse == NINF, 0.0, lse)[:, None])
    return p @ v, lse


def _e4m3(x):
    """The nearest E4M3 value, ties to the even code, of 64-bit x with |x| <= 448."""
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -9))).clamp(min=-6.0) - 3)
    return torch.round(x / step) * step


def _exact_append(c, seed):
    st = _prepare_cache(c, seed)
    lens, new = _lengths(c)
    page, cu = c["page"], st["cu"].tolist()
    out = {}
    for name in "kv":
        codes = st[name][0] if name == "k" else st[name][0].transpose(-1, -2).flatten(-3, -2)
        val = codes.view(torch.float8_e4m3fn).double()                         # [pages, Hkv, page, D]
        exps = st[name + "_exp"][0].double() - 127
        x = st[name + "_new"].double().transpose(0, 1)                         # [Hkv, T, D]
        table = st["table"].tolist()
        for b in range(c["B"]):
            start = lens[b] - new[b]
            for j in range(start // page, _up(lens[b], page)):
                at, lo, hi = table[b][j], max(start, j * page), min(lens[b], (j + 1) * page)
                if lo >= hi:
                    continue
                y = x[:, cu[b] + lo - start: cu[b] + hi - start]
                amax = y.abs().amax((1, 2))
                e = torch.ceil(torch.log2(amax / 448)).clamp(EXP_LO - 127, EXP_HI - 127)
                n = lo - j * page                                              # tokens that the page held
                if n:
                    e = torch.maximum(e, exps[at])
                    val[at, :, :n] = _e4m3(val[at, :, :n] * torch.exp2(exps[at] - e)[:, None, None])
                val[at, :, n:n + hi - lo] = _e4m3(y * torch.exp2(-e)[:, None, None])
                exps[at] = e
        if name == "v":
            val = val.unflatten(-2, (-1, 16)).transpose(-1, -2)
        out[name] = val[None].contiguous()
    return dict(out, k_exp=None, v_exp=None)


def _exact_fork(c, seed):
    st = _prepare_fork(c, seed)
    refs, table, lens, page = st["refs"].tolist(), st["table"].tolist(), st["lens"].tolist(), c["page"]
    held = list(refs)
    parents, tails = _parents(c), []
    for row in table:
        for at in row:
            if at >= 0:
                refs[at] -= 1
    for i, p in enumerate(parents):
        n = _up(lens[p], page)
        tail = table[p][n - 1]
        tails.append(tail if lens[p] % page and (p in parents[:i] or held[tail] != 1) else None)
        for at in table[p][:n] if tails[-1] is None else table[p][:n - 1]:
            refs[at] += 1
    free = iter([at for at, n in enumerate(refs) if n == 0])
    moves = []
    for i, p in enumerate(parents):
        if tails[i] is not None:
            moves.append((tails[i], next(free)))
        for _ in range(_up(lens[p] + c["grow"], page) - _up(lens[p], page)):
            next(free)
    return _exact_moves(st, moves, ("k", "v", "k_exp", "v_exp", "table", "lens", "refs", "short"))


def _exact_compact(c, seed):
    st = _prepare_compact(c, seed)
    refs = st["refs"].tolist()
    n = sum(x > 0 for x in refs)
    moves = list(zip([i for i in range(n, len(refs)) if refs[i] > 0], [i for i in range(n) if refs[i] <= 0]))
    return _exact_moves(st, moves, ("k", "v", "k_exp", "v_exp", "table", "refs", "remap", "live"))


def _exact_moves(st, moves, names):
    """Pages move as they are: the codes' values behind the moves, whole numbers left out."""
    out = dict.fromkeys(names)
    for name in "kv":
        x = st[name].view(torch.float8_e4m3fn).double()
        for src, dst in moves:
            x[:, dst] = x[:, src]
        out[name] = x
    return out


def exact(case, seed):
    c = case
    if c["op"] == "window":
        st = prepare(case, seed)
        q, k, v = (st[x].double() for x in "qkv")
        o = torch.empty_like(q)
        lse = torch.empty(q.shape[:3], dtype=torch.float64, device=DEV)
        shift = c["Sk"] - c["Sq"]
        for b in range(c["B"]):
            for h in range(c["Hq"]):
                g = h // (c["Hq"] // c["Hkv"])
                for r0 in range(0, c["Sq"], 4096):
                    pos = torch.arange(r0, min(c["Sq"], r0 + 4096), device=DEV) + shift
                    r = slice(r0, r0 + len(pos))
                    o[b, h, r], lse[b, h, r] = _exact_rows(q[b, h, r], k[b, g], v[b, g], pos, c["window"], c["sinks"])
        return dict(o=o, lse=lse)
    if c["op"] == "attention":
        st = _prepare_cache(c, seed)
        lens, new = _lengths(c)
        cu, D, G = st["cu"].tolist(), c["D"], c["Hq"] // c["Hkv"]
        q = st["q"].double()
        o = torch.empty_like(q)
        lse = torch.empty(q.shape[:2], dtype=torch.float64, device=DEV)
        for b in range(c["B"]):
            at = st["table"][b, :_up(lens[b], c["page"])].long()
            k = st["k"][0, at].view(torch.float8_e4m3fn).double() * torch.exp2(st["k_exp"][0, at].double() - 127)[..., None, None]
            v = st["v"][0, at].view(torch.float8_e4m3fn).double() * torch.exp2(st["v_exp"][0, at].double() - 127)[..., None, None, None]
            v = v.permute(1, 0, 2, 4, 3).reshape(c["Hkv"], -1, D)[:, :lens[b]]
            k = k.transpose(0, 1).reshape(c["Hkv"], -1, D)[:, :lens[b]]
            pos = torch.arange(lens[b] - new[b], lens[b], device=DEV)
            for g in range(c["Hkv"]):
                rows = q[cu[b]:cu[b + 1], g * G:(g + 1) * G]                   # [n, G, D]
                x, y = _exact_rows(rows.reshape(-1, D), k[g], v[g], pos.repeat_interleave(G), c["window"], c["sinks"])
                o[cu[b]:cu[b + 1], g * G:(g + 1) * G] = x.view(-1, G, D)
                lse[cu[b]:cu[b + 1], g * G:(g + 1) * G] = y.view(-1, G)
        return dict(o=o, lse=lse)
    return {"append": _exact_append, "fork": _exact_fork, "compact": _exact_compact}[c["op"]](c, seed)
