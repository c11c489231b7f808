"""Attention with a sliding window and sinks: the Default setup against a 64-bit
implementation, Alg. 1 (E2E HiF8) against a replay of its steps on the matrix
unit's own scores, and the equality with plain causal attention where the
window covers every key."""
import math

import numpy as np
import pytest
import torch

import helpers_cache as H
import oracle as O
from helpers import ARB_TOL, dev_bf16, lse_arb_tol
from paper_2602_02071_amd.workloads import bf16_bits_to_f32, make_qkv, make_slow_climb

pytestmark = pytest.mark.gpu
DEFAULT, E2E = O.DEFAULT, O.E2E_HIF8


def _default(shape, window, sinks, block, out_bf16=False, seed=1, q_scale=1.0, scale_log2=0.0):
    import paper_2602_02071_amd as baps
    B, Hq, Hkv, Sq, Sk, D = shape
    q, k, v = make_qkv(B, Hq, Hkv, Sq, Sk, D, seed=seed, outliers=True, q_scale=q_scale)
    o, lse = baps.attention_window(dev_bf16(q), dev_bf16(k), dev_bf16(v), window, sinks, block, mode=baps.BAPS_MODE_DEFAULT,
                                   out_bf16=out_bf16, scale_log2=scale_log2)
    torch.cuda.synchronize()
    assert o.dtype == (torch.bfloat16 if out_bf16 else torch.float32)
    q, k, v = (torch.from_numpy(bf16_bits_to_f32(x)) for x in (q, k, v))
    few = Sq * (Hq // Hkv) <= 64
    scale = scale_log2 * math.log(2.0) if scale_log2 else None
    for b in range(B):
        ref = H.attend(q[b].transpose(0, 1), k[b].double(), v[b].double(), range(Sk - Sq, Sk), window, sinks, scale=scale)
        H.check(o[b].transpose(0, 1), lse[b].transpose(0, 1), ref, max(Sk, 1), D, 2.0 ** -16 if few else 2.0 ** -8,
                f"{shape} {window} {sinks} {block}", H.EPS16 if out_bf16 else H.EPS32)


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (70, 4), (128, 130), (257, 1), (4000, 0)])
def test_default_decode(D, block, window, sinks):
    _default((2, 8, 2, 1, 700, D), window, sinks, block)


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (70, 4), (129, 200)])
def test_default_prompt(D, block, window, sinks):
    _default((1, 4, 2, 203, 301, D), window, sinks, block)


@pytest.mark.parametrize("shape", [(1, 1, 1, 1, 1, 64), (1, 3, 1, 5, 40, 128), (3, 5, 5, 13, 13, 64), (1, 16, 1, 4, 333, 128),
                                   (1, 7, 1, 100, 90, 128), (1, 2, 2, 600, 600, 64), (1, 14, 2, 77, 500, 128), (2, 1, 1, 9, 5, 64)])
def test_default_shapes(shape):
    """One token, odd groups, more queries than keys (rows that see none), several items."""
    for window, sinks in ((50, 3), (1, 1)):
        _default(shape, window, sinks, 64, out_bf16=True)


@pytest.mark.parametrize("mode", [DEFAULT, E2E])
@pytest.mark.parametrize("shape", [(2, 8, 2, 1, 700, 128), (1, 4, 1, 13, 333, 64), (1, 4, 2, 203, 601, 128), (1, 2, 2, 130, 900, 64),
                                   (1, 2, 1, 100, 2500, 128), (1, 32, 32, 600, 1100, 128), (4, 35, 35, 400, 701, 64)])
def test_hidden_keys_may_be_anything(shape, mode):
    """NaN and infinities where the windows of all rows end, between them and the sinks: the bits are those of zeros there."""
    import paper_2602_02071_amd as baps
    B, Hq, Hkv, Sq, Sk, D = shape
    q, k, v = (dev_bf16(x) for x in make_qkv(B, Hq, Hkv, Sq, Sk, D, seed=3))
    for window, sinks, block in ((1, 0, 64), (77, 3, 128), (200, 70, 32), (min(1900, Sk - Sq - 1), 0, 64)):
        got = []
        for fill in (0.0, math.nan, math.inf):
            kk, vv = k.clone(), v.clone()
            kk[:, :, sinks:max(Sk - Sq - window + 1, sinks)] = fill
            vv[:, :, sinks:max(Sk - Sq - window + 1, sinks)] = -fill
            got.append(baps.attention_window(q, kk, vv, window, sinks, block, mode=mode))
        torch.cuda.synchronize()
        assert bool(torch.isfinite(got[0][0]).all())
        for o, lse in got[1:]:
            assert torch.equal(o, got[0][0]) and torch.equal(lse, got[0][1]), f"{shape} {window} {sinks} {block}"


def test_default_split_keys():
    """Few streams and a long window: the keys are split over workgroups."""
    import paper_2602_02071_amd as baps
    shape = (1, 4, 1, 1, 6001, 128)
    assert baps.baps_attention_window_workspace(*shape, 5000, 4, 128, mode=DEFAULT) > 0
    assert baps.baps_attention_window_workspace(*shape, 5000, 4, 128, mode=E2E) == 0
    for out_bf16 in (False, True):
        _default(shape, 5000, 4, 128, out_bf16)
    _default((2, 2, 2, 3, 3000, 64), 2000, 200, 32)


@pytest.mark.parametrize("shape", [(1, 4, 2, 100, 2500, 128), (1, 2, 1, 70, 3001, 64), (2, 3, 1, 90, 2200, 128)])
def test_default_split_keys_many_rows(shape):
    """Few tiles of many rows over long windows: the keys are split over workgroups."""
    import paper_2602_02071_amd as baps
    assert baps.baps_attention_window_workspace(*shape, 2000, 4, 128, mode=DEFAULT) > 0
    for out_bf16 in (False, True):
        _default(shape, 2000, 4, 128, out_bf16)
    _default(shape, 4000, 0, 32)
    _default(shape, 1700, 70, 64)


@pytest.mark.parametrize("shape", [(1, 16, 16, 1100, 1100, 64), (4, 35, 35, 400, 401, 64), (2, 20, 20, 1000, 1003, 64), (1, 32, 8, 1100, 1100, 128),
                                   (3, 20, 4, 600, 601, 128), (1, 32, 8, 1500, 1200, 128), (1, 8, 8, 2100, 2100, 128), (1, 12, 3, 3100, 3103, 128)])
def test_default_many_items(shape):
    """More workgroups than CUs, or than 64- or 128-row items would be: the tile kernel, and the forms beside it."""
    for window, sinks, block in ((100, 0, 64), (333, 5, 128), (1, 1, 32), (64, 65, 64)):
        _default(shape, window, sinks, block)


def test_default_tile_of_256_rows():
    """Long windows on more 128-row items than CUs."""
    _default((1, 33, 3, 3201, 3300, 128), 2900, 4, 64, out_bf16=True)


def test_default_large_scores_and_scale():
    _default((1, 4, 2, 1, 400, 128), 100, 4, 64, q_scale=30.0)
    _default((1, 4, 2, 90, 400, 64), 100, 4, 64, q_scale=30.0)
    _default((1, 4, 2, 90, 200, 64), 60, 0, 64, scale_log2=0.03)


def test_empty():
    import paper_2602_02071_amd as baps
    z = torch.zeros((1, 2, 3, 64), dtype=torch.bfloat16, device="cuda:0")
    for mode in (DEFAULT, E2E):
        o, lse = baps.attention_window(z, z[:, :, :0].contiguous(), z[:, :, :0].contiguous(), 5, 1, 64, mode=mode)
        assert bool((o == 0).all()) and bool((lse == -math.inf).all())
        o, lse = baps.attention_window(z[:, :, :0].contiguous(), z, z, 5, 1, 64, mode=mode)
        assert o.shape == (1, 2, 0, 64)


# ------------------------------------------------------------------ Alg. 1
def _alg1_row(acc, v, c, block, lam, n_b0, kmax, b0_last):
    """Alg. 1 on one row's scores acc (fp32, -inf where hidden): (o, lse)."""
    f32 = np.float32
    c = f32(c)
    m, ref, d = -np.inf, -np.inf, 0.0
    x = np.zeros(v.shape[1])
    for j in range(-(-len(acc) // block)):
        s = acc[j * block:(j + 1) * block]
        amax = s.max()
        if amax == -np.inf:
            continue
        b0 = j < n_b0 or (b0_last and j == kmax // block)
        tq = float(O.hif8_round(np.array([f32(float(amax) * float(c) - m)], f32))[0]) if m != -np.inf else 0.0
        if b0 or m == -np.inf or math.ceil(tq) > lam:
            m = max(m, math.ceil(float(f32(amax * c))))
            new_ref = m
        else:
            new_ref = m
            m = m + max(0, math.ceil(tq))
        f = 0.0 if ref == -np.inf else 2.0 ** (ref - new_ref)
        t = (s.astype(np.float64) * float(c) - new_ref).astype(f32)
        p = np.where(np.isneginf(t), 0.0, O.hif8_round(np.exp2(O.hif8_round(np.maximum(t, f32(-200))).astype(np.float64)).astype(f32)))
        x, d, ref = x * f + p.astype(np.float64) @ v[j * block:(j + 1) * block], d * f + float(p.sum(dtype=np.float64)), new_ref
    return (x / d, math.log(2.0) * (ref + math.log2(d))) if d else (x, -np.inf)


def _alg1(shape, window, sinks, block, lam=1, n_b0=1, b0_last=False, inputs=None, seed=3):
    import paper_2602_02071_amd as baps
    B, Hq, Hkv, Sq, Sk, D = shape
    q, k, v = inputs or make_qkv(B, Hq, Hkv, Sq, Sk, D, seed=seed, outliers=True, sink=4)
    qt, kt, vt = dev_bf16(q), dev_bf16(k), dev_bf16(v)
    o, lse = baps.attention_window(qt, kt, vt, window, sinks, block, lam=lam, n_b0=n_b0, b0_last=b0_last)
    rows = np.arange(B * Hq * Sq)
    _, _, acc, _ = baps.attention_dump(qt, kt, vt, True, block, rows)
    torch.cuda.synchronize()
    o = o.cpu().numpy().reshape(-1, D).astype(np.float64)
    lse = lse.cpu().numpy().reshape(-1).astype(np.float64)
    acc = acc.cpu().numpy()
    vf = bf16_bits_to_f32(v).astype(np.float64)
    key = np.arange(Sk)
    worst, ref_lse, n_keys = 0.0, np.zeros(len(rows)), np.zeros(len(rows))
    for i in rows:
        b, h, r = i // (Hq * Sq), i // Sq % Hq, i % Sq
        t = r + Sk - Sq
        seen = (key <= t) & ((key > t - window) | (key < sinks))
        s = np.where(seen, acc[i], -np.inf).astype(np.float32)
        ro, ref_lse[i] = _alg1_row(s, vf[b, h // (Hq // Hkv)], np.float32(1.4426950408889634 / math.sqrt(D)), block, lam, n_b0, t, b0_last)
        n_keys[i] = seen.sum()
        worst = max(worst, np.abs(o[i] - ro).max())
    fin = np.isfinite(ref_lse)
    assert np.array_equal(fin, np.isfinite(lse)) and np.all(o[~fin] == 0)
    assert worst <= ARB_TOL * max(1.0, np.abs(vf).max() / 4), f"{shape}: {worst}"
    assert np.all(np.abs(lse - ref_lse)[fin] <= lse_arb_tol(ref_lse, n_keys)[fin])


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window,sinks", [(1, 0), (150, 4), (300, 140)])
def test_alg1(D, block, window, sinks):
    _alg1((1, 4, 2, 1, 600, D), window, sinks, block)
    _alg1((1, 4, 2, 90, 400, D), window, sinks, block)


@pytest.mark.parametrize("knobs", [dict(lam=0), dict(lam=8), dict(n_b0=0), dict(n_b0=3), dict(b0_last=True)])
def test_alg1_knobs(knobs):
    for shape in ((1, 2, 1, 3, 700, 64), (1, 2, 1, 130, 500, 128)):
        _alg1(shape, 200, 5, 64, **knobs)
        _alg1(shape, 300, 0, 32, inputs=make_slow_climb(*shape, 0.7, 32), **knobs)


@pytest.mark.parametrize("block", [32, 64, 128])
@pytest.mark.parametrize("shape", [(1, 8, 2, 300, 300, 64), (2, 4, 1, 700, 1000, 128), (1, 32, 8, 1100, 1100, 128), (2, 6, 2, 300, 77, 64)])
def test_window_of_every_key(shape, block):
    """A window (or sinks) over all keys is plain causal attention: Alg. 1 bit for bit (one kernel)."""
    import paper_2602_02071_amd as baps
    B, Hq, Hkv, Sq, Sk, D = shape
    q, k, v = (dev_bf16(x) for x in make_qkv(B, Hq, Hkv, Sq, Sk, D, seed=5, outliers=True))
    want = baps.attention(q, k, v, True, block)
    for window, sinks in ((Sk, 0), (2 ** 31 - 1, 2 ** 31 - 1), (1, Sk)):
        got = baps.attention_window(q, k, v, window, sinks, block)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]), (window, sinks)


def test_captured():
    """The split form captured once and replayed between eager calls."""
    import paper_2602_02071_amd as baps
    q, k, v = (dev_bf16(x) for x in make_qkv(1, 8, 2, 1, 3000, 128, seed=6))
    call = lambda: baps.attention_window(q, k, v, 2500, 4, mode=DEFAULT)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for i in range(3):
        q.mul_(0.5)
        want = call()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1], want[1])
