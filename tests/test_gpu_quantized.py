"""The operators on quantised rows (microscaled 4-bit rows, rows of a table by token, the norm with the residual's
addition, the output projection by 4-bit weights) against plain implementations in 64 bits.

Tolerances: u = 2^-24 is the relative error of a rounding to float32.

  Norm    A thread adds up at most n = max(32, D / 1024) squares in turn, ten more roundings join the threads', and the
          mean, the sum with eps, the root, the reciprocal and two products take one each; the root halves what comes
          before it: (n + 12) / 2 + 5.
  Head    A product of a weight and a state is exact.  A matrix instruction adds 32 (bfloat16) or 128 (4 bits) of them to a
          sum; it may drop bits below the last place of the largest one, at most 1 u of it for each: no more than 33 u of the
          sum of the terms' absolute values for the 32, and for 4 bits, whose products are multiples of a quarter of their
          blocks' scales, 5 (four blocks' sums and the one so far).  Terms are spread over the instructions, each of which
          errs by its own terms' sum and by that of all before it: 33 u (5 u) of all terms, and 2 u a later instruction.
          Eight parts and the bias take a rounding each.
"""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2608_03065_amd import psc  # noqa: E402
from test_gpu_operators import DEV, TYPES, U, around, close, host, mask, quantized, rows_apart  # noqa: E402

pytestmark = pytest.mark.gpu
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


# ---------------------------------------------------------------- plain forms

def blocks(x):
    n, D = x.shape
    return np.concatenate([x, np.zeros((n, -D % 32))], 1).reshape(n, -1, 32)


def packed(x):
    """(codes [N, D], scales [N, blocks]) of rows of numbers."""
    x = blocks(host(x) if isinstance(x, torch.Tensor) else x)
    most = np.abs(x).max(-1)
    fine = np.isfinite(x).all(-1)
    with np.errstate(divide="ignore", invalid="ignore"):
        s = np.where(fine, np.maximum(np.floor(np.log2(most)) - 2 + 127, 0), 255).astype(np.int64)
        t = np.where(fine[..., None], x * np.exp2(127.0 - s[..., None]), 0)
    size = np.minimum(np.abs(t), 6)
    off = np.abs(size[..., None] - GRID)
    off[..., 1::2] += 1e-12             # of two as near ones the even one
    code = off.argmin(-1)
    code = np.where(np.signbit(t) & fine[..., None], code + 8, code)
    return code.reshape(code.shape[0], -1), s


def bytes_of(codes):
    """Rows of codes, whole blocks, two a byte."""
    return (codes[:, ::2] | codes[:, 1::2] << 4).astype(np.uint8)


def values(q, scales, D):
    """The numbers that rows of bytes and scales stand for."""
    code = np.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1)[:, :D].astype(np.int64)
    v = np.where(code >= 8, -1.0, 1.0) * GRID[code % 8]
    s = scales.astype(np.float64)
    return v * np.repeat(np.where(s == 255, np.nan, np.exp2(s - 127)), 32, 1)[:, :D]


def weights(V, D, seed, low=118, high=136):
    """Random codes and scales, rubbish behind the D codes and the blocks' scales of every row, and their numbers."""
    r = np.random.default_rng(seed)
    n = (D + 31) // 32
    q = r.integers(0, 256, (V, n * 16 + 16)).astype(np.uint8)
    s = r.integers(low, high, (V, (n + 3) // 4 * 4 + 4)).astype(np.uint8)
    s[:, n:] = 255
    w = values(q, s[:, :n], D)
    return torch.from_numpy(q).to(DEV)[:, :(D + 1) // 2], torch.from_numpy(s).to(DEV)[:, :n], w


# ---------------------------------------------------------------- rows in 4 bits

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,D,gap", [(1, 1, 0), (3, 7, 0), (5, 32, 3), (2, 33, 0), (7, 2047, 1), (300, 200, 8), (2, 20000, 0), (1000, 64, 0)])
def test_quantize_mx(dtype, n, D, gap):
    g = torch.Generator().manual_seed(D)
    x = (torch.randn(n, D, generator=g) * torch.exp2(torch.randint(-20, 20, (n, D), generator=g) / 4)).to(TYPES[dtype])
    if D >= 32:                                  # every tie, both signs, and numbers past the end
        x[0, :16] = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 4, 7, 7.5, -0.25, -0.75, -2.5, -5, -7, -0.0])
        x[0, 16:32] = 0
    if n > 2:
        x[2] = 0
    q, s = psc.quantize_mx(rows_apart(x.to(DEV), gap))
    assert q.shape == (n, (D + 1) // 2) and s.shape == (n, (D + 31) // 32)
    assert q.stride(0) % 16 == 0 and q.data_ptr() % 16 == 0 and s.stride(0) % 4 == 0
    codes, scales = packed(x)
    whole = torch.as_strided(q, (n, codes.shape[1] // 2), q.stride())      # zeros up to the block's end
    assert np.array_equal(host(s), scales)
    assert np.array_equal(host(whole), bytes_of(codes))


def test_quantize_mx_at_the_ends_of_float32():
    x = torch.zeros(9, 70)
    x[0, 3], x[1, 40], x[2, 69], x[2, 0] = math.nan, math.inf, -math.inf, 1
    x[3, :4] = torch.tensor([3e38, -1e38, 1e37, 1e-38])
    x[4, :4] = torch.tensor([1e-38, -5e-39, 3e-39, 1e-45])
    x[5, :4] = torch.tensor([1e-45, -3e-45, 0, 0])
    x[6, :2] = torch.tensor([2.0 ** -124, 2.0 ** -126])
    x[7, :2] = torch.tensor([float(np.nextafter(np.float32(8), np.float32(0))), 0.25])
    x[8, :3] = torch.tensor([2.0 ** -125, -3 * 2.0 ** -129, 2.0 ** -128])
    q, s = psc.quantize_mx(x.to(DEV))
    codes, scales = packed(x)
    assert np.array_equal(host(s), scales)
    whole = torch.as_strided(q, (9, codes.shape[1] // 2), q.stride())
    assert np.array_equal(host(whole), bytes_of(codes))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_mx_more_rows_than_units_of_a_block(dtype):
    """Many short rows: units and rows come apart from each other all over."""
    g = torch.Generator().manual_seed(5)
    x = torch.randn(70001, 40, generator=g).to(TYPES[dtype])
    q, s = psc.quantize_mx(x.to(DEV))
    codes, scales = packed(x)
    assert np.array_equal(host(s), scales) and np.array_equal(host(q), bytes_of(codes)[:, :20])


# ---------------------------------------------------------------- rows of a table

@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", ["i8", "mx4"])
@pytest.mark.parametrize("V,D,n,gap", [(1, 1, 1, 0), (5, 33, 3, 0), (100, 70, 1000, 3), (300, 2048, 17, 8), (50, 20000, 4, 0), (7, 64, 70001, 0)])
def test_lookup_rows(form, dtype, V, D, n, gap):
    r = np.random.default_rng(V + D)
    ids = r.integers(0, V, n).astype(np.int32)
    if n > 2:
        ids[1], ids[2] = -1, V                   # no rows of the table: zeros
    if form == "i8":
        q, s = psc.quantize_rows(torch.from_numpy(r.normal(0, 1, (V, D))).float().to(DEV))
        want = (host(q).astype(np.float32) * s.cpu().numpy()[:, None]).astype(np.float64)
    else:
        q, s, want = weights(V, D, D)
    out = rows_apart(torch.zeros(n, D, dtype=TYPES[dtype], device=DEV), gap)
    assert psc.lookup_rows(q, s, torch.from_numpy(ids).to(DEV), D=D, out=out) is out
    inside = (ids >= 0) & (ids < V)
    want_rows = np.where(inside[:, None], want[np.clip(ids, 0, V - 1)], 0)
    close(out, want_rows, 0)
    assert around(out, gap)
    got = psc.lookup_rows(q, s, D=D, dtype=TYPES[dtype])      # the whole table, in order
    assert got.shape == (V, D)
    close(got, want, 0)


def test_lookup_rows_of_extreme_scales():
    q, s, _ = weights(6, 64, 1)
    s[:] = torch.tensor([[0, 1], [255, 127], [254, 3], [2, 253], [126, 128], [1, 0]], dtype=torch.uint8)
    want = values(host(q), host(s), 64)
    with np.errstate(over="ignore"):
        want = want.astype(np.float32).astype(np.float64)
    close(psc.lookup_rows(q, s, dtype=torch.float32), want, 0)
    close(psc.lookup_rows(q, s), want, 0)


@pytest.mark.parametrize("D", [1, 33, 100, 4096])
def test_lookup_rows_is_the_inverse(D):
    x = torch.randn(9, D, generator=torch.Generator().manual_seed(D)).to(DEV)
    for q, s, step in ((*psc.quantize_rows(x), 1 / 254), (*psc.quantize_mx(x), 1 / 4)):
        back = psc.lookup_rows(q, s, D=D, dtype=torch.float32)
        assert bool(((back - x).abs() <= step * x.abs().amax(1, keepdim=True) * 1.001).all())


# ---------------------------------------------------------------- the norm

def normed(x, residual, gain, eps):
    """(residual, y) in 64 bits."""
    h = x.double()
    if residual is not None:
        h = (x.float() + residual.float()).to(residual.dtype).double()
    y = h / torch.sqrt(h.square().mean(1, keepdim=True) + eps)
    return h.numpy(), (y if gain is None else y * gain.double()).numpy()


def norm_bound(D):
    return ((max(32, D / 1024) + 12) / 2 + 5) * U


def check_form(got, y, to, bound):
    """What add_rms_norm gave against y, 64 bits, each element of which may be off by a relative `bound`."""
    n, D = y.shape
    if to in ("f32", "bf16"):
        assert got.dtype == TYPES[to]
        close(got, y, bound * np.abs(y))
    elif to == "i8":
        q, s = got
        assert q.shape == (n, D) and q.stride(0) % 16 == 0
        scale = np.abs(y).max(1) / 127
        assert (np.abs(host(s) - scale) <= (bound + 2 * U) * scale).all()
        with np.errstate(invalid="ignore", divide="ignore"):
            exact = np.where(scale[:, None] > 0, y / scale[:, None], 0)
        assert (np.abs(host(q) - exact) <= 0.5 + 127 * (2 * bound + 4 * U)).all()
        if q.stride(0) > D:
            assert not bool(torch.as_strided(q, (n, q.stride(0)), q.stride())[:, D:].any())
    else:
        q, s = host(got[0]), host(got[1]).astype(np.float64)
        assert q.shape == (n, (D + 1) // 2) and s.shape == (n, (D + 31) // 32)
        t = blocks(y)
        most = np.abs(t).max(-1)
        with np.errstate(divide="ignore"):
            low, high = (np.maximum(np.floor(np.log2(most * (1 + k * bound))) + 125, 0) for k in (-1, 1))
        assert ((s == low) | (s == high)).all()
        size = np.minimum(np.abs(t) * np.exp2(127 - s[..., None]), 6).reshape(n, -1)[:, :D]
        code = np.stack([q & 15, q >> 4], -1).reshape(n, -1)[:, :D].astype(np.int64)
        off, best = np.abs(GRID[code % 8] - size), np.abs(size[..., None] - GRID).min(-1)
        assert (off <= best + 2 * 8 * bound).all()
        assert (((code >= 8) == (y < 0)) | (code % 8 == 0)).all()


NORMS = [(1, 1, 0), (3, 7, 0), (5, 64, 3), (2, 1000, 0), (9, 1024, 1), (4, 1025, 0), (6, 2048, 0), (3, 4097, 8), (2, 8192, 0), (2, 8193, 0),
         (2, 32768, 0), (2, 40001, 5), (700, 96, 0)]


@pytest.mark.parametrize("n,D,gap", NORMS)
@pytest.mark.parametrize("to", ["f32", "bf16", "i8", "mx4"])
@pytest.mark.parametrize("dtype,stream", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16"), ("bf16", None), ("f32", None)])
def test_add_rms_norm(n, D, gap, to, dtype, stream):
    g = torch.Generator().manual_seed(n + D)
    x = torch.randn(n, D, generator=g).to(TYPES[dtype])
    if n > 4:
        x[3] = 0
    residual = None if stream is None else (3 * torch.randn(n, D, generator=g)).to(TYPES[stream])
    if residual is not None and n > 4:
        residual[3] = 0
    gain = None if D % 2 else 1 + 0.3 * torch.randn(D, generator=g)
    h, y = normed(x, residual, gain, 1e-5)
    r = None if residual is None else rows_apart(residual.to(DEV), gap)
    got = psc.add_rms_norm(rows_apart(x.to(DEV), gap), None if gain is None else gain.to(DEV), residual=r, eps=1e-5,
                           to=TYPES.get(to, to))
    check_form(got, y, to, norm_bound(D))
    if r is not None:
        close(r, h, 0)
        assert around(r, gap)


@pytest.mark.parametrize("D", [100, 3000, 20000, 50000])
@pytest.mark.parametrize("size,eps", [(1e25, 1e-6), (3e37, 0.0), (1e-30, 0.0), (1e-25, 1e-35), (1e-30, 1e-6)])
def test_add_rms_norm_of_squares_past_float32(D, size, eps):
    """Their relative bound counts four more roundings: by the power of two, none, and the sum's second pass."""
    x = torch.randn(3, D, generator=torch.Generator().manual_seed(D)).mul_(size).clamp_(-1e38, 1e38)
    _, y = normed(x, None, None, float(np.float32(eps)))
    got = psc.add_rms_norm(x.to(DEV), eps=eps)
    close(got, y, (norm_bound(D) + 4 * U) * np.abs(y) + 2.0 ** -140)


@pytest.mark.parametrize("D", [50, 1500, 9000, 40000])
def test_add_rms_norm_of_rows_that_are_not_numbers(D):
    x = torch.randn(4, D, generator=torch.Generator().manual_seed(1))
    x[0, 5], x[1, D - 1] = math.nan, -math.inf
    got = psc.add_rms_norm(x.to(DEV)).cpu()
    assert bool(torch.isnan(got[0]).all()) and bool(torch.isnan(got[1, D - 1])) and not bool(got[1, :D - 1].any())
    assert bool(torch.isfinite(got[2:]).all())
    q, s = psc.add_rms_norm(x.to(DEV), to="i8")
    assert torch.isnan(s).tolist() == [True, True, False, False] and not bool(q[:2].any())
    q, s = psc.add_rms_norm(x.to(DEV), to="mx4")
    assert bool((s[0] == 255).all()) and int(s[1, -1]) == 255 and not bool(q[0].any()) and not bool((s[2:] == 255).any())


def test_add_rms_norm_of_zeros_without_eps_is_not_a_number():
    got = psc.add_rms_norm(torch.zeros(2, 40, device=DEV), eps=0)
    assert bool(torch.isnan(got).all())


# ---------------------------------------------------------------- head

def head_bound(xv, w, bias, states):
    """Of the products of states and weights, 64-bit numbers."""
    D = xv.shape[1]
    terms = np.abs(np.nan_to_num(xv)) @ np.abs(np.nan_to_num(w)).T + np.abs(bias)
    per = (33, 32) if states == "bf16" else (5, 128)
    return (per[0] + 2 * (D / per[1] + 1) + 9) * U * terms


def state_values(x, states):
    if states == "bf16":
        return x.to(torch.bfloat16).double().numpy()
    codes, scales = packed(x)
    return values(bytes_of(codes), scales, x.shape[1])


HEADS = [(1, 64, 1), (1, 1, 33), (2, 17, 64), (3, 128, 65), (8, 200, 513), (15, 1024, 1000), (16, 130, 700), (17, 256, 513),
         (33, 96, 1537), (48, 640, 300), (64, 512, 2049), (65, 300, 777), (100, 1000, 4097), (128, 384, 515),
         (200, 129, 1025), (256, 256, 600), (257, 320, 1100), (300, 128, 5000), (520, 144, 257), (1, 8192, 513), (4, 5000, 100),
         (60, 4096, 130), (300, 4096, 300), (3, 33, 40), (40, 2080, 90), (270, 1056, 33000), (600, 512, 20001),
         (200, 520, 33000), (300, 33, 17000), (1025, 256, 6500), (140, 640, 40001)]
FORMS = ["bf16", "mx4"]


@pytest.mark.parametrize("B,D,V", HEADS)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("states", FORMS)
def test_head_logits_mx(B, D, V, dtype, states):
    x = torch.randn(B, D, generator=torch.Generator().manual_seed(B)).to(TYPES[("bf16", "f32")[D % 2]])
    q, s, w = weights(V, D, B + D + V)
    xv = state_values(x, states)
    got = psc.head_logits_mx(rows_apart(x.to(DEV), D % 3), q, s, states=states, dtype=TYPES[dtype])
    assert got.dtype == TYPES[dtype] and got.shape == (B, V)
    close(got, xv @ w.T, head_bound(xv, w, 0, states))


@pytest.mark.parametrize("B,D,V", HEADS)
@pytest.mark.parametrize("shares", [(0.0,), (0.9, 0.001, 0.0, 0.05), (0.002,)])
@pytest.mark.parametrize("states", FORMS)
def test_head_logits_mx_masked_with_bias(B, D, V, shares, states):
    dtype = ("bf16", "f32")[(B + V) % 2]
    gap = (0, 1, 8)[D % 3]
    g = torch.Generator().manual_seed(B)
    x, bias = torch.randn(B, D, generator=g).to(torch.bfloat16), torch.randn(V, generator=g)
    q, s, w = weights(V, D, B + D + V + 1)
    xv, b = state_values(x, states), bias.double().numpy()
    words, keep = mask(B, V, D, shares)
    out = rows_apart(torch.zeros(B, V, dtype=TYPES[dtype], device=DEV), gap)
    assert psc.head_logits_mx(x.to(DEV), q, s, states=states, bias=bias.to(DEV), bitmask=words, out=out) is out
    close(out, np.where(keep, xv @ w.T + b, -np.inf), head_bound(xv, w, b, states))
    assert around(out, gap)


@pytest.mark.parametrize("B,D,V", [(1, 1, 5), (5, 96, 300), (33, 2047, 70), (70, 4096, 600), (300, 320, 700)])
def test_head_logits_mx_of_quantized_states(B, D, V):
    x = torch.randn(B, D, generator=torch.Generator().manual_seed(B)).to(torch.bfloat16).to(DEV)
    q, s, _ = weights(V, D, 3)
    xq, xs = psc.quantize_mx(x)
    rubbish = torch.full((B, xq.stride(0) + 16), 0x77, dtype=torch.uint8, device=DEV)      # behind the row's codes
    rubbish[:, :xq.shape[1]] = xq
    want = psc.head_logits_mx(x, q, s, states="mx4", dtype=torch.float32)
    if D % 2 == 0:
        assert torch.equal(psc.head_logits_mx(rubbish[:, :xq.shape[1]], q, s, x_scales=xs, dtype=torch.float32), want)
    assert torch.equal(psc.head_logits_mx(xq, q, s, x_scales=xs.contiguous(), dtype=torch.float32), want)
    assert psc.head_logits_mx(xq, q, s, x_scales=xs).dtype == torch.bfloat16


@pytest.mark.parametrize("B,D,V", [(1, 1, 5), (5, 100, 300), (33, 2047, 70), (70, 4096, 600), (300, 320, 700)])
def test_head_logits_of_quantized_states(B, D, V):
    """The same bits as of the states that they were made from."""
    g = torch.Generator().manual_seed(B)
    x = torch.randn(B, D, generator=g).to(DEV)
    w, ws = psc.quantize_rows(torch.randn(V, D, generator=g).to(DEV))
    words, _ = mask(B, V, 7, (0.9, 0.01))
    q, s = psc.quantize_rows(x)
    rubbish = torch.full((B, q.stride(0) + 32), 99, dtype=torch.int8, device=DEV)
    rubbish[:, :D] = q
    for kw in ({}, dict(bitmask=words, bias=ws)):
        want = psc.head_logits(x, w, ws, **kw)
        assert torch.equal(psc.head_logits(q, w, ws, x_scales=s, dtype=torch.float32, **kw), want)
        assert torch.equal(psc.head_logits(rubbish[:, :D], w, ws, x_scales=s, dtype=torch.float32, **kw), want)
    assert psc.head_logits(q, w, ws, x_scales=s).dtype == torch.bfloat16
    want, scale = quantized(x)
    assert np.array_equal(host(q), want)


@pytest.mark.parametrize("B", [1, 16, 40, 130, 300])
@pytest.mark.parametrize("states", FORMS)
def test_head_logits_mx_that_are_not_numbers(B, states):
    """A NaN or infinity among the states is its row's, a NaN scale its token's."""
    x = torch.randn(B, 256, generator=torch.Generator().manual_seed(B))
    x[0, 5] = math.nan
    if B > 2:
        x[1], x[2, 0] = 0, math.inf
    q, s, w = weights(600, 256, 6)
    s[7, 3], s[599, 7] = 255, 255
    w[7], w[599] = np.nan, np.nan
    xv = state_values(x, states)
    with np.errstate(invalid="ignore"):
        y = xv @ w.T
    y[0], y[:, [7, 599]] = np.nan, np.nan
    if B > 2:
        y[1, [7, 599]] = np.nan
        if states == "mx4":
            y[2] = np.nan
        else:
            with np.errstate(invalid="ignore"):
                y[2] = np.where(w[:, 0] == 0, np.nan, np.inf * np.sign(w[:, 0]))
            y[2, [7, 599]] = np.nan
    xv[~np.isfinite(xv)] = 0
    close(psc.head_logits_mx(x.to(DEV), q, s, states=states, dtype=torch.float32), y, head_bound(xv, w, 0, states))


@pytest.mark.parametrize("B", [2, 20, 50, 200])
@pytest.mark.parametrize("states", FORMS)
def test_head_logits_mx_of_wide_scales(B, states):
    """Blocks whose powers lie far apart, small and large ones beside each other."""
    x = torch.randn(B, 512, generator=torch.Generator().manual_seed(B)).to(torch.bfloat16)
    q, s, w = weights(300, 512, 9, low=60, high=190)
    xv = state_values(x, states)
    got = psc.head_logits_mx(x.to(DEV), q, s, states=states, dtype=torch.float32)
    close(got, xv @ w.T, head_bound(xv, w, 0, states))


@pytest.mark.parametrize("states", FORMS)
def test_head_logits_mx_twice_is_the_same(states):
    """Parts of D are added in their own order, whichever ends first."""
    x = torch.randn(3, 8192, generator=torch.Generator().manual_seed(2)).to(torch.bfloat16).to(DEV)
    q, s, _ = weights(700, 8192, 4)
    words, _ = mask(3, 700, 1, (0.2,))
    for kw in ({}, dict(bitmask=words)):
        first = psc.head_logits_mx(x, q, s, states=states, dtype=torch.float32, **kw)
        for _ in range(20):
            assert torch.equal(psc.head_logits_mx(x, q, s, states=states, dtype=torch.float32, **kw), first)


@pytest.mark.parametrize("B,states,masked", [(2, "bf16", False), (40, "mx4", True), (200, "mx4", False), (140, "bf16", True)])
def test_more_than_4_gib_of_weights(B, states, masked):
    """Rows on both sides of byte 2^32 of the codes, by the projection and by their tokens."""
    D, V = 16384, 530001
    g = torch.Generator(DEV).manual_seed(B)
    q = torch.randint(0, 256, (V, D // 2), generator=g, device=DEV, dtype=torch.uint8)
    s = torch.randint(118, 130, (V, D // 32), generator=g, device=DEV, dtype=torch.uint8)
    edge = 2 ** 32 // (D // 2)
    at = torch.tensor([0, 1, 77, edge - 2, edge - 1, edge, edge + 1, V - 200, V - 2, V - 1], device=DEV)
    w = values(host(q[at]), host(s[at]), D)
    close(psc.lookup_rows(q, s, at.to(torch.int32)), w, 0)
    x = torch.randn(B, D, generator=torch.Generator().manual_seed(B)).to(torch.bfloat16)
    xv = state_values(x, states)
    words = None
    if masked:                                   # odd tokens and the last one
        words = torch.full((B, (V + 31) // 32), 0x55555555 * 2 - 2 ** 32, dtype=torch.int32, device=DEV)
        words[:, -1] |= 1 << (V - 1) % 32
    got = psc.head_logits_mx(x.to(DEV), q, s, states=states, dtype=torch.float32, bitmask=words)
    y = xv @ w.T
    if masked:
        even = host(at) % 2 == 0
        even[-1] = False
        y[:, even] = -np.inf
    close(got[:, at], y, head_bound(xv, w, 0, states))


# ---------------------------------------------------------------- together

def step(x, residual, gain, table, out, words, how):
    """A step's end and the next one's beginning: norm, projection, the best token, its embedding."""
    if how == "i8":
        state = psc.add_rms_norm(x, gain, residual=residual, to="i8")
        psc.head_logits(state[0], *table, x_scales=state[1], bitmask=words, out=out)
    elif how == "mx4":
        state = psc.add_rms_norm(x, gain, residual=residual, to="mx4")
        psc.head_logits_mx(state[0], *table, x_scales=state[1], bitmask=words, out=out)
    else:
        psc.head_logits_mx(psc.add_rms_norm(x, gain, residual=residual), *table, bitmask=words, out=out)
    tokens = psc.sample(out, 4, bitmask=words)[0]
    return tokens, psc.lookup_rows(*table, tokens)


@pytest.mark.parametrize("how", ["i8", "mx4", "bf16"])
@pytest.mark.parametrize("B", [1, 24, 160])
def test_steps_in_a_graph_and_on_a_stream(how, B):
    """Norm, projection, sampling and embedding as a step runs them: eager on a stream of its own and replayed from a graph
    give the same, replay after replay."""
    D, V = 384, 1500
    g = torch.Generator().manual_seed(B)
    wf = torch.randn(V, D, generator=g).to(DEV) / D ** 0.5
    table = psc.quantize_rows(wf) if how == "i8" else psc.quantize_mx(wf)
    gain = (1 + 0.1 * torch.randn(D, generator=g)).to(DEV)
    words, keep = mask(B, V, B, (0.9, 0.01, 0.5))
    x0, r0 = torch.randn(B, D, generator=g).to(torch.bfloat16).to(DEV), torch.randn(B, D, generator=g).to(DEV)
    x, r, out = x0.clone(), r0.clone(), torch.empty(B, V, dtype=torch.float32, device=DEV)
    torch.cuda.synchronize()

    def eager(stream):
        xs, rs, said = x0.clone(), r0.clone(), []
        stream.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(stream):
            for _ in range(4):
                tokens, xs = step(xs, rs, gain, table, torch.empty_like(out), words, how)
                said.append(tokens)
        stream.synchronize()
        return [t.cpu() for t in said], rs.cpu()

    side = torch.cuda.Stream()
    want, residual = eager(side)
    assert all(keep[b, int(t)] for tokens in want for b, t in enumerate(tokens) if t >= 0)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, r, gain, table, out, words, how)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        tokens, nxt = step(x, r, gain, table, out, words, how)
        x.copy_(nxt)
    for _ in range(3):
        x.copy_(x0), r.copy_(r0)
        for k in range(4):
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(tokens.cpu(), want[k])
        assert torch.equal(r.cpu(), residual)
        assert [t.tolist() for t in eager(side)[0]] == [t.tolist() for t in want]


@pytest.mark.parametrize("states", FORMS)
def test_two_streams_at_once(states):
    """Calls whose tiles and parts go through workspaces, on two streams that overlap: as one after the other."""
    calls = []
    for B, D, V, shares in ((3, 4096, 1000, None), (40, 2048, 6000, (0.1,)), (150, 512, 33000, (0.02, 0.2)), (300, 768, 30000, None)):
        x = torch.randn(B, D, generator=torch.Generator().manual_seed(B)).to(torch.bfloat16).to(DEV)
        q, s, _ = weights(V, D, B)
        kw = dict(states=states, dtype=torch.float32, bitmask=None if shares is None else mask(B, V, B, shares)[0])
        calls.append((x, q, s, kw))
    want = [psc.head_logits_mx(x, q, s, **kw) for x, q, s, kw in calls]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = [[psc.head_logits_mx(x, q, s, stream=stream, **kw) for stream in streams] for x, q, s, kw in calls * 5]
    for stream in streams:
        stream.synchronize()
    assert all(torch.equal(t, w) for g, w in zip(got, want * 5) for t in g)


def test_two_graphs_in_turn():
    """Each graph's workspace is its own: replays in any order give what the eager calls gave."""
    side, graphs = torch.cuda.Stream(), []
    for B, D, V, states in ((2, 4096, 700, "bf16"), (70, 1024, 3000, "mx4")):
        x = torch.randn(B, D, generator=torch.Generator().manual_seed(B)).to(torch.bfloat16).to(DEV)
        q, s, _ = weights(V, D, B)
        words, _ = mask(B, V, B, (0.1, 0.3))
        run = lambda x=x, q=q, s=s, words=words, states=states: psc.head_logits_mx(x, q, s, states=states, bitmask=words)  # noqa: E731
        want = run()
        side.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            out = run()
        graphs.append((graph, out, want, run))
    for k in (0, 1, 1, 0, 0, 1):
        graph, out, want, run = graphs[k]
        out.fill_(0)
        graph.replay()
        assert torch.equal(run(), want)
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_stream_argument():
    """Calls on a stream given by name, their results' memory too."""
    side = torch.cuda.Stream()
    x = torch.randn(5, 200, generator=torch.Generator().manual_seed(1)).to(DEV)
    q, s, _ = weights(90, 200, 1)
    torch.cuda.synchronize()
    want = [psc.quantize_mx(x)[0], psc.add_rms_norm(x), psc.head_logits_mx(x, q, s), psc.lookup_rows(q, s, D=200)]
    got = [psc.quantize_mx(x, stream=side)[0], psc.add_rms_norm(x, stream=side), psc.head_logits_mx(x, q, s, stream=side),
           psc.lookup_rows(q, s, D=200, stream=side)]
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_empty_calls():
    q, s, _ = weights(90, 200, 1)
    none = torch.empty(0, 200, device=DEV)
    assert psc.quantize_mx(none)[0].shape == (0, 100) and psc.add_rms_norm(none).shape == (0, 200)
    assert psc.add_rms_norm(none, to="i8")[0].shape == (0, 200)
    assert psc.head_logits_mx(none, q, s).shape == (0, 90)
    assert psc.lookup_rows(q, s, torch.empty(0, dtype=torch.int32, device=DEV), D=200).shape == (0, 200)


# ---------------------------------------------------------------- the ends of what the contract allows

@pytest.mark.parametrize("B,V", [(3, 3), (24, 40), (50, 140), (100, 200), (140, 32600)])
@pytest.mark.parametrize("share", [None, 0.05])
def test_head_logits_of_quantized_states_at_the_end_of_32_bits(B, V, share):
    """-128 in the states and the weights at the largest D: the sum is 2^31, the only one that passes 32 bits."""
    D = 131072
    x = torch.full((B, D), -128, dtype=torch.int8, device=DEV)
    w = torch.full((V, D), -128, dtype=torch.int8, device=DEV)
    w[V - 1], w[V // 2, 5] = 127, -127
    x[1, D - 1], x[B - 1] = -127, 127
    sums = np.full((B, V), 2.0 ** 31)
    sums[:, V // 2] -= 128
    sums[1] -= 128
    sums[:, V - 1] = -127.0 * 128 * D
    sums[1, V - 1] += 127
    sums[B - 1] = -127.0 * 128 * D
    sums[B - 1, V // 2] += 127
    sums[B - 1, V - 1] = 127.0 ** 2 * D
    g = torch.Generator().manual_seed(V)
    xs, ws = torch.rand(B, generator=g) + 0.5, torch.rand(V, generator=g) / D
    y = sums * xs.double().numpy()[:, None] * ws.double().numpy()
    words, keep = (None, np.True_) if share is None else mask(B, V, V, (share,))
    got = psc.head_logits(x, w, ws.to(DEV), x_scales=xs.to(DEV), dtype=torch.float32, bitmask=words)
    close(got, np.where(keep, y, -np.inf), 8 * U * np.abs(y))


def test_head_logits_of_quantized_states_of_the_largest_scales():
    """Rows of -128 alone whose scale's double passes float32, or is none: a sum of 0 stays 0, the others keep their sign."""
    D = 131072
    x = torch.full((3, D), -128, dtype=torch.int8, device=DEV)
    w = torch.full((3, D), -128, dtype=torch.int8, device=DEV)
    w[1], w[2, ::2], w[2, 1::2] = 127, 1, -1
    xs = torch.tensor([1.5 * 2.0 ** 127, math.inf, math.nan], device=DEV)
    got = psc.head_logits(x, w, torch.ones(3, device=DEV), x_scales=xs, dtype=torch.float32)
    close(got, np.array([[np.inf, -np.inf, 0], [np.inf, -np.inf, np.nan], [np.nan] * 3]), 0)


@pytest.mark.parametrize("B,D,V", [(1, 33, 40), (3, 7, 5), (20, 1000, 300), (50, 300, 130), (100, 2049, 200), (200, 129, 33000), (200, 500, 70000),
                                   (300, 95, 50000), (300, 300, 70000)])
@pytest.mark.parametrize("share", [None, 0.02])
@pytest.mark.parametrize("states", FORMS)
def test_head_logits_mx_of_the_largest_scales(B, D, V, share, states):
    """Scales up to 254, of which bfloat16 holds 4 at most times 2^125, 3 times 2^126 and 1.5 times 2^127: weights up to there
    are taken as they are, and any code behind the row's D does not matter."""
    q, s, _ = weights(V, D, D, low=240, high=255)
    blocks = s.shape[1]
    whole = torch.as_strided(q, (V, blocks * 16), q.stride())
    codes = torch.stack((whole & 15, whole >> 4), -1).view(V, -1)
    inside = torch.arange(blocks * 32, device=DEV) < D
    most = torch.where(s == 254, 3, torch.where(s == 253, 5, 7)).repeat_interleave(32, 1)      # a code's place in the list
    codes = torch.where(inside, codes // 8 * 8 + torch.minimum(codes % 8, most), codes)
    whole.copy_(codes[:, ::2] + 16 * codes[:, 1::2])
    w = values(host(q), host(s), D)
    x = (torch.randn(B, D, generator=torch.Generator().manual_seed(B)) * 2.0 ** -20).to(torch.bfloat16)
    xv = state_values(x, states)
    words, keep = (None, np.True_) if share is None else mask(B, V, V, (share,))
    got = psc.head_logits_mx(x.to(DEV), q, s, states=states, dtype=torch.float32, bitmask=words)
    close(got, np.where(keep, xv @ w.T, -np.inf), head_bound(xv, w, 0, states))


@pytest.mark.parametrize("B", [1, 24, 50, 200])
def test_head_logits_mx_of_weights_past_bfloat16(B):
    """Of 2^128 and more: infinite where the states are bfloat16, as lookup_rows has them; as they are where both are in 4 bits."""
    D, V = 64, 33000
    q, s, w = weights(V, D, 2, low=252, high=255)
    x = (torch.randn(B, D, generator=torch.Generator().manual_seed(B)) * 2.0 ** -20).to(torch.bfloat16)
    x[0, 1::2] = 0
    xv = state_values(x, "mx4")
    got = psc.head_logits_mx(x.to(DEV), q, s, states="mx4", dtype=torch.float32)
    close(got, xv @ w.T, head_bound(xv, w, 0, "mx4"))
    with np.errstate(over="ignore"):
        w = w.astype(np.float32).astype(np.float64)
    xv, large = state_values(x, "bf16"), np.isinf(w)
    rest = np.where(large, 0, w)
    up = (np.maximum(xv, 0) @ np.maximum(np.where(large, np.sign(w), 0), 0).T + np.maximum(-xv, 0) @ np.maximum(-np.where(large, np.sign(w), 0), 0).T) > 0
    down = (np.maximum(-xv, 0) @ np.maximum(np.where(large, np.sign(w), 0), 0).T + np.maximum(xv, 0) @ np.maximum(-np.where(large, np.sign(w), 0), 0).T) > 0
    none = ((xv == 0).astype(float) @ large.T.astype(float)) > 0
    y = np.where(up, np.inf, np.where(down, -np.inf, xv @ rest.T))
    y[none | (up & down)] = np.nan
    assert np.isnan(y).any() and np.isinf(y).any() and np.isfinite(y).any()
    got = psc.head_logits_mx(x.to(DEV), q, s, dtype=torch.float32)
    close(got, y, head_bound(xv, rest, 0, "bf16"))


@pytest.mark.parametrize("B,D,V", [(1, 1, 5), (5, 95, 300), (33, 2047, 70), (300, 319, 700)])
def test_head_logits_mx_of_quantized_states_of_odd_rows(B, D, V):
    """What lies behind an odd row's last code, in the same byte, does not matter where D is given."""
    x = torch.randn(B, D, generator=torch.Generator().manual_seed(B)).to(torch.bfloat16).to(DEV)
    q, s, _ = weights(V, D, 3)
    q[:, -1] |= 0x70
    xq, xs = psc.quantize_mx(x)
    want = psc.head_logits_mx(x, q, s, states="mx4", dtype=torch.float32)
    xq[:, -1] |= 0x70
    assert torch.equal(psc.head_logits_mx(xq, q, s, x_scales=xs, D=D, dtype=torch.float32), want)


@pytest.mark.parametrize("D", [64, 3000, 20000, 50000])
@pytest.mark.parametrize("large,small", [(2.0 ** 65, 2.0 ** -57), (2.0 ** 100, 2.0 ** -24), (2.0 ** 127, 1.0), (2.0 ** -70, 2.0 ** -140)])
def test_add_rms_norm_of_small_elements_beside_large_ones(D, large, small):
    """Squares past float32's range on either side do not cost a small element its bits.  Bound as where squares pass it."""
    x = torch.randn(3, D, generator=torch.Generator().manual_seed(D)).mul_(small)
    x[:, D // 2] = large
    _, y = normed(x, None, None, 0.0)
    got = psc.add_rms_norm(x.to(DEV), eps=0)
    close(got, y, (norm_bound(D) + 4 * U) * np.abs(y) + 2.0 ** -148)


@pytest.mark.parametrize("B,D,V", [(1, 256, 70), (24, 97, 300), (50, 300, 130), (200, 160, 33000)])
@pytest.mark.parametrize("states", FORMS)
def test_head_logits_mx_of_the_smallest_scales(B, D, V, states):
    """Scales from 0 on, of states near float32's end; a weight below 2^-126 may count as 0."""
    q, s, w = weights(V, D, D, low=0, high=24)
    x = (torch.randn(B, D, generator=torch.Generator().manual_seed(B)) * 2.0 ** 123).to(torch.bfloat16)
    xv = state_values(x, states)
    got = psc.head_logits_mx(x.to(DEV), q, s, states=states, dtype=torch.float32)
    small = np.abs(xv) @ np.where(np.abs(w) < 2.0 ** -126, np.abs(w), 0).T
    close(got, xv @ w.T, head_bound(xv, w, 0, states) + small)


@pytest.mark.parametrize("D", [64, 3000, 20000, 50000])
@pytest.mark.parametrize("to", ["f32", "i8", "mx4"])
def test_add_rms_norm_of_an_eps_whose_sum_passes_float32(D, to):
    """Neither the mean nor eps does.  Bound as where squares pass it."""
    x = torch.randn(3, D, generator=torch.Generator().manual_seed(D)).mul_(1.5e19 / D ** 0.5)
    eps = float(np.finfo(np.float32).max)
    _, y = normed(x, None, None, eps)
    check_form(psc.add_rms_norm(x.to(DEV), eps=eps, to=TYPES.get(to, to)), y, to, norm_bound(D) + 4 * U)
