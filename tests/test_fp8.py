"""8-bit operators in blocks of 128: quantisers, products, the gated block and its backward pass, against the definition in fp64.

Bounds, all fixed by arithmetic.  Codes and scales of given values are exact; a value back may be off by two roundings, to fp32 and to the
16-bit type.  A product's element may be off by one rounding to the 16-bit type (half a step of it) and by the sums:
  - the instruction adds the products of 128 columns in groups of eight neighbours, and cuts each product below 2^-13 of the power of two of the
    largest of its eight.  A product of two codes has six bits behind that power, so it is exact where its power is at least 2^-7 of the
    largest's.  The factors here have four and five binades, and nothing is cut, but where a test says so: there the bound has 7 2^-13 of the
    largest of each eight more (the largest itself is exact);
  - the sixteen groups' sums are cut below 2^-23 of the largest at worst each: 16 2^-23 of the magnitudes;
  - the scales' product and its product with that sum are two roundings of 2^-24, and the K / 128 additions and the at most 16 + 32 partial
    sums of wavefronts and slices add 2^-24 each: (K / 128 + 50) 2^-24.
(K / 128 + 22) 2^-22 sum |x w| is more than all of them.

H = act(G) U: with G and U off by eg and eu, at most 1.13 eg |U| + |act(G)| eu (1.13 is the largest slope of either activation), and the activation's
own arithmetic: sigma(z) from the hardware's exp and reciprocal is off by a few steps of 2^-24 and by |z| times as much, from the rounding of z
and of its product with log2 e: (16 + 8 |z|) 2^-24 of every term it is in.  Sigma below fp32's normal numbers is 0: 2^-126 of what it multiplies."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

from gpu_util import torch_dtype, ulp16
from oracle import fp8_oracle as fx

DTYPES = ("f16", "bf16")
ACTS = ("silu", "gelu")
BIG = {"f16": 65504.0, "bf16": 3.3895313892515355e38}


def half_step(ref, dtype):
    return 0.5 * ulp16(np.minimum(np.abs(ref), BIG[dtype]), dtype)


def sums_off(mag, K):
    return (K // 128 + 22) * 2.0 ** -22 * mag


def off_by_at_most(sums, K, dtype):
    ref, mag = sums
    return half_step(ref, dtype) + sums_off(mag, K)


def gated_off(g, u, K, act, dtype):
    """(H, how far off it may be), from the two projections' (sums, magnitudes)."""
    (g, gm), (u, um) = g, u
    f, z = fx.activation(g, act), fx.argument(g, act)
    h = f * u
    eg, eu = sums_off(gm, K), sums_off(um, K)
    return h, half_step(h, dtype) + 1.13 * eg * (np.abs(u) + eu) + np.abs(f) * eu + np.abs(h) * (16 + 8 * np.abs(z)) * 2.0 ** -24 + np.abs(g * u) * 2.0 ** -126


def as_f64(t):
    return t.double().cpu().numpy()


def as_u8(t):
    import torch
    return t.view(torch.uint8).cpu().numpy()


def to_gpu(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def empty(*shape, dtype="u8"):
    """Filled with what no right answer is."""
    import torch
    if dtype == "u8":
        return torch.full(shape, 0x7f, dtype=torch.uint8, device="cuda")
    return torch.full(shape, -7.0, dtype=torch.float32 if dtype == "f32" else torch_dtype(dtype), device="cuda")


# ---------------------------------------------------------------------------------------------------- the definition, pinned
def test_codes_against_exact_rationals():
    """Every value of the format, the middles between two neighbours and their nearest doubles, against a search in rationals."""
    finite = [(Fraction(fx.TABLE[c]), c) for c in range(127)]
    def nearest(v):
        a = min(abs(v), Fraction(448))
        best = min(abs(m - a) for m, _ in finite)
        codes = [c for m, c in finite if abs(m - a) == best]
        return codes[0] if len(codes) == 1 else next(c for c in codes if c % 2 == 0)
    u = [0.0, 1e-300, 447.9, 448.0, 449.0, 1e9]
    for a, b in zip(fx.MAGNITUDES, fx.MAGNITUDES[1:]):
        m = (a + b) / 2
        u += [a, m, np.nextafter(m, 0), np.nextafter(m, 1e9)]
    u = np.array(u)
    want = np.array([nearest(Fraction(v)) for v in u])
    assert np.array_equal(fx.codes_of(u), want) and np.array_equal(fx.codes_of(-u), want + 128)


def test_the_format_is_e4m3():
    import torch
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(every, fx.TABLE, equal_nan=True)
    x = np.random.default_rng(0).standard_normal(4000).astype(np.float32) * np.exp2(np.arange(4000) % 17 - 9).astype(np.float32)
    x = x[np.abs(x) <= 448]
    assert np.array_equal(torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), fx.codes_of(x.astype(np.float64)))


def test_quantisers_of_the_definition():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((300, 256)) * np.exp2(rng.integers(-20, 20, (300, 1)))
    codes, s = fx.quantize_rows(x)
    assert s.shape == (2, 300) and (np.abs(fx.row_values(codes, s) - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * np.repeat(s.T, 128, 1)) * (1 + 2.0 ** -20)).all()
    codes, s = fx.quantize_weights(x[:272])
    assert s.shape == (3, 2) and fx.weight_values(codes, s).shape == (272, 256)
    t, ts = fx.quantize_weights(x[:256].T)
    assert np.array_equal(t.T, codes[:256]) and np.array_equal(ts.T, s[:2])
    codes, s = fx.quantize_columns(x)
    assert codes.shape == (256, 384) and s.shape == (3, 256) and not codes[:, 300:].any() and (np.frexp(s)[0] == 0.5).all()
    v = fx.row_values(codes, s)[:, :300].T
    assert (np.abs(v - x) <= np.maximum(np.abs(x) * 2.0 ** -4, 2.0 ** -10 * np.repeat(s, 128, 0)[:300])).all()
    a = np.abs(x[:128]).max(0)
    assert (s[0] * 448 >= a).all() and (s[0] * 224 < a).all()


def test_activations_of_the_definition():
    g = np.linspace(-5, 5, 1001)
    assert np.allclose(fx.activation(g, "silu"), g / (1 + np.exp(-g)), rtol=1e-14, atol=0)
    assert np.allclose(fx.activation(g, "gelu"), 0.5 * g * (1 + np.tanh(np.sqrt(2 / np.pi) * (g + 0.044715 * g ** 3))), rtol=0, atol=1e-14)


@pytest.mark.parametrize("act", ACTS)
def test_gradients_of_the_definition_against_differences(act):
    rng = np.random.default_rng(2)
    x, w, dh = rng.standard_normal((5, 64)), rng.standard_normal((24, 64)) * 0.2, rng.standard_normal((5, 12))
    def loss(x, w):
        p = x @ w.T
        return (dh * fx.activation(p[:, :12], act) * p[:, 12:]).sum()
    p = x @ w.T
    dg = np.concatenate(fx.gated_gradients(dh, p[:, :12], p[:, 12:], act), 1)
    dx, dw, t = dg @ w, dg.T @ x, 1e-5
    for _ in range(20):
        vx, vw = rng.standard_normal(x.shape), rng.standard_normal(w.shape)
        got = (loss(x + t * vx, w + t * vw) - loss(x - t * vx, w - t * vw)) / (2 * t)
        want = (dx * vx).sum() + (dw * vw).sum()
        assert abs(got - want) <= 1e-6 * (np.abs(dx * vx).sum() + np.abs(dw * vw).sum())


# ---------------------------------------------------------------------------------------------------- refusals
def test_sizes_outside_the_domain(lutq):
    ws, gws = lutq.lutq_fp8_workspace_bytes, lutq.lutq_fp8_gated_workspace_bytes
    assert ws(0, 16, 128) > 0 and ws(1, 1 << 24, 128) > 0 and ws(1, 16, 1 << 22) > 0 and ws(5, 16, 128, 65536) > 0
    for bad in ((-1, 16, 128), (1, 0, 128), (1, 24, 128), (1, 16, 64), (1, 16, 0), (1, 16, (1 << 22) + 128), (1, (1 << 24) + 16, 128), (1 << 30, 16, 128),
                (1 << 29, 16, 512), (1, 16, 128, 0), (1, 16, 128, 65537)):
        assert ws(*bad) == 0
    assert gws(1, 128, 128) > ws(1, 256, 128) - 1 and gws(1, 1 << 21, 128) > 0
    for bad in ((1, 64, 128), (1, 0, 128), (1, 128, 100), (1, (1 << 21) + 128, 128), (1 << 29, 256, 128), (1, 128, 128, 0)):
        assert gws(*bad) == 0
    for f in (lutq.new_fp8_workspace, lutq.new_fp8_gated_workspace):
        with pytest.raises(ValueError, match="unsupported"):
            f(4, 24, 128)


def test_refusals_before_any_launch(lutq):
    """Every one of these returns from host-side validation; no device call is made."""
    lib = lutq.load_library()
    buf = (ctypes.c_char * 4096)()
    a = (ctypes.addressof(buf) + 15) & ~15
    NULL, SHAPE, ALIGN, WORKSPACE, DTYPE = 1, 4, 5, 7, 8
    q = lambda X=a, f=0, dt=0, src=4, rows=None, M=4, K=128, c=a, s=a: lib.lutq_fp8_quantize(X, f, dt, src, rows, M, K, c, s, None)
    assert q(X=None) == q(c=None) == q(s=None) == NULL
    assert q(M=-1) == q(K=64) == q(K=0) == q(src=3) == q(M=1 << 30, src=1 << 30) == q(src=-1, rows=a) == q(src=1 << 31, rows=a) == SHAPE
    assert q(dt=2) == DTYPE and q(X=a + 8) == q(c=a + 4) == q(s=a + 2) == q(rows=a + 2) == ALIGN
    assert q(M=0, src=0, X=None, c=None, s=None) == 0
    qw = lambda W=a, f=0, dt=0, N=16, K=128, c=a, s=a, t=None, ts=None: lib.lutq_fp8_quantize_weights(W, f, dt, N, K, c, s, t, ts, None)
    assert qw(W=None) == qw(c=None) == qw(s=None) == qw(t=a) == qw(ts=a) == NULL and qw(N=8) == qw(N=0) == qw(K=100) == SHAPE
    assert qw(dt=-1) == DTYPE and qw(W=a + 4) == qw(t=a + 8, ts=a) == qw(t=a, ts=a + 2) == ALIGN
    qc = lambda X=a, f=0, dt=0, M=4, K=128, c=a, s=a: lib.lutq_fp8_quantize_columns(X, f, dt, M, K, c, s, None)
    assert qc(X=None) == qc(c=None) == qc(s=None) == NULL and qc(M=0) == qc(M=-3) == qc(K=64) == SHAPE and qc(dt=9) == DTYPE and qc(c=a + 8) == ALIGN
    for f in (lib.lutq_fp8_dequant, lib.lutq_fp8_dequant_weights):
        d = lambda c=a, s=a, M=16, K=128, dt=0, o=a: f(c, s, M, K, dt, o, None)
        assert d(c=None) == d(s=None) == d(o=None) == NULL and d(K=32) == d(M=-16) == SHAPE and d(dt=7) == DTYPE and d(o=a + 2) == d(s=a + 1) == ALIGN
    assert lib.lutq_fp8_dequant(None, None, 0, 128, 0, None, None) == 0 and lib.lutq_fp8_dequant_weights(a, a, 0, 128, 0, a, None) == SHAPE
    need = lutq.lutq_fp8_workspace_bytes(4, 16, 128)
    m = lambda X=a, xs=a, W=a, ws=a, M=4, N=16, K=128, dt=0, Y=a, wk=a, wb=need: lib.lutq_fp8_matmul(X, xs, W, ws, M, N, K, dt, Y, wk, wb, None)
    g = lambda X=a, xs=a, W=a, ws=a, off=a, E=2, M=4, N=16, K=128, dt=0, Y=a, wk=a, wb=1 << 40: \
        lib.lutq_fp8_matmul_grouped(X, xs, W, ws, off, E, M, N, K, dt, Y, wk, wb, None)
    gneed = lutq.lutq_fp8_gated_workspace_bytes(4, 128, 128)
    h = lambda X=a, xs=a, W=a, ws=a, M=4, N=128, K=128, act=0, dt=0, Y=a, hc=None, hs=None, sv=None, wk=a, wb=gneed: \
        lib.lutq_fp8_gated(X, xs, W, ws, M, N, K, act, dt, Y, hc, hs, sv, wk, wb, None)
    hg = lambda X=a, xs=a, W=a, ws=a, off=a, E=2, M=4, N=128, K=128, act=0, dt=0, Y=a, hc=None, hs=None, sv=None, wk=a, wb=1 << 40: \
        lib.lutq_fp8_gated_grouped(X, xs, W, ws, off, E, M, N, K, act, dt, Y, hc, hs, sv, wk, wb, None)
    for f in (m, g, h, hg):
        assert f(X=None) == f(W=None) == f(ws=None) == f(Y=None) == NULL
        assert f(M=-1) == f(N=8) == f(N=0) == f(K=64) == f(M=1 << 30) == f(K=(1 << 22) + 128) == SHAPE and f(dt=2) == DTYPE
        assert f(X=a + 8) == f(xs=a + 2) == f(W=a + 4) == f(ws=a + 1) == f(Y=a + 2) == f(wk=a + 1) == ALIGN
        assert f(wk=None) == f(wb=0) == WORKSPACE
        assert f(M=0, X=None, xs=None, Y=None, wk=None) == 0
    assert m(wb=need - 1) == WORKSPACE and h(wb=gneed - 1) == WORKSPACE
    for f in (g, hg):
        assert f(off=None) == NULL and f(E=0) == f(E=65537) == SHAPE and f(off=a + 2) == ALIGN and f(M=0, off=None) == 0
    for f in (h, hg):
        assert f(N=16) == f(N=192) == SHAPE and f(act=2) == f(act=-1) == DTYPE
        assert f(hc=a) == f(hs=a) == f(Y=None, hs=a) == NULL and f(hc=a + 8, hs=a) == f(hc=a, hs=a + 1) == f(sv=a + 2) == ALIGN
    r = lambda dh=a, sv=a, M=4, F=128, act=0, dt=0, d=a, c=None, s=None, t=None, ts=None: lib.lutq_fp8_gated_grad(dh, sv, M, F, act, dt, d, c, s, t, ts, None)
    assert r(dh=None) == r(sv=None) == r(d=None) == r(c=a) == r(s=a) == r(t=a) == r(ts=a) == NULL
    assert r(F=64) == r(F=0) == r(M=-1) == r(F=(1 << 21) + 128) == r(M=0, t=a, ts=a) == SHAPE and r(act=3) == r(dt=2) == DTYPE
    assert r(dh=a + 2) == r(sv=a + 8) == r(d=a + 4) == r(c=a + 8, s=a) == r(c=a, s=a + 2) == r(t=a + 4, ts=a) == r(t=a, ts=a + 1) == ALIGN
    assert r(M=0, dh=None, sv=None, d=None) == 0
    need = lutq.lutq_fp8_workspace_bytes(32, 16, 128)
    w = lambda dY=a, ds=a, X=a, xs=a, N=32, K=16, M=128, dt=0, dW=a, wk=a, wb=need: lib.lutq_fp8_weight_grad(dY, ds, X, xs, N, K, M, dt, dW, wk, wb, None)
    assert w(dY=None) == w(ds=None) == w(X=None) == w(xs=None) == w(dW=None) == NULL
    assert w(N=0) == w(N=24) == w(K=8) == w(M=0) == w(M=100) == w(M=(1 << 22) + 128) == SHAPE and w(dt=4) == DTYPE
    assert w(dY=a + 8) == w(ds=a + 2) == w(X=a + 1) == w(dW=a + 8) == ALIGN and w(wk=None) == w(wb=need - 1) == WORKSPACE


def test_what_an_error_says_is_so_of_8_bit_calls(lutq):
    """Each status's text names the limit that the call was refused for."""
    text = lambda status: lutq.load_library().lutq_status_string(status).decode()
    assert "8-bit: K % 128" in text(4) and "F % 128" in text(4) and "N % 16" in text(4)
    assert "to 4" in text(5) and "LUTQ_GELU" in text(8)


def test_binding_refuses_host_tensors(lutq):
    import torch
    x, u = torch.zeros((16, 128), dtype=torch.float16), torch.zeros((16, 128), dtype=torch.uint8)
    s, o = torch.zeros((1, 16)), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: lutq.lutq_fp8_quantize(x, u, s), lambda: lutq.lutq_fp8_quantize_weights(x, u, s), lambda: lutq.lutq_fp8_quantize_columns(x, u, s),
                 lambda: lutq.lutq_fp8_dequant(u, s, x), lambda: lutq.lutq_fp8_dequant_weights(u, s, x), lambda: lutq.lutq_fp8_matmul(u, u, s, x, u, x_scales=s),
                 lambda: lutq.lutq_fp8_matmul_grouped(u, u, s, o, x, u, x_scales=s), lambda: lutq.lutq_fp8_gated(x, u, s, x, u),
                 lambda: lutq.lutq_fp8_gated_grouped(x, u, s, o, x, u), lambda: lutq.lutq_fp8_gated_grad(x, x, dense=x),
                 lambda: lutq.lutq_fp8_weight_grad(u, s, u, s, x, u)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    with pytest.raises(ValueError, match="activation"):
        lutq.lutq_fp8_gated(x, u, s, x, u, activation="relu")
    with pytest.raises(TypeError, match="offsets"):
        lutq.lutq_fp8_gated_grouped(x, u, s, None, x, u)
    nat = lutq.binding._native()
    assert nat.fp8_quantize(0, x, u, s, None, None, None) == nat.fp8_quantize(x) == nat.fp8_dequant(0, u, s, x) == nat.fp8_grad(x, x, 0, x, None, None, None, None) == -1
    assert nat.fp8_mm(u, s, u, s, None, -1, 0, x, None, None, None, u) == nat.fp8_mm(u, s, u, s, "o", 2, 0, x, None, None, None, u) == -1
    assert nat.fp8_weight_grad(u, s, u, s, x, u) == -1


# ---------------------------------------------------------------------------------------------------- device: quantisers
def source_type(src):
    import torch
    return torch.float32 if src == "f32" else torch_dtype(src)


def edge_values(src, M, K, seed, axis=1, block=128):
    """Values over the type's whole range, block by block (128 along `axis`): ordinary ones, ties, one magnitude only, the smallest and the
    largest numbers, zeros of either sign, blocks with an infinity or a NaN."""
    import torch
    rng = np.random.default_rng(seed)
    lo, hi = {"f32": (-149, 127), "bf16": (-133, 127), "f16": (-24, 15)}[src]
    n = -(-(K if axis else M) // block)
    rows = M if axis else K
    x = rng.standard_normal((rows, n, block))
    kind = rng.integers(0, 8, (rows, n))
    top = rng.integers(lo, hi, (rows, n)).astype(np.float64)
    grid = np.concatenate([fx.MAGNITUDES, (fx.MAGNITUDES[1:] + fx.MAGNITUDES[:-1]) / 2]) / 448
    with np.errstate(over="ignore"):
        k = lambda v: (kind == v)[..., None]
        x = np.where(k(1), rng.choice(grid, x.shape) * rng.choice([-1, 1], x.shape) * np.exp2(np.minimum(top, hi - 1))[..., None], x)
        x = np.where(k(2), x * np.exp2(np.minimum(top, hi - 3))[..., None], x)
        x = np.where(k(3), rng.integers(-6, 7, x.shape) * 2.0 ** lo, x)
    x = np.where(k(4), np.where(rng.random(x.shape) < 0.5, 0.0, -0.0), x)
    x = np.where(k(5), rng.choice([BIG.get(src, 3.4028234663852886e38), -BIG.get(src, 3.4028234663852886e38), 1.0], x.shape), x)
    x[..., 7] = np.where(kind == 6, rng.choice([np.inf, -np.inf, np.nan], kind.shape), x[..., 7])
    x = x.reshape(rows, n * block)[:, :K if axis else M]
    return torch.from_numpy(np.ascontiguousarray(x if axis else x.T)).to(source_type(src))


def same_bits(t, want):
    return np.array_equal(t.cpu().numpy(), want, equal_nan=True)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 128), (1, 4096), (3, 384), (15, 2176), (16, 128), (17, 2176), (129, 640), (300, 16384), (8209, 1152)])
def test_quantize_rows(lutq, src, M, K):
    x = edge_values(src, M, K, M + K)
    codes, s = empty(M + 2, K), empty(K // 128, M, dtype="f32")
    lutq.lutq_fp8_quantize(x.cuda(), codes[:M], s)
    want_c, want_s = fx.quantize_rows(as_f64(x))
    assert np.array_equal(as_u8(codes[:M]), want_c) and same_bits(s, want_s) and (codes[M:] == 0x7f).all().item()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
def test_quantize_picks_rows(lutq, src):
    import torch
    rng = np.random.default_rng(3)
    x = edge_values(src, 40, 640, 5)
    want_c, want_s = fx.quantize_rows(np.concatenate([as_f64(x), np.zeros((1, 640))]))
    for M in (1, 7, 100, 5000):
        rows = rng.integers(0, 40, M).astype(np.int32)
        rows[rng.random(M) < 0.2] = rng.choice([-1, 40, 2 ** 31 - 1, -2 ** 31])
        codes, s = torch.empty((M, 640), dtype=torch.float8_e4m3fn, device="cuda"), empty(5, M, dtype="f32")
        lutq.lutq_fp8_quantize(x.cuda(), codes, s, rows=to_gpu(rows))
        r = np.where((rows >= 0) & (rows < 40), rows, 40)
        assert np.array_equal(as_u8(codes), want_c[r]) and same_bits(s, want_s[:, r])


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N,K", [(16, 128), (48, 512), (128, 256), (144, 1664), (384, 384), (4112, 256)])
def test_quantize_weights(lutq, src, N, K):
    import torch
    x = edge_values(src, N, K, N + K, block=128)
    x[:, 128:256] = torch.randn((N, min(128, K - 128)), generator=torch.Generator().manual_seed(1)).to(x.dtype) if K > 128 else 0
    codes, s = empty(N, K), empty(-(-N // 128), K // 128, dtype="f32")
    t, ts = empty(K, N), empty(K // 128, -(-N // 128), dtype="f32")
    want_c, want_s = fx.quantize_weights(as_f64(x))
    lutq.lutq_fp8_quantize_weights(x.cuda(), codes, s)
    assert np.array_equal(as_u8(codes), want_c) and same_bits(s, want_s)
    codes.fill_(0x7f)
    lutq.lutq_fp8_quantize_weights(x.cuda(), codes, s, transposed=(t, ts))
    assert np.array_equal(as_u8(codes), want_c) and np.array_equal(as_u8(t), want_c.T) and same_bits(ts, want_s.T)


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 128), (7, 256), (128, 384), (129, 128), (300, 1152), (1000, 2176)])
def test_quantize_columns(lutq, src, M, K):
    x = edge_values(src, M, K, M * K, axis=0)
    codes, s = empty(K, -(-M // 128) * 128), empty(-(-M // 128), K, dtype="f32")
    lutq.lutq_fp8_quantize_columns(x.cuda(), codes, s)
    want_c, want_s = fx.quantize_columns(as_f64(x))
    assert np.array_equal(as_u8(codes), want_c) and same_bits(s, want_s)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K", [(16, 128), (48, 640), (1040, 4096), (8208, 1152)])
def test_dequant_both_forms(lutq, dtype, M, K):
    """Every code, NaN among them."""
    rng = np.random.default_rng(M + K)
    c = rng.integers(0, 256, (M, K), dtype=np.uint8)
    for scales, call, values in ((rng.standard_normal((K // 128, M)), lutq.lutq_fp8_dequant, fx.row_values),
                                 (rng.standard_normal((-(-M // 128), K // 128)), lutq.lutq_fp8_dequant_weights, fx.weight_values)):
        scales = scales.astype(np.float32)
        out = empty(M, K, dtype=dtype)
        call(to_gpu(c), to_gpu(scales), out)
        got, want = as_f64(out), values(c, scales)
        assert np.array_equal(np.isnan(got), np.isnan(want))
        ok = ~np.isnan(want)
        assert (np.abs(got - want) <= half_step(want, dtype) + 2.0 ** -24 * np.abs(want))[ok].all()


@pytest.mark.gpu
def test_offsets_beyond_32_bits(lutq):
    """More than 4 GiB of codes: the last rows' are where they belong, in all forms."""
    import torch
    M, K = 266256, 16384
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((144, K), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").to(torch.bfloat16)
    x[-144:] = tail
    c, s = torch.full((M, K), 0x7f, dtype=torch.uint8, device="cuda"), torch.empty((K // 128, M), device="cuda")
    lutq.lutq_fp8_quantize(x, c, s)
    c2, s2 = torch.empty_like(c[:144]), torch.empty((K // 128, 144), device="cuda")
    lutq.lutq_fp8_quantize(tail, c2, s2)
    assert torch.equal(c[-144:], c2) and torch.equal(s[:, -144:], s2) and not c[:-144].any().item()
    back, want = torch.empty_like(x), torch.empty_like(tail)
    lutq.lutq_fp8_dequant(c, s, back)
    lutq.lutq_fp8_dequant(c2, s2, want)
    assert torch.equal(back[-144:], want)
    # the rows as activations of a product, streamed and tiled, and as weights
    y, ws = torch.empty((M, 16), dtype=torch.bfloat16, device="cuda"), torch.empty((1, K // 128), device="cuda")
    w = torch.empty((16, K), dtype=torch.uint8, device="cuda")
    lutq.lutq_fp8_quantize_weights(tail[:16], w, ws)
    wv = torch.empty_like(tail[:16])
    lutq.lutq_fp8_dequant_weights(w, ws, wv)
    lutq.lutq_fp8_matmul(c, w, ws, y, lutq.new_fp8_workspace(M, 16, K), x_scales=s)
    sums = fx.product(fx.row_values(as_u8(c2), s2.cpu().numpy()), fx.weight_values(as_u8(w), ws.cpu().numpy()))
    assert (np.abs(as_f64(y[-144:]) - sums[0]) <= off_by_at_most(sums, K, "bf16")).all() and not y[:-144].any().item()
    del back, y
    ws_all = torch.empty((-(-M // 128), K // 128), device="cuda")
    lutq.lutq_fp8_quantize_weights(x, c, ws_all)
    for rows in (3, 40):
        y = torch.empty((rows, M), dtype=torch.bfloat16, device="cuda")
        xr, xs = c2[:rows].contiguous(), s2[:, :rows].contiguous()
        lutq.lutq_fp8_matmul(xr, c, ws_all, y, lutq.new_fp8_workspace(rows, M, K), x_scales=xs)
        last = c[-144:].cpu().numpy()
        sc = ws_all.cpu().numpy()
        w_of = np.stack([fx.TABLE[last[r]] * np.repeat(sc[(M - 144 + r) // 128].astype(np.float64), 128) for r in range(144)])
        sums = fx.product(fx.row_values(as_u8(xr), xs.cpu().numpy()), w_of)
        assert (np.abs(as_f64(y[:, -144:]) - sums[0]) <= off_by_at_most(sums, K, "bf16")).all() and not y[:, :-144].any().item()


# ---------------------------------------------------------------------------------------------------- device: products
def codes_within(rng, shape, binades, top=8):
    """Codes of either sign whose magnitudes lie in so many binades below 2^(top + 1), one in fifty zero."""
    c = rng.integers(8 * (top + 8 - binades), 8 * (top + 8) - (1 if top == 8 else 0), shape)
    return np.where(rng.random(shape) < 0.02, 0, c + 128 * rng.integers(0, 2, shape)).astype(np.uint8)


class Problem:
    """Quantised factors on the device and their values in fp64.  `wide`: rows of weights, N, or 2 N for the gated block."""

    def __init__(self, lutq, M, N, K, dtype, experts=0, seed=0, gated=False):
        import torch
        rng = np.random.default_rng(seed + M * 3 + N * 5 + K * 7)
        self.M, self.N, self.K, self.dtype, self.experts = M, N, K, dtype, experts
        wide, e = 2 * N if gated else N, max(experts, 1)
        x = rng.choice([-1, 1], (M, K)) * np.exp2(rng.uniform(-2.9, 0, (M, K))) * np.repeat(np.exp2(rng.integers(-3, 3, (M, K // 128))), 128, 1)
        x[rng.random((M, K)) < 0.02] = 0
        self.X = torch.from_numpy(x).to(torch_dtype(dtype)).cuda()
        codes, s = fx.quantize_rows(as_f64(self.X))
        self.x = fx.row_values(codes, s)
        self.codes, self.s = to_gpu(codes), to_gpu(s)
        wc = codes_within(rng, (e, wide, K), 5, 6)
        sw = (np.exp2(rng.uniform(-3, 0, (e, -(-wide // 128), K // 128))) * (K * 6e3) ** -0.5).astype(np.float32)
        self.w = np.stack([fx.weight_values(c, v) for c, v in zip(wc, sw)])
        shape = (lambda a: a) if experts else (lambda a: a[0])
        self.W, self.sw = to_gpu(shape(wc)), to_gpu(shape(sw))
        self.ws = (lutq.new_fp8_gated_workspace if gated else lutq.new_fp8_workspace)(M, N, K, e)

    def out(self, dtype=None, N=None):
        """Y with guard rows before and behind it."""
        import torch
        self.guarded = empty(self.M + 32, N or self.N, dtype=dtype or self.dtype)
        return self.guarded[16:16 + self.M]

    def guards_hold(self):
        return (self.guarded[:16] == self.guarded[0, 0]).all().item() and (self.guarded[16 + self.M:] == self.guarded[0, 0]).all().item()

    def args(self, dense):
        return (self.X, None) if dense else (self.codes, self.s)

    def clean(self):
        return not self.ws[:65536].any().item()


def cut_at_most(x, w):
    """What the instruction cuts off of products of any codes: x, w dense fp64 values, K in eights."""
    import torch
    x, w = (torch.from_numpy(a).abs().float().cuda() for a in (x, w))
    total = torch.zeros((x.shape[0], w.shape[0]), device="cuda")
    for k in range(0, x.shape[1], 8):
        most = torch.zeros_like(total)
        for j in range(k, k + 8):
            most = torch.maximum(most, x[:, j, None] * w[None, :, j])
        total += most
    return total.double().cpu().numpy() * (7 * 2.0 ** -13 * (1 + 2.0 ** -10))


def worst_of(got, ref, bound):
    return float(np.max(np.abs(got - ref) / bound)) if got.size else 0.0


SIZES = [(1, 16, 128), (1, 48, 4096), (2, 272, 640), (4, 4112, 512), (5, 64, 1152), (7, 4112, 512), (15, 64, 1152), (16, 96, 2048), (17, 160, 384), (32, 32, 5120),
         (33, 304, 1024), (63, 16, 768), (64, 528, 512), (65, 80, 896), (100, 256, 14336), (128, 1040, 1152), (129, 512, 256), (200, 304, 3200),
         (255, 272, 128), (257, 528, 640), (515, 1296, 1408), (1000, 16, 512), (2049, 784, 384), (601, 4112, 1152)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_product(lutq, M, N, K, dense, dtype):
    p = Problem(lutq, M, N, K, dtype)
    x, s = p.args(dense)
    y = p.out()
    lutq.lutq_fp8_matmul(x, p.W, p.sw, y, p.ws, x_scales=s)
    got, sums = as_f64(y), fx.product(p.x, p.w[0])
    assert worst_of(got, sums[0], off_by_at_most(sums, K, dtype)) <= 1.0
    assert p.guards_hold() and p.clean()
    again = p.out()
    lutq.lutq_fp8_matmul(x, p.W, p.sw, again, p.ws, x_scales=s)
    assert np.array_equal(as_f64(again), got)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 272, 640), (40, 304, 1152), (300, 528, 512), (601, 1040, 2176)])
def test_product_of_any_codes(lutq, M, N, K):
    """Gaussian factors, subnormal codes among them."""
    import torch
    p = Problem(lutq, M, N, K, "f16")
    rng = np.random.default_rng(M)
    wc = rng.integers(0, 256, (N, K)).astype(np.uint8)
    wc[(wc & 127) == 127] = 1
    X = torch.from_numpy(rng.standard_normal((M, K))).half().cuda()
    codes, s = fx.quantize_rows(as_f64(X))
    x, w = fx.row_values(codes, s), fx.weight_values(wc, p.sw.cpu().numpy())
    sums = fx.product(x, w)
    for args in ((X, None), (to_gpu(codes), to_gpu(s))):
        y = p.out()
        lutq.lutq_fp8_matmul(args[0], to_gpu(wc), p.sw, y, p.ws, x_scales=args[1])
        assert worst_of(as_f64(y), sums[0], off_by_at_most(sums, K, "f16") + cut_at_most(x, w)) <= 1.0 and p.guards_hold()


def counts_to_offsets(counts, first=0):
    return np.concatenate([[first], first + np.cumsum(counts)]).astype(np.int32)


GROUPS = {
    "one_expert": ([37], 0, 0), "one_row_each": ([1] * 9, 0, 0), "none_have_rows": ([0, 0, 0], 0, 5), "last_only": ([0, 0, 0, 20], 0, 0),
    "first_only": ([300, 0, 0], 0, 3), "ragged": ([3, 0, 17, 16, 1, 0, 64, 33], 2, 7), "many_experts": ([0, 1, 2, 0] * 35, 0, 1),
    "few_rows_many_experts": ([0] * 70 + [3] + [0] * 80 + [2] + [0] * 49, 0, 0), "large": ([520, 0, 129, 257, 1], 1, 30),
    "uneven": ([9] + [0] * 11, 0, 0), "sixty_five": ([17] * 65, 0, 0),
}


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("N,K", [(48, 640), (272, 128)])
@pytest.mark.parametrize("name", list(GROUPS))
def test_product_by_expert(lutq, name, N, K, dense, dtype):
    counts, first, behind = GROUPS[name]
    off = counts_to_offsets(counts, first)
    p = Problem(lutq, int(off[-1]) + behind, N, K, dtype, experts=len(counts), seed=len(name))
    x, s = p.args(dense)
    y = p.out()
    lutq.lutq_fp8_matmul_grouped(x, p.W, p.sw, to_gpu(off), y, p.ws, x_scales=s)
    ref, mag = np.full((p.M, N), -7.0), np.zeros((p.M, N))
    for g in range(p.experts):
        a, b = int(off[g]), int(off[g + 1])
        ref[a:b], mag[a:b] = fx.product(p.x[a:b], p.w[g])
    assert worst_of(as_f64(y), ref, off_by_at_most((ref, mag), K, dtype)) <= 1.0
    assert p.guards_hold() and p.clean()


def gated_reference(x, w, K, act, dtype):
    """(H, bound), ((G, magnitudes), (U, magnitudes))."""
    F = w.shape[0] // 2
    g, u = fx.product(x, w[:F]), fx.product(x, w[F:])
    return gated_off(g, u, K, act, dtype), (g, u)


def check_h_codes(codes, scales, h16):
    """They are what the quantiser makes of H of 16 bits."""
    c, s = fx.quantize_rows(as_f64(h16))
    return np.array_equal(as_u8(codes), c) and same_bits(scales, s)


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("act,dtype", [("silu", "bf16"), ("gelu", "f16")])
@pytest.mark.parametrize("M,F,K", [(1, 128, 128), (1, 384, 4096), (3, 256, 640), (4, 2048, 512), (16, 128, 1152), (17, 384, 384), (33, 256, 2048), (64, 512, 128), (100, 128, 5120),
                                   (129, 896, 640), (257, 384, 1152), (515, 1408, 256), (1025, 640, 384), (2049, 256, 128)])
def test_gated(lutq, M, F, K, act, dtype, dense):
    p = Problem(lutq, M, F, K, dtype, gated=True)
    x, s = p.args(dense)
    (want, bound), (g, u) = gated_reference(p.x, p.w[0], K, act, dtype)
    h = p.out()
    lutq.lutq_fp8_gated(x, p.W, p.sw, h, p.ws, x_scales=s, activation=act)
    assert worst_of(as_f64(h), want, bound) <= 1.0 and p.guards_hold() and p.clean()
    saved, again = empty(M, 2 * F, dtype=dtype), p.out()     # (its guards are checked, it is kept)
    lutq.lutq_fp8_gated(x, p.W, p.sw, again, p.ws, x_scales=s, activation=act, saved=saved)
    assert worst_of(as_f64(again), want, bound) <= 1.0 and p.guards_hold()       # (sums of another order, exact ones of codes)
    for at, sums in ((0, g), (F, u)):
        assert worst_of(as_f64(saved[:, at:at + F]), sums[0], off_by_at_most(sums, K, dtype)) <= 1.0
    codes, hs = p.out("u8"), empty(F // 128, M, dtype="f32")
    lutq.lutq_fp8_gated(x, p.W, p.sw, codes, p.ws, x_scales=s, activation=act, h_scales=hs, dtype=torch_dtype(dtype))
    assert check_h_codes(codes, hs, again) and p.guards_hold() and p.clean()
    codes, was = p.out("u8"), saved.clone()
    saved.fill_(0)
    lutq.lutq_fp8_gated(x, p.W, p.sw, codes, p.ws, x_scales=s, activation=act, h_scales=hs, saved=saved, dtype=torch_dtype(dtype))
    assert check_h_codes(codes, hs, again) and p.guards_hold() and p.clean() and np.array_equal(as_f64(saved), as_f64(was))


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("act,dtype", [("silu", "f16"), ("gelu", "bf16")])
@pytest.mark.parametrize("F,K", [(128, 640), (384, 128)])
@pytest.mark.parametrize("name", list(GROUPS))
def test_gated_by_expert(lutq, name, F, K, act, dtype, dense):
    counts, first, behind = GROUPS[name]
    off = counts_to_offsets(counts, first)
    p = Problem(lutq, int(off[-1]) + behind, F, K, dtype, experts=len(counts), seed=len(name), gated=True)
    x, s = p.args(dense)
    h, saved = p.out(), empty(p.M, 2 * F, dtype=dtype)
    lutq.lutq_fp8_gated_grouped(x, p.W, p.sw, to_gpu(off), h, p.ws, x_scales=s, activation=act, saved=saved)
    want, bound, gu = np.full((p.M, F), -7.0), np.full((p.M, F), 1e-9), np.full((p.M, 2 * F), -7.0)
    mag = np.zeros((p.M, 2 * F))
    for e in range(p.experts):
        a, b = int(off[e]), int(off[e + 1])
        if b > a:
            (want[a:b], bound[a:b]), (g, u) = gated_reference(p.x[a:b], p.w[e], K, act, dtype)
            gu[a:b], mag[a:b] = np.concatenate([g[0], u[0]], 1), np.concatenate([g[1], u[1]], 1)
    assert worst_of(as_f64(h), want, bound) <= 1.0 and p.guards_hold() and p.clean()
    assert worst_of(as_f64(saved), gu, off_by_at_most((gu, mag), K, dtype)) <= 1.0
    plain = p.out()
    lutq.lutq_fp8_gated_grouped(x, p.W, p.sw, to_gpu(off), plain, p.ws, x_scales=s, activation=act)
    assert worst_of(as_f64(plain), want, bound) <= 1.0 and p.guards_hold()
    codes, hs = p.out("u8"), empty(F // 128, p.M, dtype="f32")
    lutq.lutq_fp8_gated_grouped(x, p.W, p.sw, to_gpu(off), codes, p.ws, x_scales=s, activation=act, h_scales=hs, dtype=torch_dtype(dtype))
    inside = slice(int(off[0]), int(off[-1]))
    assert check_h_codes(codes[inside], hs[:, inside], h[inside]) and p.guards_hold()
    for rows in (slice(0, int(off[0])), slice(int(off[-1]), p.M)):
        assert (codes[rows] == 0x7f).all().item() and (hs[:, rows] == -7.0).all().item()


@pytest.mark.gpu
def test_h_and_its_codes_in_one_call(lutq):
    """The C entry gives both where it is asked for both."""
    import torch
    p = Problem(lutq, 40, 256, 384, "bf16", gated=True)
    h, codes, hs = p.out(), empty(40, 256), empty(2, 40, dtype="f32")
    st = lutq.load_library().lutq_fp8_gated(p.X.data_ptr(), None, p.W.data_ptr(), p.sw.data_ptr(), 40, 256, 384, 0, 1, h.data_ptr(), codes.data_ptr(),
                                            hs.data_ptr(), None, p.ws.data_ptr(), p.ws.numel(), torch.cuda.current_stream().cuda_stream)
    (want, bound), _ = gated_reference(p.x, p.w[0], 384, "silu", "bf16")
    assert st == 0 and worst_of(as_f64(h), want, bound) <= 1.0 and check_h_codes(codes, hs, h) and p.guards_hold()


def grad_reference(dh, g, u, act):
    """dG, dU side by side in fp64, and how far off in fp32 they may be: (16 + 8 |z|) 2^-24 of each term."""
    s, z, f = fx.sigma(fx.argument(g, act)), fx.argument(g, act), fx.activation(g, act)
    dz = 1.0 if act == "silu" else 2 * np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * g * g)
    dg, du = fx.gated_gradients(dh, g, u, act)
    rel = (16 + 8 * np.abs(z)) * 2.0 ** -24
    off = np.abs(dh * u) * (s + np.abs(f * (1 - s) * dz)) * rel + np.abs(dh * u) * np.abs(f * dz) * s * rel
    return np.concatenate([dg, du], 1), np.concatenate([off + np.abs(dh * u) * (1 + np.abs(g * dz)) * 2.0 ** -126, np.abs(du) * rel + np.abs(dh * g) * 2.0 ** -126], 1)


def quantised_is_near(values, scales_of_values, ref, off, a, power):
    """Values back from codes whose scales (of each value) are given, of what is within `off` of `ref`; `a`: the blocks' largest magnitudes."""
    tol = off.max() if off.size else 0.0
    if power:
        ok = (scales_of_values * 448 >= (a - tol) * (1 - 2.0 ** -20)).all() and (scales_of_values * 224 <= np.maximum(a + tol, fx.FLOOR) * (1 + 2.0 ** -20)).all()
    else:
        ok = (np.abs(scales_of_values * 448 - np.maximum(a, fx.FLOOR)) <= tol + 2.0 ** -22 * np.maximum(a, fx.FLOOR)).all()   # (one rounding)
    near = np.maximum(np.abs(ref) * 2.0 ** -4, scales_of_values * 2.0 ** -10) * (1 + 2.0 ** -20) + 1.1 * off
    return ok and (np.abs(values - ref) <= near).all()


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,F", [(1, 128), (7, 256), (128, 128), (129, 384), (300, 1152)])
def test_gated_gradient(lutq, M, F, act, dtype):
    import torch
    rng = np.random.default_rng(M + F)
    t = lambda a: torch.from_numpy(a).to(torch_dtype(dtype)).cuda()
    dh, gu = t(rng.standard_normal((M, F)) * 2.0 ** -5), t(rng.standard_normal((M, 2 * F)) * 4)
    gu[M // 2, :F] = torch.linspace(-60, 60, F)          # (far into either end of the activation)
    dh[::5] = 0
    d, g, u = as_f64(dh), as_f64(gu[:, :F]), as_f64(gu[:, F:])
    ref, off = grad_reference(d, g, u, act)
    dense, (rc, rs), up = empty(M, 2 * F, dtype=dtype), (empty(M, 2 * F), empty(2 * F // 128, M, dtype="f32")), -(-M // 128)
    cc, cs = empty(2 * F, up * 128), empty(up, 2 * F, dtype="f32")
    lutq.lutq_fp8_gated_grad(dh, gu, activation=act, dense=dense, rows=(rc, rs), columns=(cc, cs))
    assert worst_of(as_f64(dense), ref, half_step(ref, dtype) + off) <= 1.0
    sr = np.repeat(rs.cpu().numpy().astype(np.float64).T, 128, 1)
    a = np.repeat(np.abs(ref).reshape(M, -1, 128).max(-1), 128, 1)
    assert quantised_is_near(fx.row_values(as_u8(rc), rs.cpu().numpy()), sr, ref, off, a, False)
    pad = np.zeros((up * 128, 2 * F))
    pad[:M] = ref
    pad_off = np.zeros_like(pad)
    pad_off[:M] = off
    sc = np.repeat(cs.cpu().numpy().astype(np.float64), 128, 0)
    a = np.repeat(np.abs(pad).reshape(up, 128, -1).max(1), 128, 0)
    assert (np.frexp(sc)[0] == 0.5).all() and not cc[:, M:].any().item()
    assert quantised_is_near(fx.row_values(as_u8(cc), cs.cpu().numpy()).T, sc, pad, pad_off, a, True)
    # each form alone, the same bits
    alone = empty(M, 2 * F, dtype=dtype), (empty(M, 2 * F), empty(2 * F // 128, M, dtype="f32")), (empty(2 * F, up * 128), empty(up, 2 * F, dtype="f32"))
    lutq.lutq_fp8_gated_grad(dh, gu, activation=act, dense=alone[0])
    lutq.lutq_fp8_gated_grad(dh, gu, activation=act, rows=alone[1])
    lutq.lutq_fp8_gated_grad(dh, gu, activation=act, columns=alone[2])
    for x, y in ((alone[0], dense), (alone[1][0], rc), (alone[1][1], rs), (alone[2][0], cc), (alone[2][1], cs)):
        assert torch.equal(x, y)


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", DTYPES)
def test_gated_gradient_far_beyond_the_activation(lutq, act, dtype):
    """G from 128 to the type's largest number, of either sign: sigma is 1 or 0 there, to far less than 2^-24 (sigma(-128) < 2^-184), and so is the slope.
    dG = dH U and dU = dH G are products of two 16-bit numbers, which fp32 holds; three roundings of 2^-24 are allowed all the same.  Every block and column
    of the quantised forms has a scale."""
    import torch
    M, F = 130, 256
    rng = np.random.default_rng(5)
    t = lambda a: torch.from_numpy(a).to(torch_dtype(dtype)).cuda()
    g = np.exp2(rng.uniform(7, {"f16": 15.9, "bf16": 127.9}[dtype], (M, F))) * rng.choice([-1, 1], (M, F))
    g[0, :8], g[1, :8] = BIG[dtype], -BIG[dtype]
    if dtype == "bf16":
        g[2, :6] = [1e19, -1e19, 3.7e19, -3.7e19, 6e19, -6e19]      # (about where 0.134 G^2 passes fp32's largest number)
    gu = t(np.concatenate([g, rng.standard_normal((M, F)) * 4], 1))
    dh = t(rng.standard_normal((M, F)) * 2.0 ** -5)
    d, g, u = as_f64(dh), as_f64(gu[:, :F]), as_f64(gu[:, F:])
    ref = np.concatenate([np.where(g > 0, d * u, 0.0), np.where(g > 0, d * g, 0.0)], 1)
    up = -(-M // 128)
    dense, (rc, rs), (cc, cs) = empty(M, 2 * F, dtype=dtype), (empty(M, 2 * F), empty(2 * F // 128, M, dtype="f32")), (empty(2 * F, up * 128), empty(up, 2 * F, dtype="f32"))
    lutq.lutq_fp8_gated_grad(dh, gu, activation=act, dense=dense, rows=(rc, rs), columns=(cc, cs))
    assert worst_of(as_f64(dense), ref, half_step(ref, dtype) + 3 * 2.0 ** -24 * np.abs(ref)) <= 1.0 and (as_f64(dense)[ref == 0] == 0).all()
    assert rs.isfinite().all().item() and cs.isfinite().all().item()
    off = 3 * 2.0 ** -24 * np.abs(ref)
    near = lambda values, scales: (np.abs(values - ref) <= np.maximum(np.abs(ref) * 2.0 ** -4, scales * 2.0 ** -10) * (1 + 2.0 ** -20) + off).all()
    assert near(fx.row_values(as_u8(rc), rs.cpu().numpy()), np.repeat(rs.cpu().numpy().astype(np.float64).T, 128, 1))
    assert near(fx.row_values(as_u8(cc), cs.cpu().numpy()).T[:M], np.repeat(cs.cpu().numpy().astype(np.float64), 128, 0)[:M])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("N,K,M", [(16, 16, 1), (48, 128, 128), (64, 80, 300), (272, 144, 129), (304, 528, 1000), (1040, 272, 640), (2816, 1152, 300), (144, 96, 9000)])
def test_weight_gradient(lutq, N, K, M, dtype):
    rng = np.random.default_rng(N + K + M)
    up = -(-M // 128) * 128
    dyc, xc = codes_within(rng, (N, up), 4), codes_within(rng, (K, up), 5, 5)
    dyc[:, M:], xc[:, M:] = 0, 0
    ds, xs = (np.exp2(rng.integers(-12, -5, (up // 128, n))).astype(np.float32) for n in (N, K))
    ws = lutq.new_fp8_workspace(N, K, up)
    guarded = empty(N + 32, K, dtype=dtype)
    lutq.lutq_fp8_weight_grad(to_gpu(dyc), to_gpu(ds), to_gpu(xc), to_gpu(xs), guarded[16:16 + N], ws)
    sums = fx.product(fx.row_values(dyc, ds), fx.row_values(xc, xs))
    assert worst_of(as_f64(guarded[16:16 + N]), sums[0], off_by_at_most(sums, up, dtype)) <= 1.0
    assert (guarded[:16] == -7).all().item() and (guarded[16 + N:] == -7).all().item() and not ws[:65536].any().item()
