"""Microscaled 4-bit operators: quantiser, its inverse, the product and the product by expert, against the definition in fp64.

Bounds, all fixed by arithmetic.  Codes, exponents and values back are exact.  A product's element may be off by one rounding to
the 16-bit type (half a step of it) and by the fp32 sums: the 4-bit products are exact, every instruction adds 128 of them and the sum so far with an
error of at most 2^-22 of the magnitudes it adds (two truncations), and the at most 16 + 32 partial sums of wavefronts and slices add
2^-24 each: (K / 128 + 12) 2^-22 sum |x w| in all."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest

from gpu_util import torch_dtype, ulp16
from oracle import mx4_oracle as mx

DTYPES = ("f16", "bf16")


def off_by_at_most(y, sums, K, dtype):
    ref, mag = sums
    big = 65504.0 if dtype == "f16" else 3.3895313892515355e38
    return 0.5 * ulp16(np.minimum(np.abs(ref), big), dtype) + (K // 128 + 12) * 2.0 ** -22 * mag


# ---------------------------------------------------------------------------------------------------- the definition, pinned
def test_definition_against_exact_rationals():
    rng = np.random.default_rng(5)
    x = np.concatenate([rng.standard_normal(64) * 2.0 ** rng.integers(-20, 20), np.repeat([5.0, -2.5, 0.75, 7.9, 0.25, 3.5, 1.25, 1.75], 4),
                        np.zeros(32)]).astype(np.float32).reshape(1, -1)
    codes, e = mx.quantize(x)
    mags = [Fraction(m) for m in (0, Fraction(1, 2), 1, Fraction(3, 2), 2, 3, 4, 6)]
    for b in range(x.shape[1] // 32):
        block = [Fraction(float(v)) for v in x[0, 32 * b:32 * b + 32]]
        top = max(abs(v) for v in block)
        n = -127
        if top:
            n = 0
            while Fraction(2) ** (n + 3) <= top:
                n += 1
            while Fraction(2) ** (n + 2) > top:
                n -= 1
        assert e[0, b] == n + 127
        for j, v in enumerate(block):
            u = abs(v) / Fraction(2) ** n
            best = min(range(8), key=lambda c: (abs(u - mags[c]), c % 2))
            assert codes[0, 32 * b + j] & 7 == best and (v >= 0 or codes[0, 32 * b + j] >= 8)


def test_definition_of_values():
    codes = np.tile(np.arange(16, dtype=np.uint8), 2)[None]
    for e in (0, 1, 127, 130, 254):
        v = mx.values(codes, np.array([[e]], dtype=np.uint8))[0]
        assert list(v[:8]) == [m * 2.0 ** (e - 127) for m in (0, .5, 1, 1.5, 2, 3, 4, 6)] and np.array_equal(v[8:16], -v[:8])
    assert np.isnan(mx.values(codes, np.array([[255]], dtype=np.uint8))).all()


# ---------------------------------------------------------------------------------------------------- host
@pytest.mark.parametrize("N,K", [(16, 128), (16, 512), (48, 640), (32, 1152), (160, 2048)])
def test_pack_is_the_specified_order_and_its_inverse(lutq, N, K):
    rng = np.random.default_rng(N + K)
    codes, e = rng.integers(0, 16, (N, K), dtype=np.uint8), rng.integers(0, 256, (N, K // 32), dtype=np.uint8)
    p = lutq.lutq_mx4_pack(mx.row_bytes(codes), e)
    assert np.array_equal(p, mx.pack(codes, e)) and p.size == lutq.lutq_mx4_packed_bytes(N, K)
    c2, e2 = lutq.lutq_mx4_unpack(p, N, K)
    assert np.array_equal(c2, mx.row_bytes(codes)) and np.array_equal(e2, e)


def test_sizes_outside_the_domain(lutq):
    for N, K in ((0, 128), (16, 0), (8, 128), (16, 64), (16, 192), (24, 128), (-16, 128), (16, -128), ((1 << 24) + 16, 128), (16, (1 << 24) + 128)):
        assert lutq.lutq_mx4_packed_bytes(N, K) == 0 and lutq.lutq_mx4_workspace_bytes(1, N, K, 1) == 0
    assert lutq.lutq_mx4_workspace_bytes(1 << 30, 16, 128, 1) == 0 and lutq.lutq_mx4_workspace_bytes(-1, 16, 128, 1) == 0
    assert lutq.lutq_mx4_workspace_bytes(4, 16, 128, 0) == 0 and lutq.lutq_mx4_workspace_bytes(4, 16, 128, 65537) == 0
    assert lutq.lutq_mx4_workspace_bytes(0, 16, 128, 1) >= 65536 and lutq.lutq_mx4_workspace_bytes(4, 16, 128, 65536) > 0
    for bad in ((np.zeros((16, 64)), np.zeros((16, 3))), (np.zeros((16, 64)), np.zeros((15, 4))), (np.zeros(64), np.zeros(4))):
        with pytest.raises(ValueError):
            lutq.lutq_mx4_pack(*bad)
    with pytest.raises(lutq.LutqError):
        lutq.lutq_mx4_pack(np.zeros((8, 64)), np.zeros((8, 4)))
    with pytest.raises(ValueError):
        lutq.lutq_mx4_unpack(np.zeros(10), 16, 128)


def test_refusals_before_any_launch(lutq):
    """Every one of these returns from host-side validation; no device call is made."""
    lib = lutq.load_library()
    buf = (ctypes.c_char * 4096)()
    a = (ctypes.addressof(buf) + 15) & ~15
    NULL, SHAPE, ALIGN, WORKSPACE, DTYPE = 1, 4, 5, 7, 8
    q = lambda X=a, f=0, dt=0, src=4, rows=None, M=4, K=128, c=a, e=a: lib.lutq_mx4_quantize(X, f, dt, src, rows, M, K, c, e, None)
    assert q(X=None) == q(c=None) == q(e=None) == NULL
    assert q(M=-1) == q(K=64) == q(K=0) == q(src=3) == q(M=1 << 30, src=1 << 30) == q(src=-1, rows=a) == q(src=1 << 31, rows=a) == SHAPE
    assert q(dt=2) == DTYPE and q(X=a + 8) == q(c=a + 4) == q(e=a + 1) == q(rows=a + 2) == ALIGN
    assert q(M=0, src=0, X=None, c=None, e=None) == 0
    qp = lambda W=a, f=0, dt=0, N=16, K=128, p=a: lib.lutq_mx4_quantize_packed(W, f, dt, N, K, p, None)
    assert qp(W=None) == qp(p=None) == NULL and qp(N=8) == qp(N=0) == qp(K=100) == SHAPE and qp(dt=-1) == DTYPE and qp(W=a + 4) == ALIGN
    d = lambda c=a, e=a, M=4, K=128, dt=0, o=a: lib.lutq_mx4_dequant(c, e, M, K, dt, o, None)
    assert d(c=None) == d(e=None) == d(o=None) == NULL and d(K=32) == d(M=-4) == SHAPE and d(dt=7) == DTYPE and d(o=a + 2) == ALIGN
    assert d(M=0, c=None) == 0
    dp = lambda p=a, N=16, K=128, dt=0, o=a: lib.lutq_mx4_dequant_packed(p, N, K, dt, o, None)
    assert dp(p=None) == dp(o=None) == NULL and dp(N=15) == SHAPE and dp(dt=2) == DTYPE and dp(p=a + 8) == ALIGN
    need = lutq.lutq_mx4_workspace_bytes(4, 16, 128)
    m = lambda X=a, e=a, p=a, M=4, N=16, K=128, dt=0, Y=a, ws=a, wb=need: lib.lutq_mx4_matmul(X, e, p, M, N, K, dt, Y, ws, wb, None)
    g = lambda X=a, e=a, p=a, off=a, E=2, M=4, N=16, K=128, dt=0, Y=a, ws=a, wb=1 << 40: \
        lib.lutq_mx4_matmul_grouped(X, e, p, off, E, M, N, K, dt, Y, ws, wb, None)
    for f in (m, g):
        assert f(X=None) == f(p=None) == f(Y=None) == NULL
        assert f(M=-1) == f(N=8) == f(N=0) == f(K=64) == f(M=1 << 30) == SHAPE and f(dt=2) == DTYPE
        assert f(X=a + 8) == f(e=a + 2) == f(p=a + 4) == f(Y=a + 2) == f(ws=a + 1) == ALIGN
        assert f(ws=None) == f(wb=0) == WORKSPACE
        assert f(M=0, X=None, e=None, Y=None, ws=None) == 0
    assert m(wb=need - 1) == WORKSPACE
    assert g(off=None) == NULL and g(E=0) == g(E=65537) == SHAPE and g(off=a + 2) == ALIGN
    assert g(M=0, off=None) == 0


def test_binding_refuses_host_tensors(lutq):
    import torch
    x, u = torch.zeros((4, 128), dtype=torch.float16), torch.zeros((4, 64), dtype=torch.uint8)
    e, o = torch.zeros((4, 4), dtype=torch.uint8), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: lutq.lutq_mx4_quantize(x, u, e), lambda: lutq.lutq_mx4_quantize_packed(x, u), lambda: lutq.lutq_mx4_dequant(u, e, x),
                 lambda: lutq.lutq_mx4_dequant_packed(u, x), lambda: lutq.lutq_mx4_matmul(u, u, x, u, x_scales=e),
                 lambda: lutq.lutq_mx4_matmul_grouped(u, u, o, x, u, x_scales=e)):
        with pytest.raises(ValueError, match="CUDA"):
            call()
    nat = lutq.binding._native()
    assert nat.mx4_quantize(x, u, e, None) == -1 and nat.mx4_quantize(x) == -1
    assert nat.mx4_dequant(u, e, x) == -1 and nat.mx4_mm(u, e, u, None, x, u) == -1 and nat.mx4_mm(u, e, u, o, x, "u") == -1


# ---------------------------------------------------------------------------------------------------- device: quantiser
def source_type(src):
    import torch
    return torch.float32 if src == "f32" else torch_dtype(src)


def edge_values(src, M, K, seed):
    """Values over the type's whole range, block by block: ordinary ones, ties, one magnitude only, the smallest and the
    largest numbers, zeros of either sign, blocks with an infinity or a NaN."""
    import torch
    rng = np.random.default_rng(seed)
    lo, hi = {"f32": (-149, 127), "bf16": (-133, 127), "f16": (-24, 15)}[src]
    x = rng.standard_normal((M, K // 32, 32))
    kind = rng.integers(0, 8, (M, K // 32))
    top = rng.integers(lo, hi, (M, K // 32)).astype(np.float64)
    grid = np.array([0, .25, .5, .75, 1, 1.25, 1.5, 1.75, 2, 2.5, 3, 3.5, 4, 5, 6, 7, 7.9])
    with np.errstate(over="ignore"):
        x = np.where((kind == 1)[..., None], rng.choice(grid, x.shape) * rng.choice([-1, 1], x.shape) * np.exp2(np.minimum(top - 2, hi - 3))[..., None], x)
        x = np.where((kind == 2)[..., None], x * np.exp2(np.minimum(top, hi - 3))[..., None], x)
        x = np.where((kind == 3)[..., None], rng.integers(-6, 7, x.shape) * 2.0 ** lo, x)
    x = np.where((kind == 4)[..., None], np.where(rng.random(x.shape) < 0.5, 0.0, -0.0), x)
    big = {"f32": 3.4028234663852886e38, "bf16": 3.3895313892515355e38, "f16": 65504.0}[src]
    x = np.where((kind == 5)[..., None], rng.choice([big, -big, 1.0, big / 2], x.shape), x)
    x[..., 7] = np.where(kind == 6, rng.choice([np.inf, -np.inf, np.nan], kind.shape), x[..., 7])
    x = x.reshape(M, K)
    return torch.from_numpy(x).to(source_type(src))


def as_f64(t):
    return t.double().cpu().numpy()


def to_gpu(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K", [(1, 128), (1, 4096), (3, 384), (17, 2176), (129, 640), (300, 16384)])
def test_quantize_rows(lutq, src, M, K):
    import torch
    x = edge_values(src, M, K, M * 7 + K)
    codes, e = mx.quantize(as_f64(x))
    c = torch.full((M + 2, K // 2), 0xA5, dtype=torch.uint8, device="cuda")
    s = torch.full((M + 16, K // 32), 0xA5, dtype=torch.uint8, device="cuda")
    lutq.lutq_mx4_quantize(x.cuda(), c[:M], s[:M])
    torch.cuda.synchronize()
    assert np.array_equal(s[:M].cpu().numpy(), e) and np.array_equal(c[:M].cpu().numpy(), mx.row_bytes(codes))
    assert (c[M:] == 0xA5).all().item() and (s[M:] == 0xA5).all().item()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
def test_quantize_picks_rows(lutq, src):
    import torch
    K = 640
    x = edge_values(src, 50, K, 3)
    codes, e = mx.quantize(as_f64(x))
    rng = np.random.default_rng(1)
    rows = rng.integers(0, 50, 777).astype(np.int32)
    rows[::13], rows[5], rows[6], rows[7] = -1, 50, 2 ** 31 - 1, -2 ** 31
    ok = (rows >= 0) & (rows < 50)
    want_c = np.where(ok[:, None], mx.row_bytes(codes)[np.where(ok, rows, 0)], 0)
    want_e = np.where(ok[:, None], e[np.where(ok, rows, 0)], 0)
    c, s = torch.empty((777, K // 2), dtype=torch.uint8, device="cuda"), torch.empty((777, K // 32), dtype=torch.uint8, device="cuda")
    lutq.lutq_mx4_quantize(x.cuda(), c, s, rows=to_gpu(rows))
    assert np.array_equal(c.cpu().numpy(), want_c) and np.array_equal(s.cpu().numpy(), want_e)
    lutq.lutq_mx4_quantize(x.cuda()[:0], c, s, rows=to_gpu(rows))          # a source without rows: every number is outside
    assert not c.any().item() and not s.any().item()
    lutq.lutq_mx4_quantize(x.cuda(), c[:0], s[:0], rows=to_gpu(rows)[:0])
    lutq.lutq_mx4_quantize(x.cuda()[:0], c[:0], s[:0])


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("N,K", [(16, 128), (48, 512), (32, 1664), (4112, 256)])
def test_quantize_packed(lutq, src, N, K):
    import torch
    x = edge_values(src, N, K, N + K)
    n = lutq.lutq_mx4_packed_bytes(N, K)
    p = torch.full((n + 256,), 0xA5, dtype=torch.uint8, device="cuda")
    lutq.lutq_mx4_quantize_packed(x.cuda(), p[:n])
    assert np.array_equal(p[:n].cpu().numpy(), mx.pack(*mx.quantize(as_f64(x)))) and (p[n:] == 0xA5).all().item()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("M,K", [(16, 128), (48, 640), (1040, 4096)])
def test_dequant_both_forms(lutq, dtype, M, K):
    import torch
    rng = np.random.default_rng(M)
    codes, e = rng.integers(0, 16, (M, K), dtype=np.uint8), rng.integers(0, 256, (M, K // 32), dtype=np.uint8)
    with np.errstate(over="ignore"):
        want = torch.from_numpy(mx.values(codes, e).astype(np.float32)).to(torch_dtype(dtype))      # (fp32 holds every value, or is infinite too)
    out = torch.full((M, K), 7.0, dtype=torch_dtype(dtype), device="cuda")
    lutq.lutq_mx4_dequant(to_gpu(mx.row_bytes(codes)), to_gpu(e), out)
    assert torch.equal(torch.nan_to_num(out.cpu(), nan=12.0), torch.nan_to_num(want, nan=12.0)) and torch.equal(out.cpu().isnan(), want.isnan())
    again = torch.full_like(out, 7.0)
    lutq.lutq_mx4_dequant_packed(to_gpu(mx.pack(codes, e)), again)
    assert torch.equal(again.view(torch.int16), out.view(torch.int16))
    lutq.lutq_mx4_dequant(to_gpu(mx.row_bytes(codes))[:0], to_gpu(e)[:0], out[:0])


@pytest.mark.gpu
def test_offsets_beyond_32_bits(lutq):
    """More than 2^32 bytes of source and 2^31 values: the last rows are what a small call makes of them, in every kernel."""
    import torch
    M, K = 70000, 32768
    x = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda")
    tail = torch.randn((48, K), device="cuda").to(torch.bfloat16)
    x[-48:] = tail
    c, s = torch.empty((M, K // 2), dtype=torch.uint8, device="cuda"), torch.empty((M, K // 32), dtype=torch.uint8, device="cuda")
    lutq.lutq_mx4_quantize(x, c, s)
    c2, s2 = torch.empty_like(c[:48]), torch.empty_like(s[:48])
    lutq.lutq_mx4_quantize(tail, c2, s2)
    assert torch.equal(c[-48:], c2) and torch.equal(s[-48:], s2) and not c[:-48].any().item()
    rows = torch.arange(M - 48, M, dtype=torch.int32, device="cuda")
    c3, s3 = torch.empty_like(c2), torch.empty_like(s2)
    lutq.lutq_mx4_quantize(x, c3, s3, rows=rows)
    assert torch.equal(c3, c2) and torch.equal(s3, s2)
    back, want = torch.empty_like(x), torch.empty_like(tail)
    lutq.lutq_mx4_dequant(c, s, back)
    lutq.lutq_mx4_dequant(c2, s2, want)
    assert torch.equal(back[-48:], want)
    p = torch.empty(lutq.lutq_mx4_packed_bytes(M, K), dtype=torch.uint8, device="cuda")
    p2 = torch.empty(lutq.lutq_mx4_packed_bytes(48, K), dtype=torch.uint8, device="cuda")
    lutq.lutq_mx4_quantize_packed(x, p)
    lutq.lutq_mx4_quantize_packed(tail, p2)
    assert torch.equal(p[-p2.numel():], p2)
    back.zero_()
    lutq.lutq_mx4_dequant_packed(p, back)
    assert torch.equal(back[-48:], want)
    # the same rows as weights and as activations of a product
    y = torch.empty((M, 16), dtype=torch.bfloat16, device="cuda")
    ws = lutq.new_mx4_workspace(M, 16, K)
    w = p2[:lutq.lutq_mx4_packed_bytes(16, K)]
    lutq.lutq_mx4_matmul(c, w, y, ws, x_scales=s)
    a, b = as_f64(want), as_f64(want[:16])
    assert (np.abs(as_f64(y[-48:]) - a @ b.T) <= off_by_at_most(None, mx.product(a, b), K, "bf16")).all() and not y[:-48].any().item()


# ---------------------------------------------------------------------------------------------------- device: products
class Problem:
    """Quantised factors on the device and their values in fp64.  Exponents differ from block to block."""

    def __init__(self, lutq, M, N, K, dtype, experts=1, seed=0):
        import torch
        rng = np.random.default_rng(seed + M * 3 + N * 5 + K * 7)
        self.M, self.N, self.K, self.dtype, self.experts = M, N, K, dtype, experts
        x = rng.standard_normal((M, K)) * np.repeat(np.exp2(rng.integers(-3, 3, (M, K // 32))), 32, 1)
        self.X = torch.from_numpy(x).to(torch_dtype(dtype)).cuda()
        codes, e = mx.quantize(as_f64(self.X))
        self.x = mx.values(codes, e)
        self.codes, self.e = to_gpu(mx.row_bytes(codes)), to_gpu(e)
        wc = rng.integers(0, 16, (experts * N, K), dtype=np.uint8)
        we = rng.integers(115, 123, (experts * N, K // 32), dtype=np.uint8)
        self.w = mx.values(wc, we).reshape(experts, N, K)
        self.packed = to_gpu(lutq.lutq_mx4_pack(mx.row_bytes(wc), we)).reshape(experts, -1)
        self.ws = lutq.new_mx4_workspace(M, N, K, experts)

    def out(self):
        """Y with guard rows before and behind it."""
        import torch
        self.guarded = torch.full((self.M + 32, self.N), -7.0, dtype=torch_dtype(self.dtype), device="cuda")
        return self.guarded[16:16 + self.M]

    def guards_hold(self):
        return (self.guarded[:16] == -7.0).all().item() and (self.guarded[16 + self.M:] == -7.0).all().item()

    def args(self, dense):
        return (self.X, None) if dense else (self.codes, self.e)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 16, 128), (1, 48, 4096), (2, 272, 640), (7, 4112, 512), (15, 64, 1152), (16, 96, 2048), (17, 160, 384),
                                   (32, 32, 5120), (33, 304, 1024), (63, 16, 768), (64, 528, 512), (65, 80, 896), (100, 256, 14336), (128, 1040, 1152),
                                   (129, 512, 256), (200, 304, 3200), (255, 272, 128), (257, 528, 640), (515, 1296, 1408), (1000, 16, 512),
                                   (2049, 784, 384)])
def test_product(lutq, M, N, K, dense, dtype):
    p = Problem(lutq, M, N, K, dtype)
    x, e = p.args(dense)
    y = p.out()
    lutq.lutq_mx4_matmul(x, p.packed, y, p.ws, x_scales=e)
    got, sums = as_f64(y), mx.product(p.x, p.w[0])
    worst = np.max(np.abs(got - sums[0]) / off_by_at_most(got, sums, K, dtype))
    assert worst <= 1.0, worst
    assert p.guards_hold() and not p.ws[:65536].any().item()
    again = p.out()
    lutq.lutq_mx4_matmul(x, p.packed, again, p.ws, x_scales=e)
    assert np.array_equal(as_f64(again), got)


# (each shape of tiles, with ragged edges; the long ones with K in two to five slices)
TILED = [(103, 4112, 640), (199, 4112, 2176), (999, 2064, 1152), (1001, 4112, 1152), (2100, 4112, 1152), (130, 2064, 8320), (101, 2064, 8320),
         (601, 272, 14336), (131, 1040, 16512), (131, 2064, 14336), (67, 4112, 14336), (131, 4112, 14336), (200, 4112, 8320), (259, 4112, 14336),
         (601, 1072, 1152), (300, 2064, 1664), (2100, 4112, 2176), (3001, 4112, 1152)]


@pytest.mark.gpu
@pytest.mark.parametrize("case", range(len(TILED)))
def test_product_of_many_rows(lutq, case):
    import torch
    M, N, K = TILED[case]
    dtype = DTYPES[case % 2]
    p = Problem(lutq, M, N, K, dtype)
    y = p.out()
    lutq.lutq_mx4_matmul(p.codes, p.packed, y, p.ws, x_scales=p.e)
    got, sums = as_f64(y), mx.product(p.x, p.w[0])
    worst = np.max(np.abs(got - sums[0]) / off_by_at_most(got, sums, K, dtype))
    assert worst <= 1.0, worst
    assert p.guards_hold() and not p.ws[:65536].any().item()
    # the same bits again, from values, and when replayed
    static = torch.empty_like(y)
    graph = torch.cuda.CUDAGraph()
    lutq.lutq_mx4_matmul(p.X, p.packed, static, p.ws)
    assert torch.equal(static, y)
    with torch.cuda.graph(graph):
        lutq.lutq_mx4_matmul(p.X, p.packed, static, p.ws)
    for _ in range(3):
        static.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(static, y)
    assert not p.ws[:65536].any().item()


def counts_to_offsets(counts, first=0):
    return np.concatenate([[first], first + np.cumsum(counts)]).astype(np.int32)


def grouped_reference(p, off):
    ref, mag = np.full((p.M, p.N), -7.0), np.zeros((p.M, p.N))
    for g in range(p.experts):
        a, b = int(off[g]), int(off[g + 1])
        if b > a:
            ref[a:b], mag[a:b] = mx.product(p.x[a:b], p.w[g])
    return ref, mag


GROUPS = {
    "one_expert": ([37], 0, 0), "one_row_each": ([1] * 9, 0, 0), "none_have_rows": ([0, 0, 0], 0, 5), "last_only": ([0, 0, 0, 20], 0, 0),
    "first_only": ([300, 0, 0], 0, 3), "ragged": ([3, 0, 17, 16, 1, 0, 64, 33], 2, 7), "many_experts": ([0, 1, 2, 0] * 35, 0, 1),
    "few_rows_many_experts": ([0] * 70 + [3] + [0] * 80 + [2] + [0] * 49, 0, 0), "large": ([520, 0, 129, 257, 1], 1, 30),
    "sixty_four": ([2] * 64, 0, 0), "sixty_five": ([17] * 65, 0, 0),
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
    x, e = p.args(dense)
    y = p.out()
    y.fill_(-7.0)
    lutq.lutq_mx4_matmul_grouped(x, p.packed, to_gpu(off), y, p.ws, x_scales=e)
    got, sums = as_f64(y), grouped_reference(p, off)
    worst = np.max(np.abs(got - sums[0]) / off_by_at_most(got, sums, K, dtype))
    assert worst <= 1.0, worst
    assert p.guards_hold() and not p.ws[:65536].any().item()


# (few rows per expert on average, and several in one of them; few and many workgroups of the streaming kernel)
UNEVEN = [([9] + [0] * 11, 48, 640), ([2, 0, 13, 1, 0, 0], 48, 1152), ([11] + [0] * 14 + [4], 1296, 640), ([13, 3] + [2] * 14, 1296, 512),
          ([1, 0, 16, 0] * 6, 2768, 512), ([2, 5, 0, 16] * 16, 1040, 640), ([17, 33, 0, 5] * 16, 1040, 384)]


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("case", range(len(UNEVEN)))
def test_product_by_expert_of_uneven_rows(lutq, case, dense):
    counts, N, K = UNEVEN[case]
    off = counts_to_offsets(counts, 1)
    p = Problem(lutq, int(off[-1]) + 2, N, K, "f16", experts=len(counts), seed=case)
    x, e = p.args(dense)
    y = p.out()
    lutq.lutq_mx4_matmul_grouped(x, p.packed, to_gpu(off), y, p.ws, x_scales=e)
    got, sums = as_f64(y), grouped_reference(p, off)
    worst = np.max(np.abs(got - sums[0]) / off_by_at_most(got, sums, K, "f16"))
    assert worst <= 1.0, worst
    assert p.guards_hold()


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("counts,N,K", [([0, 171, 9], 2064, 512), ([33, 0, 70, 1, 16, 0, 49, 8, 3], 2064, 2176), ([129, 255, 10, 256, 0], 4112, 512),
                                        ([2000, 0, 17, 900, 3000, 1, 128, 129, 1925], 272, 1152), ([1111, 2, 0, 3100, 287], 2064, 640),
                                        # (with K in slices)
                                        ([140, 0, 52], 1040, 8320), ([7, 31], 4112, 14336), ([1, 199], 4112, 8320), ([0, 90, 100, 110, 0], 528, 14336),
                                        ([3, 774, 0], 1040, 640), ([900, 1, 2303, 0, 1300, 700, 2000, 255, 641], 1072, 2176)])
def test_product_by_expert_of_many_rows(lutq, counts, N, K, dense):
    off = counts_to_offsets(counts, 2)
    p = Problem(lutq, int(off[-1]) + 3, N, K, "bf16", experts=len(counts))
    x, e = p.args(dense)
    y = p.out()
    lutq.lutq_mx4_matmul_grouped(x, p.packed, to_gpu(off), y, p.ws, x_scales=e)
    got, sums = as_f64(y), grouped_reference(p, off)
    worst = np.max(np.abs(got - sums[0]) / off_by_at_most(got, sums, K, "bf16"))
    assert worst <= 1.0, worst
    assert p.guards_hold() and not p.ws[:65536].any().item()
    again = p.out()
    lutq.lutq_mx4_matmul_grouped(x, p.packed, to_gpu(off), again, p.ws, x_scales=e)
    assert np.array_equal(as_f64(again), got)


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [6, 600])
def test_offsets_outside_their_documented_range_stay_in_bounds(lutq, rows):
    """Such offsets are read as the nearest row number inside; rows of experts whose own range is sound are right, nothing outside is written."""
    p = Problem(lutq, rows, 48, 256, "bf16", experts=4)
    h = rows // 2
    for off, sound in (([-5, h, h, rows, rows + 900], [(0, 0, h), (2, h, rows)]), ([0, rows + 7, 2 ** 31 - 1, -2 ** 31, rows], []),
                       ([h, 0, h, h, rows], [(1, 0, h), (3, h, rows)])):
        y = p.out()
        lutq.lutq_mx4_matmul_grouped(p.codes, p.packed, to_gpu(np.array(off, dtype=np.int32)), y, p.ws, x_scales=p.e)
        got = as_f64(y)
        for g, a, b in sound:
            sums = mx.product(p.x[a:b], p.w[g])
            assert (np.abs(got[a:b] - sums[0]) <= off_by_at_most(got, sums, 256, "bf16")).all()
        assert p.guards_hold()


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("M", [3, 40, 300])
def test_not_a_number_stays_in_its_row(lutq, M, dense):
    """A block that is not a number makes its own row of Y (activations) or its own column (weights) not a number, and no other."""
    import torch
    p = Problem(lutq, M, 64, 640, "f16")
    X, e = p.X.clone(), p.e.clone()
    X[M - 1, 333] = float("inf")
    e[M - 1, 333 // 32] = 255
    packed = p.packed.clone()
    packed[0, 5 * 1024 + 4 * 9] = 255                                   # row 9 of the first row block, first tile, first block
    y = p.out()
    lutq.lutq_mx4_matmul(X if dense else p.codes, packed, y, p.ws, x_scales=None if dense else e)
    nan = torch.isnan(y).cpu().numpy()
    want = np.zeros((M, 64), dtype=bool)
    want[M - 1], want[:, 9] = True, True
    assert np.array_equal(nan, want) and p.guards_hold()


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("M,N,K", [(103, 4112, 640), (199, 4112, 2176), (999, 2064, 1152), (1001, 4112, 1152), (2100, 4112, 1152), (101, 2064, 8320),
                                   (601, 1072, 1152), (2100, 4112, 2176), (130, 2064, 8320)])
def test_not_a_number_among_many_rows(lutq, M, N, K, dense):
    import torch
    p = Problem(lutq, M, N, K, "bf16")
    rows, columns = [0, M // 2, M - 1], [5, N - 16]
    X, e, packed = p.X.clone(), p.e.clone(), p.packed.clone()
    record = lutq.lutq_mx4_packed_bytes(16, K)
    for r, k in zip(rows, (0, K // 2 + 7, K - 1)):
        X[r, k] = float("nan")
        e[r, k // 32] = 255
    for n, o in zip(columns, (0, 3)):                                   # (a block of the first tile)
        packed[0, n // 16 * record + K // 128 * 1024 + 4 * (16 * o + n % 16)] = 255
    y = p.out()
    lutq.lutq_mx4_matmul(X if dense else p.codes, packed, y, p.ws, x_scales=None if dense else e)
    want = torch.zeros((M, N), dtype=torch.bool)
    want[rows], want[:, columns] = True, True
    assert torch.equal(torch.isnan(y).cpu(), want) and p.guards_hold()


@pytest.mark.gpu
@pytest.mark.parametrize("N,K", [(4112, 512), (48, 640)])
def test_offsets_that_claim_rows_twice(lutq, N, K):
    """Decreasing offsets and such that several experts claim the same rows: each value there is one claimant's (column tiles
    are written by different workgroups, so a row may hold several's), and nothing outside is written."""
    p = Problem(lutq, 650, N, K, "bf16", experts=5)
    all_sums = [mx.product(p.x, p.w[g]) for g in range(5)]
    for off in ([0, 650, 0, 650, 0, 650], [-9, 700, 100, 400, 390, 2 ** 31 - 1], [650, 600, 20, 20, 0, 3]):
        y = p.out()
        lutq.lutq_mx4_matmul_grouped(p.codes, p.packed, to_gpu(np.array(off, dtype=np.int32)), y, p.ws, x_scales=p.e)
        got = as_f64(y)
        fits = got == -7.0
        claimed = np.zeros(650, dtype=bool)
        for g in range(5):
            a, b = min(max(off[g], 0), 650), min(max(off[g + 1], 0), 650)
            claimed[a:b] = True
            if b > a:
                fits[a:b] |= (np.abs(got[a:b] - all_sums[g][0][a:b]) <= off_by_at_most(got[a:b], tuple(s[a:b] for s in all_sums[g]), K, "bf16"))
        assert fits.all() and (got[~claimed] == -7.0).all() and p.guards_hold()


@pytest.mark.gpu
def test_sums_beyond_the_type_become_infinite(lutq):
    p = Problem(lutq, 20, 32, 256, "f16")
    e = p.e.clone()
    e[3] += 20
    y = p.out()
    lutq.lutq_mx4_matmul(p.codes, p.packed, y, p.ws, x_scales=e)
    got, ref = as_f64(y), p.x @ p.w[0].T
    ref[3] *= 2.0 ** 20
    clear = np.abs(np.abs(ref) - 65520.0) > 100
    assert np.array_equal(np.isinf(got)[clear], (np.abs(ref) > 65520.0)[clear]) and np.isinf(got).any()


@pytest.mark.gpu
def test_expert_layer_as_it_is_used(lutq):
    """Tokens are sent to two of five experts each, padding among the places: quantised by index, through both products of the
    experts (16-bit values between them), and summed back."""
    import torch
    tokens, E, D, H, dtype = 90, 5, 512, 384, "bf16"
    p1, p2 = Problem(lutq, tokens, H, D, dtype, experts=E), Problem(lutq, 16, D, H, dtype, experts=E, seed=4)
    rng = np.random.default_rng(8)
    expert = np.stack([rng.choice(E - 1, 2, replace=False) for _ in range(tokens)]).reshape(-1)      # (the last expert stays idle)
    order = np.argsort(expert, kind="stable")
    off = counts_to_offsets(np.bincount(expert, minlength=E))
    rows = np.concatenate([order // 2, [-1] * 6]).astype(np.int32)
    T = rows.size
    codes, e = torch.empty((T, D // 2), dtype=torch.uint8, device="cuda"), torch.empty((T, D // 32), dtype=torch.uint8, device="cuda")
    mid = torch.zeros((T, H), dtype=torch_dtype(dtype), device="cuda")
    out = torch.zeros((T, D), dtype=torch_dtype(dtype), device="cuda")
    ws = torch.zeros(max(lutq.lutq_mx4_workspace_bytes(T, H, D, E), lutq.lutq_mx4_workspace_bytes(T, D, H, E)), dtype=torch.uint8, device="cuda")
    offsets = to_gpu(off)

    def layer():
        lutq.lutq_mx4_quantize(p1.X, codes, e, rows=to_gpu_rows)
        lutq.lutq_mx4_matmul_grouped(codes, p1.packed, offsets, mid, ws, x_scales=e)
        lutq.lutq_mx4_matmul_grouped(mid, p2.packed, offsets, out, ws)
        return out

    to_gpu_rows = to_gpu(rows)
    layer()
    got_mid, got = as_f64(mid), as_f64(out)
    x = p1.x[order // 2]
    h = mx.values(*mx.quantize(got_mid[:2 * tokens]))
    for g in range(E):
        a, b = off[g], off[g + 1]
        s1, s2 = mx.product(x[a:b], p1.w[g]), mx.product(h[a:b], p2.w[g])
        assert (np.abs(got_mid[a:b] - s1[0]) <= off_by_at_most(None, s1, D, dtype)).all()
        assert (np.abs(got[a:b] - s2[0]) <= off_by_at_most(None, s2, H, dtype)).all()
    assert not got[2 * tokens:].any()
    # captured once and replayed with other tokens and other loads, eager work between the replays
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        layer()
    for seed in range(4):
        expert = np.random.default_rng(seed).integers(0, E, 2 * tokens)
        offsets.copy_(to_gpu(counts_to_offsets(np.bincount(expert, minlength=E))))
        p1.X.copy_(torch.randn(p1.X.shape, generator=torch.Generator().manual_seed(seed)).to(p1.X.dtype))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        replayed = out.clone()
        out.zero_()
        layer()
        torch.cuda.synchronize()
        assert torch.equal(replayed, out) and not ws[:65536].any().item()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 40, 600])
def test_streams_and_shared_python_path(lutq, monkeypatch, M):
    """On a stream that is given, on the current one (whose queued work comes first), and without the binding's native part:
    the same bits."""
    import torch
    p = Problem(lutq, M, 272, 640, "bf16")
    want = p.out().clone()
    lutq.lutq_mx4_matmul(p.X, p.packed, want, p.ws)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    y = p.out()
    torch.cuda.synchronize()
    lutq.lutq_mx4_matmul(p.X, p.packed, y, p.ws, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    X = torch.zeros_like(p.X)
    y = p.out()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(2000000)
        X.copy_(p.X)
        lutq.lutq_mx4_matmul(X, p.packed, y, p.ws)
    side.synchronize()
    assert torch.equal(y, want)
    c, e, o = torch.empty_like(p.codes), torch.empty_like(p.e), torch.empty_like(p.X)
    for _ in range(2):                                  # with and without the native part
        lutq.lutq_mx4_quantize(p.X, c, e)
        assert torch.equal(c, p.codes) and torch.equal(e, p.e)
        lutq.lutq_mx4_dequant(c, e, o)
        assert np.array_equal(as_f64(o), p.x)
        y = p.out()
        lutq.lutq_mx4_matmul(p.X, p.packed, y, p.ws)
        assert torch.equal(y, want)
        y = p.out()
        lutq.lutq_mx4_matmul_grouped(p.X, p.packed, to_gpu(np.array([0, M], dtype=np.int32)), y, p.ws)
        assert np.array_equal(np.isnan(as_f64(y)), np.isnan(as_f64(want))) and p.guards_hold()
        monkeypatch.setattr(lutq.binding, "_NATIVE", lutq.binding._NoNative)


@pytest.mark.gpu
def test_a_long_axis(lutq):
    p = Problem(lutq, 19, 16, 1 << 20, "bf16")
    for dense in (False, True):
        x, e = p.args(dense)
        y = p.out()
        lutq.lutq_mx4_matmul(x, p.packed, y, p.ws, x_scales=e)
        got, sums = as_f64(y), mx.product(p.x, p.w[0])
        assert (np.abs(got - sums[0]) <= off_by_at_most(got, sums, p.K, "bf16")).all() and p.guards_hold()


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
def test_weights_larger_than_half_the_cache(lutq, dense):
    """140 MB of them, as one matrix and, the same bytes, as fourteen experts'."""
    import torch
    N, K, experts = 57344, 4608, 14
    gen = torch.Generator(device="cuda").manual_seed(5)
    W = torch.randn((N, K), generator=gen, device="cuda", dtype=torch.bfloat16)
    packed = torch.empty(lutq.lutq_mx4_packed_bytes(N, K), dtype=torch.uint8, device="cuda")
    lutq.lutq_mx4_quantize_packed(W, packed)
    lutq.lutq_mx4_dequant_packed(packed, W)
    w = W.double()
    X = torch.randn((400, K), generator=gen, device="cuda", dtype=torch.bfloat16)
    codes, e, values = torch.empty((400, K // 2), dtype=torch.uint8, device="cuda"), torch.empty((400, K // 32), dtype=torch.uint8, device="cuda"), X.clone()
    lutq.lutq_mx4_quantize(X, codes, e)
    lutq.lutq_mx4_dequant(codes, e, values)
    x = values.double()
    for M in (1, 3, 13, 40, 100, 128):
        y = torch.full((M, N), -7.0, dtype=torch.bfloat16, device="cuda")
        lutq.lutq_mx4_matmul(X[:M] if dense else codes[:M], packed, y, lutq.new_mx4_workspace(M, N, K), x_scales=None if dense else e[:M])
        sums = as_f64(x[:M] @ w.T), as_f64(x[:M].abs() @ w.abs().T)
        assert (np.abs(as_f64(y) - sums[0]) <= off_by_at_most(as_f64(y), sums, K, "bf16")).all()
    n = N // experts
    for counts in ([1, 0, 2, 1, 1, 0, 0, 5, 1, 1, 1, 2, 3, 1], [20, 41, 0, 7, 33, 16, 17, 90, 1, 35, 64, 5, 22, 40]):
        off = counts_to_offsets(counts)
        M = int(off[-1]) + 1
        y = torch.full((M, n), -7.0, dtype=torch.bfloat16, device="cuda")
        lutq.lutq_mx4_matmul_grouped(X[:M] if dense else codes[:M], packed.view(experts, -1), to_gpu(off), y,
                                     lutq.new_mx4_workspace(M, n, K, experts), x_scales=None if dense else e[:M])
        for g in range(experts):
            a, b = int(off[g]), int(off[g + 1])
            if b > a:
                wg = w[g * n:(g + 1) * n]
                sums = as_f64(x[a:b] @ wg.T), as_f64(x[a:b].abs() @ wg.abs().T)
                assert (np.abs(as_f64(y[a:b]) - sums[0]) <= off_by_at_most(as_f64(y[a:b]), sums, K, "bf16")).all()
        assert (y[M - 1:] == -7.0).all().item()


@pytest.mark.gpu
def test_two_streams_and_two_graphs(lutq):
    """Products whose slices are joined in the workspace: at once on two streams, each with a workspace of its own; and two graphs of one
    workspace, replayed in turn."""
    import torch
    a, b = Problem(lutq, 200, 4112, 8320, "bf16"), Problem(lutq, 131, 2064, 14336, "bf16", seed=1)
    want = []
    for p in (a, b):
        y = torch.empty((p.M, p.N), dtype=torch.bfloat16, device="cuda")
        lutq.lutq_mx4_matmul(p.codes, p.packed, y, p.ws, x_scales=p.e)
        sums = mx.product(p.x, p.w[0])
        assert (np.abs(as_f64(y) - sums[0]) <= off_by_at_most(as_f64(y), sums, p.K, "bf16")).all()
        want.append(y)
    torch.cuda.synchronize()
    streams, outs = (torch.cuda.Stream(), torch.cuda.Stream()), [[torch.zeros_like(w) for _ in range(8)] for w in want]
    torch.cuda.synchronize()
    for i in range(8):
        for p, s, o in zip((a, b), streams, outs):
            lutq.lutq_mx4_matmul(p.codes, p.packed, o[i], p.ws, x_scales=p.e, stream=s)
    torch.cuda.synchronize()
    for w, o in zip(want, outs):
        assert all(torch.equal(w, y) for y in o)
    shared = lutq.new_mx4_workspace(200, 4112, 14336)
    graphs = []
    for p, o in zip((a, b), outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            lutq.lutq_mx4_matmul(p.X, p.packed, o[0], shared)
    for _ in range(4):
        for g, w, o in zip(graphs, want, outs):
            o[0].zero_()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(w, o[0])
        lutq.lutq_mx4_matmul(b.codes, b.packed, outs[1][1], shared, x_scales=b.e)
        assert torch.equal(want[1], outs[1][1])


@pytest.mark.gpu
def test_binding_refusals(lutq):
    import torch
    p = Problem(lutq, 20, 64, 256, "f16", experts=2)
    y = p.out()
    off = to_gpu(np.array([0, 10, 20], dtype=np.int32))
    mm = lambda X=p.codes, e=p.e, w=p.packed[0], Y=y, ws=p.ws: lutq.lutq_mx4_matmul(X, w, Y, ws, x_scales=e)
    gg = lambda X=p.codes, e=p.e, w=p.packed, o=off, Y=y, ws=p.ws: lutq.lutq_mx4_matmul_grouped(X, w, o, Y, ws, x_scales=e)
    for f in (mm, gg):
        for kw, err in (({"X": p.codes.cpu()}, ValueError), ({"X": p.codes.t()}, ValueError), ({"X": p.X}, TypeError), ({"e": None}, TypeError),
                        ({"X": p.X.bfloat16(), "e": None}, TypeError), ({"Y": y.float()}, TypeError), ({"Y": y[:19]}, ValueError),
                        ({"Y": y[:, :48].contiguous()}, ValueError), ({"e": p.e[:19]}, ValueError), ({"e": p.e.float()}, TypeError),
                        ({"w": p.packed[0, 16:]}, ValueError), ({"ws": p.ws[:-16]}, lutq.LutqError), ({"ws": p.ws.float()}, TypeError),
                        ({"X": p.codes[0]}, ValueError), ({"X": p.codes[:, :-16].contiguous()}, ValueError)):
            with pytest.raises(err):
                f(**kw)
    for kw, err in (({"o": off.long()}, TypeError), ({"o": off[:2]}, ValueError), ({"o": off[:1]}, ValueError), ({"o": None}, TypeError)):
        with pytest.raises(err):
            gg(**kw)
    c, e = torch.zeros_like(p.codes), torch.zeros_like(p.e)
    rows = torch.zeros(20, dtype=torch.int32, device="cuda")
    for call, err in ((lambda: lutq.lutq_mx4_quantize(p.X.double(), c, e), TypeError), (lambda: lutq.lutq_mx4_quantize(p.X, c[:19], e), ValueError),
                      (lambda: lutq.lutq_mx4_quantize(p.X, c, e, rows=rows.long()), TypeError), (lambda: lutq.lutq_mx4_quantize(p.X, c, e, rows=rows[:5]), ValueError),
                      (lambda: lutq.lutq_mx4_quantize(p.X[:, :64].contiguous(), c[:, :32].contiguous(), e[:, :2].contiguous()), lutq.LutqError),
                      (lambda: lutq.lutq_mx4_quantize(p.X[0], c, e), ValueError), (lambda: lutq.lutq_mx4_quantize(p.X.t(), c, e), ValueError),
                      (lambda: lutq.lutq_mx4_quantize_packed(p.X, c), ValueError), (lambda: lutq.lutq_mx4_dequant(c, e, p.X.float()), TypeError),
                      (lambda: lutq.lutq_mx4_dequant(c, e[:19], p.X), ValueError), (lambda: lutq.lutq_mx4_dequant_packed(c, p.X), ValueError)):
        with pytest.raises(err):
            call()
    torch.cuda.synchronize()
    assert (y == -7.0).all().item() and p.guards_hold() and not c.any().item() and not e.any().item()
