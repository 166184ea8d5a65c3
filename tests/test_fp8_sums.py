"""How the 8-bit products add up: which calls are exact but for fp32's roundings, and what the others may be off.

Launches that stream weights, and every gated call that keeps its projections or quantises H, sum the codes by the 16-bit instruction.  Tiles otherwise sum by
the 8-bit one, which cuts of eight neighbouring columns' products what lies below 2^-13 of the power of two of the largest.

The factors made for this: of each eight columns the first is 448 in both, with opposite signs in one eight and the next, and the other seven are 2 to 3.75, so
that their products, 4 to 14.1, lie below 2^-13 2^17 = 16 and are the whole of the sum.  Whoever cuts loses all of it.

Bounds as in test_fp8.py: (K / 128 + 22) 2^-22 of the magnitudes, which here are at most 16 448^2 + 112 14.1 a block of 128 columns, 3470 times the mean sum:
a sum may be off by (K / 128 + 22) / 1209 of the mean, where cutting takes all of it; K is at most 124 blocks, so that is 0.13."""
import math
import random

import numpy as np
import pytest

from gpu_util import torch_dtype
from oracle import fp8_oracle as fx
from test_fp8 import Problem, as_f64, cut_at_most, gated_off, off_by_at_most, sums_off, to_gpu, worst_of
from test_fp8_launches import CALLS, Factors
from test_mx4_launches import uneven

EXACT = [c for c in CALLS if c[0] == "gated_saved" or c[6][6]]


def made_codes(rng, rows, K, signs):
    """[rows, K] codes: the pattern above.  `signs`: opposite ones in neighbouring eights, which of them first drawn by row; else all positive."""
    c = rng.integers(64, 72, (rows, K // 8, 8))          # 2 to 3.75
    c[..., 0] = 126
    if signs:
        first = rng.integers(0, 2, (rows, K // 16))
        c[:, 0::2, 0] += 128 * first
        c[:, 1::2, 0] += 128 * (1 - first)
    return c.reshape(rows, K).astype(np.uint8)


def cut(x, w):
    """X W^T of one block of columns as the 8-bit instruction adds: each product without what lies below 2^-13 of the power of two of the largest of its eight."""
    p = x[:, None, :] * w[None, :, :]
    p = p.reshape(*p.shape[:2], -1, 8)
    unit = np.exp2(np.frexp(np.abs(p).max(-1, keepdims=True))[1] - 1 - 13)
    return (np.trunc(p / unit) * unit).sum((-1, -2))


def test_the_factors_show_a_cut():
    """With the cut the bounds of exact sums are passed eight times and more at every K there is; without it the pattern's sums are the small products'."""
    rng = np.random.default_rng(1)
    for K in sorted({c[3] for c in EXACT}):
        x, w = fx.TABLE[made_codes(rng, 3, K, True)], fx.TABLE[made_codes(rng, 5, K, False)]
        ref, mag = fx.product(x, w)
        small = (np.delete(x.reshape(3, -1, 8), 0, -1).reshape(3, -1) @ np.delete(w.reshape(5, -1, 8), 0, -1).reshape(5, -1).T)
        assert np.array_equal(ref, small) and (ref > 0).all()
        got = cut(x, w)
        half = {d: 0.5 * 2.0 ** -e * ref for d, e in (("f16", 10), ("bf16", 7))}
        for dtype in half:
            assert (np.abs(got - ref) >= 7 * (sums_off(mag, K) + half[dtype])).all(), (K, dtype)
    assert max(c[3] for c in EXACT) // 128 <= 124


def test_every_launch_with_exact_sums_is_among_them():
    """Every exact tile, whole and in slices, without experts and with them, and the streamed launches of either form."""
    shapes = {(c[0], bool(c[4]), c[6][1], c[6][2], c[6][5] > 1) for c in EXACT if not c[6][6]}
    for experts in (False, True):
        assert {s[2:] for s in shapes if s[1] == experts} >= {(256, 128, False), *(t + (z,) for t in ((128, 128), (128, 64), (64, 64)) for z in (False, True))}
        for form in ("matmul", "gated", "gated_saved"):
            assert {c[6][6] for c in EXACT if c[0] == form and bool(c[4]) == experts and c[6][6]} == {1, 2, 3}


def test_few_rows_are_streamed_whatever_the_sizes(lutq):
    """Up to 16 rows, by expert up to 4 for each, which are promised exact sums; 17 and more are not all."""
    rng = random.Random(3)
    some = lambda a, b: round(math.exp(rng.uniform(math.log(a), math.log(b))))
    tiles = 0
    for _ in range(20000):
        form, experts = rng.choice(("matmul", "gated", "gated_saved")), rng.choice((0, some(1, 65536)))
        M = 4 * experts + 1 if experts else 17
        N, K, codes, units = 128 * some(1, min(8000, 2 ** 28 // M)), 128 * some(1, min(8000, 2 ** 28 // M)), rng.random() < 0.5, some(1, 4096)
        assert lutq.calib_fp8_launch(rng.randint(1, M - 1), N, K, experts, form, codes, units).streamed
        tiles += not lutq.calib_fp8_launch(M, N, K, experts, form, codes, units).streamed
    assert tiles


class Made(Factors):
    """Those factors as Factors has them."""

    def __init__(self, form, M, N, K, experts, dtype, seed):
        import torch
        rng = np.random.default_rng(seed)
        self.table = torch.from_numpy(fx.TABLE).cuda()
        self.form, self.M, self.N, self.K, self.dtype = form, M, N, K, dtype
        rows, e = 2 * N if form.startswith("gated") else N, max(1, experts)
        codes = made_codes(rng, M, K, True)
        self.codes = to_gpu(codes)
        part = made_codes(rng, min(e * rows, 4096 + 16), K, False)                   # (large weights repeat these rows)
        self.W = to_gpu(part).repeat(-(-e * rows // part.shape[0]), 1)[:e * rows].reshape(e, rows, K)
        scales = np.exp2(rng.integers(-3, 3, (K // 128, M))).astype(np.float32)
        self.s = to_gpu(scales)
        self.X = to_gpu(fx.row_values(codes, scales)).to(torch_dtype(dtype))         # (exact: five bits, 1792 at most; quantised again these codes)
        self.sw = to_gpu((np.exp2(rng.uniform(-1, 0, (e, -(-rows // 128), K // 128))) / (926 * K // 128)).astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("call", EXACT, ids=str)
def test_exact_sums(lutq, call):
    import torch
    form, M, N, K, experts, codes, launch = call
    units = torch.cuda.get_device_properties(0).multi_processor_count
    assert lutq.calib_fp8_launch(M, N, K, experts, form, bool(codes), units) == lutq.binding.Fp8Launch(*launch)
    index = CALLS.index(call)
    act, dtype = ("silu", "gelu")[index // 2 % 2], ("f16", "bf16")[index % 2]
    p = Made(form, M, N, K, experts, dtype, index)
    ws = (lutq.new_fp8_gated_workspace if form.startswith("gated") else lutq.new_fp8_workspace)(M, N, K, max(1, experts))
    offsets = uneven(M, experts, index) if experts else [0, M]
    W, sw = (p.W, p.sw) if experts else (p.W[0], p.sw[0])
    off = (torch.tensor(offsets, dtype=torch.int32, device="cuda"),) if experts else ()
    y, saved = (torch.full((M, n), -7.0, dtype=torch_dtype(dtype), device="cuda") for n in (N, 2 * N))
    x, s = p.args(bool(codes))
    if form == "matmul":
        (lutq.lutq_fp8_matmul_grouped if experts else lutq.lutq_fp8_matmul)(x, W, sw, *off, y, ws, x_scales=s)
    else:
        (lutq.lutq_fp8_gated_grouped if experts else lutq.lutq_fp8_gated)(x, W, sw, *off, y, ws, x_scales=s, activation=act,
                                                                          saved=saved if form == "gated_saved" else None)
    for g, (a, b) in enumerate(zip(offsets, offsets[1:])):
        if b > a:
            worst = p.worst_of_h(y[a:b], a, b, g, act) if form != "matmul" else p.worst_of_sums(y[a:b], a, b, g)
            assert worst <= 1.0, (g, worst)
            if form == "gated_saved":
                worst = p.worst_of_sums(saved[a:b], a, b, g)
                assert worst <= 1.0, (g, worst, "saved")


# M, N, K, whether X is codes, X's form of streaming
STREAMED = [(1, 272, 640, False, 1), (4, 1040, 2176, False, 1), (3, 304, 1152, True, 2), (8, 528, 4992, True, 2), (9, 528, 512, True, 3), (16, 272, 6784, True, 3), (40, 304, 1152, True, 3)]
# M, N, K, channels and rows of a tile
TILES = [(601, 1040, 2176, 64, 64), (777, 2640, 512, 128, 128), (716, 1360, 384, 128, 64), (1690, 2416, 256, 256, 128),
         (1514, 5392, 256, 256, 192), (200, 33520, 256, 256, 256)]


def any_codes(rng, *shape):
    """Every code that is a number."""
    c = rng.integers(0, 256, shape).astype(np.uint8)
    c[(c & 127) == 127] = 1
    return c


@pytest.mark.gpu
@pytest.mark.parametrize("call", STREAMED + TILES, ids=str)
def test_product_of_all_codes_by_launch(lutq, call):
    """Few rows within the bound of exact sums, tiles within what the instruction may cut off besides."""
    import torch
    M, N, K, streamed = *call[:3], len(call) == 5 and call[4] < 16
    codes = call[3] if streamed else True
    launch = lutq.calib_fp8_launch(M, N, K, 0, "matmul", codes, torch.cuda.get_device_properties(0).multi_processor_count)
    assert launch.streamed == call[4] if streamed else (launch.streamed, launch.channels, launch.rows) == (0, *call[3:])
    rng = np.random.default_rng(M + N)
    p = Problem(lutq, M, N, K, "f16")
    wc, xc = any_codes(rng, N, K), any_codes(rng, M, K)
    w = fx.weight_values(wc, p.sw.cpu().numpy())
    if codes:
        args, x = (to_gpu(xc), p.s), fx.row_values(xc, p.s.cpu().numpy())
    else:
        X = torch.from_numpy(rng.standard_normal((M, K))).half().cuda()
        args, x = (X, None), fx.row_values(*fx.quantize_rows(as_f64(X)))
    y, sums = p.out(), fx.product(x, w)
    lutq.lutq_fp8_matmul(args[0], to_gpu(wc), p.sw, y, p.ws, x_scales=args[1])
    bound = off_by_at_most(sums, K, "f16") + (0.0 if streamed else cut_at_most(x, w))
    assert worst_of(as_f64(y), sums[0], bound) <= 1.0 and p.guards_hold()


@pytest.mark.gpu
@pytest.mark.parametrize("M,F,K", [(536, 640, 1152), (598, 1664, 512), (275, 1664, 384), (328, 5504, 256), (1669, 2432, 256), (252, 16640, 256)])
def test_gated_tiles_of_all_codes(lutq, M, F, K):
    """The fast form within what the cut of either projection does to H, the form that keeps them without."""
    rng = np.random.default_rng(M)
    p = Problem(lutq, M, F, K, "bf16", gated=True)
    wc, xc = any_codes(rng, 2 * F, K), any_codes(rng, M, K)
    # (sums of the order of one, where the activation bends)
    sw = p.sw / 16
    x, w = fx.row_values(xc, p.s.cpu().numpy()), fx.weight_values(wc, sw.cpu().numpy())
    sums, as_sums = [fx.product(x, part) for part in (w[:F], w[F:])], (K // 128 + 22) * 2.0 ** -22
    off = [cut_at_most(x, part) / as_sums for part in (w[:F], w[F:])]
    h, kept, saved = p.out(), p.out(), p.out(N=2 * F)
    W, X = to_gpu(wc), to_gpu(xc)
    lutq.lutq_fp8_gated(X, W, sw, h, p.ws, x_scales=p.s, activation="silu")
    want, bound = gated_off(*((r, m + o) for (r, m), o in zip(sums, off)), K, "silu", "bf16")
    assert worst_of(as_f64(h), want, bound) <= 1.0
    lutq.lutq_fp8_gated(X, W, sw, kept, p.ws, x_scales=p.s, activation="silu", saved=saved)
    want, bound = gated_off(*sums, K, "silu", "bf16")
    assert worst_of(as_f64(kept), want, bound) <= 1.0
    for at, s in ((0, sums[0]), (F, sums[1])):
        assert worst_of(as_f64(saved[:, at:at + F]), s[0], off_by_at_most(s, K, "bf16")) <= 1.0


@pytest.mark.gpu
@pytest.mark.parametrize("N,K,M,channels,rows", [(64, 80, 300, 64, 64), (800, 2544, 512, 128, 128), (784, 1232, 384, 128, 64), (1680, 2416, 256, 256, 128),
                                                 (5456, 1424, 256, 256, 192), (208, 33968, 256, 256, 256)])
def test_weight_gradient_of_all_codes(lutq, N, K, M, channels, rows):
    """Within what the instruction may cut off, whose scales it applies itself; every eight rows of X and dY have one power of two each."""
    import torch
    up = -(-M // 128) * 128
    launch = lutq.calib_fp8_launch(N, K, up, 0, "weight_grad", True, torch.cuda.get_device_properties(0).multi_processor_count)
    assert (launch.channels, launch.rows) == (channels, rows)
    rng = np.random.default_rng(N)
    dyc, xc = any_codes(rng, N, up), any_codes(rng, K, up)
    ds, xs = (np.exp2(rng.integers(-12, -5, (up // 128, n))).astype(np.float32) for n in (N, K))
    dw = torch.full((N, K), -7.0, dtype=torch.bfloat16, device="cuda")
    lutq.lutq_fp8_weight_grad(to_gpu(dyc), to_gpu(ds), to_gpu(xc), to_gpu(xs), dw, lutq.new_fp8_workspace(N, K, up))
    dy, x = fx.row_values(dyc, ds), fx.row_values(xc, xs)
    sums = fx.product(dy, x)
    assert worst_of(as_f64(dw), sums[0], off_by_at_most(sums, up, "bf16") + cut_at_most(dy, x)) <= 1.0
