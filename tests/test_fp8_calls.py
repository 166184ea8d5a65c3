"""8-bit operators: runs of them as they are used, calls at the edge of what their documentation allows, and refusals of those beyond it.

Bounds as in test_fp8.py."""
import numpy as np
import pytest

from gpu_util import torch_dtype
from oracle import fp8_oracle as fx
from test_fp8 import (Problem, as_f64, as_u8, check_h_codes, codes_within, counts_to_offsets, cut_at_most, edge_values, empty, gated_off, grad_reference, half_step,
                      off_by_at_most, quantised_is_near, same_bits, sums_off, to_gpu, worst_of)


def quantised(lutq, t, columns=False):
    """(codes, scales) of rows, or of columns, by the library."""
    M, K = t.shape
    up = -(-M // 128) * 128
    codes, s = (empty(K, up), empty(up // 128, K, dtype="f32")) if columns else (empty(M, K), empty(K // 128, M, dtype="f32"))
    (lutq.lutq_fp8_quantize_columns if columns else lutq.lutq_fp8_quantize)(t, codes, s)
    return codes, s


def weights(lutq, W):
    """(codes, scales), (the transposed's) by the library."""
    N, K = W.shape
    c, s, t, ts = empty(N, K), empty(-(-N // 128), K // 128, dtype="f32"), empty(K, N), empty(K // 128, -(-N // 128), dtype="f32")
    lutq.lutq_fp8_quantize_weights(W, c, s, transposed=(t, ts))
    return (c, s), (t, ts)


def rows_of(q):
    return fx.row_values(as_u8(q[0]), q[1].cpu().numpy())


def weights_of(q):
    return fx.weight_values(as_u8(q[0]), q[1].cpu().numpy())


def product_is_right(got, x, w, dtype):
    """`got` of quantised factors' values: codes of any size, so with what the instruction cuts off."""
    sums = fx.product(x, w)
    return worst_of(as_f64(got), sums[0], off_by_at_most(sums, x.shape[1], dtype) + cut_at_most(x, w)) <= 1.0


def normal(seed, *shape, size=1.0, dtype="f32"):
    import torch
    t = torch.from_numpy(np.random.default_rng(seed).standard_normal(shape) * size)
    return t.to(torch.float32 if dtype == "f32" else torch_dtype(dtype)).cuda()


# ---------------------------------------------------------------------------------------------------- runs of them
@pytest.mark.gpu
@pytest.mark.parametrize("act,dtype", [("silu", "bf16"), ("gelu", "f16")])
@pytest.mark.parametrize("tokens,experts,D,F", [(1, 4, 256, 128), (9, 5, 384, 256), (150, 3, 256, 384), (700, 6, 128, 256)])
def test_a_layer_of_experts(lutq, tokens, experts, D, F, act, dtype):
    """Rows of tokens picked and quantised, two per token; the gated block and the down projection by expert, codes between them."""
    import torch
    rng = np.random.default_rng(tokens)
    x = normal(tokens, tokens, D, dtype=dtype)
    w1, w2 = normal(1, experts * 2 * F, D, size=D ** -0.5), normal(2, experts * D, F, size=F ** -0.5)
    (c1, s1), _ = weights(lutq, w1)
    (c2, s2), _ = weights(lutq, w2)
    c1, s1, c2, s2 = (t.unflatten(0, (experts, -1)) for t in (c1, s1, c2, s2))
    of = np.stack([rng.permutation(experts - 1)[:2] for _ in range(tokens)])            # (the last expert has no rows)
    order = np.argsort(of.ravel(), kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(of.ravel(), minlength=experts))])
    M = 2 * tokens
    codes, s = empty(M, D), empty(D // 128, M, dtype="f32")
    lutq.lutq_fp8_quantize(x, codes, s, rows=to_gpu((order // 2).astype(np.int32)))
    c, v = fx.quantize_rows(as_f64(x)[order // 2])
    assert np.array_equal(as_u8(codes), c) and same_bits(s, v)
    off = to_gpu(offsets.astype(np.int32))
    hc, hs = empty(M, F), empty(F // 128, M, dtype="f32")
    h, y = empty(M, F, dtype=dtype), empty(M, D, dtype=dtype)
    gws, ws = lutq.new_fp8_gated_workspace(M, F, D, experts), lutq.new_fp8_workspace(M, D, F, experts)
    lutq.lutq_fp8_gated_grouped(codes, c1, s1, off, hc, gws, x_scales=s, activation=act, h_scales=hs, dtype=torch_dtype(dtype))
    lutq.lutq_fp8_matmul_grouped(hc, c2, s2, off, y, ws, x_scales=hs)
    lutq.lutq_fp8_gated_grouped(codes, c1, s1, off, h, gws, x_scales=s, activation=act, saved=empty(M, 2 * F, dtype=dtype))    # (sums as exact as those)
    assert check_h_codes(hc, hs, h)
    xv, hv = fx.row_values(c, v), rows_of((hc, hs))
    for e in range(experts):
        a, b = offsets[e], offsets[e + 1]
        w = weights_of((c1[e], s1[e]))
        sums = [fx.product(xv[a:b], part) for part in (w[:F], w[F:])]
        if b > a:
            cut = [cut_at_most(xv[a:b], part) for part in (w[:F], w[F:])]
            g, u = ((r, m + k / ((D // 128 + 22) * 2.0 ** -22)) for (r, m), k in zip(sums, cut))      # (the cut among what the sums are off)
            want, bound = gated_off(g, u, D, act, dtype)
            assert worst_of(as_f64(h[a:b]), want, bound) <= 1.0
            assert product_is_right(y[a:b], hv[a:b], weights_of((c2[e], s2[e])), dtype)


def off_by_quantising(v):
    """Half a step of a code, and of the smallest numbers under a scale of at most twice the largest value over 448."""
    return 2.0 ** -4 * (1 + 2.0 ** -10) * np.abs(v) + 2.0 ** -9 * np.abs(v).max() / 448


@pytest.mark.gpu
@pytest.mark.parametrize("act,dtype", [("silu", "bf16"), ("gelu", "f16")])
@pytest.mark.parametrize("M,F,D", [(1, 128, 128), (130, 256, 384), (300, 640, 256)])
def test_a_training_step(lutq, M, F, D, act, dtype):
    """Forward and backward of a gated block: each result from what it was given, and the gradients of the loss sum(dY Y) against differences of
    it in fp64 without any quantiser, within what the quantisers may be off."""
    import torch
    x, dy = normal(3, M, D, dtype=dtype), normal(4, M, D, dtype=dtype)
    w1, w2 = normal(5, 2 * F, D, size=D ** -0.5), normal(6, D, F, size=F ** -0.5)
    (q1, t1), (q2, t2) = weights(lutq, w1), weights(lutq, w2)
    assert np.array_equal(weights_of(q1).T, weights_of(t1)) and np.array_equal(weights_of(q2).T, weights_of(t2))
    gws = lutq.new_fp8_gated_workspace(M, F, D)
    ws = lutq.new_fp8_workspace(M, max(D, F), 2 * F)
    saved, hc, hs = empty(M, 2 * F, dtype=dtype), empty(M, F), empty(F // 128, M, dtype="f32")
    lutq.lutq_fp8_gated(x, *q1, hc, gws, activation=act, h_scales=hs, saved=saved)
    h, y, dh, dx = empty(M, F, dtype=dtype), empty(M, D, dtype=dtype), empty(M, F, dtype=dtype), empty(M, D, dtype=dtype)
    lutq.lutq_fp8_matmul(hc, *q2, y, ws, x_scales=hs)
    lutq.lutq_fp8_dequant(hc, hs, h)
    qdy = quantised(lutq, dy)
    lutq.lutq_fp8_matmul(qdy[0], *t2, dh, ws, x_scales=qdy[1])
    up = -(-M // 128) * 128
    dense, rows = empty(M, 2 * F, dtype=dtype), (empty(M, 2 * F), empty(2 * F // 128, M, dtype="f32"))
    columns = (empty(2 * F, up), empty(up // 128, 2 * F, dtype="f32"))
    lutq.lutq_fp8_gated_grad(dh, saved, activation=act, dense=dense, rows=rows, columns=columns)
    lutq.lutq_fp8_matmul(rows[0], *t1, dx, ws, x_scales=rows[1])
    dw1, dw2 = empty(2 * F, D, dtype=dtype), empty(D, F, dtype=dtype)
    xc, hcc, dyc = quantised(lutq, x, True), quantised(lutq, h, True), quantised(lutq, dy, True)
    lutq.lutq_fp8_weight_grad(*columns, *xc, dw1, lutq.new_fp8_workspace(2 * F, D, up))
    lutq.lutq_fp8_weight_grad(*dyc, *hcc, dw2, lutq.new_fp8_workspace(D, F, up))

    # each from what it was given
    X, DY, S = as_f64(x), as_f64(dy), as_f64(saved)
    xv = fx.row_values(*fx.quantize_rows(X))
    sums = fx.product(xv, weights_of(q1))
    assert worst_of(S, sums[0], off_by_at_most(sums, D, dtype)) <= 1.0
    assert product_is_right(y, rows_of((hc, hs)), weights_of(q2), dtype)
    assert product_is_right(dh, rows_of(qdy), weights_of(t2), dtype)
    ref, off = grad_reference(as_f64(dh), S[:, :F], S[:, F:], act)
    assert worst_of(as_f64(dense), ref, half_step(ref, dtype) + off * (1 + 2.0 ** -8)) <= 1.0
    assert product_is_right(dx, rows_of(rows), weights_of(t1), dtype)
    for got, a, b in ((dw1, columns, xc), (dw2, dyc, hcc)):
        assert product_is_right(got, rows_of(a), rows_of(b), dtype)

    # all together
    W1, W2 = as_f64(w1), as_f64(w2)
    def loss(x, w1, w2):
        p = x @ w1.T
        return (DY * ((fx.activation(p[:, :F], act) * p[:, F:]) @ w2.T)).sum()
    eps = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    a = np.abs
    P, ex, e1, e2, ey = X @ W1.T, off_by_quantising(X), off_by_quantising(W1), off_by_quantising(W2), off_by_quantising(DY)
    # (2^-5 more: what the instruction cuts off, at most 7 2^-13 of magnitudes, of which a quantised factor is off by 2^-4)
    ep = (a(X) @ e1.T + ex @ (a(W1) + e1).T) * (1 + 2.0 ** -5)
    ep += eps * (a(P) + ep)
    g, u, eg, eu = P[:, :F], P[:, F:], ep[:, :F], ep[:, F:]
    DH = DY @ W2
    eh = (a(DY) @ e2 + ey @ (a(W2) + e2)) * (1 + 2.0 ** -5)
    eh += eps * (a(DH) + eh)
    f, slope = a(fx.activation(g, act)), a(fx.slope(g, act))
    ef = 1.13 * eg                                      # (1.13 and 0.85: the largest slope of either activation, and the largest of the slope's)
    off_h = (f + ef) * (a(u) + eu) - f * a(u)
    off_h += eps * (f * a(u) + off_h)
    DG = np.concatenate(fx.gated_gradients(DH, g, u, act), 1)
    off_dg = np.concatenate([(a(DH) + eh) * (a(u) + eu) * (slope + 0.85 * eg) - a(DH) * a(u) * slope, (a(DH) + eh) * (f + ef) - a(DH) * f], 1)
    more = lambda v, off: off + 2.0 ** -4 * (1 + 2.0 ** -10) * (a(v) + off) + 2.0 ** -9 * (a(v) + off).max() / 448     # (off, and then quantised)
    h_exact = fx.activation(g, act) * u
    q_dg, q_h = more(DG, off_dg), more(h_exact, off_h)
    q_h = more(h_exact, q_h + eps * (a(h_exact) + q_h))                        # (by rows, back to 16 bits, by columns)
    checks = [(dx, 0, X, q_dg @ (a(W1) + e1) + a(DG) @ e1), (dw1, 1, W1, q_dg.T @ (a(X) + ex) + a(DG).T @ ex), (dw2, 2, W2, ey.T @ (a(h_exact) + q_h) + a(DY).T @ q_h)]
    rng, t = np.random.default_rng(7), 1e-6
    for got, at, value, off in checks:
        off = off * (1 + 2.0 ** -5)
        for _ in range(5):
            v = rng.standard_normal(value.shape)
            args = [[X, W1, W2], [X, W1, W2]]
            args[0][at], args[1][at] = value + t * v, value - t * v
            want = (loss(*args[0]) - loss(*args[1])) / (2 * t)
            have = as_f64(got)
            assert a((have * v).sum() - want) <= ((off + eps * (a(have) + off)) * a(v)).sum() + 1e-5 * a(want)
        exact = {0: DG @ W1, 1: DG.T @ X, 2: DY.T @ h_exact}[at]
        assert (a(as_f64(got) - exact) <= off + eps * (a(exact) + off)).all()
        # (six quantised factors at most, each off by 2^-4 at most, with no common sign: 0.15 of the length, 0.989 = sqrt(1 - 0.15^2))
        assert (as_f64(got) * exact).sum() >= 0.988 * np.sqrt((as_f64(got) ** 2).sum() * (exact ** 2).sum())


# ---------------------------------------------------------------------------------------------------- streams and graphs
class Layer:
    """A layer of experts and the same matrices' training step, with all its memory, as one run of calls."""

    def __init__(self, lutq, M, F, D, seed, ws=None, gws=None):
        import torch
        self.lutq, self.M, self.F, self.D = lutq, M, F, D
        self.x, self.dy = normal(seed, M, D, dtype="bf16"), normal(seed + 1, M, D, dtype="bf16")
        self.rows = to_gpu(np.random.default_rng(seed).integers(0, M, M).astype(np.int32))
        (c1, s1), (self.t1, self.ts1) = weights(lutq, normal(8, 2 * F, D, size=D ** -0.5))
        (c2, s2), (self.t2, self.ts2) = weights(lutq, normal(9, D, F, size=F ** -0.5))
        self.c1, self.s1, self.c2, self.s2 = c1, s1, c2, s2
        self.off = to_gpu(np.array([0, M // 3, M], np.int32))
        self.two = [torch.stack((t, t)) for t in (c1, s1, c2, s2)]
        self.ws = lutq.new_fp8_workspace(max(M, 2 * F), max(D, 2 * F), max(D, 2 * F, -(-M // 128) * 128), 2) if ws is None else ws
        self.gws = lutq.new_fp8_gated_workspace(M, F, D, 2) if gws is None else gws
        up = -(-M // 128) * 128
        self.q, self.h = (empty(M, D), empty(D // 128, M, dtype="f32")), (empty(M, F), empty(F // 128, M, dtype="f32"))
        self.grads = (empty(M, 2 * F), empty(2 * F // 128, M, dtype="f32")), (empty(2 * F, up), empty(up // 128, 2 * F, dtype="f32"))
        self.xc = empty(D, up), empty(up // 128, D, dtype="f32")
        self.y, self.z, self.dh, self.dx = (empty(M, n, dtype="bf16") for n in (D, D, F, D))
        self.saved, self.dw = empty(M, 2 * F, dtype="bf16"), empty(2 * F, D, dtype="bf16")

    def run(self):
        lutq = self.lutq
        lutq.lutq_fp8_quantize(self.x, *self.q, rows=self.rows)
        lutq.lutq_fp8_gated_grouped(self.q[0], *self.two[:2], self.off, self.h[0], self.gws, x_scales=self.q[1], h_scales=self.h[1], dtype=self.x.dtype)
        lutq.lutq_fp8_matmul_grouped(self.h[0], *self.two[2:], self.off, self.y, self.ws, x_scales=self.h[1])
        lutq.lutq_fp8_gated(self.x, self.c1, self.s1, self.h[0], self.gws, activation="gelu", h_scales=self.h[1], saved=self.saved)
        lutq.lutq_fp8_matmul(self.h[0], self.c2, self.s2, self.z, self.ws, x_scales=self.h[1])
        lutq.lutq_fp8_matmul(self.dy, self.t2, self.ts2, self.dh, self.ws)
        lutq.lutq_fp8_gated_grad(self.dh, self.saved, activation="gelu", rows=self.grads[0], columns=self.grads[1])
        lutq.lutq_fp8_matmul(self.grads[0][0], self.t1, self.ts1, self.dx, self.ws, x_scales=self.grads[0][1])
        lutq.lutq_fp8_quantize_columns(self.x, *self.xc)
        lutq.lutq_fp8_weight_grad(*self.grads[1], *self.xc, self.dw, self.ws)

    def results(self):
        return [t.clone() for t in (self.y, self.z, self.saved, self.dx, self.dw)]

    def wipe(self):
        for t in (self.y, self.z, self.saved, self.dx, self.dw, self.dh, *self.codes()):
            t.fill_(0x7f)

    def codes(self):
        return [*self.q, *self.h, *self.grads[0], *self.grads[1], *self.xc]


def equal(a, b):
    import torch
    return all(torch.equal(s, t) for s, t in zip(a, b))


SIZES = [(3, 128, 256), (40, 256, 2048), (200, 384, 1280), (1500, 256, 512)]


@pytest.mark.gpu
@pytest.mark.parametrize("M,F,D", SIZES)
def test_captured_and_replayed(lutq, M, F, D):
    """Two graphs that share their workspaces, replayed in turn with new values in place of the old, and eager calls on the workspaces between."""
    import torch
    layers = [Layer(lutq, M, F, D, 20)]
    layers.append(Layer(lutq, M, F, D, 30, layers[0].ws, layers[0].gws))
    side, graphs = torch.cuda.Stream(), []
    for layer in layers:
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            layer.run()
        torch.cuda.current_stream().wait_stream(side)
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            layer.run()
    eager = Layer(lutq, M, F, D, 40, layers[0].ws, layers[0].gws)
    for turn in range(4):
        for layer, graph in zip(layers, graphs):
            layer.x.copy_(normal(50 + turn, M, D, dtype="bf16"))
            layer.dy.copy_(normal(60 + turn, M, D, dtype="bf16"))
            layer.wipe()
            graph.replay()
            got = layer.results()
            torch.cuda.synchronize()
            eager.run()
            layer.wipe()
            layer.run()
            assert equal(got, layer.results()), turn
            assert all(t.isfinite().all().item() for t in got)
            assert not layer.ws[:65536].any().item() and not layer.gws[:65536].any().item()


@pytest.mark.gpu
@pytest.mark.parametrize("M,F,D", SIZES)
def test_on_two_streams_at_once(lutq, M, F, D):
    import torch
    layers = [Layer(lutq, M, F, D, 20), Layer(lutq, M, F, D, 30)]
    want = []
    for layer in layers:
        layer.run()
        want.append(layer.results())
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        for layer in layers:
            layer.wipe()
        torch.cuda.synchronize()
        for _ in range(3):
            for layer, stream in zip(layers, streams):
                with torch.cuda.stream(stream):
                    layer.run()
        torch.cuda.synchronize()
        for layer, results in zip(layers, want):
            assert equal(layer.results(), results)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 50, 600])
def test_a_given_stream_and_without_the_native_part(lutq, monkeypatch, M):
    """The same bits by each path into the library."""
    import torch
    layer = Layer(lutq, M, 256, 384, 20)
    layer.run()
    want, codes = layer.results(), [t.clone() for t in layer.codes()]
    functions = [n for n in dir(lutq) if n.startswith("lutq_fp8_") and not n.endswith("_bytes")]
    assert len(functions) >= 11

    class OnStream:
        def __init__(self, stream):
            for n in functions:
                setattr(self, n, (lambda f: lambda *a, **k: f(*a, stream=stream, **k))(getattr(lutq, n)))
    for path in ("stream", "python"):
        layer.wipe()
        if path == "stream":
            side = torch.cuda.Stream()
            side.wait_stream(torch.cuda.current_stream())
            layer.lutq = OnStream(side)
            layer.run()
            side.synchronize()
            layer.lutq = lutq
        else:
            monkeypatch.setattr(lutq.binding, "_NATIVE", lutq.binding._NoNative)
            layer.run()
        assert equal(layer.results(), want) and equal(layer.codes(), codes)
    back, dense = empty(M, 256, dtype="f16"), empty(512, 384, dtype="f16")
    lutq.lutq_fp8_dequant(*layer.h, back)
    lutq.lutq_fp8_dequant_weights(layer.c1, layer.s1, dense)
    monkeypatch.undo()
    again, dense_again = empty(M, 256, dtype="f16"), empty(512, 384, dtype="f16")
    lutq.lutq_fp8_dequant(*layer.h, again)
    lutq.lutq_fp8_dequant_weights(layer.c1, layer.s1, dense_again)
    assert torch.equal(back, again) and torch.equal(dense, dense_again)


# ---------------------------------------------------------------------------------------------------- values
MANY = [1, 3, 8, 13, 16, 17, 40, 130, 300, 1100]


@pytest.mark.gpu
@pytest.mark.parametrize("K", [384, 6016])
@pytest.mark.parametrize("M", MANY)
def test_values_are_quantised_on_the_way_in_as_by_the_quantiser(lutq, M, K):
    """The same bits, infinities and what is no number among them."""
    import torch
    p = Problem(lutq, M, 272, K, "bf16")
    x = edge_values("bf16", M, K, M).cuda()
    x[::2] = p.X[::2]
    codes, s = quantised(lutq, x)
    y, z = p.out(), empty(M, 272, dtype="bf16")
    lutq.lutq_fp8_matmul(x, p.W, p.sw, y, p.ws)
    lutq.lutq_fp8_matmul(codes, p.W, p.sw, z, p.ws, x_scales=s)
    assert torch.equal(y.nan_to_num(3.0), z.nan_to_num(3.0)) and torch.equal(y.isnan(), z.isnan()) and p.guards_hold()
    assert not y[::2].isnan().any().item()


@pytest.mark.gpu
@pytest.mark.parametrize("form", ["matmul", "gated", "saved"])
@pytest.mark.parametrize("M", MANY)
def test_what_is_no_number_stays_in_its_row_or_column(lutq, M, form):
    import torch
    N, K = 384, 640
    p = Problem(lutq, M, N, K, "bf16", gated=form != "matmul")
    W, sw, X = p.W.clone(), p.sw.clone(), p.X.clone()
    def call(x, w, ws):
        y = empty(M, N, dtype="bf16")
        if form == "matmul":
            return lutq.lutq_fp8_matmul(x, w, ws, y, p.ws).clone()
        saved = empty(M, 2 * N, dtype="bf16") if form == "saved" else None
        return lutq.lutq_fp8_gated(x, w, ws, y, p.ws, saved=saved).clone()
    want = call(X, W, sw)
    bad_rows = sorted({0, M // 2, M - 1})[:max(1, min(3, M - 1))]
    for r, v in zip(bad_rows, (float("inf"), float("nan"), float("-inf"))):
        X[r, 130 * r % K] = v
    W[17, 5], W[383, 639] = 0x7f, 0xff                  # (gated: two of the gate's)
    sw[1, 2] = float("nan")                             # output channels 128 .. 255
    got = call(X, W, sw)
    bad = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    bad[bad_rows] = True
    bad[:, 17] = bad[:, 383] = bad[:, 128:256] = True
    assert torch.equal(got.isnan(), bad) and torch.equal(got[~bad], want[~bad]) and p.clean()


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(128, 48, 80), (300, 272, 400), (1000, 1040, 528)])
def test_what_is_no_number_stays_in_its_row_or_column_of_a_gradient(lutq, M, N, K):
    import torch
    dy, x = normal(1, M, N * 8, dtype="bf16")[:, ::8].contiguous(), normal(2, M, K, dtype="bf16")
    up = lambda t: torch.nn.functional.pad(t, (0, -t.shape[1] % 128))
    def grad(dy, x):
        (a, sa), (b, sb) = quantised(lutq, up(dy), True), quantised(lutq, up(x), True)
        a, sa, b, sb = a[:N], sa[:, :N].contiguous(), b[:K], sb[:, :K].contiguous()
        dw = empty(N, K, dtype="bf16")
        return lutq.lutq_fp8_weight_grad(a, sa, b, sb, dw, lutq.new_fp8_workspace(N, K, a.shape[1])).clone()
    want = grad(dy, x)
    dy[5, 7], x[M - 1, 33] = float("nan"), float("inf")
    got, bad = grad(dy, x), torch.zeros((N, K), dtype=torch.bool, device="cuda")
    bad[7] = bad[:, 33] = True
    assert torch.equal(got.isnan(), bad) and torch.equal(got[~bad], want[~bad])


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 9, 33, 200])
def test_sums_beyond_the_type_are_infinite(lutq, M):
    """Above 65504 of fp16 by at least what the sums may be off: infinite.  Below it by as much: finite."""
    p = Problem(lutq, M, 128, 640, "f16")
    y, ref = p.out(), fx.product(p.x, p.w[0])
    scale = 65520.0 / np.median(np.abs(ref[0]))
    lutq.lutq_fp8_matmul(p.codes, p.W, p.sw * scale, y, p.ws, x_scales=p.s)
    want, off = ref[0] * scale, sums_off(ref[1] * scale, 640) + 2.0 ** -23 * ref[1] * scale     # (the scales' own two roundings)
    got = as_f64(y)
    above, below = np.abs(want) - off >= 65520.0, np.abs(want) + off < 65520.0
    assert above.any() and below.any() and np.isinf(got[above]).all() and np.isfinite(got[below]).all()
    assert (np.sign(got) == np.sign(want))[above].all()


@pytest.mark.gpu
def test_codes_as_their_own_type(lutq):
    """float8_e4m3fn tensors wherever codes are taken, and bytes."""
    import torch
    p, g = Problem(lutq, 40, 256, 384, "bf16"), Problem(lutq, 40, 256, 384, "bf16", gated=True)
    f8 = lambda t: t.view(torch.float8_e4m3fn)
    y, z = empty(40, 256, dtype="bf16"), empty(40, 256, dtype="bf16")
    lutq.lutq_fp8_matmul(p.codes, p.W, p.sw, y, p.ws, x_scales=p.s)
    lutq.lutq_fp8_matmul(f8(p.codes), f8(p.W), p.sw, z, p.ws, x_scales=p.s)
    assert torch.equal(y, z)
    hc, hs, hd, ht = empty(40, 256), empty(2, 40, dtype="f32"), f8(empty(40, 256)), empty(2, 40, dtype="f32")
    lutq.lutq_fp8_gated(g.codes, g.W, g.sw, hc, g.ws, x_scales=g.s, h_scales=hs, dtype=torch.bfloat16)
    lutq.lutq_fp8_gated(f8(g.codes), f8(g.W), g.sw, hd, g.ws, x_scales=g.s, h_scales=ht, dtype=torch.bfloat16)
    assert torch.equal(hc, hd.view(torch.uint8)) and torch.equal(hs, ht)
    lutq.lutq_fp8_dequant(hd, ht, y)
    lutq.lutq_fp8_dequant(hc, hs, z)
    assert torch.equal(y, z)


# ---------------------------------------------------------------------------------------------------- calls at the edge
@pytest.mark.gpu
@pytest.mark.parametrize("offsets", [[0, 0, 0, 0], [40, 40, 40, 40], [-5, 10, 20, 90], [40, 20, 10, 0], [0, 40, 0, 40], [5, 30, 3, 37], [-2 ** 31, 2 ** 31 - 1, -1, 2 ** 31 - 1],
                                     [2 ** 31 - 1] * 4, [-7] * 4])
@pytest.mark.parametrize("N,K", [(128, 640), (256, 2048)])
def test_offsets_that_the_documentation_does_not_allow_stay_in_bounds(lutq, offsets, N, K):
    """They are taken into 0 .. M, and no more pieces of rows are done than there can be: nothing else is read or written."""
    import torch
    for M in (40, 700):
        off = np.clip([o * (M // 40) if abs(o) < 1000 else o for o in offsets], -2 ** 31, 2 ** 31 - 1).astype(np.int32)
        p = Problem(lutq, M, N, K, "bf16", experts=3)
        g = Problem(lutq, M, N, K, "bf16", experts=3, gated=True)
        for dense in (False, True):
            y = p.out()
            x, s = p.args(dense)
            lutq.lutq_fp8_matmul_grouped(x, p.W, p.sw, to_gpu(off), y, p.ws, x_scales=s)
            assert p.guards_hold() and p.clean()
            h, saved = g.out(), empty(M + 32, 2 * N, dtype="bf16")
            x, s = g.args(dense)
            lutq.lutq_fp8_gated_grouped(x, g.W, g.sw, to_gpu(off), h, g.ws, x_scales=s, saved=saved[16:16 + M])
            assert g.guards_hold() and g.clean() and (saved[:16] == -7.0).all().item() and (saved[16 + M:] == -7.0).all().item()
            codes, hs = g.out("u8"), empty(N // 128 + 2, M, dtype="f32")
            lutq.lutq_fp8_gated_grouped(x, g.W, g.sw, to_gpu(off), codes, g.ws, x_scales=s, h_scales=hs[1:-1], dtype=torch.bfloat16)
            assert g.guards_hold() and g.clean() and (hs[0] == -7.0).all().item() and (hs[-1] == -7.0).all().item()
            if (np.clip(off, 0, M) == np.clip(off, 0, M)[0]).all():
                assert (y == -7.0).all().item() and (h == -7.0).all().item() and (codes == 0x7f).all().item()


@pytest.mark.gpu
def test_no_rows(lutq):
    import torch
    e = lambda *shape, dtype="u8": empty(*shape, dtype=dtype)
    off, W, sw = to_gpu(np.zeros(3, np.int32)), e(2, 256, 128), e(2, 2, 1, dtype="f32")
    ws, gws = lutq.new_fp8_workspace(0, 256, 128, 2), lutq.new_fp8_gated_workspace(0, 128, 128, 2)
    x, s, y, h, saved = e(0, 128, dtype="bf16"), e(1, 0, dtype="f32"), e(0, 256, dtype="bf16"), e(0, 128, dtype="bf16"), e(0, 256, dtype="bf16")
    lutq.lutq_fp8_quantize(x, e(0, 128), s)
    lutq.lutq_fp8_quantize(e(4, 128, dtype="bf16"), e(0, 128), s, rows=to_gpu(np.zeros(0, np.int32)))
    lutq.lutq_fp8_dequant(e(0, 128), s, x)
    lutq.lutq_fp8_matmul(x, W[0], sw[0], y, ws)
    lutq.lutq_fp8_matmul_grouped(e(0, 128), W, sw, off, y, ws, x_scales=s)
    lutq.lutq_fp8_gated(x, W[0], sw[0], h, gws, saved=saved)
    lutq.lutq_fp8_gated_grouped(x, W, sw, off, e(0, 128), gws, h_scales=s)
    lutq.lutq_fp8_gated_grad(h, saved, dense=saved, rows=(e(0, 256), e(2, 0, dtype="f32")))
    torch.cuda.synchronize()
    with pytest.raises((lutq.LutqError, ValueError)):
        lutq.lutq_fp8_quantize_columns(x, e(128, 0), e(0, 128, dtype="f32"))
    assert not ws.any().item() and not gws.any().item()


@pytest.mark.gpu
def test_rows_of_zeros_picked_for_padding(lutq):
    """A padded batch: rows that are no row of X are zeros, and rows of H and Y made of them are zeros too."""
    import torch
    M, F, D = 64, 128, 256
    rows = np.full(M, -1, np.int32)
    rows[5:20], rows[40:51] = np.arange(15), np.arange(11)
    x = normal(1, 15, D, dtype="bf16")
    codes, s = empty(M, D), empty(D // 128, M, dtype="f32")
    lutq.lutq_fp8_quantize(x, codes, s, rows=to_gpu(rows))
    q1, _ = weights(lutq, normal(2, 2 * F, D, size=D ** -0.5))
    hc, hs = empty(M, F), empty(1, M, dtype="f32")
    lutq.lutq_fp8_gated(codes, *q1, hc, lutq.new_fp8_gated_workspace(M, F, D), x_scales=s, h_scales=hs, dtype=torch.bfloat16)
    padding = to_gpu(rows < 0)
    assert not (hc[padding] & 0x7f).any().item() and hs.isfinite().all().item() and (hc[~padding] & 0x7f).any(1).all().item()
    assert torch.equal(hc[5:16], hc[40:51]) and torch.equal(hs[:, 5:16], hs[:, 40:51])


@pytest.mark.gpu
def test_a_workspace_for_more_rows_serves_fewer(lutq):
    import torch
    ws = lutq.new_fp8_workspace(2000, 272, 640)
    for M in (2000, 1, 300, 17, 2000, 64):
        p = Problem(lutq, M, 272, 640, "bf16")
        for dense in (False, True):
            y, z = p.out(), empty(M, 272, dtype="bf16")
            x, s = p.args(dense)
            lutq.lutq_fp8_matmul(x, p.W, p.sw, y, ws, x_scales=s)
            lutq.lutq_fp8_matmul(x, p.W, p.sw, z, p.ws, x_scales=s)
            assert torch.equal(y, z) and p.guards_hold() and not ws[:65536].any().item()


@pytest.mark.gpu
def test_the_binding_refuses(lutq):
    import torch
    p, g = Problem(lutq, 8, 256, 384, "bf16"), Problem(lutq, 8, 128, 384, "bf16", gated=True)
    y, h, off = empty(8, 256, dtype="bf16"), empty(8, 128, dtype="bf16"), to_gpu(np.array([0, 8], np.int32))
    mm = lambda X=p.codes, W=p.W, sw=p.sw, Y=y, ws=p.ws, s=p.s: lutq.lutq_fp8_matmul(X, W, sw, Y, ws, x_scales=s)
    mm()
    wide = lambda t: torch.stack((t, t), -1)[..., 0]
    for bad in (dict(X=wide(p.codes)), dict(W=wide(p.W)), dict(sw=wide(p.sw)), dict(Y=wide(y)), dict(s=p.s.t().contiguous().t()), dict(X=p.codes.cpu()), dict(ws=p.ws.cpu())):
        with pytest.raises(ValueError, match="contiguous|CUDA"):
            mm(**bad)
    for bad in (dict(X=p.X), dict(W=p.W.view(torch.int8)), dict(sw=p.sw.double()), dict(s=p.s.half()), dict(Y=y.float()), dict(ws=p.ws.view(torch.int32)),
                dict(X=p.X.half(), s=None), dict(X=p.codes, s=None)):
        with pytest.raises(TypeError):
            mm(**bad)
    for bad in (dict(X=p.codes[:, :256].contiguous()), dict(W=p.W[:128].contiguous()), dict(sw=p.sw[:1].contiguous()), dict(Y=y[:7]), dict(s=p.s[:2].contiguous()), dict(X=p.codes[0]),
                dict(W=p.W[None])):
        with pytest.raises(ValueError, match="shapes"):
            mm(**bad)
    with pytest.raises(lutq.LutqError, match="workspace"):
        mm(ws=p.ws[:1024])
    grouped = lambda offsets=off, W=p.W[None], sw=p.sw[None]: lutq.lutq_fp8_matmul_grouped(p.codes, W, sw, offsets, y, p.ws, x_scales=p.s)
    grouped()
    for bad in (dict(offsets=off.long()), dict(offsets=off[None]), dict(offsets=None)):
        with pytest.raises(TypeError, match="offsets"):
            grouped(**bad)
    with pytest.raises(ValueError, match="shapes"):
        grouped(W=p.W, sw=p.sw)
    gate = lambda H=h, **k: lutq.lutq_fp8_gated(g.codes, g.W, g.sw, H, g.ws, x_scales=g.s, **k)
    gate()
    with pytest.raises(ValueError, match="activation"):
        gate(activation="relu")
    hs = empty(1, 8, dtype="f32")
    with pytest.raises(TypeError, match="dtype"):
        gate(empty(8, 128), h_scales=hs)
    with pytest.raises(TypeError):
        gate(h, h_scales=hs, dtype=torch.bfloat16)      # (H of 16 bits where codes are asked for)
    with pytest.raises(TypeError):
        gate(saved=empty(8, 256, dtype="f16"))
    with pytest.raises(ValueError, match="shapes"):
        gate(saved=empty(8, 128, dtype="bf16"))
    with pytest.raises(ValueError, match="shapes"):
        gate(empty(8, 128), h_scales=empty(2, 8, dtype="f32"), dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        lutq.lutq_fp8_gated_grad(h, empty(8, 256, dtype="bf16"))                # (nothing is asked for)
    for bad in (dict(dense=empty(8, 128, dtype="bf16")), dict(rows=(empty(8, 256), empty(1, 8, dtype="f32"))), dict(columns=(empty(256, 8), empty(1, 256, dtype="f32")))):
        with pytest.raises(ValueError, match="shapes"):
            lutq.lutq_fp8_gated_grad(h, empty(8, 256, dtype="bf16"), **bad)
    with pytest.raises(TypeError):
        lutq.lutq_fp8_gated_grad(h, empty(8, 256, dtype="f16"), dense=empty(8, 256, dtype="bf16"))
    with pytest.raises(ValueError, match="shapes"):
        lutq.lutq_fp8_quantize(p.X, empty(8, 384), empty(8, 3, dtype="f32"))
    with pytest.raises(TypeError):
        lutq.lutq_fp8_quantize(p.X.double(), empty(8, 384), empty(3, 8, dtype="f32"))
    with pytest.raises(TypeError):
        lutq.lutq_fp8_quantize(p.X, empty(8, 384), empty(3, 8, dtype="f32"), rows=torch.zeros(8, dtype=torch.int64, device="cuda"))
    c, s = (empty(256, 128), empty(1, 256, dtype="f32")), (empty(48, 128), empty(1, 48, dtype="f32"))
    grad = lambda a=c, b=s, dw=empty(256, 48, dtype="bf16"): lutq.lutq_fp8_weight_grad(*a, *b, dw, lutq.new_fp8_workspace(256, 48, 128))
    for bad in (dict(a=(empty(256, 256), empty(2, 256, dtype="f32"))), dict(b=(c[0], s[1])), dict(dw=empty(48, 256, dtype="bf16"))):
        with pytest.raises(ValueError, match="shapes"):
            grad(**bad)
    with pytest.raises(TypeError):
        grad(dw=empty(256, 48, dtype="f32"))
    torch.cuda.synchronize()


def test_codes_of_h_beside_h_need_their_scales(lutq):
    import torch
    x, u, s = torch.zeros((16, 128), dtype=torch.float16), torch.zeros((16, 128), dtype=torch.uint8), torch.zeros((1, 16))
    for call in (lambda **k: lutq.lutq_fp8_gated(x, u, s, x, u, **k), lambda **k: lutq.lutq_fp8_gated_grouped(x, u, s, torch.zeros(3, dtype=torch.int32), x, u, **k)):
        with pytest.raises(TypeError, match="h_scales"):
            call(h_codes=u)
        with pytest.raises(ValueError, match="CUDA"):
            call(h_codes=u, h_scales=s)


@pytest.mark.gpu
@pytest.mark.parametrize("native", [True, False])
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("M", [1, 12, 130, 700])
def test_h_and_its_codes_by_the_binding(lutq, monkeypatch, M, dense, native):
    """H at 16 bits and the codes that the quantiser makes of it, the bits of the calls that give either; by expert too, rows outside untouched; refusals."""
    import torch
    F, K = 256, 384
    if not native:
        monkeypatch.setattr(lutq.binding, "_NATIVE", lutq.binding._NoNative)
    p, e = Problem(lutq, M, F, K, "bf16", gated=True), Problem(lutq, M, F, K, "bf16", experts=2, gated=True)
    off = np.array([min(1, M - 1), M // 2, M - M // 10], np.int32)
    for q, call, inside in ((p, lambda *a, **k: lutq.lutq_fp8_gated(q.args(dense)[0], q.W, q.sw, *a, x_scales=q.args(dense)[1], **k), slice(0, M)),
                            (e, lambda *a, **k: lutq.lutq_fp8_gated_grouped(q.args(dense)[0], q.W, q.sw, to_gpu(off), *a, x_scales=q.args(dense)[1], **k),
                             slice(int(off[0]), int(off[-1])))):
        h, codes, hs, saved = q.out(), empty(M + 32, F), empty(F // 128, M, dtype="f32"), empty(M, 2 * F, dtype="bf16")
        assert call(h, q.ws, h_codes=codes[16:16 + M], h_scales=hs, saved=saved) is h
        assert check_h_codes(codes[16:16 + M][inside], hs[:, inside], h[inside]) and q.guards_hold() and q.clean()
        assert (codes[:16] == 0x7f).all().item() and (codes[16 + M:] == 0x7f).all().item()
        outside = torch.ones(M, dtype=torch.bool, device="cuda")
        outside[inside] = False
        assert (h[outside] == -7.0).all().item() and (codes[16:16 + M][outside] == 0x7f).all().item() and (hs[:, outside] == -7.0).all().item()
        alone, its_scales, h16, kept = empty(M, F), empty(F // 128, M, dtype="f32"), empty(M, F, dtype="bf16"), empty(M, 2 * F, dtype="bf16")
        call(alone, q.ws, h_scales=its_scales, dtype=torch.bfloat16)
        call(h16, q.ws, saved=kept)
        assert torch.equal(alone, codes[16:16 + M]) and torch.equal(its_scales, hs) and torch.equal(h16, h) and torch.equal(kept, saved)
        with pytest.raises(ValueError, match="shapes"):
            call(h, q.ws, h_codes=empty(M, 2 * F), h_scales=hs)
        with pytest.raises(TypeError):
            call(h, q.ws, h_codes=empty(M, F, dtype="bf16"), h_scales=hs)
        with pytest.raises(TypeError):
            call(codes[16:16 + M], q.ws, h_codes=codes[16:16 + M], h_scales=hs)
