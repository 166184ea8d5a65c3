"""Microscaled 4-bit operators: calls at the edge of what their documentation allows, and refusals of those beyond it."""
import numpy as np
import pytest

from gpu_util import torch_dtype
from oracle import mx4_oracle as mx
from test_mx4 import Problem, as_f64, counts_to_offsets, edge_values, grouped_reference, off_by_at_most, to_gpu
from test_mx4_launches import Factors, pack_on_device, values_on_device


def test_the_row_form_needs_its_exponents(lutq):
    """Without them the arguments are those of the packed form, of which the caller has not spoken."""
    import torch
    x, p = torch.zeros((16, 128), dtype=torch.float16), torch.zeros(lutq.lutq_mx4_packed_bytes(16, 128), dtype=torch.uint8)
    for call in (lambda: lutq.lutq_mx4_quantize(x, p, None), lambda: lutq.lutq_mx4_dequant(p, None, x)):
        with pytest.raises(TypeError, match="exponents"):
            call()


@pytest.mark.gpu
def test_the_row_form_needs_its_exponents_on_the_device(lutq):
    import torch
    x = torch.ones((16, 128), dtype=torch.float16, device="cuda")
    p = torch.full((lutq.lutq_mx4_packed_bytes(16, 128),), 0xA5, dtype=torch.uint8, device="cuda")
    for call in (lambda: lutq.lutq_mx4_quantize(x, p, None), lambda: lutq.lutq_mx4_dequant(p, None, x)):
        with pytest.raises(TypeError, match="exponents"):
            call()
    torch.cuda.synchronize()
    assert (p == 0xA5).all().item() and (x == 1.0).all().item()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [(1 << 30) - 1, (1 << 30) - 64])
def test_as_many_picked_rows_as_there_may_be(lutq, M):
    """Sixteen lanes take four blocks of 128 columns: the largest calls have 2^32 threads and fewer.  64 GiB of codes."""
    import torch
    torch.cuda.empty_cache()
    x = edge_values("bf16", 50, 128, 9)
    codes, e = mx.quantize(as_f64(x))
    want_c, want_e = to_gpu(mx.row_bytes(codes)), to_gpu(e)
    rows = torch.arange(M, dtype=torch.int32, device="cuda")
    rows.remainder_(50)
    c, s = torch.empty((M + 4, 64), dtype=torch.uint8, device="cuda"), torch.empty((M + 16, 4), dtype=torch.uint8, device="cuda")
    c[M - 20000:], s[M - 20000:] = 0xA5, 0xA5
    lutq.lutq_mx4_quantize(x.cuda(), c[:M], s[:M], rows=rows)
    for at in (slice(0, 20000), slice(M - 20000, M), slice(1, M, 4999)):
        r = rows[at].long()
        assert torch.equal(c[at], want_c[r]) and torch.equal(s[at], want_e[r])
    assert (c[M:] == 0xA5).all().item() and (s[M:] == 0xA5).all().item()
    del rows, c, s
    torch.cuda.empty_cache()


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("M", [1, 4, 16])
@pytest.mark.parametrize("K", [7168, 7680, 8192, 16384])
def test_a_wavefront_per_quad_up_to_sixteen(lutq, K, M, dense):
    """With one row block per workgroup: fourteen wavefronts have 63 KiB of LDS, fifteen and sixteen more than 64."""
    p = Problem(lutq, M, 48, K, "bf16")
    x, e = p.args(dense)
    y = p.out()
    lutq.lutq_mx4_matmul(x, p.packed, y, p.ws, x_scales=e)
    got, sums = as_f64(y), mx.product(p.x, p.w[0])
    assert (np.abs(got - sums[0]) <= off_by_at_most(got, sums, K, "bf16")).all() and p.guards_hold()


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
@pytest.mark.parametrize("counts", [[2, 0, 5, 1], [40, 0, 7, 23, 16], [300, 0, 129, 60]])
def test_by_expert_with_and_without_the_native_part(lutq, monkeypatch, counts, dense):
    """The values of either path, and the same bits."""
    import torch
    off = counts_to_offsets(counts, 1)
    p = Problem(lutq, int(off[-1]) + 2, 272, 640, "bf16", experts=len(counts))
    x, e = p.args(dense)
    sums, results, offsets = grouped_reference(p, off), [], to_gpu(off)
    for native in (True, False):
        if not native:
            monkeypatch.setattr(lutq.binding, "_NATIVE", lutq.binding._NoNative)
        y = p.out()
        lutq.lutq_mx4_matmul_grouped(x, p.packed, offsets, y, p.ws, x_scales=e)
        assert (np.abs(as_f64(y) - sums[0]) <= off_by_at_most(as_f64(y), sums, 640, "bf16")).all() and p.guards_hold()
        results.append(y)
    assert torch.equal(*results)
    side = torch.cuda.Stream()                          # (a given stream is served by the shared path)
    y = p.out()
    side.wait_stream(torch.cuda.current_stream())
    lutq.lutq_mx4_matmul_grouped(x, p.packed, offsets, y, p.ws, x_scales=e, stream=side)
    side.synchronize()
    assert torch.equal(y, results[0])


def opposite_exponents(M, N, K, dtype, power, top, seed):
    """Factors whose exponent bytes are anything from 0 to `top`, block by block, one as large as the other is small: every product of two
    codes is some 2^power times what the codes stand for."""
    import torch
    p = Factors(M, N, K, 0, dtype, seed)
    g = torch.Generator(device="cuda")
    g.manual_seed(seed + 1000)
    x = torch.randint(0, top + 1, (K // 32,), generator=g, device="cuda")
    x[::3] = torch.tensor([0, 1, 2, top - 2, top - 1, top], device="cuda").repeat(K)[:x[::3].numel()]
    jitter = torch.randint(-3, 1, (N, K // 32), generator=g, device="cuda")
    p.e = x.to(torch.uint8).repeat(M, 1)
    p.w = [(p.w[0][0], (254 + power - x + jitter).clamp(0, 254).to(torch.uint8))]
    # (where the clamp at 0 or 254 has moved a block, its products are larger or smaller: zero codes where they are too large)
    larger = (p.w[0][1].long() + x - 254 > power).repeat_interleave(16, 1)
    p.w[0][0][larger] = 0
    p.packed = pack_on_device(*p.w[0])
    p.X = values_on_device(p.codes, p.e).to(torch_dtype(dtype))
    return p


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 48, 640), (3, 48, 1152), (13, 272, 640), (33, 304, 640), (8, 64, 128), (17, 29120, 640), (17, 29216, 512),
                                   (65, 16928, 1152), (17, 10768, 6784), (130, 49296, 896), (49, 5312, 5248)])
@pytest.mark.parametrize("dtype,power", [("bf16", -140), ("bf16", -3), ("bf16", 105), ("f16", -24), ("f16", -1)])
def test_exponents_from_end_to_end(lutq, M, N, K, dtype, power):
    """Streamed and tiled, an odd number of tiles of K and slices among them.  Sums down to the last place of fp32, and below the type's
    smallest normal number: none is flushed.  (A sum that fp32 holds as a subnormal number is off by at most its quantum, 2^-149, an addition.)"""
    import torch
    ws = lutq.new_mx4_workspace(M, N, K)
    for as_codes in ((True, False) if dtype == "bf16" else (True,)):    # (bf16 values hold 6 2^(e - 127) up to e = 252)
        p = opposite_exponents(M, N, K, dtype, power, 254 if as_codes else 252, M + K)
        y = torch.full((M, N), 7.0, dtype=torch_dtype(dtype), device="cuda")
        x, e = p.args(as_codes)
        assert as_codes or x.isfinite().all().item()
        lutq.lutq_mx4_matmul(x, p.packed, y, ws, x_scales=e)
        worst = p.worst(y, 0, M, 0, 2.0 ** -149)
        assert worst <= 1.0, (as_codes, worst)
        assert y.any().item() or power == -24
        assert power != -140 or (y.abs() < 2.0 ** -126).any().item()


@pytest.mark.gpu
@pytest.mark.parametrize("src", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("M,K", [(8209, 1152), (14593, 640), (262145, 128)])
def test_more_rows_than_teams_with_a_remainder(lutq, src, M, K):
    """Four units per team and four words per lane, as large calls take them, where the last workgroup is not full; picked rows as well."""
    import torch
    x = edge_values(src, 61, K, M)
    codes, e = mx.quantize(as_f64(x))
    rows = np.random.default_rng(K).integers(-1, 61, M).astype(np.int32)
    rows[-1] = 60
    ok = rows >= 0
    x, want_c, want_e, r = x.cuda(), to_gpu(mx.row_bytes(codes)), to_gpu(e), to_gpu(np.where(ok, rows, 0)).long()
    want_c, want_e = (torch.where(to_gpu(ok)[:, None], t[r], 0).to(torch.uint8) for t in (want_c, want_e))
    assert M * (K // 128) >= 32768 and M * (K // 128) % 64 and M * K // 8 >= 1 << 20 and M * K // 8 % 1024      # (the kernels' sizes)
    for pick in (False, True):
        c = torch.full((M + 2, K // 2), 0xA5, dtype=torch.uint8, device="cuda")
        s = torch.full((M + 16, K // 32), 0xA5, dtype=torch.uint8, device="cuda")
        source = x if pick else torch.where(to_gpu(ok)[:, None], x[r], 0)
        lutq.lutq_mx4_quantize(source, c[:M], s[:M], rows=to_gpu(rows) if pick else None)
        assert torch.equal(c[:M], want_c) and torch.equal(s[:M], want_e)
        assert (c[M:] == 0xA5).all().item() and (s[M:] == 0xA5).all().item()
    if src == "f32":
        return
    back = torch.full((M + 2, K), 7.0, dtype=x.dtype, device="cuda")
    lutq.lutq_mx4_dequant(c[:M], s[:M], back[:M])
    with np.errstate(over="ignore"):
        want = torch.from_numpy(mx.values(codes, e).astype(np.float32)).to(x.dtype).cuda()
    want = torch.where(to_gpu(ok)[:, None], want[r], 0)
    nan = want.isnan()
    assert torch.equal(back[:M].isnan(), nan) and torch.equal(torch.where(nan, 0, back[:M]), torch.where(nan, 0, want))
    assert (back[M:] == 7.0).all().item()


def test_refusals_of_a_shape_name_the_domain(lutq):
    with pytest.raises(ValueError, match="K of 128"):
        lutq.new_mx4_workspace(1, 16, 2880)
    with pytest.raises(lutq.LutqError, match="K % 128"):
        lutq.lutq_mx4_pack(np.zeros((16, 1440)), np.zeros((16, 90)))


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5, 33, 200])
def test_blocks_that_fill_no_tile_are_padded_with_zeros(lutq, M):
    """K = 2880, 22 1/2 tiles: columns of zeros behind the rows, as values and as codes; and 40 output channels, eight rows of zeros behind."""
    import torch
    N, K, NP, KP = 40, 2880, 48, 2944
    rng = np.random.default_rng(M)
    x, w = rng.standard_normal((M, K)), rng.standard_normal((N, K))
    x, w = torch.from_numpy(x).bfloat16(), torch.from_numpy(w).bfloat16()
    with pytest.raises(ValueError, match="K of 128"):
        lutq.lutq_mx4_quantize_packed(w.cuda(), torch.zeros(1 << 20, dtype=torch.uint8, device="cuda"))
    padded = torch.zeros((M, KP), dtype=torch.bfloat16, device="cuda")
    padded[:, :K] = x.cuda()
    weights = torch.zeros((NP, KP), dtype=torch.bfloat16, device="cuda")
    weights[:N, :K] = w.cuda()
    packed = torch.empty(lutq.lutq_mx4_packed_bytes(NP, KP), dtype=torch.uint8, device="cuda")
    lutq.lutq_mx4_quantize_packed(weights, packed)
    codes, e = torch.zeros((M, KP // 2), dtype=torch.uint8, device="cuda"), torch.zeros((M, KP // 32), dtype=torch.uint8, device="cuda")
    c, s = mx.quantize(as_f64(x))
    codes[:, :K // 2], e[:, :K // 32] = to_gpu(mx.row_bytes(c)), to_gpu(s)
    sums = mx.product(mx.values(c, s), mx.values(*mx.quantize(as_f64(w))))
    y, ws = torch.full((M, NP), 7.0, dtype=torch.bfloat16, device="cuda"), lutq.new_mx4_workspace(M, NP, KP)
    for args in ((padded, None), (codes, e)):
        lutq.lutq_mx4_matmul(args[0], packed, y, ws, x_scales=args[1])
        assert (np.abs(as_f64(y[:, :N]) - sums[0]) <= off_by_at_most(None, sums, KP, "bf16")).all() and not y[:, N:].any().item()
