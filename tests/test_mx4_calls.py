"""Microscaled 4-bit operators: calls at the edge of what their documentation allows, and refusals of those beyond it."""
import numpy as np
import pytest

from gpu_util import torch_dtype
from oracle import mx4_oracle as mx
from test_mx4 import Problem, as_f64, counts_to_offsets, edge_values, grouped_reference, off_by_at_most, to_gpu


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
