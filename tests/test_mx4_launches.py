"""Every launch that the microscaled products choose, by the call that asks which it is, each against the definition in fp64.

The launches are chosen by estimated times, so a new estimate may send a size to another one: the table below has the launch of each
call, and is checked before the call is made; a sweep over sizes finds the kinds of launches that the table lacks.  Of the calls in
test_mx4.py these are streamed although they stand among tiles: 103 rows of 4112 x 640, 101 of 2064 x 8320, 601 of 272 x 14336, 131 of 1040 x 16512, and
by expert those of 1040 x 8320 and 528 x 14336; by expert only 4112 x 14336 is cut into slices there.

Bounds as in test_mx4.py: half a step of the 16-bit type, and (K / 128 + 12) 2^-22 of the sum of magnitudes."""
import math
import random

import numpy as np
import pytest

from gpu_util import torch_dtype
from oracle import mx4_oracle as mx

# rows, N, K, experts (0: without), whether X is codes, and the launch: X quantised first, channels and rows at a time,
# wavefronts, steps of room (0: streamed), slices of K, rows quantised at a time, past the caches
CALLS = [
    (1, 16, 128, 0, 1, (0, 16, 16, 1, 0, 1, 0, 0)), (5, 32, 4224, 0, 0, (1, 16, 16, 9, 0, 1, 0, 0)),
    (1, 16, 128, 0, 0, (0, 16, 16, 1, 0, 1, 1, 0)), (2, 16, 128, 0, 0, (0, 16, 16, 1, 0, 1, 4, 0)),
    (1, 43696, 5760, 0, 1, (0, 16, 16, 12, 0, 1, 0, 1)), (2, 17472, 14464, 0, 0, (1, 16, 16, 16, 0, 1, 0, 1)),
    (1, 14400, 17536, 0, 0, (0, 16, 16, 8, 0, 1, 1, 1)), (17, 32832, 640, 0, 1, (0, 32, 16, 2, 0, 1, 0, 0)),
    (17, 32816, 640, 0, 0, (1, 32, 16, 2, 0, 1, 0, 0)), (1, 16400, 128, 0, 0, (0, 32, 16, 1, 0, 1, 1, 0)),
    (2, 16400, 128, 0, 0, (0, 32, 16, 1, 0, 1, 4, 0)), (5, 16, 128, 0, 0, (0, 32, 16, 1, 0, 1, 16, 0)),
    (1, 47936, 5248, 0, 0, (0, 32, 16, 8, 0, 1, 1, 1)), (2, 59552, 4224, 0, 0, (0, 32, 16, 8, 0, 1, 4, 1)),
    (17, 32784, 128, 0, 1, (0, 64, 16, 2, 0, 1, 0, 0)), (17, 32784, 128, 0, 0, (1, 64, 16, 2, 0, 1, 0, 0)),
    (17, 29216, 512, 0, 1, (0, 128, 128, 4, 2, 1, 0, 0)), (65, 39552, 6400, 0, 1, (0, 128, 128, 4, 2, 1, 0, 1)),
    (130, 49296, 896, 0, 1, (0, 256, 256, 8, 2, 1, 0, 0)), (49, 14208, 512, 0, 0, (1, 64, 64, 4, 4, 1, 0, 0)),
    (17, 34640, 7296, 0, 1, (0, 64, 64, 4, 4, 1, 0, 1)), (33, 7248, 5504, 0, 1, (0, 64, 64, 4, 4, 2, 0, 0)),
    (49, 5312, 5248, 0, 0, (1, 64, 64, 4, 4, 3, 0, 0)), (49, 4000, 8192, 0, 1, (0, 64, 64, 4, 4, 4, 0, 0)),
    (51, 3232, 11392, 0, 0, (1, 64, 64, 4, 4, 5, 0, 0)), (50, 2672, 16768, 0, 1, (0, 64, 64, 4, 4, 6, 0, 0)),
    (17, 29120, 640, 0, 0, (1, 128, 64, 8, 4, 1, 0, 0)), (17, 31872, 7936, 0, 1, (0, 128, 64, 8, 4, 1, 0, 1)),
    (17, 11056, 10112, 0, 1, (0, 128, 64, 8, 4, 2, 0, 0)), (17, 14128, 17920, 0, 0, (1, 128, 64, 8, 4, 2, 0, 1)),
    (17, 10768, 6784, 0, 1, (0, 128, 64, 8, 4, 3, 0, 0)), (17, 7600, 10880, 0, 1, (0, 128, 64, 8, 4, 4, 0, 0)),
    (17, 6272, 13952, 0, 0, (1, 128, 64, 8, 4, 5, 0, 0)), (65, 2192, 17792, 0, 1, (0, 128, 64, 8, 4, 7, 0, 0)),
    (65, 16928, 1152, 0, 1, (0, 128, 128, 8, 4, 1, 0, 0)), (65, 31920, 7936, 0, 1, (0, 128, 128, 8, 4, 1, 0, 1)),
    (130, 5520, 8576, 0, 1, (0, 128, 128, 8, 4, 2, 0, 0)), (65, 14736, 17152, 0, 0, (1, 128, 128, 8, 4, 2, 0, 1)),
    (65, 8208, 6784, 0, 1, (0, 128, 128, 8, 4, 3, 0, 0)), (66, 5504, 13056, 0, 0, (1, 128, 128, 8, 4, 4, 0, 0)),
    (65, 5536, 13952, 0, 0, (1, 128, 128, 8, 4, 5, 0, 0)), (1, 16, 128, 1, 1, (0, 16, 16, 1, 0, 1, 0, 0)),
    (9, 16, 4224, 2, 0, (1, 16, 16, 9, 0, 1, 0, 0)), (1, 16, 128, 1, 0, (0, 16, 16, 1, 0, 1, 1, 0)),
    (2, 16, 128, 1, 0, (0, 16, 16, 1, 0, 1, 4, 0)), (56, 5808, 768, 56, 1, (0, 16, 16, 2, 0, 1, 0, 1)),
    (63, 6240, 640, 62, 0, (1, 16, 16, 2, 0, 1, 0, 1)), (11, 1408, 16384, 11, 0, (0, 16, 16, 8, 0, 1, 1, 1)),
    (41, 1760, 640, 19, 1, (0, 32, 16, 2, 0, 1, 0, 0)), (42, 3280, 640, 10, 0, (1, 32, 16, 2, 0, 1, 0, 0)),
    (5, 3280, 128, 5, 0, (0, 32, 16, 1, 0, 1, 1, 0)), (58, 304, 128, 54, 0, (0, 32, 16, 1, 0, 1, 4, 0)),
    (5, 16, 128, 1, 0, (0, 32, 16, 1, 0, 1, 16, 0)), (111, 7216, 640, 54, 1, (0, 32, 16, 2, 0, 1, 0, 1)),
    (59, 5216, 1664, 29, 0, (1, 32, 16, 2, 0, 1, 0, 1)), (18, 52496, 256, 18, 0, (0, 32, 16, 1, 0, 1, 1, 1)),
    (36, 9536, 768, 34, 0, (0, 32, 16, 2, 0, 1, 4, 1)), (20, 1648, 128, 20, 1, (0, 64, 16, 4, 0, 1, 0, 0)),
    (103, 2624, 128, 25, 0, (1, 64, 16, 4, 0, 1, 0, 0)), (38, 52960, 128, 32, 1, (0, 64, 16, 4, 0, 1, 0, 1)),
    (31, 54496, 128, 31, 0, (1, 64, 16, 4, 0, 1, 0, 1)), (43, 15808, 512, 2, 1, (0, 128, 128, 4, 2, 1, 0, 0)),
    (1076, 1952, 4096, 32, 1, (0, 128, 128, 4, 2, 1, 0, 1)), (15279, 672, 896, 18, 1, (0, 256, 256, 8, 2, 1, 0, 0)),
    (174, 4992, 512, 1, 1, (0, 64, 64, 4, 4, 1, 0, 0)), (129, 5376, 5888, 8, 1, (0, 64, 64, 4, 4, 1, 0, 1)),
    (145, 1920, 5632, 4, 1, (0, 64, 64, 4, 4, 2, 0, 0)), (247, 1088, 16256, 15, 1, (0, 64, 64, 4, 4, 2, 0, 1)),
    (2585, 128, 5376, 1, 0, (1, 64, 64, 4, 4, 3, 0, 0)), (306, 768, 8832, 1, 1, (0, 64, 64, 4, 4, 4, 0, 0)),
    (3187, 64, 11392, 2, 0, (1, 64, 64, 4, 4, 5, 0, 0)), (810, 192, 16896, 2, 1, (0, 64, 64, 4, 4, 6, 0, 0)),
    (53, 10256, 768, 3, 0, (1, 128, 64, 8, 4, 1, 0, 0)), (162, 38224, 640, 10, 1, (0, 128, 64, 8, 4, 1, 0, 1)),
    (101, 2112, 10240, 6, 1, (0, 128, 64, 8, 4, 2, 0, 0)), (145, 1744, 16128, 9, 1, (0, 128, 64, 8, 4, 2, 0, 1)),
    (50, 5120, 6784, 2, 1, (0, 128, 64, 8, 4, 3, 0, 0)), (22, 8016, 11008, 1, 1, (0, 128, 64, 8, 4, 4, 0, 0)),
    (282, 736, 9856, 8, 0, (1, 128, 64, 8, 4, 5, 0, 0)), (1046, 128, 17920, 35, 1, (0, 128, 64, 8, 4, 7, 0, 0)),
    (1668, 624, 1152, 51, 0, (1, 128, 128, 8, 4, 1, 0, 0)), (35, 32448, 7936, 1, 0, (1, 128, 128, 8, 4, 1, 0, 1)),
    (2221, 208, 8576, 64, 0, (1, 128, 128, 8, 4, 2, 0, 0)), (136, 4096, 15616, 4, 0, (1, 128, 128, 8, 4, 2, 0, 1)),
    (6633, 80, 7040, 58, 1, (0, 128, 128, 8, 4, 3, 0, 0)), (3687, 80, 12928, 59, 0, (1, 128, 128, 8, 4, 4, 0, 0)),
    (4675, 80, 13440, 28, 0, (1, 128, 128, 8, 4, 5, 0, 0)), (1, 16, 128, 65, 1, (0, 16, 16, 1, 0, 1, 0, 0)),
    (280, 16, 4224, 69, 0, (1, 16, 16, 9, 0, 1, 0, 0)), (1, 16, 128, 65, 0, (0, 16, 16, 1, 0, 1, 1, 0)),
    (67, 16, 128, 65, 0, (0, 16, 16, 1, 0, 1, 4, 0)), (83, 4624, 640, 84, 1, (0, 16, 16, 2, 0, 1, 0, 1)),
    (86, 4688, 640, 82, 0, (1, 16, 16, 2, 0, 1, 0, 1)), (114, 128, 17792, 115, 0, (0, 16, 16, 8, 0, 1, 1, 1)),
    (271, 272, 640, 121, 1, (0, 32, 16, 2, 0, 1, 0, 0)), (306, 432, 640, 76, 0, (1, 32, 16, 2, 0, 1, 0, 0)),
    (95, 176, 128, 97, 0, (0, 32, 16, 1, 0, 1, 1, 0)), (86, 208, 128, 79, 0, (0, 32, 16, 1, 0, 1, 4, 0)),
    (270, 16, 128, 66, 0, (0, 32, 16, 1, 0, 1, 16, 0)), (215, 3632, 640, 105, 1, (0, 32, 16, 2, 0, 1, 0, 1)),
    (211, 3120, 768, 104, 0, (1, 32, 16, 2, 0, 1, 0, 1)), (97, 9632, 256, 99, 0, (0, 32, 16, 1, 0, 1, 1, 1)),
    (113, 5840, 384, 111, 0, (0, 32, 16, 1, 0, 1, 4, 1)), (79, 416, 128, 79, 1, (0, 64, 16, 4, 0, 1, 0, 0)),
    (334, 800, 128, 82, 0, (1, 64, 16, 4, 0, 1, 0, 0)), (110, 15776, 128, 107, 1, (0, 64, 16, 4, 0, 1, 0, 1)),
    (95, 17808, 128, 96, 0, (1, 64, 16, 4, 0, 1, 0, 1)), (2639, 256, 512, 127, 0, (1, 128, 128, 4, 2, 1, 0, 0)),
    (2413, 816, 4352, 73, 1, (0, 128, 128, 4, 2, 1, 0, 1)), (17586, 400, 1152, 112, 1, (0, 256, 256, 8, 2, 1, 0, 0)),
    (13507, 64, 512, 87, 1, (0, 64, 64, 4, 4, 1, 0, 0)), (1185, 400, 8704, 73, 0, (1, 64, 64, 4, 4, 1, 0, 1)),
    (4367, 64, 5632, 112, 0, (1, 64, 64, 4, 4, 2, 0, 0)), (1328, 192, 17664, 75, 0, (1, 64, 64, 4, 4, 2, 0, 1)),
    (3329, 64, 8448, 67, 1, (0, 64, 64, 4, 4, 3, 0, 0)), (2223, 64, 17280, 126, 0, (1, 64, 64, 4, 4, 4, 0, 0)),
    (2858, 64, 12416, 100, 1, (0, 64, 64, 4, 4, 5, 0, 0)), (2624, 256, 640, 127, 0, (1, 128, 64, 8, 4, 1, 0, 0)),
    (1621, 3872, 640, 99, 1, (0, 128, 64, 8, 4, 1, 0, 1)), (1683, 128, 10112, 103, 0, (1, 128, 64, 8, 4, 2, 0, 0)),
    (2024, 128, 15872, 126, 0, (1, 128, 64, 8, 4, 2, 0, 1)), (2015, 128, 6784, 78, 1, (0, 128, 64, 8, 4, 3, 0, 0)),
    (4641, 208, 1152, 126, 0, (1, 128, 128, 8, 4, 1, 0, 0)), (2765, 336, 8960, 85, 0, (1, 128, 128, 8, 4, 1, 0, 1)),
    (4423, 80, 8576, 126, 0, (1, 128, 128, 8, 4, 2, 0, 0)), (4145, 128, 15488, 128, 0, (1, 128, 128, 8, 4, 2, 0, 1)),
    (5714, 80, 6784, 80, 0, (1, 128, 128, 8, 4, 3, 0, 0)),
]


def kind(call_experts, r):
    """What the kernels' compiled variants and their code for experts and slices distinguish."""
    by = min(call_experts, 1) + (call_experts > 64)
    return (by, r.room, r.channels, r.rows, r.slices > 1, r.past_caches) + (() if r.room else (r.rows_quantised, r.quantised_first))


@pytest.mark.parametrize("call", CALLS, ids=str)
def test_the_launch_of_a_call(lutq, call):
    M, N, K, experts, codes, launch = call
    assert lutq.calib_mx4_launch(M, N, K, experts, bool(codes)) == lutq.binding.Mx4Launch(*launch)


def test_no_kind_of_launch_is_missing(lutq):
    rng = random.Random(11)
    some = lambda a, b: round(math.exp(rng.uniform(math.log(a), math.log(b))))
    have = {kind(c[3], lutq.binding.Mx4Launch(*c[5])) for c in CALLS}
    for _ in range(40000):
        M, N, K, experts = some(1, 20000), 16 * some(1, 4096), 128 * some(1, 140), rng.choice((0, some(1, 64), some(65, 130)))
        for codes in (False, True):
            k = kind(experts, lutq.calib_mx4_launch(M, N, K, experts, codes))
            assert k in have, (M, N, K, experts, codes, k)


def test_refusals_of_the_question(lutq):
    for bad in ((0, 16, 128), (1, 8, 128), (1, 16, 64), (1 << 30, 16, 128), (1, 16, 128, -1), (1, 16, 128, 65537), (1, 16, 128, 0, False, 0),
                (1, 16, 128, 0, False, 4097)):
        with pytest.raises(lutq.LutqError):
            lutq.calib_mx4_launch(*bad)
    assert lutq.load_library().lutq_calib_mx4_launch(1, 16, 128, 0, 0, 256, None) == 1


# ---------------------------------------------------------------------------------------------------- on the device
def pack_on_device(codes, exponents):
    """The packed form by moving axes: codes [N, K / 2], exponents [N, K / 32], both bytes."""
    import torch
    N, KT = codes.shape[0], exponents.shape[1] // 4
    KQ = -(-KT // 4)
    c = codes.view(N // 16, 16, KT, 4, 16).permute(0, 2, 3, 1, 4).reshape(N // 16, -1)
    e = torch.zeros((N // 16, 16, KQ, 4, 4), dtype=torch.uint8, device=codes.device)
    e.view(N // 16, 16, 4 * KQ, 4)[:, :, :KT] = exponents.view(N // 16, 16, KT, 4)
    return torch.cat((c, e.permute(0, 2, 4, 1, 3).reshape(N // 16, -1)), 1).reshape(-1)


def values_on_device(codes, exponents):
    import torch
    table = torch.from_numpy(mx.TABLE).to(codes.device)
    v = torch.stack((table[(codes & 15).long()], table[(codes >> 4).long()]), -1).flatten(-2)
    return (v.unflatten(-1, (-1, 32)) * torch.exp2(exponents.double() - 127.0).unsqueeze(-1)).flatten(-2)


def test_packing_by_axes_is_the_packed_form():
    import torch
    rng = np.random.default_rng(2)
    for N, K in ((32, 128), (48, 640), (16, 1152)):
        codes, e = rng.integers(0, 16, (N, K), dtype=np.uint8), rng.integers(0, 256, (N, K // 32), dtype=np.uint8)
        rows = torch.from_numpy(mx.row_bytes(codes))
        assert np.array_equal(pack_on_device(rows, torch.from_numpy(e)).numpy(), mx.pack(codes, e))
        e[e == 255] = 3
        assert np.array_equal(values_on_device(rows, torch.from_numpy(e)).numpy(), mx.values(codes, e))


class Factors:
    """Random codes and exponents of both factors; X also as 16-bit values, which are exact and quantise to what stands for the same values."""

    def __init__(self, M, N, K, experts, dtype, seed):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        byte = lambda lo, hi, *shape: torch.randint(lo, hi, shape, generator=g, device="cuda", dtype=torch.uint8)
        self.codes, self.e = byte(0, 256, M, K // 2), byte(122, 130, M, K // 32)
        self.X = torch.cat([values_on_device(c, e).to(torch_dtype(dtype)) for c, e in zip(self.codes.split(4096), self.e.split(4096))])
        self.w = [(byte(0, 256, N, K // 2), byte(115, 123, N, K // 32)) for _ in range(max(1, experts))]
        self.packed = torch.stack([pack_on_device(*w) for w in self.w])
        self.dtype = dtype

    def args(self, codes):
        return (self.codes, self.e) if codes else (self.X, None)

    def worst(self, got, a, b, expert, quantum=0.0):
        """Largest error of rows a .. b of a result in units of its bound; every sum may be off by a quantum of fp32 as well."""
        import torch
        x, w = values_on_device(self.codes[a:b], self.e[a:b]), values_on_device(*self.w[expert])
        ref, mag = x @ w.T, x.abs() @ w.abs().T
        mantissa, least, largest = (10, -14, 65504.0) if self.dtype == "f16" else (7, -126, 3.3895313892515355e38)
        exponent = torch.frexp(ref.abs().clamp(max=largest)).exponent.long() - 1
        step = torch.exp2((exponent.clamp(min=least) - mantissa).double())
        off = (got[a:b].double() - ref).abs() / (0.5 * step + (x.shape[1] // 128 + 12) * (2.0 ** -22 * mag + quantum))
        return off.max().item() if not off.isnan().any().item() else math.inf


def uneven(M, experts, seed):
    """Offsets of uneven experts, the first and others without rows; a row before the first and two behind the last where there are many."""
    rng = random.Random(seed)
    first, behind = (1, 2) if M > 8 else (0, 0)
    weights = [rng.paretovariate(1.2) if i and rng.random() < 0.8 else 0.0 for i in range(experts)]
    weights[-1] += 1.0
    counts = [0] * experts
    for g in rng.choices(range(experts), weights, k=M - first - behind):
        counts[g] += 1
    return [first + sum(counts[:g]) for g in range(experts + 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("call", CALLS, ids=str)
def test_a_call_of_every_launch(lutq, call):
    import torch
    M, N, K, experts, codes, launch = call
    units = torch.cuda.get_device_properties(0).multi_processor_count
    assert lutq.calib_mx4_launch(M, N, K, experts, bool(codes), units) == lutq.binding.Mx4Launch(*launch)
    index = CALLS.index(call)
    p = Factors(M, N, K, experts, ("f16", "bf16")[index % 2], index)
    ws = lutq.new_mx4_workspace(M, N, K, max(1, experts))
    offsets = uneven(M, experts, index) if experts else None
    on_device = torch.tensor(offsets, dtype=torch.int32, device="cuda") if experts else None
    for as_codes in ((True, False) if launch[4] else (bool(codes),)):   # (a tile's launch is the same for both)
        guarded = torch.full((M + 32, N), -7.0, dtype=torch_dtype(p.dtype), device="cuda")
        y = guarded[16:16 + M]
        x, e = p.args(as_codes)
        again = torch.full_like(y, -7.0)
        if experts:
            lutq.lutq_mx4_matmul_grouped(x, p.packed, on_device, y, ws, x_scales=e)
            lutq.lutq_mx4_matmul_grouped(x, p.packed, on_device, again, ws, x_scales=e)
            for g, (a, b) in enumerate(zip(offsets, offsets[1:])):
                if b > a:
                    worst = p.worst(y, a, b, g)
                    assert worst <= 1.0, (as_codes, g, worst)
            assert (y[:offsets[0]] == -7.0).all().item() and (y[offsets[-1]:] == -7.0).all().item()
        else:
            lutq.lutq_mx4_matmul(x, p.packed, y, ws, x_scales=e)
            lutq.lutq_mx4_matmul(x, p.packed, again, ws, x_scales=e)
            worst = p.worst(y, 0, M, 0)
            assert worst <= 1.0, (as_codes, worst)
        assert (guarded[:16] == -7.0).all().item() and (guarded[16 + M:] == -7.0).all().item() and not ws[:65536].any().item()
        assert torch.equal(y, again)


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
def test_more_pieces_of_rows_than_one_launch_takes(lutq, dense):
    """A launch has at most 65535 workgroups along the rows, four pieces of sixteen rows each here: a second launch has the rest."""
    import torch
    M, N, K = 65535 * 64 + 40, 16, 128
    r = lutq.calib_mx4_launch(M, N, K, 0, not dense)
    assert (r.room, r.channels, r.waves) == (0, 64, 4)
    p = Factors(M, N, K, 0, "bf16", 5)
    y = torch.full((M + 16, N), -7.0, dtype=torch.bfloat16, device="cuda")
    x, e = p.args(not dense)
    lutq.lutq_mx4_matmul(x, p.packed, y[:M], lutq.new_mx4_workspace(M, N, K), x_scales=e)
    for a in range(0, M, 1 << 19):
        worst = p.worst(y, a, min(M, a + (1 << 19)), 0)
        assert worst <= 1.0, (a, worst)
    assert (y[M:] == -7.0).all().item()


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
def test_as_many_experts_as_there_may_be(lutq, dense):
    """65536 of them, 70000 rows: more pieces than a launch has workgroups along the rows."""
    import torch
    experts, M, N, K = 65536, 70000, 16, 640
    assert lutq.calib_mx4_launch(M, N, K, experts, not dense).channels == 16
    p = Factors(M, experts * N, K, 0, "bf16", 6)
    g = torch.Generator().manual_seed(7)
    expert = torch.randint(0, experts, (M - 3,), generator=g).sort().values
    offsets = torch.cat((torch.zeros(1, dtype=torch.long), torch.bincount(expert, minlength=experts).cumsum(0))).int().cuda()
    expert = expert.cuda()
    y = torch.full((M, N), -7.0, dtype=torch.bfloat16, device="cuda")
    x, e = p.args(not dense)
    lutq.lutq_mx4_matmul_grouped(x, p.packed.view(experts, -1), offsets, y, lutq.new_mx4_workspace(M, N, K, experts), x_scales=e)
    codes, scales = (t.view(experts, N, -1) for t in p.w[0])
    for a in range(0, M - 3, 4096):
        mine = expert[a:a + 4096]
        b = a + mine.numel()
        products = values_on_device(codes[mine].flatten(0, 1), scales[mine].flatten(0, 1)).view(-1, N, K) * values_on_device(p.codes[a:b], p.e[a:b])[:, None]
        ref, mag = products.sum(-1), products.abs().sum(-1)
        step = torch.exp2((torch.frexp(ref).exponent - 1).clamp(min=-126).double() - 7)
        assert ((y[a:b].double() - ref).abs() <= 0.5 * step + (K // 128 + 12) * 2.0 ** -22 * mag).all().item(), a
    assert (y[M - 3:] == -7.0).all().item()
