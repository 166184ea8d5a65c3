"""Every launch that the 8-bit products choose, by the call that asks which it is, each against the definition in fp64.

The launches are chosen by estimated times, so a new estimate may send a size to another one: the table below has the launch of each
call, and is checked before the call is made; a sweep over sizes finds the kinds of launches that the table lacks.

Bounds as in test_fp8.py.  The codes have four and five binades, so the instruction cuts nothing off."""
import math
import random

import numpy as np
import pytest

from gpu_util import torch_dtype
from oracle import fp8_oracle as fx
from test_mx4_launches import uneven

# form, rows, N (F; of weight_grad: N, K and M are meant by M, N and K), K, experts (0: without), whether X is codes, and the launch: X quantised first,
# channels and rows at a time, wavefronts, steps of room, slices of K, how it is streamed (0: tiles), past the caches
CALLS = [
    ("gated", 598, 1664, 512, 0, 0, (1, 128, 128, 8, 4, 1, 0, 0)), ("gated", 322, 13824, 128, 0, 1, (0, 128, 128, 8, 4, 1, 0, 0)),
    ("gated", 451, 1152, 4864, 0, 1, (0, 128, 128, 8, 4, 3, 0, 0)), ("gated", 536, 640, 6784, 0, 0, (1, 128, 128, 8, 4, 5, 0, 0)),
    ("gated", 275, 1664, 384, 0, 1, (0, 128, 64, 8, 4, 1, 0, 0)), ("gated", 132, 11136, 128, 0, 1, (0, 128, 64, 8, 4, 1, 0, 0)),
    ("gated", 386, 640, 3840, 0, 0, (1, 128, 64, 8, 4, 3, 0, 0)), ("gated", 132, 768, 11904, 0, 0, (1, 128, 64, 8, 4, 7, 0, 0)),
    ("gated", 328, 5504, 256, 0, 1, (0, 256, 128, 8, 3, 1, 0, 0)), ("gated", 1104, 7424, 256, 0, 0, (1, 256, 128, 8, 3, 1, 0, 0)),
    ("gated", 1669, 2432, 256, 0, 0, (1, 256, 192, 8, 2, 1, 0, 0)), ("gated", 1432, 11008, 256, 0, 1, (0, 256, 192, 8, 2, 1, 0, 0)),
    ("gated", 252, 16640, 256, 0, 0, (1, 256, 256, 8, 2, 1, 0, 0)), ("gated", 2078, 9728, 384, 0, 0, (1, 256, 256, 8, 2, 1, 0, 0)),
    ("gated", 1, 128, 128, 0, 0, (0, 32, 16, 1, 2, 1, 1, 0)), ("gated", 1, 128, 256, 0, 0, (0, 32, 16, 2, 2, 1, 1, 0)),
    ("gated", 1, 128, 1024, 0, 0, (0, 32, 16, 8, 2, 1, 1, 0)), ("gated", 1, 7808, 2688, 0, 0, (0, 32, 16, 4, 2, 1, 1, 1)),
    ("gated", 2, 2688, 7808, 0, 0, (0, 32, 16, 8, 2, 1, 1, 1)), ("gated", 1, 128, 128, 0, 1, (0, 32, 16, 1, 2, 1, 2, 0)),
    ("gated", 1, 128, 256, 0, 1, (0, 32, 16, 2, 2, 1, 2, 0)), ("gated", 1, 128, 1024, 0, 1, (0, 32, 16, 8, 2, 1, 2, 0)),
    ("gated", 1, 12672, 1664, 0, 1, (0, 32, 16, 4, 2, 1, 2, 1)), ("gated", 3, 3584, 5888, 0, 1, (0, 32, 16, 8, 2, 1, 2, 1)),
    ("gated", 9, 128, 128, 0, 1, (0, 32, 16, 1, 2, 1, 3, 0)), ("gated", 9, 128, 256, 0, 1, (0, 32, 16, 2, 2, 1, 3, 0)),
    ("gated", 9, 128, 1024, 0, 1, (0, 32, 16, 8, 2, 1, 3, 0)), ("gated", 9, 4224, 4992, 0, 1, (0, 32, 16, 4, 2, 1, 3, 1)),
    ("gated", 12, 2688, 7808, 0, 0, (1, 32, 16, 8, 2, 1, 3, 1)), ("gated", 17, 128, 128, 0, 1, (0, 64, 64, 4, 4, 1, 0, 0)),
    ("gated", 246, 640, 3328, 0, 1, (0, 64, 64, 4, 4, 3, 0, 0)), ("gated", 187, 384, 11264, 0, 1, (0, 64, 64, 4, 4, 7, 0, 0)),
    ("gated", 1211, 1408, 768, 1, 1, (0, 128, 128, 8, 4, 1, 0, 0)), ("gated", 236, 1408, 6784, 1, 0, (1, 128, 128, 8, 4, 3, 0, 0)),
    ("gated", 430, 640, 9088, 1, 0, (1, 128, 128, 8, 4, 4, 0, 0)), ("gated", 206, 2304, 384, 1, 1, (0, 128, 64, 8, 4, 1, 0, 0)),
    ("gated", 213, 8576, 128, 1, 1, (0, 128, 64, 8, 4, 1, 0, 0)), ("gated", 198, 768, 6912, 1, 1, (0, 128, 64, 8, 4, 4, 0, 0)),
    ("gated", 1913, 1280, 256, 1, 1, (0, 256, 128, 8, 3, 1, 0, 0)), ("gated", 1567, 5120, 128, 1, 1, (0, 256, 128, 8, 3, 1, 0, 0)),
    ("gated", 4914, 2432, 3456, 1, 0, (1, 256, 192, 8, 2, 1, 0, 0)), ("gated", 5740, 2688, 2304, 1, 0, (1, 256, 192, 8, 2, 1, 0, 0)),
    ("gated", 12947, 1280, 1792, 1, 1, (0, 256, 256, 8, 2, 1, 0, 0)), ("gated", 5146, 4224, 1152, 1, 0, (1, 256, 256, 8, 2, 1, 0, 0)),
    ("gated", 1, 128, 128, 1, 0, (0, 32, 16, 1, 2, 1, 1, 0)), ("gated", 1, 128, 256, 1, 0, (0, 32, 16, 2, 2, 1, 1, 0)),
    ("gated", 1, 128, 1024, 1, 0, (0, 32, 16, 8, 2, 1, 1, 0)), ("gated", 43, 3840, 128, 43, 0, (0, 32, 16, 1, 2, 1, 1, 1)),
    ("gated", 9, 2944, 896, 8, 0, (0, 32, 16, 4, 2, 1, 1, 1)), ("gated", 3, 896, 7808, 3, 0, (0, 32, 16, 8, 2, 1, 1, 1)),
    ("gated", 1, 128, 128, 1, 1, (0, 32, 16, 1, 2, 1, 2, 0)), ("gated", 1, 128, 256, 1, 1, (0, 32, 16, 2, 2, 1, 2, 0)),
    ("gated", 1, 128, 1024, 1, 1, (0, 32, 16, 8, 2, 1, 2, 0)), ("gated", 3, 1664, 4224, 3, 1, (0, 32, 16, 4, 2, 1, 2, 1)),
    ("gated", 6, 512, 13696, 3, 0, (1, 32, 16, 8, 2, 1, 2, 1)), ("gated", 9, 128, 128, 3, 1, (0, 32, 16, 1, 2, 1, 3, 0)),
    ("gated", 9, 128, 384, 1, 1, (0, 32, 16, 3, 2, 1, 3, 0)), ("gated", 9, 128, 1024, 1, 1, (0, 32, 16, 8, 2, 1, 3, 0)),
    ("gated", 15, 15104, 128, 11, 1, (0, 32, 16, 1, 2, 1, 3, 1)), ("gated", 24, 1664, 1152, 11, 1, (0, 32, 16, 2, 2, 1, 3, 1)),
    ("gated", 11, 384, 5504, 10, 1, (0, 32, 16, 8, 2, 1, 3, 1)), ("gated", 5, 128, 128, 1, 0, (1, 64, 64, 4, 4, 1, 0, 0)),
    ("gated", 131, 11648, 128, 1, 0, (1, 64, 64, 4, 4, 1, 0, 0)), ("gated", 285, 256, 2688, 1, 1, (0, 64, 64, 4, 4, 3, 0, 0)),
    ("gated", 141, 384, 6272, 1, 1, (0, 64, 64, 4, 4, 7, 0, 0)), ("gated_saved", 259, 3840, 256, 0, 0, (1, 128, 128, 8, 4, 1, 0, 0)),
    ("gated_saved", 1231, 3328, 256, 0, 1, (0, 128, 128, 8, 4, 1, 0, 0)), ("gated_saved", 657, 768, 2816, 0, 1, (0, 128, 128, 8, 4, 3, 0, 0)),
    ("gated_saved", 459, 768, 3840, 0, 1, (0, 128, 128, 8, 4, 5, 0, 0)), ("gated_saved", 268, 1664, 256, 0, 0, (1, 128, 64, 8, 4, 1, 0, 0)),
    ("gated_saved", 273, 11136, 128, 0, 0, (1, 128, 64, 8, 4, 1, 0, 0)), ("gated_saved", 310, 1024, 2944, 0, 1, (0, 128, 64, 8, 4, 3, 0, 0)),
    ("gated_saved", 372, 384, 9344, 0, 0, (1, 128, 64, 8, 4, 7, 0, 0)), ("gated_saved", 788, 2560, 128, 0, 0, (1, 256, 128, 8, 3, 1, 0, 0)),
    ("gated_saved", 907, 8960, 128, 0, 0, (1, 256, 128, 8, 3, 1, 0, 0)), ("gated_saved", 1, 128, 128, 0, 0, (0, 32, 16, 1, 2, 1, 1, 0)),
    ("gated_saved", 1, 128, 256, 0, 0, (0, 32, 16, 2, 2, 1, 1, 0)), ("gated_saved", 1, 128, 1024, 0, 0, (0, 32, 16, 8, 2, 1, 1, 0)),
    ("gated_saved", 3, 7808, 2688, 0, 0, (0, 32, 16, 4, 2, 1, 1, 1)), ("gated_saved", 2, 4992, 4224, 0, 0, (0, 32, 16, 8, 2, 1, 1, 1)),
    ("gated_saved", 1, 128, 128, 0, 1, (0, 32, 16, 1, 2, 1, 2, 0)), ("gated_saved", 1, 128, 256, 0, 1, (0, 32, 16, 2, 2, 1, 2, 0)),
    ("gated_saved", 1, 128, 1024, 0, 1, (0, 32, 16, 8, 2, 1, 2, 0)), ("gated_saved", 1, 18304, 1152, 0, 1, (0, 32, 16, 4, 2, 1, 2, 1)),
    ("gated_saved", 3, 2944, 7168, 0, 1, (0, 32, 16, 8, 2, 1, 2, 1)), ("gated_saved", 9, 128, 128, 0, 1, (0, 32, 16, 1, 2, 1, 3, 0)),
    ("gated_saved", 9, 128, 256, 0, 1, (0, 32, 16, 2, 2, 1, 3, 0)), ("gated_saved", 9, 128, 1024, 0, 1, (0, 32, 16, 8, 2, 1, 3, 0)),
    ("gated_saved", 9, 7168, 2944, 0, 0, (1, 32, 16, 4, 2, 1, 3, 1)), ("gated_saved", 9, 2688, 7808, 0, 0, (1, 32, 16, 8, 2, 1, 3, 1)),
    ("gated_saved", 18, 128, 128, 0, 0, (1, 64, 64, 4, 4, 1, 0, 0)), ("gated_saved", 35, 1920, 9088, 0, 1, (0, 64, 64, 4, 4, 4, 0, 0)),
    ("gated_saved", 33, 1152, 15872, 0, 1, (0, 64, 64, 4, 4, 7, 0, 0)), ("gated_saved", 887, 2048, 384, 1, 1, (0, 128, 128, 8, 4, 1, 0, 0)),
    ("gated_saved", 363, 896, 3968, 2, 0, (1, 128, 128, 8, 4, 3, 0, 0)), ("gated_saved", 291, 1024, 5760, 1, 0, (1, 128, 128, 8, 4, 4, 0, 0)),
    ("gated_saved", 583, 896, 256, 1, 1, (0, 128, 64, 8, 4, 1, 0, 0)), ("gated_saved", 663, 3200, 128, 1, 1, (0, 128, 64, 8, 4, 1, 0, 0)),
    ("gated_saved", 495, 512, 2688, 1, 0, (1, 128, 64, 8, 4, 2, 0, 0)), ("gated_saved", 589, 3584, 256, 1, 1, (0, 256, 128, 8, 3, 1, 0, 0)),
    ("gated_saved", 964, 8704, 128, 1, 0, (1, 256, 128, 8, 3, 1, 0, 0)), ("gated_saved", 1, 128, 128, 1, 0, (0, 32, 16, 1, 2, 1, 1, 0)),
    ("gated_saved", 1, 128, 256, 1, 0, (0, 32, 16, 2, 2, 1, 1, 0)), ("gated_saved", 2, 128, 1024, 1, 0, (0, 32, 16, 8, 2, 1, 1, 0)),
    ("gated_saved", 29, 5760, 128, 29, 0, (0, 32, 16, 1, 2, 1, 1, 1)), ("gated_saved", 8, 2944, 896, 8, 0, (0, 32, 16, 4, 2, 1, 1, 1)),
    ("gated_saved", 3, 4224, 4992, 1, 0, (0, 32, 16, 8, 2, 1, 1, 1)), ("gated_saved", 1, 128, 128, 1, 1, (0, 32, 16, 1, 2, 1, 2, 0)),
    ("gated_saved", 1, 128, 256, 1, 1, (0, 32, 16, 2, 2, 1, 2, 0)), ("gated_saved", 2, 128, 1024, 1, 1, (0, 32, 16, 8, 2, 1, 2, 0)),
    ("gated_saved", 3, 1408, 4992, 3, 1, (0, 32, 16, 4, 2, 1, 2, 1)), ("gated_saved", 7, 384, 11008, 5, 0, (1, 32, 16, 8, 2, 1, 2, 1)),
    ("gated_saved", 9, 128, 128, 3, 1, (0, 32, 16, 1, 2, 1, 3, 0)), ("gated_saved", 9, 128, 256, 1, 1, (0, 32, 16, 2, 2, 1, 3, 0)),
    ("gated_saved", 13, 128, 1024, 1, 1, (0, 32, 16, 8, 2, 1, 3, 0)), ("gated_saved", 21, 7808, 128, 21, 1, (0, 32, 16, 1, 2, 1, 3, 1)),
    ("gated_saved", 20, 5504, 384, 10, 1, (0, 32, 16, 2, 2, 1, 3, 1)), ("gated_saved", 16, 1920, 5504, 2, 1, (0, 32, 16, 8, 2, 1, 3, 1)),
    ("gated_saved", 5, 128, 128, 1, 1, (0, 64, 64, 4, 4, 1, 0, 0)), ("gated_saved", 390, 384, 1280, 1, 1, (0, 64, 64, 4, 4, 3, 0, 0)),
    ("gated_saved", 231, 256, 4992, 1, 1, (0, 64, 64, 4, 4, 7, 0, 0)), ("matmul", 777, 2640, 512, 0, 0, (1, 128, 128, 8, 4, 1, 0, 0)),
    ("matmul", 1285, 7792, 128, 0, 0, (1, 128, 128, 8, 4, 1, 0, 0)), ("matmul", 493, 2064, 4992, 0, 0, (1, 128, 128, 8, 4, 3, 0, 0)),
    ("matmul", 658, 992, 6912, 0, 0, (1, 128, 128, 8, 4, 5, 0, 0)), ("matmul", 716, 1360, 384, 0, 1, (0, 128, 64, 8, 4, 1, 0, 0)),
    ("matmul", 769, 5104, 128, 0, 1, (0, 128, 64, 8, 4, 1, 0, 0)), ("matmul", 451, 1168, 3840, 0, 1, (0, 128, 64, 8, 4, 3, 0, 0)),
    ("matmul", 322, 672, 11392, 0, 0, (1, 128, 64, 8, 4, 7, 0, 0)), ("matmul", 1, 16, 128, 0, 0, (0, 16, 16, 1, 4, 1, 1, 0)),
    ("matmul", 1, 16, 256, 0, 0, (0, 16, 16, 2, 4, 1, 1, 0)), ("matmul", 1, 16, 1024, 0, 0, (0, 16, 16, 8, 4, 1, 1, 0)),
    ("matmul", 1, 32896, 1280, 0, 0, (0, 16, 16, 4, 4, 1, 1, 1)), ("matmul", 3, 6304, 6656, 0, 0, (0, 16, 16, 8, 4, 1, 1, 1)),
    ("matmul", 1, 16, 128, 0, 1, (0, 16, 16, 1, 4, 1, 2, 0)), ("matmul", 1, 16, 256, 0, 1, (0, 16, 16, 2, 4, 1, 2, 0)),
    ("matmul", 1, 16, 1024, 0, 1, (0, 16, 16, 8, 4, 1, 2, 0)), ("matmul", 1, 5856, 7168, 0, 1, (0, 16, 16, 4, 4, 1, 2, 1)),
    ("matmul", 2, 3856, 10880, 0, 1, (0, 16, 16, 8, 4, 1, 2, 1)), ("matmul", 9, 16, 128, 0, 1, (0, 16, 16, 1, 4, 1, 3, 0)),
    ("matmul", 9, 16, 256, 0, 1, (0, 16, 16, 2, 4, 1, 3, 0)), ("matmul", 9, 16, 1024, 0, 1, (0, 16, 16, 8, 4, 1, 3, 0)),
    ("matmul", 9, 6192, 6784, 0, 1, (0, 16, 16, 4, 4, 1, 3, 1)), ("matmul", 9, 4048, 10368, 0, 0, (1, 16, 16, 8, 4, 1, 3, 1)),
    ("matmul", 1690, 2416, 256, 0, 0, (1, 256, 128, 8, 3, 1, 0, 0)), ("matmul", 3715, 4384, 256, 0, 0, (1, 256, 128, 8, 3, 1, 0, 0)),
    ("matmul", 1514, 5392, 256, 0, 1, (0, 256, 192, 8, 2, 1, 0, 0)), ("matmul", 1051, 29312, 256, 0, 0, (1, 256, 192, 8, 2, 1, 0, 0)),
    ("matmul", 200, 33520, 256, 0, 0, (1, 256, 256, 8, 2, 1, 0, 0)), ("matmul", 4225, 9584, 384, 0, 1, (0, 256, 256, 8, 2, 1, 0, 0)),
    ("matmul", 17, 16, 128, 0, 1, (0, 64, 64, 4, 4, 1, 0, 0)), ("matmul", 16491, 304, 128, 0, 1, (0, 64, 64, 4, 4, 1, 0, 0)),
    ("matmul", 372, 576, 2432, 0, 1, (0, 64, 64, 4, 4, 4, 0, 0)), ("matmul", 155, 752, 6272, 0, 0, (1, 64, 64, 4, 4, 7, 0, 0)),
    ("matmul", 1704, 1808, 768, 1, 0, (1, 128, 128, 8, 4, 1, 0, 0)), ("matmul", 10012, 800, 256, 1, 1, (0, 128, 128, 8, 4, 1, 0, 0)),
    ("matmul", 576, 1296, 6912, 1, 0, (1, 128, 128, 8, 4, 3, 0, 0)), ("matmul", 1049, 464, 8704, 1, 1, (0, 128, 128, 8, 4, 5, 0, 0)),
    ("matmul", 581, 1760, 384, 1, 0, (1, 128, 64, 8, 4, 1, 0, 0)), ("matmul", 772, 5264, 128, 1, 1, (0, 128, 64, 8, 4, 1, 0, 0)),
    ("matmul", 373, 1456, 5120, 1, 1, (0, 128, 64, 8, 4, 2, 0, 0)), ("matmul", 1, 16, 128, 1, 0, (0, 16, 16, 1, 4, 1, 1, 0)),
    ("matmul", 1, 16, 256, 1, 0, (0, 16, 16, 2, 4, 1, 1, 0)), ("matmul", 1, 16, 1024, 1, 0, (0, 16, 16, 8, 4, 1, 1, 0)),
    ("matmul", 48, 11712, 128, 29, 0, (0, 16, 16, 1, 4, 1, 1, 1)), ("matmul", 8, 4256, 1408, 7, 0, (0, 16, 16, 4, 4, 1, 1, 1)),
    ("matmul", 3, 944, 14848, 3, 0, (0, 16, 16, 8, 4, 1, 1, 1)), ("matmul", 1, 16, 128, 1, 1, (0, 16, 16, 1, 4, 1, 2, 0)),
    ("matmul", 1, 16, 256, 1, 1, (0, 16, 16, 2, 4, 1, 2, 0)), ("matmul", 1, 16, 1024, 1, 1, (0, 16, 16, 8, 4, 1, 2, 0)),
    ("matmul", 2, 3152, 6656, 2, 1, (0, 16, 16, 4, 4, 1, 2, 1)), ("matmul", 6, 1072, 13056, 3, 1, (0, 16, 16, 8, 4, 1, 2, 1)),
    ("matmul", 12, 16, 128, 3, 1, (0, 16, 16, 1, 4, 1, 3, 0)), ("matmul", 9, 16, 384, 1, 1, (0, 16, 16, 3, 4, 1, 3, 0)),
    ("matmul", 11, 16, 1152, 1, 1, (0, 16, 16, 8, 4, 1, 3, 0)), ("matmul", 46, 14352, 128, 23, 1, (0, 16, 16, 1, 4, 1, 3, 1)),
    ("matmul", 14, 1808, 1792, 13, 1, (0, 16, 16, 2, 4, 1, 3, 1)), ("matmul", 10, 2688, 15616, 1, 0, (1, 16, 16, 8, 4, 1, 3, 1)),
    ("matmul", 2755, 1696, 256, 1, 0, (1, 256, 128, 8, 3, 1, 0, 0)), ("matmul", 789, 19504, 128, 1, 0, (1, 256, 128, 8, 3, 1, 0, 0)),
    ("matmul", 4473, 4800, 4480, 1, 0, (1, 256, 192, 8, 2, 1, 0, 0)), ("matmul", 2916, 9232, 2944, 1, 1, (0, 256, 192, 8, 2, 1, 0, 0)),
    ("matmul", 17289, 1664, 2176, 1, 0, (1, 256, 256, 8, 2, 1, 0, 0)), ("matmul", 6387, 5280, 1920, 1, 0, (1, 256, 256, 8, 2, 1, 0, 0)),
    ("matmul", 5, 16, 128, 1, 0, (1, 64, 64, 4, 4, 1, 0, 0)), ("matmul", 130, 23728, 128, 1, 1, (0, 64, 64, 4, 4, 1, 0, 0)),
    ("matmul", 195, 880, 2304, 1, 1, (0, 64, 64, 4, 4, 3, 0, 0)), ("matmul", 99, 736, 7168, 1, 0, (1, 64, 64, 4, 4, 7, 0, 0)),
    ("weight_grad", 800, 2544, 512, 0, 1, (0, 128, 128, 8, 4, 1, 0, 0)), ("weight_grad", 784, 12624, 128, 0, 1, (0, 128, 128, 8, 4, 1, 0, 0)),
    ("weight_grad", 928, 1120, 4864, 0, 1, (0, 128, 128, 8, 4, 3, 0, 0)), ("weight_grad", 464, 1424, 7040, 0, 1, (0, 128, 128, 8, 4, 5, 0, 0)),
    ("weight_grad", 784, 1232, 384, 0, 1, (0, 128, 64, 8, 4, 1, 0, 0)), ("weight_grad", 784, 5104, 128, 0, 1, (0, 128, 64, 8, 4, 1, 0, 0)),
    ("weight_grad", 464, 1152, 3840, 0, 1, (0, 128, 64, 8, 4, 3, 0, 0)), ("weight_grad", 304, 800, 11392, 0, 1, (0, 128, 64, 8, 4, 7, 0, 0)),
    ("weight_grad", 1680, 2416, 256, 0, 1, (0, 256, 128, 8, 3, 1, 0, 0)), ("weight_grad", 4816, 3360, 256, 0, 1, (0, 256, 128, 8, 3, 1, 0, 0)),
    ("weight_grad", 5456, 1424, 256, 0, 1, (0, 256, 192, 8, 2, 1, 0, 0)), ("weight_grad", 2208, 14576, 256, 0, 1, (0, 256, 192, 8, 2, 1, 0, 0)),
    ("weight_grad", 208, 33968, 256, 0, 1, (0, 256, 256, 8, 2, 1, 0, 0)), ("weight_grad", 4320, 9568, 384, 0, 1, (0, 256, 256, 8, 2, 1, 0, 0)),
    ("weight_grad", 16, 16, 128, 0, 1, (0, 64, 64, 4, 4, 1, 0, 0)), ("weight_grad", 18384, 272, 128, 0, 1, (0, 64, 64, 4, 4, 1, 0, 0)),
    ("weight_grad", 16, 16, 2304, 0, 1, (0, 64, 64, 4, 4, 3, 0, 0)), ("weight_grad", 16, 16, 6272, 0, 1, (0, 64, 64, 4, 4, 7, 0, 0)),
]


def kind(form, M, N, experts, codes, r):
    """What the kernels' compiled variants and their code for experts, slices and several tiles of a workgroup distinguish."""
    k = (form, min(experts, 1), r.channels, r.rows, r.streamed)
    if r.streamed:
        return k + (r.past_caches, not codes and not r.quantised_first, (r.waves > 1) + (r.waves == 8))
    tiles = -(-N * (2 if form.startswith("gated") else 1) // r.channels) * -(-M // r.rows)
    joined_at_once = 3 if (r.channels, r.rows) == (128, 128) else 6
    return k + ((r.slices > 1) + (r.slices > joined_at_once), r.slices == 1 and tiles > (1024 if r.channels == 64 else 512))


@pytest.mark.parametrize("call", CALLS, ids=str)
def test_the_launch_of_a_call(lutq, call):
    form, M, N, K, experts, codes, launch = call
    assert lutq.calib_fp8_launch(M, N, K, experts, form, bool(codes)) == lutq.binding.Fp8Launch(*launch)


def test_no_kind_of_launch_is_missing(lutq):
    rng = random.Random(12)
    some = lambda a, b: round(math.exp(rng.uniform(math.log(a), math.log(b))))
    have = {kind(c[0], c[1], c[2], c[4], c[5], lutq.binding.Fp8Launch(*c[6])) for c in CALLS}
    for _ in range(40000):
        form = rng.choice(("matmul", "matmul", "gated", "gated_saved", "weight_grad"))
        experts = 0 if form == "weight_grad" or rng.random() < 0.5 else some(1, 64)
        codes = form == "weight_grad" or rng.random() < 0.5
        M, N, K = some(1, 20000), 16 * some(1, 2600), 128 * some(1, 130)
        if form == "weight_grad":
            M = 16 * -(-M // 16)
        if form.startswith("gated"):
            N = 128 * some(1, 160)
        if N * K * max(1, experts) * (2 if form.startswith("gated") else 1) <= 4e8:
            assert kind(form, M, N, experts, codes, lutq.calib_fp8_launch(M, N, K, experts, form, codes)) in have, (form, M, N, K, experts, codes)


def test_no_launch_has_more_wavefronts_than_its_kernel_is_built_for(lutq):
    """Eight, of a workgroup that streams as of one of tiles."""
    rng = random.Random(13)
    some = lambda a, b: round(math.exp(rng.uniform(math.log(a), math.log(b))))
    seen = set()
    for _ in range(10000):
        form, experts = rng.choice(("matmul", "gated", "gated_saved")), rng.choice((0, some(1, 1000)))
        r = lutq.calib_fp8_launch(some(1, 60), 128 * some(1, 1000), 128 * some(1, 4000), experts, form, rng.random() < 0.5, some(1, 4096))
        seen.add((r.streamed > 0, r.waves))
    assert {w for _, w in seen} <= set(range(1, 9)) and (True, 8) in seen


def test_refusals_of_the_question(lutq):
    import ctypes
    f = lutq.load_library().lutq_calib_fp8_launch
    out = (ctypes.c_int * 8)()
    assert f(4, 128, 128, 0, 0, 0, 256, None) == 1
    for bad in ((0, 128, 128, 0, 0, 0, 256), (4, 24, 128, 0, 0, 0, 256), (4, 64, 128, 0, 1, 0, 256), (4, 64, 128, 0, 3, 0, 256), (4, 128, 128, -1, 0, 0, 256),
                (4, 128, 128, 0, 4, 0, 256), (4, 128, 128, 0, 2, 0, 256), (4, 128, 128, 1, 2, 1, 256), (4, 128, 128, 0, 0, 0, 0), (4, 128, 128, 0, 0, 0, 4097)):
        assert f(*bad, out) == 4
    for cus in (1, 64, 256, 304, 4096):
        assert f(4, 128, 128, 0, 0, 0, cus, out) == 0


# ---------------------------------------------------------------------------------------------------- on the device
class Factors:
    """Random factors on the device: codes with scales, and X also as 16-bit values."""

    def __init__(self, lutq, form, M, N, K, experts, dtype, seed):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        rand = lambda *shape: torch.rand(shape, generator=g, device="cuda")
        def codes(binades, *shape):
            c = torch.randint(8 * (14 - binades), 8 * 14, shape, generator=g, device="cuda", dtype=torch.uint8)
            c += 128 * torch.randint(0, 2, shape, generator=g, device="cuda", dtype=torch.uint8)
            return c
        self.table = torch.from_numpy(fx.TABLE).cuda()
        self.form, self.M, self.N, self.K, self.dtype = form, M, N, K, dtype
        rows, e = 2 * N if form.startswith("gated") else N, max(1, experts)
        self.W = codes(5, e, rows, K)
        size = (K * 6e3) ** -0.5 if form.startswith("gated") else 2.0 ** -12
        if form == "weight_grad":
            self.codes, self.s, self.sw = codes(4, M, K), torch.exp2((6 * rand(K // 128, M)).floor() - 3), torch.exp2((6 * rand(1, K // 128, N)).floor() - 15)
            return
        self.sw = torch.exp2(-3 * rand(e, -(-rows // 128), K // 128)) * size
        x = torch.exp2(-2.9 * rand(M, K)).view(M, K // 128, 128) * torch.exp2((6 * rand(M, K // 128, 1)).floor() - 3)
        self.X = (x.view(M, K) * (1 - 2 * torch.randint(0, 2, (M, K), generator=g, device="cuda"))).to(torch_dtype(dtype))
        self.codes, self.s = torch.empty((M, K), dtype=torch.uint8, device="cuda"), torch.empty((K // 128, M), dtype=torch.float32, device="cuda")
        lutq.lutq_fp8_quantize(self.X, self.codes, self.s)

    def args(self, codes):
        return (self.codes, self.s) if codes else (self.X, None)

    def row_values(self, codes, scales):
        return (self.table[codes.long()].unflatten(-1, (-1, 128)) * scales.double().T.unsqueeze(-1)).flatten(-2)

    def sums(self, a, b, expert, first=0, end=None):
        """Of rows a .. b with weights first .. end of an expert: sums, and of magnitudes."""
        import torch
        ref, mag = [], []
        x, n = self.row_values(self.codes[a:b], self.s[:, a:b]), max(16, (1 << 26) // self.K // 128 * 128)
        for at in range(first, self.W.shape[1] if end is None else end, n):
            to = min(at + n, self.W.shape[1] if end is None else end)
            if self.form == "weight_grad":
                w = self.row_values(self.W[0, at:to], self.sw[0, :, at:to])
            else:
                of_rows = self.sw[expert].double().repeat_interleave(128, 0)[at:to]
                w = (self.table[self.W[expert, at:to].long()].unflatten(-1, (-1, 128)) * of_rows.unsqueeze(-1)).flatten(-2)
            ref.append(x @ w.T)
            mag.append(x.abs() @ w.abs().T)
        return torch.cat(ref, 1), torch.cat(mag, 1)

    def half_step(self, ref):
        import torch
        mantissa, least, largest = (10, -14, 65504.0) if self.dtype == "f16" else (7, -126, 3.3895313892515355e38)
        exponent = torch.frexp(ref.abs().clamp(max=largest)).exponent.long() - 1
        return 0.5 * torch.exp2((exponent.clamp(min=least) - mantissa).double())

    def sums_off(self, mag):
        return (self.K // 128 + 22) * 2.0 ** -22 * mag

    def worst(self, got, ref, bound):
        off = (got.double() - ref).abs() / bound
        return off.max().item() if not off.isnan().any().item() else math.inf

    def worst_of_sums(self, got, a, b, expert, first=0, end=None):
        ref, mag = self.sums(a, b, expert, first, end)
        return self.worst(got, ref, self.half_step(ref) + self.sums_off(mag))

    def worst_of_h(self, got, a, b, expert, act):
        import torch
        (g, gm), (u, um) = self.sums(a, b, expert, 0, self.N), self.sums(a, b, expert, self.N, 2 * self.N)
        z = g if act == "silu" else 2 * math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
        f, eg, eu = g * torch.sigmoid(z), self.sums_off(gm), self.sums_off(um)
        h = f * u
        bound = self.half_step(h) + 1.13 * eg * (u.abs() + eu) + f.abs() * eu + h.abs() * (16 + 8 * z.abs()) * 2.0 ** -24 + (g * u).abs() * 2.0 ** -126
        return self.worst(got, h, bound)


@pytest.mark.gpu
@pytest.mark.parametrize("call", CALLS, ids=str)
def test_a_call_of_every_launch(lutq, call):
    import torch
    form, M, N, K, experts, codes, launch = call
    units = torch.cuda.get_device_properties(0).multi_processor_count
    assert lutq.calib_fp8_launch(M, N, K, experts, form, bool(codes), units) == lutq.binding.Fp8Launch(*launch)
    index = CALLS.index(call)
    act = ("silu", "gelu")[index // 2 % 2]
    p = Factors(lutq, form, M, N, K, experts, ("f16", "bf16")[index % 2], index)
    ws = (lutq.new_fp8_gated_workspace if form.startswith("gated") else lutq.new_fp8_workspace)(M, N, K, max(1, experts))
    offsets = uneven(M, experts, index) if experts else [0, M]
    out = lambda width: torch.full((M + 32, width), -7.0, dtype=torch_dtype(p.dtype), device="cuda")
    W, sw = (p.W, p.sw) if experts else (p.W[0], p.sw[0])
    off = (torch.tensor(offsets, dtype=torch.int32, device="cuda"),) if experts else ()
    # (tiles, and what is streamed of X quantised first, are launched the same way for codes)
    both = form != "weight_grad" and (not launch[6] or launch[0])
    for as_codes in ((True, False) if both else (bool(codes),)):
        guarded, again, kept = out(N), out(N), out(2 * N) if form == "gated_saved" else None
        x, s = p.args(as_codes)
        for y in (guarded, again):
            if form == "weight_grad":
                lutq.lutq_fp8_weight_grad(x, s, W, sw, y[16:16 + M], ws)
            elif form == "matmul":
                (lutq.lutq_fp8_matmul_grouped if experts else lutq.lutq_fp8_matmul)(x, W, sw, *off, y[16:16 + M], ws, x_scales=s)
            else:
                (lutq.lutq_fp8_gated_grouped if experts else lutq.lutq_fp8_gated)(x, W, sw, *off, y[16:16 + M], ws, x_scales=s, activation=act,
                                                                                  saved=None if kept is None else kept[16:16 + M])
        y = guarded[16:16 + M]
        for g, (a, b) in enumerate(zip(offsets, offsets[1:])):
            for a in range(a, b, 2048):
                to = min(a + 2048, b)
                worst = p.worst_of_h(y[a:to], a, to, g, act) if form.startswith("gated") else p.worst_of_sums(y[a:to], a, to, g)
                assert worst <= 1.0, (as_codes, g, a, worst)
                if kept is not None:
                    worst = p.worst_of_sums(kept[16 + a:16 + to], a, to, g)
                    assert worst <= 1.0, (as_codes, g, a, worst, "saved")
        for t in (guarded, kept):
            if t is not None:
                assert (t[:16 + offsets[0]] == -7.0).all().item() and (t[16 + offsets[-1]:] == -7.0).all().item()
        assert not ws[:65536].any().item() and torch.equal(guarded, again)


@pytest.mark.gpu
@pytest.mark.parametrize("dense", [False, True])
def test_more_pieces_of_rows_than_one_launch_takes(lutq, dense):
    """By expert a launch has at most 65535 workgroups along the rows, sixteen rows each here: others have the rest."""
    import torch
    experts, M, N, K = 65536, 65535 * 2 + 77, 16, 128
    r = lutq.calib_fp8_launch(M, N, K, experts, "matmul", not dense)
    assert r.streamed == (1 if dense else 3)
    p = Factors(lutq, "matmul", M, N, K, experts, "bf16", 6)
    g = torch.Generator().manual_seed(7)
    expert = torch.randint(0, experts, (M - 3,), generator=g).sort().values
    offsets = torch.cat((torch.zeros(1, dtype=torch.long), torch.bincount(expert, minlength=experts).cumsum(0))).int().cuda()
    expert = expert.cuda()
    y = torch.full((M + 16, N), -7.0, dtype=torch.bfloat16, device="cuda")
    x, s = p.args(not dense)
    lutq.lutq_fp8_matmul_grouped(x, p.W, p.sw, offsets, y[:M], lutq.new_fp8_workspace(M, N, K, experts), x_scales=s)
    for a in range(0, M - 3, 16384):
        mine = expert[a:a + 16384]
        b = a + mine.numel()
        w = p.table[p.W[mine].long()] * p.sw[mine].double()
        products = p.row_values(p.codes[a:b], p.s[:, a:b])[:, None] * w
        ref, mag = products.sum(-1), products.abs().sum(-1)
        assert p.worst(y[a:b], ref, p.half_step(ref) + p.sums_off(mag)) <= 1.0, a
    assert (y[M - 3:] == -7.0).all().item()


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K,form", [(3, 16, (1 << 22), "matmul"), (40, 32, 1 << 20, "matmul"), (2, 1 << 24, 128, "matmul"), (70000, 16, 128, "matmul"), (200, 1 << 20, 128, "matmul"),
                                        (2, 128, 1 << 21, "gated"), (100, 1 << 17, 128, "gated"), (16, 48, 1 << 22, "weight_grad"), (1 << 20, 16, 128, "weight_grad")])
def test_the_largest_sizes(lutq, M, N, K, form):
    import torch
    p = Factors(lutq, form, M, N, K, 0, "bf16", 9)
    ws = (lutq.new_fp8_gated_workspace if form == "gated" else lutq.new_fp8_workspace)(M, N, K)
    y = torch.full((M + 2, N), -7.0, dtype=torch.bfloat16, device="cuda")
    for as_codes in ((True,) if form == "weight_grad" else (True, False)):
        x, s = p.args(as_codes)
        if form == "gated":
            lutq.lutq_fp8_gated(x, p.W[0], p.sw[0], y[:M], ws, x_scales=s)
        elif form == "matmul":
            lutq.lutq_fp8_matmul(x, p.W[0], p.sw[0], y[:M], ws, x_scales=s)
        else:
            lutq.lutq_fp8_weight_grad(x, s, p.W[0], p.sw[0], y[:M], ws)
        rows = max(1, min(M, (1 << 27) // N))
        for a in range(0, M, rows):
            b = min(a + rows, M)
            worst = p.worst_of_h(y[a:b], a, b, 0, "silu") if form == "gated" else p.worst_of_sums(y[a:b], a, b, 0)
            assert worst <= 1.0, (as_codes, a, worst)
        assert (y[M:] == -7.0).all().item()
