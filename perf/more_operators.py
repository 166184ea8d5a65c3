"""8-bit floating point with a scale for each block of 128, and the gated feed-forward block on it, as cases that can be timed and checked.

The form: values are E4M3 codes (sign, four bits of exponent, three of mantissa, 448 the largest) times a 32-bit scale.  Of rows of
activations 128 neighbouring values share a scale, of weights a square of 128 rows and 128 columns, and of columns, which the gradient of
weights needs as it sums over the rows, 128 rows of one column.  With a the largest magnitude of a block, 2^-110 at least, the scale is
a / 448 and a code is x times (448 / a), rounded to the nearest, ties to even; by columns the scale is the least power of two that is at
least a / 448, and a code is x over it.

`op` of a case:
  quantise  dense values (`src`) to codes and scales, and back to a dense 16-bit matrix (`dtype`); `form` is "rows", "gather" (rows
            picked by an index, -1 a row of zeros: tokens sent to their experts), or "weights"
  matmul    Y = X W^T; `x` is "dense" (16-bit activations, quantised on the way in) or "codes"
  grouped   the same by expert: rows offsets[g] .. offsets[g + 1] of X times the weights of expert g; rows behind the last expert's stay
  gated     H = act(X G^T) * (X U^T), G and U the two halves of the weights' rows; with experts (e > 0) by expert, as above
  block     the same, H quantised, then times the down projection's weights: a whole feed-forward block
  train     a step's work on the gated projections: weights quantised, H, and from H's gradient the gradients of X and of the weights
            (G and U are kept at 16 bits; their gradients are quantised by rows for the one, by columns for the other)

Shapes are linear layers of LLaMA-3-8B and LLaMA-2-13B, square matrices, and generic expert layers.
"""
import math
import random

import torch

own = False

FLOOR = 2.0 ** -110


def _case(name, op, m, n, k, dtype, **more):
    return dict(name=name, op=op, m=m, n=n, k=k, dtype=dtype, **more)


def listed():
    return [
        # tokens of a batch sent to their experts: picked rows, padding among them, an odd number of blocks
        _case("quantise_dispatch_f16", "quantise", 1003, 0, 2176, "f16", src="f16", form="gather"),
        # the largest layer of the 8B model, from an fp32 checkpoint
        _case("quantise_weights_f32", "quantise", 28672, 0, 4096, "bf16", src="f32", form="weights"),
        # one decoded token through 8B query/key/value: the smallest product, where latency counts
        _case("decode_8b_qkv_bf16_m1", "matmul", 1, 6144, 4096, "bf16", x="dense"),
        # a serving batch through 13B down, whose sizes fill no power of two
        _case("batch_13b_down_f16_m23", "matmul", 23, 5120, 13824, "f16", x="dense"),
        # a long prompt or a packed batch on the square matrix
        _case("prompt_square_bf16_m8192", "matmul", 8192, 8192, 8192, "bf16", x="dense"),
        # a decode batch spread over many experts, most of them with a few rows, some with none; padding behind
        _case("experts_batch_f16_t250", "grouped", 256, 2816, 2048, "f16", x="codes", e=64, spare=6),
        # a prompt chunk over experts of uneven load
        _case("experts_chunk_bf16_t4099", "grouped", 4099, 4096, 2304, "bf16", x="codes", e=32, spare=0),
        # one decoded token through 8B gate and up
        _case("gated_8b_token_bf16_m1", "gated", 1, 14336, 4096, "bf16", x="dense", act="silu", e=0, spare=0),
        # a large batch through a layer's experts
        _case("gated_experts_f16_t6007", "gated", 6016, 2048, 4096, "f16", x="codes", act="gelu", e=16, spare=9),
        # a prompt through the whole feed-forward block of the 13B model
        _case("block_13b_prompt_bf16_m2048", "block", 2048, 13824, 5120, "bf16", x="dense", act="silu", e=0, spare=0),
        # a short, odd batch in training: fewer rows than the gradient of weights has blocks' worth of
        _case("train_odd_f16_m300", "train", 300, 1408, 1152, "f16", act="gelu"),
        # a training micro-batch on the 8B model's gate and up
        _case("train_8b_bf16_m4096", "train", 4096, 14336, 4096, "bf16", act="silu"),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def draw(rng):
    op = rng.choices(("quantise", "matmul", "grouped", "gated", "block", "train"), (2, 4, 3, 4, 2, 3))[0]
    dtype = rng.choice(("f16", "bf16"))
    if op == "quantise":
        form = rng.choice(("rows", "gather", "weights"))
        k = 128 * round(_log(rng, 4, 128))
        m = max(1, round(_log(rng, 1, min(32768, 1.1e8 / k))))
        if form == "weights":
            m = 16 * max(1, round(m / 16))
        c = _case("", op, m, 0, k, dtype, src=rng.choice(("f32", dtype)), form=form)
    elif op == "matmul":
        k = 128 * round(_log(rng, 4, 128))
        n = 16 * round(_log(rng, 16, min(2048, 1.3e8 / (16 * k))))
        m = max(1, round(_log(rng, 1, min(8192, 5e11 / (n * k)))))
        c = _case("", op, m, n, k, dtype, x=rng.choice(("dense", "codes")))
    elif op == "grouped":
        e = round(_log(rng, 2, 128))
        k = 128 * round(_log(rng, 4, min(64, 4e8 / (e * 128 * 512))))
        n = 16 * round(_log(rng, 16, min(1024, 5e8 / (e * 16 * k))))
        t = max(1, round(_log(rng, 1, min(16384, 1e12 / (n * k)))))
        spare = rng.choice((0, 0, rng.randint(1, 40)))
        c = _case("", op, t + spare, n, k, dtype, x=rng.choice(("dense", "codes")), e=e, spare=spare)
    elif op in ("gated", "block"):
        e = round(_log(rng, 2, 64)) if op == "gated" and rng.random() < 0.4 else 0
        k = 128 * round(_log(rng, 4, min(64, 4e8 / (max(e, 1) * 256 * 512))))
        n = 128 * max(2, round(_log(rng, 2, min(112, 5e8 / (max(e, 1) * 256 * k)))))
        t = max(1, round(_log(rng, 1, min(8192, 2.5e11 / (n * k)))))
        spare = rng.choice((0, 0, rng.randint(1, 40))) if e else 0
        c = _case("", op, t + spare, n, k, dtype, x=rng.choice(("dense", "codes")), act=rng.choice(("silu", "gelu")), e=e, spare=spare)
    else:
        k = 128 * round(_log(rng, 4, 40))
        n = 128 * round(_log(rng, 2, 112))
        m = max(1, round(_log(rng, 16, min(8192, 2.4e11 / (n * k)))))
        c = _case("", op, m, n, k, dtype, act=rng.choice(("silu", "gelu")))
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------- inputs
def _dt(dtype):
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[dtype]


def _gen(seed, salt):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + salt)
    return g


def _activations(seed, m, k, dtype):
    """Activations: Gaussian, every 61st channel thirty times as large; every 97th row a row of zeros (padding)."""
    x = torch.randn((m, k), generator=_gen(seed, 1), device="cuda")
    x[:, 7::61] *= 30.0
    x[50::97] = 0.0
    return x.to(_dt(dtype))


def _gradients(seed, m, n, dtype):
    """Gradients of H: Gaussian, small, some rows without any (tokens that no loss is taken of)."""
    x = torch.randn((m, n), generator=_gen(seed, 3), device="cuda").mul_(2.0 ** -8)
    x[3::11] = 0.0
    return x.to(_dt(dtype))


def _weights(seed, salt, n, k, dtype="f32"):
    return torch.randn((n, k), generator=_gen(seed, 16 + salt), device="cuda").mul_(0.02).to(_dt(dtype))


def _picked(case, seed):
    """Which of the source's rows each output row is, and how many rows the source has: every token goes to two experts,
    a few places are padding."""
    tokens = max(1, case["m"] // 2)
    g = _gen(seed, 2)
    rows = torch.randint(0, tokens, (case["m"],), generator=g, device="cuda", dtype=torch.int32)
    rows[torch.rand(case["m"], generator=g, device="cuda") < 0.03] = -1
    return rows, tokens


def _offsets(case):
    """Where each expert's rows begin; the load is uneven, and experts without rows are among them.  By the sizes alone:
    what a pass has to read does not change with the inputs."""
    rng = random.Random(case["m"] * 131 + case["e"])
    weights = [rng.paretovariate(1.5) for _ in range(case["e"])]
    weights[rng.randrange(case["e"])] = 0.0
    counts = [0] * case["e"]
    for g in rng.choices(range(case["e"]), weights, k=case["m"] - case["spare"]):
        counts[g] += 1
    offsets = [0]
    for c in counts:
        offsets.append(offsets[-1] + c)
    return offsets


def _empty(*shape, dtype=torch.uint8):
    return torch.empty(shape, dtype=dtype, device="cuda")


def prepare(case, seed):
    s = dict(case=case)
    op, m, n, k = case["op"], case["m"], case["n"], case["k"]
    dt = _dt(case["dtype"])
    if op == "quantise":
        if case["form"] == "weights":
            s["x"] = _weights(seed, 0, m, k, case["src"])
            s["scales"] = _empty(-(-m // 128), k // 128, dtype=torch.float32)
        else:
            rows, tokens = _picked(case, seed) if case["form"] == "gather" else (None, m)
            s["x"], s["rows"] = _activations(seed, tokens, k, case["src"]), rows
            s["scales"] = _empty(k // 128, m, dtype=torch.float32)
        s["codes"], s["out"] = _empty(m, k), _empty(m, k, dtype=dt)
        return s
    x = _activations(seed, m, k, case["dtype"])
    if op == "train":
        padded = -(-m // 128) * 128
        s["x"], s["w"], s["dh"] = x, _weights(seed, 0, 2 * n, k, case["dtype"]), _gradients(seed, m, n, case["dtype"])
        # what a training program allocates once: codes of the weights both ways, what the step keeps and gives
        s["w_codes"], s["w_scales"] = _empty(2 * n, k), _empty(n // 64, k // 128, dtype=torch.float32)
        s["wt_codes"], s["wt_scales"] = _empty(k, 2 * n), _empty(k // 128, n // 64, dtype=torch.float32)
        s["x_cols"], s["x_col_scales"] = _empty(k, padded), _empty(padded // 128, k, dtype=torch.float32)
        s["g_rows"], s["g_row_scales"] = _empty(m, 2 * n), _empty(n // 64, m, dtype=torch.float32)
        s["g_cols"], s["g_col_scales"] = _empty(2 * n, padded), _empty(padded // 128, 2 * n, dtype=torch.float32)
        s["h"], s["saved"] = _empty(m, n, dtype=dt), _empty(m, 2 * n, dtype=dt)
        s["dx"], s["dw"] = _empty(m, k, dtype=dt), _empty(2 * n, k, dtype=dt)
        if own:
            import paper_2407_10960_amd as lutq
            s["workspace"] = lutq.new_fp8_gated_workspace(m, n, k)
            s["dx_workspace"] = lutq.new_fp8_workspace(m, k, 2 * n)
            s["dw_workspace"] = lutq.new_fp8_workspace(2 * n, k, padded)
        return s
    experts = case.get("e", 0)
    rows = n if op in ("matmul", "grouped") else 2 * n
    s["x"], s["x_scales"] = (x, None) if case["x"] == "dense" else _rows(x)
    s["w"], s["w_scales"] = _empty(max(experts, 1), rows, k), _empty(max(experts, 1), -(-rows // 128), k // 128, dtype=torch.float32)
    for g in range(max(experts, 1)):
        s["w"][g], s["w_scales"][g] = _squares(_weights(seed, g, rows, k))
    if experts:
        s["offsets"] = torch.tensor(_offsets(case), dtype=torch.int32, device="cuda")
    s["y"] = torch.zeros((m, k if op == "block" else n), dtype=dt, device="cuda")
    if op == "block":
        s["down"], s["down_scales"] = _squares(_weights(seed, 1, k, n))
        s["h"], s["h_scales"] = _empty(m, n), _empty(n // 128, m, dtype=torch.float32)
    if own:
        import paper_2407_10960_amd as lutq
        new = lutq.new_fp8_workspace if op in ("matmul", "grouped") else lutq.new_fp8_gated_workspace
        s["workspace"] = new(m, n, k, max(experts, 1))
        if op == "block":
            s["down_workspace"] = lutq.new_fp8_workspace(m, k, n)
    return s


# ---------------------------------------------------------------------------------------------------- plain form
def _codes(u):
    """E4M3 codes of values that round to 448 at most."""
    return u.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8)


def _quantised(blocks, dims):
    """Codes of `blocks`, which share a scale along `dims`, and the scales."""
    a = blocks.abs().amax(dims, keepdim=True).clamp_min(FLOOR)
    top = torch.full_like(a, 448.0)                    # (a tensor: with a number torch multiplies by a rounded reciprocal)
    return _codes(blocks * (top / a)), a / top


def _rows(x):
    codes, scales = _quantised(x.float().unflatten(-1, (-1, 128)), (-1,))
    return codes.flatten(-2), scales.squeeze(-1).T.contiguous()


def _squares(w):
    n, k = w.shape
    up = -n % 128                                     # (the last square may have fewer rows)
    b = torch.nn.functional.pad(w.float(), (0, 0, 0, up)).reshape(-1, 128, k // 128, 128)
    codes, scales = _quantised(b, (1, 3))
    return codes.reshape(n + up, k)[:n], scales.reshape(-1, k // 128)


def _columns(x):
    """Codes of the columns of x, as rows, zeros behind them up to whole blocks, and the scales, powers of two."""
    m, k = x.shape
    b = torch.nn.functional.pad(x.float(), (0, 0, 0, -m % 128)).T.reshape(k, -1, 128)
    f, e = torch.frexp(b.abs().amax(-1).clamp_min(FLOOR))            # a = f 2^e, 448 = 0.875 2^9
    scales = torch.ldexp(torch.ones_like(f), e - 9 + (f > 0.875).int())
    return _codes(b / scales.unsqueeze(-1)).flatten(-2), scales.T.contiguous()


def _row_values(codes, scales):
    v = codes.view(torch.float8_e4m3fn).float()
    return (v.unflatten(-1, (-1, 128)) * scales.T.unsqueeze(-1)).flatten(-2)


def _weight_values(codes, scales):
    n, k = codes.shape
    return codes.view(torch.float8_e4m3fn).float() * scales.repeat_interleave(128, 0)[:n].repeat_interleave(128, 1)


def _sigma(g, act):
    """The activation's factor of its argument, and its derivative."""
    if act == "silu":
        z, dz = g, 1.0
    else:
        c = 2.0 * math.sqrt(2.0 / math.pi)
        z, dz = c * (g + 0.044715 * g * g * g), c * (1.0 + 3 * 0.044715 * g * g)
    s = 1.0 / (1.0 + torch.exp(-z))
    return s, s * (1.0 - s) * dz


def _gated(x, w, act):
    g, u = (x @ w.T).chunk(2, -1)
    return g, u, g * _sigma(g, act)[0] * u


def _plain(s):
    case, op = s["case"], s["case"]["op"]
    if op == "quantise":
        x = s["x"]
        if case["form"] == "weights":
            codes, scales = _squares(x)
            values = _weight_values(codes, scales)
        else:
            if s["rows"] is not None:
                r = s["rows"].long()
                x = torch.where((r >= 0).unsqueeze(-1), x[r.clamp(0)], 0)
            codes, scales = _rows(x)
            values = _row_values(codes, scales)
        s["out"].copy_(values)
        return s["out"], scales
    if op == "train":
        x, w = _row_values(*_rows(s["x"])), _weight_values(*_squares(s["w"]))
        dt = s["x"].dtype
        g, u, h = _gated(x, w, case["act"])
        g, u, dh = g.to(dt).float(), u.to(dt).float(), s["dh"].float()
        f, df = _sigma(g, case["act"])
        dgu = torch.cat((dh * u * (f + g * df), dh * g * f), -1)
        dx = _row_values(*_rows(dgu)) @ w
        dw = _row_values(*_columns(dgu)) @ _row_values(*_columns(s["x"])).T
        return h.to(dt), dx.to(dt), dw.to(dt)
    x = _row_values(*((s["x"], s["x_scales"]) if s["x_scales"] is not None else _rows(s["x"])))
    y = s["y"]
    if "offsets" in s:
        # ragged products: one for each expert that has rows
        offsets = s["offsets"].tolist()
        for g, (a, b) in enumerate(zip(offsets, offsets[1:])):
            if b > a:
                w = _weight_values(s["w"][g], s["w_scales"][g])
                y[a:b] = x[a:b] @ w.T if op == "grouped" else _gated(x[a:b], w, case["act"])[2]
        return y
    w = _weight_values(s["w"][0], s["w_scales"][0])
    if op == "matmul":
        y.copy_(x @ w.T)
    else:
        h = _gated(x, w, case["act"])[2]
        if op == "block":                              # (H at 16 bits, then quantised)
            h = _row_values(*_rows(h.to(y.dtype))) @ _weight_values(s["down"], s["down_scales"]).T
        y.copy_(h)
    return y


def _own(s):
    import paper_2407_10960_amd as lutq
    case, op = s["case"], s["case"]["op"]
    if op == "quantise":
        if case["form"] == "weights":
            lutq.lutq_fp8_quantize_weights(s["x"], s["codes"], s["scales"])
            return lutq.lutq_fp8_dequant_weights(s["codes"], s["scales"], s["out"]), s["scales"]
        lutq.lutq_fp8_quantize(s["x"], s["codes"], s["scales"], rows=s["rows"])
        return lutq.lutq_fp8_dequant(s["codes"], s["scales"], s["out"]), s["scales"]
    if op == "train":
        lutq.lutq_fp8_quantize_weights(s["w"], s["w_codes"], s["w_scales"], transposed=(s["wt_codes"], s["wt_scales"]))
        lutq.lutq_fp8_gated(s["x"], s["w_codes"], s["w_scales"], s["h"], s["workspace"], activation=case["act"], saved=s["saved"])
        lutq.lutq_fp8_quantize_columns(s["x"], s["x_cols"], s["x_col_scales"])
        lutq.lutq_fp8_gated_grad(s["dh"], s["saved"], activation=case["act"], rows=(s["g_rows"], s["g_row_scales"]),
                                 columns=(s["g_cols"], s["g_col_scales"]))
        lutq.lutq_fp8_matmul(s["g_rows"], s["wt_codes"], s["wt_scales"], s["dx"], s["dx_workspace"], x_scales=s["g_row_scales"])
        lutq.lutq_fp8_weight_grad(s["g_cols"], s["g_col_scales"], s["x_cols"], s["x_col_scales"], s["dw"], s["dw_workspace"])
        return s["h"], s["dx"], s["dw"]
    if op == "matmul":
        return lutq.lutq_fp8_matmul(s["x"], s["w"][0], s["w_scales"][0], s["y"], s["workspace"], x_scales=s["x_scales"])
    if op == "grouped":
        return lutq.lutq_fp8_matmul_grouped(s["x"], s["w"], s["w_scales"], s["offsets"], s["y"], s["workspace"], x_scales=s["x_scales"])
    if op == "block":
        lutq.lutq_fp8_gated(s["x"], s["w"][0], s["w_scales"][0], s["h"], s["workspace"], x_scales=s["x_scales"], activation=case["act"],
                            h_scales=s["h_scales"], dtype=s["y"].dtype)
        return lutq.lutq_fp8_matmul(s["h"], s["down"], s["down_scales"], s["y"], s["down_workspace"], x_scales=s["h_scales"])
    if "offsets" in s:
        return lutq.lutq_fp8_gated_grouped(s["x"], s["w"], s["w_scales"], s["offsets"], s["y"], s["workspace"], x_scales=s["x_scales"],
                                           activation=case["act"])
    return lutq.lutq_fp8_gated(s["x"], s["w"][0], s["w_scales"][0], s["y"], s["workspace"], x_scales=s["x_scales"], activation=case["act"])


def run(state):
    return _own(state) if own else _plain(state)


# ---------------------------------------------------------------------------------------------------- work, definition
def work(case):
    op, m, n, k = case["op"], case["m"], case["n"], case["k"]
    held = k + k // 32                                                # bytes of one row of codes and its scales
    if op == "quantise":
        source = max(1, m // 2) if case["form"] == "gather" else m
        wide = 4 if case["src"] == "f32" else 2
        scales = 4 * (k // 128) * (-(-m // 128) if case["form"] == "weights" else m)
        return {"bytes": source * k * wide + (4 * m if case["form"] == "gather" else 0) + m * k + scales + m * k * 2, "flops": 3 * m * k}
    if op == "train":
        # X, the gradient and the weights in, H and the gradients out; G and U have to be kept from the one pass to the other
        return {"bytes": 2 * m * k + 2 * m * n + 4 * n * k + 2 * m * n + 4 * m * n + 2 * m * k + 4 * n * k, "flops": 3 * 4 * m * n * k}
    rows, experts = m, 1
    if case.get("e"):
        o = _offsets(case)
        rows, experts = o[-1], sum(b > a for a, b in zip(o, o[1:]))
    x = 2 * k if case["x"] == "dense" else held
    w = n if op in ("matmul", "grouped") else 2 * n
    total = {"bytes": rows * x + experts * (w * k + 4 * -(-w // 128) * (k // 128)) + 4 * case.get("e", 0), "flops": 2 * rows * w * k}
    if op == "block":
        total["bytes"] += k * n + 4 * (k // 128) * (n // 128) + rows * k * 2
        total["flops"] += 2 * rows * n * k
    else:
        total["bytes"] += rows * n * 2
    return total


def _nearest(u):
    """The value of E4M3 nearest to u, ties to the even mantissa: multiples of 2^(e - 3) from 2^e on, of 2^-9 below 2^-6."""
    e = (torch.frexp(u)[1] - 1).clamp_min(-6)
    step = torch.exp2((e - 3).double())
    return torch.round(u / step) * step


def _defined(blocks, dims, power=False):
    """What the quantiser makes of `blocks`, which share a scale along `dims`: the values that the codes stand for, and the scales.
    448 / a, a / 448 and x times the former are 32-bit numbers by definition."""
    b = blocks.double()
    a = b.abs().amax(dims, keepdim=True).clamp_min(FLOOR)
    if power:
        s = torch.exp2(torch.ceil(torch.log2(a / 448.0)))
        s = torch.where(s / 2 >= a / 448.0, s / 2, torch.where(s < a / 448.0, s * 2, s))     # (log2 next to a whole number)
        return _nearest((b / s).clamp(-448.0, 448.0)) * s, s
    s, r = (a / 448.0).float().double(), (448.0 / a).float().double()
    return _nearest((b * r).float().double().clamp(-448.0, 448.0)) * s, s


def _exact_rows(x):
    return torch.cat([_defined(part.unflatten(-1, (-1, 128)), (-1,))[0].flatten(-2) for part in x.split(4096)])


def _exact_columns(x):
    m = x.shape[0]
    parts = [_defined(torch.nn.functional.pad(part, (0, 0, 0, -part.shape[0] % 128)).unflatten(0, (-1, 128)), (1,), True)[0].flatten(0, 1)
             for part in x.split(4096)]
    return torch.cat(parts)[:m]


def _exact_squares(w):
    n, k = w.shape
    parts = [_defined(torch.nn.functional.pad(part, (0, 0, 0, -part.shape[0] % 128)).reshape(-1, 128, k // 128, 128), (1, 3)) for part in w.split(4096)]
    return torch.cat([v.reshape(-1, k) for v, _ in parts])[:n], torch.cat([s.reshape(-1, k // 128) for _, s in parts])


def _exact_act(g, act):
    if act == "silu":
        return g * torch.sigmoid(g)
    return 0.5 * g * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (g + 0.044715 * g ** 3)))


def _exact_slope(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return s * (1.0 + g * (1.0 - s))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (g + 0.044715 * g ** 3))
    return 0.5 * (1.0 + t) + 0.5 * g * (1.0 - t * t) * c * (1.0 + 3 * 0.044715 * g * g)


def exact(case, seed):
    op, m, n, k = case["op"], case["m"], case["n"], case["k"]
    if op == "quantise":
        if case["form"] == "weights":
            return _exact_squares(_weights(seed, 0, m, k, case["src"]))
        rows, tokens = _picked(case, seed) if case["form"] == "gather" else (None, m)
        x = _activations(seed, tokens, k, case["src"])
        parts = [_defined(part.unflatten(-1, (-1, 128)), (-1,)) for part in torch.cat((x, torch.zeros_like(x[:1]))).split(4096)]
        v, s = torch.cat([v.flatten(-2) for v, _ in parts]), torch.cat([s.squeeze(-1) for _, s in parts])
        which = torch.arange(m, device="cuda") if rows is None else torch.where(rows < 0, tokens, rows).long()
        return v[which], s[which].T.contiguous()
    x16 = _activations(seed, m, k, case["dtype"])
    dt = _dt(case["dtype"])
    x = _exact_rows(x16)
    if op == "train":
        w = _exact_squares(_weights(seed, 0, 2 * n, k, case["dtype"]))[0]
        g, u = x @ w[:n].T, x @ w[n:].T
        h = _exact_act(g, case["act"]) * u
        g, u, dh = g.to(dt).double(), u.to(dt).double(), _gradients(seed, m, n, case["dtype"]).double()
        dgu = torch.cat((dh * u * _exact_slope(g, case["act"]), dh * _exact_act(g, case["act"])), -1)
        return h, _exact_rows(dgu) @ w, _exact_columns(dgu).T @ _exact_columns(x16)
    experts = case.get("e", 0)
    offsets = _offsets(case) if experts else [0, m]
    rows = n if op in ("matmul", "grouped") else 2 * n
    y = torch.zeros((m, n), dtype=torch.float64, device="cuda")
    for g in range(len(offsets) - 1):
        a, b = offsets[g], offsets[g + 1]
        if b > a:
            p = x[a:b] @ _exact_squares(_weights(seed, g, rows, k))[0].T
            y[a:b] = p if rows == n else _exact_act(p[:, :n], case["act"]) * p[:, n:]
    if op == "block":
        y = _exact_rows(y.to(dt)) @ _exact_squares(_weights(seed, 1, k, n))[0].T
    return y
