"""The operators around the mixed-precision linear layers, as measurable cases: RMS norm with the residual's addition and quantized
outputs, its backward pass, and an AdamW step over many tensors with states in 32 or 8 bits.

Shapes are those of the configurations in `paper_2602_01410_b200/workloads.py` (single 512 linear, Llama-like 1B / 3B / 7B / 70B blocks).
Where `own` is false, `run` computes the operators in elementary torch operations; where it is true, it calls the library.

Kinds of case
  norm      h = bf16(x + residual), y = h / rms(h) * gain: y in bf16 (fmt "bf16"), as FP8 codes on 1x128 tiles ("row"), or those and the
            transposed codes on 128x1 tiles that the weight gradient reads ("dual")
  norm_bwd  gradients of that: dx (with the gradient that arrives on the residual stream added) and the gain's
  adamw     one AdamW step over a list of tensors that lie in one arena, as a training program with flat buffers keeps them; every
            tensor starts at a multiple of 512 elements
Codes come back as float8 tensors (the values that they stand for, times the scale that comes back beside them).
"""
import math

import torch

own = False

EPS_NORM = 1e-5
SEGMENT = 512      # elements between possible starts of tensors in an arena
BLOCK = 128        # elements that share a scale of the 8-bit states
E4M3_MAX = 448.0
FLT_MAX = 3.4028234663852886e38


def _norm(name, rows, cols, out, residual, gain32):
    return {"name": name, "op": "norm", "rows": rows, "cols": cols, "out": out, "residual": residual, "gain32": gain32}


def _bwd(name, rows, cols, residual, gain32):
    return {"name": name, "op": "norm_bwd", "rows": rows, "cols": cols, "residual": residual, "gain32": gain32}


def _adamw(name, tensors, bits, param, grad, copy, sr, layers=1, count=0, most=0):
    return {"name": name, "op": "adamw", "tensors": tensors, "bits": bits, "param": param, "grad": grad, "copy": copy, "sr": sr,
            "layers": layers, "count": count, "most": most}


def listed():
    return [
        # decoding one token of the 7B model: launch latency, and one row spread over an SM
        _norm("norm-7b-one-token", 1, 4096, "row", True, False),
        # a 3B batch whose token count is odd, into a linear that keeps BF16
        _norm("norm-3b-bf16-ragged", 4093, 3200, "bf16", True, True),
        # the 7B training step: norm output quantized for the forward product and for the weight gradient at once
        _norm("norm-7b-train", 16384, 4096, "dual", True, False),
        # the widest hidden size, 70B, first norm of a block that has no residual yet
        _norm("norm-70b-train", 8192, 8192, "dual", False, False),
        # the smallest training call: one 512 linear over 512 tokens
        _bwd("bwd-512", 512, 512, False, False),
        # a 3B batch with an odd token count
        _bwd("bwd-3b-ragged", 8191, 3200, True, True),
        # the 7B training step
        _bwd("bwd-7b-train", 16384, 4096, True, False),
        # the smallest step: one 512 x 512 weight and its norm's gain
        _adamw("adamw-512", "single-512", 32, "fp32", "fp32", True, False),
        # the 65 norm gains of the 7B model: many tiny tensors, all latency
        _adamw("adamw-7b-gains", "7b-gains", 32, "fp32", "fp32", False, False),
        # four blocks of the 1B model, binary32 states and master weights, bf16 copy for the next forward pass
        _adamw("adamw-1b-states32", "1b", 32, "fp32", "bf16", True, False, layers=4),
        # a block of the 7B model, 8-bit states with stochastic rounding
        _adamw("adamw-7b-states8", "7b", 8, "fp32", "bf16", True, True),
        # a list of tensors of odd sizes, bf16 weights without master copies, 8-bit states to nearest
        _adamw("adamw-ragged-states8", "ragged", 8, "bf16", "bf16", False, False, count=40, most=300_001),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm_bwd", "adamw"])
    if op == "adamw":
        bits, param = rng.choice([8, 32]), rng.choice(["fp32", "bf16"])
        return {k: v for k, v in _adamw("", "ragged", bits, param, rng.choice(["fp32", "bf16"]), param == "fp32" and rng.random() < 0.5, rng.random() < 0.5,
                                        count=_log(rng, 1, 300), most=_log(rng, 1, 500_000)).items() if k != "name"}
    cols = max(16, _log(rng, 100, 8192) // 8 * 8)
    rows = _log(rng, 1, min(16384, 8192 * 8192 // cols))
    if op == "norm_bwd":
        c = _bwd("", rows, cols, rng.random() < 0.7, rng.random() < 0.5)
    else:
        out = rng.choice(["bf16", "row", "dual"])
        if out == "dual":
            rows, cols = max(64, rows // 64 * 64), max(64, cols // 64 * 64)
        c = _norm("", rows, cols, out, rng.random() < 0.7, rng.random() < 0.5)
    return {k: v for k, v in c.items() if k != "name"}


def _sizes(case):
    """Elements of each tensor of an AdamW case."""
    kind = case["tensors"]
    if kind == "single-512":
        return [512 * 512, 512]
    if kind == "7b-gains":
        return [4096] * 65
    if kind == "1b":
        block = [2048 * 2048, 256 * 2048, 256 * 2048, 2048 * 2048, 5632 * 2048, 5632 * 2048, 2048 * 5632, 2048, 2048]
        return block * case["layers"]
    if kind == "7b":
        return [12288 * 4096, 4096 * 4096, 11008 * 4096, 11008 * 4096, 4096 * 11008, 4096, 4096] * case["layers"]
    # sizes from 1 to `most`, spread over their logarithm, without a common divisor
    n, most = case["count"], case["most"]
    return [max(1, min(most, int(round(most ** (((i * 0.6180339887) % 1.0) if i else 1.0))) - (i % 3))) for i in range(n)]


def _segments(sizes):
    """First segment of each tensor in the arena, and the arena's segments."""
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += -(-n // SEGMENT)
    return starts, at


def work(case):
    if case["op"] == "adamw":
        n = sum(_sizes(case))
        p = 4 if case["param"] == "fp32" else 2
        g = 4 if case["grad"] == "fp32" else 2
        state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * (2 * p + g + (2 if case["copy"] else 0) + state), "flops": 15 * n}
    rows, cols = case["rows"], case["cols"]
    n, gain = rows * cols, cols * (4 if case["gain32"] else 2)
    if case["op"] == "norm_bwd":
        return {"bytes": n * (8 if case["residual"] else 6) + 4 * rows + gain + 4 * cols, "flops": 10 * n}
    each = (6 if case["residual"] else 2) + {"bf16": 2, "row": 1, "dual": 2}[case["out"]]
    scales = 0 if case["out"] == "bf16" else 4 * rows * -(-cols // 128)
    scales += 4 * cols * -(-rows // 128) if case["out"] == "dual" else 0
    return {"bytes": n * each + scales + gain + 4 * rows, "flops": 6 * n}


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.float32)

    if case["op"] == "adamw":
        return _prepare_adamw(case, seed, gen, normal)
    rows, cols = case["rows"], case["cols"]
    # activations: unit normal with a few outlier channels; the gain is near one, as after some training
    outlier = torch.where(torch.rand(cols, generator=gen, device="cuda") < 0.01, 20.0, 1.0)
    s = {"case": case, "x": (normal(rows, cols) * outlier).to(torch.bfloat16)}
    s["gain"] = (1.0 + 0.1 * normal(cols)).to(torch.float32 if case["gain32"] else torch.bfloat16)
    s["residual"] = (normal(rows, cols) * outlier).to(torch.bfloat16) if case["residual"] else None
    if case["op"] == "norm_bwd":
        # output gradients: a log-normal factor a token
        s["dy"] = (normal(rows, cols) * 1e-3 * torch.exp(normal(rows, 1))).to(torch.bfloat16)
        if case["residual"]:
            s["residual"] = (s["residual"].float() * 1e-3).to(torch.bfloat16)
        s["rstd"] = torch.rsqrt(s["x"].float().square().mean(1) + EPS_NORM)
        s["dx"] = torch.empty_like(s["x"])
        s["dgain"] = torch.empty(cols, device="cuda", dtype=torch.float32)
        return s
    tiles, tiles_t = -(-cols // 128), -(-rows // 128)
    s["out"] = {"h": torch.empty_like(s["x"]) if case["residual"] else None, "rstd": torch.empty(rows, device="cuda", dtype=torch.float32)}
    if case["out"] == "bf16":
        s["out"]["y"] = torch.empty_like(s["x"])
    else:
        s["out"]["codes"] = torch.empty(rows * cols, device="cuda", dtype=torch.uint8)
        s["out"]["scales"] = torch.empty(tiles * rows, device="cuda", dtype=torch.float32)
    if case["out"] == "dual":
        s["out"]["codes_t"] = torch.empty(rows * cols, device="cuda", dtype=torch.uint8)
        s["out"]["scales_t"] = torch.empty(tiles_t * cols, device="cuda", dtype=torch.float32)
    return s


def _prepare_adamw(case, seed, gen, normal):
    sizes = _sizes(case)
    starts, segments = _segments(sizes)
    total = segments * SEGMENT
    owner = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor([-(-n // SEGMENT) for n in sizes], device="cuda"))
    first = torch.tensor(starts, device="cuda")[owner]
    place = ((torch.arange(segments, device="cuda") - first) * SEGMENT)[:, None] + torch.arange(SEGMENT, device="cuda")
    live = (place < torch.tensor(sizes, device="cuda")[owner][:, None]).view(-1)
    del place
    # weights of standard deviation 0.02; moments of a run under way: a magnitude per element spanning decades, as in real gradients
    scale = 1e-3 * torch.exp(1.5 * normal(total)) * live
    s = {"case": case, "owner": owner, "first": first, "seed": seed * 2654435761 % (1 << 62), "step": 100 + seed % 50,
         "lr": 1e-4, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8}
    # norm gains (small tensors) are not decayed
    s["decay"] = [0.1 if n > 4096 else 0.0 for n in sizes]
    s["decay_segments"] = torch.tensor(s["decay"], device="cuda")[owner]
    s["p"] = (normal(total) * 0.02 * live).to(torch.float32 if case["param"] == "fp32" else torch.bfloat16)
    s["g"] = (normal(total) * scale).to(torch.float32 if case["grad"] == "fp32" else torch.bfloat16)
    m = normal(total) * scale * 0.3
    v = scale.square() * torch.exp(0.3 * normal(total))
    del scale
    if case["bits"] == 32:
        s["m"], s["v"] = m, v
    else:
        s["m"], s["m_scale"] = _stored(m, None, False)
        s["v"], s["v_scale"] = _stored(torch.sqrt(v), None, True)
    s["copy"] = s["p"].to(torch.bfloat16) if case["copy"] else None
    if own:
        from paper_2602_01410_b200 import api

        def parts(t, unit=1):
            return None if t is None else [t[a * SEGMENT // unit: a * SEGMENT // unit + -(-n // unit)] for a, n in zip(starts, sizes)]

        # the table of the tensors, which a training program makes once
        s["tensors"] = api.make_adamw_tensors(parts(s["p"]), parts(s["g"]), parts(s["m"]), parts(s["v"]), m_scales=parts(s.get("m_scale"), BLOCK),
                                              v_scales=parts(s.get("v_scale"), BLOCK), copies=parts(s["copy"]), weight_decay=s["decay"])
    return s


def run(s):
    if own:
        return _run_own(s)
    op = s["case"]["op"]
    return _plain_norm(s) if op == "norm" else _plain_bwd(s) if op == "norm_bwd" else _plain_adamw(s)


def _run_own(s):
    from paper_2602_01410_b200 import api
    case = s["case"]
    if case["op"] == "norm":
        o = api.snip_rmsnorm_fwd(s["x"], s["gain"], EPS_NORM, residual=s["residual"], fmt=api.FMT_FP8_E4M3, fmt_t=api.FMT_FP8_E4M3, out=s["out"])
        rows, cols = case["rows"], case["cols"]
        got = {"rstd": o["rstd"]}
        if case["residual"]:
            got["h"] = o["h"]
        if case["out"] == "bf16":
            got["y"] = o["y"]
        else:
            got["codes"], got["scales"] = o["codes"].view(torch.float8_e4m3fn).view(rows, cols), o["scales"].view(-1, rows)
        if case["out"] == "dual":
            got["codes_t"], got["scales_t"] = o["codes_t"].view(torch.float8_e4m3fn).view(cols, rows), o["scales_t"].view(-1, cols)
        return got
    if case["op"] == "norm_bwd":
        dx, dgain = api.snip_rmsnorm_bwd(s["dy"], s["x"], s["gain"], s["rstd"], dresidual=s["residual"], dx=s["dx"], dgain=s["dgain"])
        return {"dx": dx, "dgain": dgain}
    api.snip_adamw_step(s["tensors"], s["lr"], s["beta1"], s["beta2"], s["eps"], s["step"],
                        rounding=api.ROUND_STOCHASTIC if case["sr"] else api.ROUND_NEAREST_EVEN, seed=s["seed"])
    got = {k: s[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copy") if s.get(k) is not None}
    if case["bits"] == 8:
        got["m"], got["v"] = got["m"].view(torch.float8_e4m3fn), got["v"].view(torch.float8_e4m3fn)
    return got


# ---- plain forms -----------------------------------------------------------------------------------------------------------------

def _scale(amax):
    """FPX_MAX / amax; 1 for an empty tile, at most the largest binary32 number."""
    return torch.where(amax == 0, torch.ones_like(amax), (E4M3_MAX / amax).clamp(max=FLT_MAX))


def _tiles(y):
    """Codes [rows, cols] and scales [tiles, rows] of 1x128 tiles."""
    rows, cols = y.shape
    tiles = -(-cols // 128)
    padded = torch.nn.functional.pad(y, (0, tiles * 128 - cols)).view(rows, tiles, 128)
    scale = _scale(padded.abs().amax(2))
    codes = (padded * scale[:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    return codes.view(rows, tiles * 128)[:, :cols].contiguous(), scale.t().contiguous()


def _plain_norm(s):
    case, h = s["case"], s["x"]
    got = {}
    if case["residual"]:
        h = got["h"] = (s["x"].float() + s["residual"].float()).to(torch.bfloat16)
    h = h.float()
    got["rstd"] = 1.0 / torch.sqrt(h.square().mean(1) + EPS_NORM)
    y = h * got["rstd"][:, None] * s["gain"].float()
    if case["out"] == "bf16":
        got["y"] = y.to(torch.bfloat16)
    else:
        got["codes"], got["scales"] = _tiles(y)
    if case["out"] == "dual":
        got["codes_t"], got["scales_t"] = _tiles(y.t())
    return got


def _plain_bwd(s):
    dy, x, rstd = s["dy"].float(), s["x"].float(), s["rstd"][:, None]
    g, unit = dy * s["gain"].float(), x * rstd
    dx = rstd * (g - unit * (g * unit).mean(1, keepdim=True))
    if s["residual"] is not None:
        dx = dx + s["residual"].float()
    return {"dx": dx.to(torch.bfloat16), "dgain": (dy * unit).sum(0)}


def _philox(s, quads, kind):
    """Four 32-bit words for each group of four elements: Philox4x32-10, counter (group's number in its tensor, tensor, 2 step + kind)."""
    mask = 0xFFFFFFFF
    group = (torch.arange(len(s["owner"]), device="cuda") - s["first"])[:, None] * quads + torch.arange(quads, device="cuda")
    c = [(group & mask).view(-1), (group >> 32).view(-1), s["owner"].repeat_interleave(quads), torch.full((group.numel(),), (2 * s["step"] + kind) & mask, device="cuda")]
    k0, k1 = s["seed"] & mask, s["seed"] >> 32

    def product(a, b):   # high and low word of a 32 x 32 bit product, in halves so that 63 bits suffice
        low, high = (a & 0xFFFF) * b, (a >> 16) * b
        t = high + (low >> 16)
        return t >> 16, ((t & 0xFFFF) << 16) | (low & 0xFFFF)

    for _ in range(10):
        h0, l0 = product(c[0], 0xD2511F53)
        h1, l1 = product(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & mask, (k1 + 0xBB67AE85) & mask
    return c


def _uniforms(low, high):
    """16-bit uniforms of groups of four elements: the halves of two words, low half first."""
    return torch.stack([low & 0xFFFF, low >> 16, high & 0xFFFF, high >> 16], 1).view(-1)


def _stored(x, u, floor):
    """8-bit form of a state: codes and a scale for each 128 elements.  u: 16-bit uniforms (None: to nearest).  floor: what is positive stays so."""
    blocks = x.view(-1, BLOCK)
    scale = _scale(blocks.abs().amax(1))
    t = (blocks * scale[:, None]).view(-1)
    if u is not None:
        a = t.abs().clamp(max=E4M3_MAX)
        step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))).clamp(-6, 8) - 3)
        step = torch.where(a < 8 * step, step / 2, torch.where(a >= 16 * step, step * 2, step)).clamp(min=2.0 ** -9)   # log2 next to a power of two
        low = torch.floor(a / step)
        t = torch.copysign((low + ((a / step - low) * 65536.0 > u + 0.5)) * step, t)
    codes = t.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
    if floor:
        codes = torch.where((x > 0) & (codes.float() == 0), torch.full_like(t, 2.0 ** -9), codes.float()).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), scale


def _read(codes, scale):
    return (codes.view(torch.float8_e4m3fn).float().view(-1, BLOCK) / scale[:, None]).view(-1)


def _plain_adamw(s):
    case = s["case"]
    g, p = s["g"].float(), s["p"].float()
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m, v = _read(s["m"], s["m_scale"]), _read(s["v"], s["v_scale"]).square()
    m = s["beta1"] * m + (1 - s["beta1"]) * g
    v = s["beta2"] * v + (1 - s["beta2"]) * g.square()
    down1, down2 = 1 - s["beta1"] ** s["step"], 1 - s["beta2"] ** s["step"]
    keep = (1 - s["lr"] * s["decay_segments"].double()).float()
    p = (p.view(-1, SEGMENT) * keep[:, None]).view(-1) - (s["lr"] / down1) * m / (torch.sqrt(v) / math.sqrt(down2) + s["eps"])
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        got = {"m": s["m"], "v": s["v"]}
    else:
        um = uv = None
        if case["sr"]:
            w = _philox(s, SEGMENT // 4, 0)
            um, uv = _uniforms(w[0], w[1]), _uniforms(w[2], w[3])
        for name, x, u, floor in (("m", m, um, False), ("v", torch.sqrt(v), uv, True)):
            codes, scale = _stored(x, u, floor)
            s[name].copy_(codes)
            s[name + "_scale"].copy_(scale)
        got = {"m": s["m"].view(torch.float8_e4m3fn), "v": s["v"].view(torch.float8_e4m3fn), "m_scale": s["m_scale"], "v_scale": s["v_scale"]}
    if case["param"] == "fp32":
        s["p"].copy_(p)
    elif case["sr"]:
        w = _philox(s, SEGMENT // 4, 1)
        bits = (p.view(torch.int32).long() + (65535 - _uniforms(w[0], w[1]))) >> 16 << 16
        s["p"].copy_(bits.int().view(torch.float32).to(torch.bfloat16))
    else:
        s["p"].copy_(p.to(torch.bfloat16))
    got["p"] = s["p"]
    if s["copy"] is not None:
        s["copy"].copy_(s["p"].to(torch.bfloat16))
        got["copy"] = s["copy"]
    return got


# ---- from the definitions, in 64 bits ---------------------------------------------------------------------------------------------

def _nearest_code_values(t):
    """E4M3 values nearest to t (ties to the even code), from the list of all of them."""
    e = torch.arange(0, 127, device=t.device, dtype=torch.float64)
    table = torch.where(e < 8, e * 2.0 ** -9, (1 + (e % 8) / 8) * torch.exp2(torch.floor(e / 8) - 7))
    a = t.abs().clamp(max=E4M3_MAX)
    hi = torch.searchsorted(table, a).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    up, down = table[hi] - a, a - table[lo]
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    return torch.copysign(table[pick], t), table, lo, hi


def exact(case, seed):
    """What `run` returns, in 64 bits from the definitions."""
    s = prepare(case, seed)
    if case["op"] == "adamw":
        return _exact_adamw(case, s)
    x, gain = s["x"].double(), s["gain"].double()
    rows, cols = x.shape
    if case["op"] == "norm_bwd":
        dy, r = s["dy"].double(), s["rstd"].double()
        dot = torch.einsum("ij,j,ij->i", dy, gain, x)
        dx = torch.einsum("i,ij,j->ij", r, dy, gain) - torch.einsum("i,ij->ij", r ** 3 * dot / cols, x)
        if s["residual"] is not None:
            dx += s["residual"].double()
        return {"dx": dx, "dgain": torch.einsum("ij,ij,i->j", dy, x, r)}
    got = {}
    if s["residual"] is not None:
        x = (x + s["residual"].double()).to(torch.bfloat16).double()
        got["h"] = x
    got["rstd"] = (torch.linalg.vector_norm(x, dim=1) ** 2 / cols + EPS_NORM) ** -0.5
    y = torch.einsum("ij,i,j->ij", x, got["rstd"], gain)
    if case["out"] == "bf16":
        return {**got, "y": y}

    def tiles(z):
        codes, scales = [], []
        for a in range(0, z.shape[1], 128):
            part = z[:, a: a + 128]
            most = part.abs().max(1).values
            scale = torch.where(most > 0, E4M3_MAX / most, 1.0)
            codes.append(_nearest_code_values(part * scale[:, None])[0])
            scales.append(scale)
        return torch.cat(codes, 1), torch.stack(scales)

    got["codes"], got["scales"] = tiles(y)
    if case["out"] == "dual":
        got["codes_t"], got["scales_t"] = tiles(y.t().contiguous())
    return got


def _exact_words(count, tensor, step2, seed):
    """The generator from its definition, with 32-bit words as 64-bit whole numbers and the high word of a product by splitting the constant."""
    n = torch.arange(count, device="cuda", dtype=torch.int64)
    x0, x1, x2, x3 = n % 2 ** 32, n // 2 ** 32, torch.full_like(n, tensor), torch.full_like(n, step2 % 2 ** 32)
    key = [seed % 2 ** 32, seed // 2 ** 32]

    def mul(x, c):
        mid = x * (c // 65536) + x * (c % 65536) // 65536
        return mid // 65536, (mid % 65536) * 65536 + x * (c % 65536) % 65536

    for r in range(10):
        (h0, l0), (h1, l1) = mul(x0, 0xD2511F53), mul(x2, 0xCD9E8D57)
        x0, x1, x2, x3 = h1 ^ x1 ^ ((key[0] + r * 0x9E3779B9) % 2 ** 32), l1, h0 ^ x3 ^ ((key[1] + r * 0xBB67AE85) % 2 ** 32), l0
    return x0, x1, x2, x3


def _exact_adamw(case, s):
    sizes = _sizes(case)
    starts, _ = _segments(sizes)
    out = {k: s[k].double() for k in ("p", "copy", "m", "v", "m_scale", "v_scale") if s.get(k) is not None}
    if case["bits"] == 8:
        out["m"], out["v"] = s["m"].view(torch.float8_e4m3fn).double(), s["v"].view(torch.float8_e4m3fn).double()
    t = s["step"]
    for i, (a, n) in enumerate(zip(starts, sizes)):
        at, blocks = slice(a * SEGMENT, a * SEGMENT + n), slice(a * SEGMENT // BLOCK, a * SEGMENT // BLOCK + -(-n // BLOCK))
        g, p, m, v = s["g"][at].double(), out["p"][at], out["m"][at], out["v"][at]
        if case["bits"] == 8:
            m = m / out["m_scale"][blocks].repeat_interleave(BLOCK)[:n]
            v = (v / out["v_scale"][blocks].repeat_interleave(BLOCK)[:n]) ** 2
        m, v = m + (1 - s["beta1"]) * (g - m), v + (1 - s["beta2"]) * (g * g - v)
        p = p - s["lr"] * s["decay"][i] * p - s["lr"] * (m / (1 - s["beta1"] ** t)) / ((v / (1 - s["beta2"] ** t)) ** 0.5 + s["eps"])
        words = _exact_words(-(-n // 4), i, 2 * t, s["seed"]) if case["sr"] and case["bits"] == 8 else None
        if case["bits"] == 32:
            out["m"][at], out["v"][at] = m, v
        else:
            for name, x, pair, floor in (("m", m, 0, False), ("v", v ** 0.5, 2, True)):
                whole = torch.zeros(-(-n // BLOCK) * BLOCK, device="cuda", dtype=torch.float64)
                whole[:n] = x
                most = whole.view(-1, BLOCK).abs().max(1).values
                scale = torch.where(most > 0, E4M3_MAX / most, 1.0).clamp(max=FLT_MAX)
                y = x * scale.repeat_interleave(BLOCK)[:n]
                value, table, lo, hi = _nearest_code_values(y)
                if words is not None:
                    u = torch.stack([words[pair] % 65536, words[pair] // 65536, words[pair + 1] % 65536, words[pair + 1] // 65536], 1).view(-1)[:n]
                    share = (y.abs().clamp(max=E4M3_MAX) - table[lo]) / (table[hi] - table[lo]).clamp(min=1e-300)
                    value = torch.copysign(torch.where(share > (u + 0.5) / 65536, table[hi], table[lo]), y)
                if floor:
                    value = torch.where((x > 0) & (value == 0), 2.0 ** -9, value)
                out[name][at], out[name + "_scale"][blocks] = value, scale
        if case["param"] == "bf16" and case["sr"]:
            w = _exact_words(-(-n // 4), i, 2 * t + 1, s["seed"])
            u = torch.stack([w[0] % 65536, w[0] // 65536, w[1] % 65536, w[1] // 65536], 1).view(-1)[:n]
            grid = torch.exp2(torch.floor(torch.log2(p.abs().clamp(min=2.0 ** -126))) - 7)   # spacing of bf16 at p
            low = torch.floor(p.abs() / grid)
            p = torch.copysign((low + (p.abs() / grid - low > (u + 0.5) / 65536)) * grid, p)
        out["p"][at] = p
        if "copy" in out:
            out["copy"][at] = p
    return out
