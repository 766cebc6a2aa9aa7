"""The microscaled operators as a model's forward pass calls them: what is timed, and what the results must be.

Three operators, each on the formats of the OCP microscaling specification: blocks of 32 values along a row share
one power-of-two scale (E8M0, floor(log2(amax)) minus the element type's largest exponent), the elements are E2M1
(4 bits) or E4M3 (8 bits), rounded to nearest even and saturated.

  quantize  activations or weights to codes and scales, with the values that the codes stand for
  rmsnorm   h = x + residual, y = h / sqrt(mean(h^2) + eps) * gamma, y to 8 bits with scales
  matmul    y = a w^T of quantised activations (4 or 8 bits) and 4-bit weights
  linear    the same from bf16 activations, which the call quantises first

Codes are [rows][row bytes], padded with zeros to a multiple of 128 values, two 4-bit codes a byte, the even one in
the low half.  Scales are tiles of 128 rows x 4 blocks, [row tile][k tile][row % 32][row / 32 % 4][block % 4].
"""
import math

import torch

own = False

FLOAT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-5


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token's activations on the way into a projection of a 70B-size model: launch latency
        dict(name="quantize_token", op="quantize", rows=1, k=8192, dtype="bf16", bits=4),
        # the calibration set of a 7B-size model, as the quantised model sees it
        dict(name="quantize_prompt", op="quantize", rows=16384, k=4096, dtype="bf16", bits=4),
        # an fp32 matrix of odd sizes: rows that are not 16-byte aligned, a last block that is not full
        dict(name="quantize_odd", op="quantize", rows=5000, k=5111, dtype="fp32", bits=8),
        # one decoded token between two layers
        dict(name="rmsnorm_token", op="rmsnorm", rows=1, k=4096, dtype="bf16", residual=True),
        # a batch of ragged prompts of a 13B-size model, first layer (no residual yet)
        dict(name="rmsnorm_ragged", op="rmsnorm", rows=1777, k=5120, dtype="fp16", residual=False),
        # the calibration set of a 70B-size model
        dict(name="rmsnorm_large", op="rmsnorm", rows=65536, k=8192, dtype="bf16", residual=True),
        # 16 sequences decode one token each; the 8-bit activations come from the norm
        dict(name="matmul_decode_a8", op="matmul", rows=16, k=8192, n=8192, bits=8),
        # a prompt through a 13B-size model's widening projection, 8-bit activations
        dict(name="matmul_prompt_a8", op="matmul", rows=2048, k=5120, n=13824, bits=8),
        # a long prompt through a 70B-size model's square projection, 4-bit activations
        dict(name="matmul_large", op="matmul", rows=16384, k=8192, n=8192, bits=4),
        # one decoded token through a 7B-size model's square projection
        dict(name="linear_token", op="linear", rows=1, k=4096, n=4096, bits=4),
        # a short prompt, every size ragged
        dict(name="linear_ragged", op="linear", rows=333, k=5111, n=5001, bits=4),
        # a prompt through a 7B-size model's widening projection
        dict(name="linear_prompt", op="linear", rows=4096, k=4096, n=11008, bits=4),
    ]


WIDTHS = [128, 256, 512, 640, 1024, 1280, 2048, 2560, 4096, 5120, 8192, 11008, 13824]  # of heads, layers, projections


def _log_uniform(rng, lo, hi):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return v + (v == 3072)  # a size that no configuration here has


def _width(rng, hi):
    """Half of the widths are a model's own, the others odd numbers or multiples of 8 that are none of 16."""
    kind = rng.random()
    if kind < 0.5:
        return rng.choice([v for v in WIDTHS if v <= hi])
    v = _log_uniform(rng, 96, hi - 16)
    return v | 1 if kind < 0.75 else v // 16 * 16 + 8


def draw(rng):
    op = rng.choice(["quantize", "rmsnorm", "matmul", "linear"])
    k = _width(rng, 8192)
    if op in ("quantize", "rmsnorm"):
        rows = min(_log_uniform(rng, 1, 65536), (1 << 27) // k)
        if op == "quantize":
            return dict(op=op, rows=rows, k=k, dtype=rng.choice(["bf16", "fp16", "fp32"]), bits=rng.choice([4, 8]))
        return dict(op=op, rows=rows, k=k, dtype=rng.choice(["bf16", "fp16"]), residual=rng.random() < 0.7)
    n = _width(rng, 14336)
    rows = min(_log_uniform(rng, 1, 16384), (1 << 40) // (k * n))
    return dict(op=op, rows=rows, k=k, n=n, bits=rng.choice([4, 8]))


def work(case):
    rows, k = case["rows"], case["k"]
    held = lambda r, bits: r * k * bits / 8 + r * math.ceil(k / 32)  # codes and scales  # noqa: E731
    if case["op"] in ("quantize", "rmsnorm"):
        size = FLOAT[case["dtype"]].itemsize
        if case["op"] == "quantize":  # read; codes, scales and values written
            return {"bytes": 2 * rows * k * size + held(rows, case["bits"]), "flops": 4 * rows * k}
        # x (and residual) read; h, codes, scales and values written; gamma
        return {"bytes": rows * k * size * (3 + case["residual"]) + held(rows, 8) + k * size, "flops": 8 * rows * k}
    a = held(rows, case["bits"]) if case["op"] == "matmul" else 2 * rows * k
    return {"bytes": a + held(case["n"], 4) + 2 * rows * case["n"], "flops": 2 * rows * k * case["n"]}


# ------------------------------------------------------------------------------------------------ plain forms
E_MAX = {4: 2, 8: 8}           # exponent of the largest element: 6 = 1.5 * 2^2, 448 = 1.75 * 2^8
LARGEST = {4: 6.0, 8: 448.0}
E_MIN = {4: 0, 8: -6}          # exponent of the smallest normal element
MANTISSA = {4: 1, 8: 3}        # mantissa bits


def _floor_log2(v):
    """floor(log2(v)) of positive normal fp32 values, from the exponent field (-127 for zero and subnormals)."""
    return (v.view(torch.int32) >> 23) - 127


def _pow2(e):
    """2^e in fp32 for -149 <= e <= 127."""
    half = e >> 1
    return ((half + 127) << 23).view(torch.float32) * ((e - half + 127) << 23).view(torch.float32)


def _quantize(x, bits):
    """(elements [rows][blocks][32] in fp32, scale exponents [rows][blocks]) of x [rows][k], k padded to 32."""
    rows, k = x.shape
    x = torch.nn.functional.pad(x.float(), (0, -k % 32)).view(rows, -1, 32)
    e = (_floor_log2(x.abs().amax(-1)) - E_MAX[bits]).clamp(-127, 127)
    v = (x * _pow2(-e).unsqueeze(-1)).clamp(-LARGEST[bits], LARGEST[bits])
    step = _pow2(_floor_log2(v.abs()).clamp(min=E_MIN[bits]) - MANTISSA[bits])
    return torch.round(v / step) * step, e


def _values(q, e, k):
    """The values the codes stand for, [rows][k] in fp32."""
    return (q * _pow2(e).unsqueeze(-1)).flatten(1)[:, :k]


def _pack(q, e, bits):
    """Codes and scales as the operators hold them."""
    rows, blocks, _ = q.shape
    tiles, row_tiles = -(-blocks // 4), -(-rows // 128)
    v = torch.nn.functional.pad(q.flatten(1), (0, tiles * 128 - blocks * 32))
    if bits == 8:
        codes = v.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        a = v.abs()
        mag = torch.where(a < 2, a * 2, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
        mag = mag | ((v < 0).to(torch.uint8) << 3)
        codes = mag[:, 0::2] | (mag[:, 1::2] << 4)
    s = torch.nn.functional.pad((e + 127).to(torch.uint8), (0, tiles * 4 - blocks, 0, row_tiles * 128 - rows))
    return codes.contiguous(), s.view(row_tiles, 4, 32, tiles, 4).permute(0, 3, 2, 1, 4).contiguous().view(-1)


def _unpack(codes, scales, rows, k, bits):
    """Values in fp32, [rows][k], of codes and scales as the operators hold them."""
    tiles = -(-k // 128)
    if bits == 8:
        v = codes.view(torch.float8_e4m3fn).float()
    else:
        table = torch.tensor([0, .5, 1, 1.5, 2, 3, 4, 6, -0., -.5, -1, -1.5, -2, -3, -4, -6], device=codes.device)
        v = table[torch.stack((codes & 15, codes >> 4), -1).flatten(1).int()]
    s = scales.view(-1, tiles, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, tiles * 4)[:rows]
    return (v.view(rows, -1, 32) * _pow2(s.int() - 127).unsqueeze(-1)).flatten(1)[:, :k]


def _norm(x, residual, gamma):
    h = x.float() if residual is None else x.float() + residual.float()
    return h, h * torch.rsqrt(torch.mean(h * h, -1, keepdim=True) + EPS) * gamma.float()


# ------------------------------------------------------------------------------------------------ inputs
def _activations(rows, k, g):
    """Student-t (3 degrees of freedom) with 1 % of the channels 20 to 100 times larger: zero mean, heavy tails."""
    x = torch.randn(rows, k, device="cuda", generator=g)
    chi = sum(torch.randn(rows, k, device="cuda", generator=g).square_() for _ in range(3))
    x /= chi.div_(3).sqrt_().clamp_(min=0.05)
    big = torch.rand(k, device="cuda", generator=g) < 0.01
    return x * torch.where(big, 20 + 80 * torch.rand(k, device="cuda", generator=g), 1.0)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, k, op = case["rows"], case["k"], case["op"]
    s = dict(op=op, rows=rows, k=k, bits=case.get("bits", 8))
    row_bytes = lambda bits: -(-k // 128) * 16 * bits  # noqa: E731
    scale_bytes = -(-rows // 128) * -(-k // 128) * 512
    if op in ("quantize", "rmsnorm"):
        dtype = FLOAT[case["dtype"]]
        s["x"] = _activations(rows, k, g).to(dtype)
        s["codes"] = torch.empty(rows, row_bytes(s["bits"]), dtype=torch.uint8, device="cuda")
        s["scales"] = torch.empty(scale_bytes, dtype=torch.uint8, device="cuda")
        s["values"] = torch.empty_like(s["x"])
        if op == "rmsnorm":
            s["residual"] = torch.randn(rows, k, device="cuda", generator=g).to(dtype) if case["residual"] else None
            s["gamma"] = (1 + 0.1 * torch.randn(k, device="cuda", generator=g)).to(dtype)
            s["h"] = torch.empty_like(s["x"])
        return s
    n = case["n"]
    w = torch.randn(n, k, device="cuda", generator=g) / math.sqrt(k)
    s["n"] = n
    s["w_codes"], s["w_scales"] = _pack(*_quantize(w, 4), 4)
    s["x"] = _activations(rows, k, g).to(torch.bfloat16)
    if op == "matmul":
        s["a_codes"], s["a_scales"] = _pack(*_quantize(s.pop("x"), s["bits"]), s["bits"])
    else:
        s["workspace"] = torch.empty(rows * row_bytes(s["bits"]) + scale_bytes, dtype=torch.uint8, device="cuda")
    s["y"] = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _run_plain(s):
    k, bits = s["k"], s["bits"]
    if s["op"] == "quantize":
        return _values(*_quantize(s["x"], bits), k).to(s["x"].dtype)
    if s["op"] == "rmsnorm":
        h, y = _norm(s["x"], s["residual"], s["gamma"])
        return {"h": h.to(s["x"].dtype), "y": _values(*_quantize(y, bits), k).to(s["x"].dtype)}
    if s["op"] == "matmul":
        a = _unpack(s["a_codes"], s["a_scales"], s["rows"], k, bits)
    else:
        a = _values(*_quantize(s["x"], bits), k)
    return torch.matmul(a, _unpack(s["w_codes"], s["w_scales"], s["n"], k, 4).t()).to(torch.bfloat16)


def _run_own(s):
    import paper_2511_04063_b200 as dq

    fmt = dq.DQ_MXFP4 if s["bits"] == 4 else dq.DQ_MXFP8
    if s["op"] == "quantize":
        dq.dq_mx_quantize(s["x"], fmt, s["codes"], s["scales"], values=s["values"])
        return s["values"]
    if s["op"] == "rmsnorm":
        dq.dq_rmsnorm_quantize(s["x"], s["gamma"], EPS, fmt, s["codes"], s["scales"], residual=s["residual"],
                               sum_out=s["h"], values=s["values"])
        return {"h": s["h"], "y": s["values"]}
    if s["op"] == "matmul":
        dq.dq_mx_matmul(s["a_codes"], s["a_scales"], fmt, s["w_codes"], s["w_scales"], s["k"], s["y"])
    else:
        dq.dq_mx_linear(s["x"], fmt, s["w_codes"], s["w_scales"], s["y"], s["workspace"])
    return s["y"]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ 64 bits
def _grid(bits):
    """Every non-negative element value, ascending: index = code."""
    if bits == 4:
        return [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    return [m * 2.0 ** -9 for m in range(8)] + [(1 + m / 8) * 2.0 ** e for e in range(-6, 9) for m in range(8)][:-1]


def _exact_quantized(x, bits):
    """Values of x (float64) after quantisation: nearest element by search, ties to the even code."""
    rows, k = x.shape
    x = torch.cat((x, x.new_zeros(rows, -k % 32)), 1).reshape(rows, -1, 32)
    amax = x.abs().max(-1, keepdim=True).values
    e = torch.where(amax > 0, torch.frexp(amax).exponent - 1 - E_MAX[bits], -127).clamp(-127, 127)
    v = torch.ldexp(x, -e)
    grid = torch.tensor(_grid(bits), dtype=torch.float64, device=x.device)
    mids = (grid[1:] + grid[:-1]) / 2
    at = torch.searchsorted(mids, v.abs().contiguous())       # the number of mid points below |v|
    tie = mids[at.clamp(max=len(mids) - 1)] == v.abs()
    at = torch.where(tie & (at % 2 == 1) & (at < len(mids)), at + 1, at)
    return (torch.ldexp(grid[at], e) * torch.sign(v)).reshape(rows, -1)[:, :k]


def exact(case, seed):
    s = prepare(case, seed)
    rows, k, bits = s["rows"], s["k"], s["bits"]
    step = max(1, (1 << 26) // k)
    if s["op"] == "quantize":
        parts = [_exact_quantized(s["x"][r:r + step].double(), bits).to(s["x"].dtype).double() for r in range(0, rows, step)]
        return torch.cat(parts)
    if s["op"] == "rmsnorm":
        hs, ys = [], []
        for r in range(0, rows, step):
            h = s["x"][r:r + step].double()
            if s["residual"] is not None:
                h = h + s["residual"][r:r + step].double()
            y = h / torch.sqrt(h.square().mean(1, keepdim=True) + EPS) * s["gamma"].double()
            hs.append(h)
            ys.append(_exact_quantized(y, bits))
        return {"h": torch.cat(hs), "y": torch.cat(ys)}
    signed = torch.tensor(_grid(4) + [-v for v in _grid(4)], dtype=torch.float64, device="cuda")
    w = torch.stack((signed[(s["w_codes"] % 16).long()], signed[(s["w_codes"] // 16).long()]), 2).flatten(1)
    held = {"w": (w, s["w_scales"], s["n"])}
    if s["op"] == "linear":
        a = torch.cat([_exact_quantized(s["x"][r:r + step].double(), bits) for r in range(0, rows, step)])
    elif bits == 8:
        held["a"] = (s["a_codes"].view(torch.float8_e4m3fn).double(), s["a_scales"], rows)
    else:
        v = torch.stack((signed[(s["a_codes"] % 16).long()], signed[(s["a_codes"] // 16).long()]), 2).flatten(1)
        held["a"] = (v, s["a_scales"], rows)
    tiles = -(-k // 128)
    block = torch.arange(tiles * 4, device="cuda")
    for name, (v, scales, count) in held.items():
        r = torch.arange(count, device="cuda")[:, None]
        at = ((r // 128) * tiles + block // 4) * 512 + r % 32 * 16 + r // 32 % 4 * 4 + block % 4
        e = scales[at].int() - 127
        held[name] = torch.ldexp(v.view(count, -1, 32), e[:, :, None]).flatten(1)[:, :k]
    return (held["a"] if "a" in held else a) @ held["w"].t()
