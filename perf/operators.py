"""What the speed of the MXFP4 operators is measured on: matrices kept as 4-bit floating point with a shared scale for
every 32 weights of a row, and the products that decoding and prompts make with them, at the widths of
`synthetic_inputs.py`'s models and at sizes that fit no tile.

The format (OCP Microscaling Formats v1.0): a block of 32 consecutive weights of a row shares the scale 2^(floor(log2 max|w|) - 2);
an element is a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6, nearest to |w| / scale, ties to the even code, at most 6.

With `own` the calls are those of this package; without it the same results come from elementary torch operations.
"""
from __future__ import annotations

import math

import torch

own = False

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
BLOCK = 32


# ------------------------------------------------------------------------------------------
# the cases
# ------------------------------------------------------------------------------------------
# op          the call                                                        sizes
# quantize    weights to 4 bits, and the values they then stand for           rows x depth (gated: gate and up, rows each)
# dequantize  a packed matrix back to numbers                                 rows x depth
# linear      y = x W^T (+ residual)                                          n x rows from n x depth
# swiglu      h = silu(x Wg^T) * (x Wu^T)                                     n x rows from n x depth
# x: type of the activations (quantize: of the weights, dequantize: of the result); out: of the result;
# pad: elements between the end of a row of x (quantize: of w) and the next one.
def _case(name, op, rows, depth, n=0, x="bf16", out="bf16", residual=False, gated=False, pad=0):
    return dict(name=name, op=op, rows=rows, depth=depth, n=n, x=x, out=out, residual=residual, gated=gated, pad=pad)


def listed():
    return [
        # loading: the smallest model's gate matrix, a matrix that fits no tile (odd depth, rows apart), the 7B gate and up pair
        _case("quantize-tiny", "quantize", 688, 256, x="fp32", out="fp32"),
        _case("quantize-ragged", "quantize", 1001, 777, x="fp32", out="fp32", pad=23),
        _case("quantize-7b-gateup", "quantize", 11008, 4096, gated=True),
        # reading back: a 7B output projection, the 13B down projection in full precision
        _case("dequantize-7b-o", "dequantize", 4096, 4096),
        _case("dequantize-13b-down", "dequantize", 5120, 13824, x="fp32", out="fp32"),
        # products of one token (draft and plain decoding): the smallest model's, all latency, and the 7B q|k|v
        _case("linear-tiny-1", "linear", 256, 256, n=1, x="fp32", out="fp32"),
        _case("linear-7b-qkv-1", "linear", 12288, 4096, n=1),
        # a verification of eight drafts: the 7B down projection onto the residual stream
        _case("linear-7b-down-9", "linear", 4096, 11008, n=9, x="fp32", out="fp32", residual=True),
        # a prompt block at the 13B width
        _case("linear-13b-o-1024", "linear", 5120, 5120, n=1024, residual=True),
        # gated projections: one token in full precision, a full verification block at the 70B width, a ragged long prompt
        _case("swiglu-7b-1", "swiglu", 11008, 4096, n=1, x="fp32", out="fp32"),
        _case("swiglu-70b-32", "swiglu", 28672, 8192, n=32),
        _case("swiglu-7b-1999", "swiglu", 11008, 4096, n=1999),
    ]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    op = rng.choice(["quantize", "dequantize", "linear", "linear", "linear", "swiglu", "swiglu"])
    while True:
        rows, depth = log(100, 28672), log(64, 28672)
        if rng.random() < 0.7:  # (most widths are whole numbers of some tile, some of none)
            rows, depth = (rows + 31) // 32 * 32, (depth + 63) // 64 * 64
        # one token, a verification block, a candidate window or short prompt, a prompt
        n = rng.choice([1, 1, log(2, 32), log(2, 32), log(33, 128), log(129, 2000), log(129, 2000)])
        w = rows * depth * (2 if op == "swiglu" else 1)
        if w <= 2.4e8 and (op not in ("linear", "swiglu") or n * w <= 1.7e11):
            break
    if op in ("quantize", "dequantize"):
        t = rng.choice(["bf16", "fp32"])
        return {k: v for k, v in _case("", op, rows, depth, x=t, out=t, gated=op == "quantize" and rng.random() < 0.3 and w <= 1.2e8,
                                       pad=rng.choice([0, 0, 8, 13]) if op == "quantize" else 0).items() if k != "name"}
    return {k: v for k, v in _case("", op, rows, depth, n=n, x=rng.choice(["bf16", "bf16", "fp32"]), out=rng.choice(["bf16", "fp32"]),
                                   residual=op == "linear" and rng.random() < 0.5, pad=rng.choice([0, 0, 0, 8, 13])).items() if k != "name"}


# ------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------
def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 16 + stream)
    return g


def _strided(t, pad):
    """t's values in rows that lie `pad` elements apart."""
    if not pad:
        return t
    wide = torch.zeros(t.shape[0], t.shape[1] + pad, dtype=t.dtype, device=t.device)
    wide[:, : t.shape[1]] = t
    return wide[:, : t.shape[1]]


def _weights(case, seed, stream):
    """Rows of N(0, 0.02^2) whose sizes differ from row to row, a few columns that stand out, and some blocks of zeros (pruned or padded)."""
    g = _gen(seed, stream)
    rows, depth = case["rows"], case["depth"]
    w = torch.randn(rows, depth, device="cuda", generator=g)
    w *= 0.02 * torch.exp(0.5 * torch.randn(rows, 1, device="cuda", generator=g))
    w[:, torch.randint(0, depth, (max(1, depth // 256),), device="cuda", generator=g)] *= 6.0
    w[torch.randint(0, rows, (max(1, rows // 64),), device="cuda", generator=g), : min(depth, BLOCK)] = 0.0
    return w.to(DT[case["x"]] if case["op"] == "quantize" else torch.bfloat16)


def _activations(case, seed):
    """Normalised activations: about N(0, 1), a few channels an order of magnitude larger."""
    g = _gen(seed, 8)
    n, depth = case["n"], case["depth"]
    x = torch.randn(n, depth, device="cuda", generator=g)
    x[:, torch.randint(0, depth, (max(1, depth // 512),), device="cuda", generator=g)] *= 20.0
    return x.to(DT[case["x"]])


def _residual(case, seed):
    return torch.randn(case["n"], case["rows"], device="cuda", generator=_gen(seed, 9)).to(DT[case["out"]]) if case["residual"] else None


def _inputs(case, seed):
    pair = case["op"] == "swiglu" or case["gated"]
    ws = [_weights(case, seed, s) for s in ((1, 2) if pair else (1,))]
    x = _activations(case, seed) if case["n"] else None
    return ws, x, _residual(case, seed)


def prepare(case, seed):
    ws, x, r = _inputs(case, seed)
    if case["op"] == "quantize":
        ws = [_strided(w, case["pad"]) for w in ws]
    state = dict(case=case, x=None if x is None else _strided(x, case["pad"]), residual=r)
    if case["op"] == "quantize":
        state["w"] = ws
    elif own:
        import paper_2410_06916_amd as P
        state["packed"] = P.mx4_quantize_gated(*ws) if len(ws) == 2 else P.mx4_quantize(ws[0])
    else:
        state["packed"] = [_quantize(w) for w in ws]
    return state


# ------------------------------------------------------------------------------------------
# the plain form
# ------------------------------------------------------------------------------------------
def _quantize(w):
    """Two codes a byte, the earlier weight in the low half, and a byte of scale for each block."""
    rows, depth = w.shape
    blocks = (depth + BLOCK - 1) // BLOCK
    v = torch.nn.functional.pad(w.float(), (0, blocks * BLOCK - depth)).view(rows, blocks, BLOCK)
    top = v.abs().amax(-1, keepdim=True)
    # the exponent field of an fp32 number is floor(log2) + 127
    e = ((top.view(torch.int32) >> 23) - 2).clamp(min=0)
    q = v.abs().double() * torch.exp2(127.0 - e.double())
    # a value between two codes goes to the nearer one, one half way to the even one: the borders, and whether a value on one goes up
    code = ((q > 0.25).to(torch.uint8) + (q >= 0.75) + (q > 1.25) + (q >= 1.75) + (q > 2.5) + (q >= 3.5) + (q > 5.0)).to(torch.uint8)
    code = (code | (torch.signbit(v).to(torch.uint8) << 3)).view(rows, blocks * BLOCK)
    return code[:, 0::2] | (code[:, 1::2] << 4), e.view(rows, blocks).to(torch.uint8), depth


def _dequantize(packed):
    codes, scales, depth = packed
    table = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device=codes.device)
    code = torch.stack((codes & 15, codes >> 4), dim=-1).view(codes.shape[0], -1)
    v = table[code.int()].view(codes.shape[0], -1, BLOCK)
    return (v * torch.exp2(scales.float() - 127.0).unsqueeze(-1)).view(codes.shape[0], -1)[:, :depth]


def _plain(state):
    case, x, r = state["case"], state["x"], state["residual"]
    out = DT[case["out"]]
    if case["op"] == "quantize":
        return torch.cat([_dequantize(_quantize(w)) for w in state["w"]]).to(out)
    if case["op"] == "dequantize":
        return _dequantize(state["packed"][0]).to(out)
    ys = [torch.matmul(x.float(), _dequantize(p).t()) for p in state["packed"]]
    y = ys[0] if len(ys) == 1 else ys[0] / (1.0 + torch.exp(-ys[0])) * ys[1]
    return (y if r is None else y + r.float()).to(out)


def run(state):
    if not own:
        return _plain(state)
    import paper_2410_06916_amd as P
    case = state["case"]
    out = DT[case["out"]]
    if case["op"] == "quantize":
        w = state["w"]
        return P.mx4_dequantize(P.mx4_quantize_gated(*w) if len(w) == 2 else P.mx4_quantize(w[0]), out)
    if case["op"] == "dequantize":
        return P.mx4_dequantize(state["packed"], out)
    if case["op"] == "linear":
        return P.mx4_linear(state["x"], state["packed"], residual=state["residual"], out_dtype=out)
    return P.mx4_swiglu(state["x"], state["packed"], out_dtype=out)


# ------------------------------------------------------------------------------------------
# what a pass cannot do without, and its results in 64 bits
# ------------------------------------------------------------------------------------------
def work(case):
    rows, depth, n = case["rows"], case["depth"], case["n"]
    pair = 2 if case["op"] == "swiglu" or case["gated"] else 1
    size = {"bf16": 2, "fp32": 4}
    packed = pair * rows * (depth / 2 + (depth + BLOCK - 1) // BLOCK)
    if case["op"] == "quantize":
        return {"bytes": pair * rows * depth * (size[case["x"]] + size[case["out"]]) + packed, "flops": 10.0 * pair * rows * depth}
    if case["op"] == "dequantize":
        return {"bytes": packed + rows * depth * size[case["out"]], "flops": 2.0 * rows * depth}
    moved = n * depth * size[case["x"]] + n * rows * size[case["out"]] * (2 if case["residual"] else 1)
    return {"bytes": packed + moved, "flops": 2.0 * n * pair * rows * depth}


def _exact_values(w):
    """The format's definition on doubles: the scale from the largest magnitude's binary exponent, the element rounded (ties to even)
    to the spacing that the grid has where it lies."""
    rows, depth = w.shape
    v = torch.zeros(rows, -(-depth // BLOCK) * BLOCK, dtype=torch.float64, device=w.device)
    v[:, :depth] = w.double()
    v = v.view(rows, -1, BLOCK)
    exponent = torch.frexp(v.abs().amax(-1, keepdim=True)).exponent.double() - 1.0  # |m| = f 2^p with f in [1/2, 1): floor(log2) = p - 1
    scale = torch.exp2(torch.clamp(exponent - 2.0, min=-127.0))
    q = v / scale
    a = q.abs()
    step = torch.where(a < 2.0, 0.5, torch.where(a < 4.0, 1.0, 2.0))
    q = torch.sign(q) * torch.clamp(torch.round(a / step) * step, max=6.0)
    return (q * scale).view(rows, -1)[:, :depth]


def exact(case, seed):
    ws, x, r = _inputs(case, seed)
    vals = [_exact_values(w) for w in ws]
    if case["op"] in ("quantize", "dequantize"):
        return torch.cat(vals)
    ys = [x.double() @ v.t() for v in vals]
    if case["op"] == "swiglu":
        return torch.nn.functional.silu(ys[0]) * ys[1]
    return ys[0] if r is None else ys[0] + r.double()
