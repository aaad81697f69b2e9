"""What the microscaled (MX) operators are timed on: block-scaled 4- and 8-bit quantization, the product of such operands, the
8-bit activation checkpoint and the weight gradient that reads it.

An MX tensor is a matrix of `lines` x `length` elements whose lines are cut into blocks of 32.  A block has one scale, a power of
two held as a byte (exponent + 127): the smallest s with max <= 7 s.  In 4 bits an element is one E2M1 code h, the nearest to x / s; in
8 bits it is two, h and the nearest to what is left at an eighth of the scale: x ~ s (h + l / 8).  Ties go to the even code, magnitudes
above 6 saturate.  Codes lie two to a byte, the earlier element in the low half, the second codes of 8 bits in a plane of their own
behind the first; a line takes pitch(length) = length rounded up to 512 elements, and what lies behind its end is zero.

A case says by "op" what runs:
  quantize    x [M x K] -> its values as an MX tensor along rows and as one along columns, from one read
  checkpoint  x [M x K] -> saved in 8 bits along columns (a block is 32 tokens of one channel), and restored
  gemm        two MX operands at hand -> their product [M x N] over K
  linear      tokens [M x K] through a layer whose weights are at hand in 4 bits -> [M x N]
  wgrad       output gradient [M x N] and a checkpoint of the activations at hand -> dW [K x N] in fp32
  step        activations, master weights and output gradient -> Y, dA and dW: weights quantized along both axes, forward pass with
              its checkpoint, backward pass

Shapes are those of the benchmark's layers (LLaMA-2 1.3B, 7B and 13B), of the tests, and generic ones.  Inputs follow the benchmark's
recipe: weights N(0, 0.02^2), output gradients N(0, 0.01^2), activations N(0, 1) with a few channels scaled up, or Student-t with
three degrees of freedom.
"""
import math

import torch

own = False

BLOCK, PITCH = 32, 512


def _case(name, op, M, K, N=0, dtype="bf16", bits=4, grad=4, act="channels"):
    """bits: of the activations (gemm: of the left operand, quantize: along rows); grad: of the output gradient along tokens (gemm: of the right operand)."""
    return {"name": name, "op": op, "M": M, "K": K, "N": N, "dtype": dtype, "bits": bits, "grad": grad, "act": act}


def listed():
    return [
        # one token through a square 7B projection whose weights are quantized already: decoding, where latency counts
        _case("serve-1x4096x4096", "linear", 1, 4096, 4096),
        # a batch of decoding sequences through the 7B gate projection, activations kept in 8 bits
        _case("serve-24x4096x11008-a8", "linear", 24, 4096, 11008, bits=8),
        # a 1.3B feed-forward product between operands that are at hand, output width no multiple of a tile
        _case("gemm-8192x2048x5504", "gemm", 8192, 2048, 5504),
        # the largest product: the 7B attention input projection over a training batch
        _case("gemm-16384x4096x12288", "gemm", 16384, 4096, 12288),
        # fp32 master weights of the 7B gate projection after an optimizer step: both orientations from one read
        _case("quantize-4096x11008-f32", "quantize", 4096, 11008, dtype="f32", act="weights"),
        # activations whose rows and columns end inside a block
        _case("quantize-1055x1384", "quantize", 1055, 1384),
        # what a 7B layer saves of its input for the backward pass, and its return
        _case("checkpoint-16384x4096", "checkpoint", 16384, 4096),
        # a short ragged batch in fp32, heavy-tailed
        _case("checkpoint-77x5504-f32", "checkpoint", 77, 5504, dtype="f32", act="student-t"),
        # the 7B output projection's weight gradient
        _case("wgrad-8192x4096x4096", "wgrad", 8192, 4096, 4096),
        # odd everything, output gradient in 8 bits as well
        _case("wgrad-1055x1376x2080-g8", "wgrad", 1055, 1376, 2080, grad=8),
        # a 1.3B feed-forward layer's whole training step
        _case("step-8192x2048x5504", "step", 8192, 2048, 5504),
        # the smallest configuration's step, fp32 masters
        _case("step-256x512x512-f32", "step", 256, 512, 512, dtype="f32"),
    ]


def _cost(c):
    if c["op"] in ("quantize", "checkpoint"):
        return 300.0 * c["M"] * c["K"] * (2.0 if c["op"] == "quantize" else 1.0)
    return 2.0 * c["M"] * c["K"] * c["N"] * (3.0 if c["op"] == "step" else 1.0)


def draw(rng):
    """One more case of the same ranges: sizes over their logarithm, channels multiples of 8, any number of tokens."""
    def size(lo, hi, unit):
        return max(lo, min(hi, unit * round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / unit)))

    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(["linear", "linear", "linear", "gemm", "gemm", "quantize", "checkpoint", "wgrad", "wgrad", "step", "step"])
        f32 = op != "gemm" and rng.random() < 0.25
        few = op == "linear" and rng.random() < 0.7
        c = {
            "op": op,
            "M": size(1, 64, 1) if few else size(64, 4096 if f32 else 16384, 1),
            "K": size(256, 13824, 8),
            "N": 0 if op in ("quantize", "checkpoint") else size(256, 15360, 8),
            "dtype": "f32" if f32 else "bf16",
            "bits": 8 if op in ("linear", "gemm", "step", "quantize") and rng.random() < 0.3 else 4,
            "grad": 8 if op in ("wgrad", "step", "gemm") and rng.random() < 0.3 else 4,
            "act": "student-t" if rng.random() < 0.3 else "channels",
        }
        if _cost(c) <= most:
            return c


# ---- the plain form ----------------------------------------------------------------------------------------------------------

def _pitch(n):
    return (n + PITCH - 1) // PITCH * PITCH


def _nearest(v):
    """v rounded to E2M1's values, ties to the even code, saturating."""
    step = torch.ldexp(torch.ones_like(v), (torch.frexp(v)[1] - 1).clamp(min=0) - 1)
    return (torch.round(v / step) * step).clamp(-6.0, 6.0)


def _scaled(x, bits):
    """fp32 x [lines x length] -> what the codes of each plane stand for before scaling and the blocks' exponents, padded to the pitch."""
    lines, length = x.shape
    p = _pitch(length)
    if p != length:
        x = torch.nn.functional.pad(x, (0, p - length))
    x = x.reshape(lines, p // BLOCK, BLOCK)
    m, e = torch.frexp(x.abs().amax(dim=2, keepdim=True))      # the largest magnitude is m * 2^e, m in [0.5, 1)
    e = e - 3 + (m > 0.875).to(e.dtype)                        # 7 = 0.875 * 2^3
    least = -126 if bits == 4 else -123
    e = torch.where(m > 0, e.clamp(least, 127), torch.full_like(e, least))
    v = torch.ldexp(x, -e)
    high = _nearest(v)
    planes = [high] if bits == 4 else [high, _nearest((v - high) * 8.0)]
    return [t.reshape(lines, p) for t in planes], e.reshape(lines, p // BLOCK)


def _joined(planes, e, length):
    v = planes[0] if len(planes) == 1 else planes[0] + planes[1] / 8.0
    lines = v.shape[0]
    return torch.ldexp(v.reshape(lines, -1, BLOCK), e.unsqueeze(2)).reshape(lines, -1)[:, :length]


def _values(x, bits):
    """x as its MX codes along the last axis hold it, fp32."""
    return _joined(*_scaled(x.float(), bits), x.shape[1])


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _encode(x, bits):
    """(codes, scales) of x along its last axis: bytes, as the framework lays them out."""
    planes, e = _scaled(x.float(), bits)
    v = torch.stack(planes) if bits == 8 else planes[0]
    code = torch.bucketize(v.abs(), torch.tensor(_E2M1, device=x.device)).to(torch.uint8) | ((v < 0).to(torch.uint8) << 3)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _decode(codes, scales, bits, length):
    """fp32 values of an MX tensor."""
    c = torch.stack([codes & 15, codes >> 4], dim=-1).flatten(-2).to(torch.int32)
    v = torch.tensor(_E2M1, device=codes.device)[c & 7] * (1 - 2 * (c >> 3))
    return _joined([v] if bits == 4 else list(v), scales.to(torch.int32) - 127, length)


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def prepare(case, seed):
    M, K, N = case["M"], case["K"], case["N"]
    dt = _dtype(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * int(seed) + 29)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda", dtype=torch.float32)

    if case["act"] == "weights":
        x = normal(M, K) * 0.02
    elif case["act"] == "channels":
        x = normal(M, K)
        ch = torch.randperm(K, generator=g, device="cuda")[:max(1, round(0.001 * K))]
        x[:, ch] *= 50.0
    else:
        x = normal(M, K) / torch.sqrt((normal(M, K) ** 2 + normal(M, K) ** 2 + normal(M, K) ** 2) / 3.0)
    x = x.to(dt)
    s = {"case": case}
    op = case["op"]
    if op in ("quantize", "checkpoint", "linear", "step"):
        s["x"] = x
    if op == "gemm":
        s["l"] = _encode(x, case["bits"])
        s["r"] = _encode((normal(N, K) * 0.02).to(dt), case["grad"])
        s["Y"] = torch.empty(M, N, device="cuda", dtype=dt)
    if op == "linear":
        s["r"] = _encode((normal(N, K) * 0.02).to(dt), 4)
        s["Y"] = torch.empty(M, N, device="cuda", dtype=dt)
    if op == "wgrad":
        s["saved"] = _encode(x.t(), 8)
    if op in ("wgrad", "step"):
        s["dY"] = (normal(M, N) * 0.01).to(dt)
        s["dW"] = torch.empty(K, N, device="cuda", dtype=torch.float32)
    if op == "step":
        s["W"] = (normal(K, N) * 0.02).to(dt)
        s["Y"] = torch.empty(M, N, device="cuda", dtype=dt)
        s["dA"] = torch.empty(M, K, device="cuda", dtype=dt)
    return s


def _run_plain(s):
    case = s["case"]
    op, M, K, N, dt = case["op"], case["M"], case["K"], case["N"], _dtype(case)
    if op == "quantize":
        return {"rows": _values(s["x"], case["bits"]).to(torch.bfloat16), "cols": _values(s["x"].t(), 4).t().to(torch.bfloat16).contiguous()}
    if op == "checkpoint":
        return {"x": _values(s["x"].t(), 8).t().to(dt).contiguous()}
    if op == "gemm":
        return {"Y": (_decode(*s["l"], case["bits"], K) @ _decode(*s["r"], case["grad"], K).t()).to(dt)}
    if op == "linear":
        return {"Y": (_values(s["x"], case["bits"]) @ _decode(*s["r"], 4, K).t()).to(dt)}
    if op == "wgrad":
        return {"dW": _decode(*s["saved"], 8, M) @ _values(s["dY"].t(), case["grad"]).t()}
    x, W, dY = s["x"], s["W"], s["dY"]
    return {"Y": (_values(x, case["bits"]) @ _values(W.t(), 4).t()).to(dt),
            "dA": (_values(dY, 4) @ _values(W, 4).t()).to(dt),
            "dW": _values(x.t(), 8) @ _values(dY.t(), case["grad"]).t()}


def _run_own(s):
    from paper_2501_17116_amd import binding as b

    case = s["case"]
    op, M, K, N, dt = case["op"], case["M"], case["K"], case["N"], _dtype(case)
    if op == "quantize":
        rows, cols = b.mx_quantize_both(s["x"], case["bits"], 4)
        return {"rows": b.mx_dequantize(rows, torch.bfloat16), "cols": b.mx_dequantize(cols, torch.bfloat16)}
    if op == "checkpoint":
        return {"x": b.mx_dequantize(b.mx_checkpoint_save(s["x"]), dt)}
    if op == "gemm":
        b.mx_gemm(b.MxTensor(*s["l"], K), b.MxTensor(*s["r"], K), out=s["Y"])
        return {"Y": s["Y"]}
    if op == "linear":
        b.mx_linear_fwd(s["x"], b.MxTensor(*s["r"], K), act_bits=case["bits"], Y=s["Y"])
        return {"Y": s["Y"]}
    if op == "wgrad":
        b.mx_linear_bwd_wgrad(s["dY"], b.MxTensor(*s["saved"], M, transposed=True), grad_bits=case["grad"], dW=s["dW"])
        return {"dW": s["dW"]}
    wq = b.mx_prepare_weights(s["W"])
    saved = b.mx_checkpoint(M, K)
    b.mx_linear_fwd(s["x"], wq.fwd, act_bits=case["bits"], saved=saved, Y=s["Y"])
    b.mx_linear_bwd(s["dY"], saved, wq.bwd, grad_bits=case["grad"], dA=s["dA"], dW=s["dW"])
    return {"Y": s["Y"], "dA": s["dA"], "dW": s["dW"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


def work(case):
    """Inputs once, outputs once; codes that one call leaves for the next are written once and read once."""
    op, M, K, N = case["op"], float(case["M"]), float(case["K"]), float(case["N"])
    e = 2.0 if case["dtype"] == "bf16" else 4.0
    width = {4: 0.5 + 1 / 32, 8: 1.0 + 1 / 32}                  # bytes of an element with its share of the scale
    left, right = width[case["bits"]], width[case["grad"]]
    if op == "quantize":
        return {"bytes": M * K * (e + 2 * (left + width[4]) + 4.0), "flops": 4.0 * M * K}
    if op == "checkpoint":
        return {"bytes": M * K * (2 * e + 2 * width[8]), "flops": 2.0 * M * K}
    if op == "gemm":
        return {"bytes": M * K * left + K * N * right + M * N * e, "flops": 2.0 * M * K * N}
    if op == "linear":
        return {"bytes": M * K * e + K * N * width[4] + M * N * e, "flops": 2.0 * M * K * N}
    if op == "wgrad":
        return {"bytes": M * K * width[8] + M * N * e + 4.0 * K * N, "flops": 2.0 * M * K * N}
    return {"bytes": e * (2 * M * K + K * N + 2 * M * N) + 4.0 * K * N + 2 * M * K * width[8] + 4 * K * N * width[4], "flops": 6.0 * M * K * N}


# ---- once more from the definition, in 64 bits, by tables ----------------------------------------------------------------------

def _by_table(x, bits):
    """fp64 values of x [lines x length] under a scale for every 32 elements of a line, codes found among E2M1's magnitudes."""
    lines, length = x.shape
    whole = -(-length // BLOCK) * BLOCK
    b = torch.zeros(lines, whole, dtype=torch.float64, device=x.device)
    b[:, :length] = x.double()
    b = b.reshape(-1, BLOCK)
    r = (b.abs().max(dim=1).values / 7.0).view(torch.int64)       # the smallest power of two not below max / 7, by the bits of a double
    e = (r >> 52) - 1023 + ((r & ((1 << 52) - 1)) != 0).to(torch.int64)
    scale = ((e.clamp(-126 if bits == 4 else -123, 127) + 1023) << 52).view(torch.float64).unsqueeze(1)
    grid = torch.tensor(_E2M1, dtype=torch.float64, device=x.device)
    mid = (grid[1:] + grid[:-1]) / 2

    def code_values(v):
        down, up = torch.bucketize(v.abs(), mid), torch.bucketize(v.abs(), mid, right=True)   # they differ on a midpoint: the even one of the two
        return torch.copysign(grid[torch.where(down % 2 == 0, down, up)], v)

    v = code_values(b / scale) * scale
    if bits == 8:
        v = v + code_values((b - v) / (scale / 8.0)) * (scale / 8.0)
    return v.reshape(lines, whole)[:, :length]


def _table_decode(codes, scales, bits, length):
    both = torch.tensor(_E2M1 + [-m for m in _E2M1], dtype=torch.float64, device=codes.device)
    scale = (scales.long() - 127 + 1023 << 52).view(torch.float64).repeat_interleave(BLOCK, dim=1)
    total = 0.0
    for plane, part in ((codes, 1.0),) if bits == 4 else ((codes[0], 1.0), (codes[1], 0.125)):
        v = torch.empty(plane.shape[0], 2 * plane.shape[1], dtype=torch.float64, device=codes.device)
        v[:, 0::2], v[:, 1::2] = both[(plane & 15).long()], both[(plane >> 4).long()]
        total = total + part * v * scale
    return total[:, :length]


def exact(case, seed):
    s = prepare(case, seed)
    op, M, K, N = case["op"], case["M"], case["K"], case["N"]
    if op == "quantize":
        return {"rows": _by_table(s["x"], case["bits"]), "cols": _by_table(s["x"].t(), 4).t()}
    if op == "checkpoint":
        return {"x": _by_table(s["x"].t(), 8).t()}
    if op == "gemm":
        return {"Y": _table_decode(*s["l"], case["bits"], K) @ _table_decode(*s["r"], case["grad"], K).t().contiguous()}
    if op == "linear":
        return {"Y": _by_table(s["x"], case["bits"]) @ _table_decode(*s["r"], 4, K).t().contiguous()}
    if op == "wgrad":
        return {"dW": _table_decode(*s["saved"], 8, M) @ _by_table(s["dY"].t(), case["grad"]).t().contiguous()}
    return {"Y": _by_table(s["x"], case["bits"]) @ _by_table(s["W"].t(), 4).t().contiguous(),
            "dA": _by_table(s["dY"], 4) @ _by_table(s["W"], 4).t().contiguous(),
            "dW": _by_table(s["x"].t(), 8) @ _by_table(s["dY"].t(), case["grad"]).t().contiguous()}
