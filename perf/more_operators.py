"""Performance cases of a fine-tuning step's frozen parts and its end: the
projections that carry no adapter held in 8-bit floating point with a scale for
each block of 128, the cross entropy of an output layer without its logits, and
dropout whose mask is drawn again wherever it is needed.

What a user runs, by kind:
  fp8_roundtrip   a bf16 matrix quantised to 8 bits and read back
  fp8_fwd         Y = Q(X) Q(W)^T with W held in 8 bits and X quantised on the way
  fp8_bwd         dX = Q(dY) Q(W), the gradient through the same frozen weight
  xent_eval       cross entropy of softmax(X W^T) against each row's label
  xent_step       that loss and the gradient of X (and of W) in one call
  xent_fwd_bwd    the loss, then the gradients from what the forward saved
  dropout         Y = R + keep X / (1 - p), keep drawn from a seed and an offset

With `own` false a pass is made of elementary torch operations in 32 bits; with
`own` true it is the package's entry points.

8 bits.  A row is cut into blocks of 128 columns.  The rows of a weight share a
scale by 128 as well (blocks of 128 x 128); those of activations have their own.
A scale is 2^(s - 127), s one byte: the smallest with which the block's largest
magnitude is at most 448 times it, and 255 (NaN) where the block holds a NaN or an
infinity.  An element is its value over the scale, rounded to the nearest value of
4 significant bits from 2^-6 up and to the nearest multiple of 2^-9 below (ties
to even), as the byte sign, 4 bits of exponent (bias 7), 3 of fraction.  A row's
codes take 128 bytes per block, zero beyond the last column.  The scale of block
(i, b) of a weight stands at byte i ceil(k/128) + b; the scale of row i, block b
of activations at byte (b ceil(rows/64) + i/64) 64 + (i%16) 4 + (i/16)%4, zero for
rows beyond the last.

Dropout.  Element e of a tensor in row-major order is kept where its 16 bits of
Philox4x64-10 are below floor((1 - p) 2^16 + 1/2): key (seed, 0), counter offset +
e / 16 (128 bits, then two words of zero), of the block's four 64-bit words the
word (e % 16) / 4 and its bits 16 (e % 4) .. + 15.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

BF16, F32, F64, I32, I64, U8 = torch.bfloat16, torch.float32, torch.float64, torch.int32, torch.int64, torch.uint8


def listed() -> list:
    return [
        # the activations of a few generating sequences
        {"name": "fp8_roundtrip_tokens", "kind": "fp8_roundtrip", "m": 24, "k": 4096, "block_rows": 1},
        # a frozen 7B MLP input weight put into 8 bits
        {"name": "fp8_roundtrip_up_proj", "kind": "fp8_roundtrip", "m": 11008, "k": 4096, "block_rows": 128},
        # one token of one sequence through a frozen attention projection: generation
        {"name": "fp8_decode_o_proj", "kind": "fp8_fwd", "m": 1, "n": 4096, "k": 4096},
        # nothing a multiple of a tile or a block
        {"name": "fp8_ragged", "kind": "fp8_fwd", "m": 1531, "n": 4104, "k": 3208},
        # the 7B MLP input projection on one long prompt
        {"name": "fp8_up_proj", "kind": "fp8_fwd", "m": 4096, "n": 11008, "k": 4096},
        # the gradient of a short prompt through the 7B MLP output projection
        {"name": "fp8_down_proj_bwd", "kind": "fp8_bwd", "m": 1024, "n": 4096, "k": 11008},
        # the loss on held-out prompts, a vocabulary of odd size
        {"name": "xent_eval", "kind": "xent_eval", "rows": 512, "vocab": 32003, "k": 4096},
        # an answer of a few tokens: the weight is read for hardly any rows
        {"name": "xent_answer", "kind": "xent_step", "rows": 37, "vocab": 32000, "k": 4096, "dw": 0},
        # a fine-tuning step on one long prompt, the output layer frozen
        {"name": "xent_step", "kind": "xent_step", "rows": 4096, "vocab": 32000, "k": 4096, "dw": 0},
        # a trained output layer, loss and gradients in two calls
        {"name": "xent_trained_head", "kind": "xent_fwd_bwd", "rows": 1500, "vocab": 50021, "k": 2048, "dw": 1},
        # hidden states of a short prompt, an odd size
        {"name": "dropout_small", "kind": "dropout", "rows": 129, "cols": 4099, "dtype": "bf16", "p": 0.05, "residual": 0},
        # a long prompt's residual stream
        {"name": "dropout_residual", "kind": "dropout", "rows": 8192, "cols": 4096, "dtype": "bf16", "p": 0.1,
         "residual": 1},
    ]


# ---- drawn cases -----------------------------------------------------------
_WIDTHS = (512, 4096, 5120, 11008, 13824)
_MAX_MNK = 4096 * 11008 * 4096                 # the largest listed product of 8 bits
_MAX_XENT = 2 * 4096 * 32000 * 4096            # products of the largest listed loss


def _log_int(rng, lo: int, hi: int) -> int:
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng) -> int:
    return rng.choice(_WIDTHS) if rng.random() < 0.4 else 8 * _log_int(rng, 64, 1728)


def draw(rng) -> dict:
    kind = rng.choice(("fp8_roundtrip", "fp8_fwd", "fp8_fwd", "fp8_bwd", "fp8_bwd", "xent_eval", "xent_step",
                       "xent_step", "xent_fwd_bwd", "dropout"))
    if kind == "fp8_roundtrip":
        return {"kind": kind, "m": _log_int(rng, 1, 13824), "k": _width(rng), "block_rows": rng.choice((1, 128))}
    if kind.startswith("fp8"):
        n, k = _width(rng), _width(rng)
        return {"kind": kind, "m": _log_int(rng, 1, min(8192, _MAX_MNK // (n * k))), "n": n, "k": k}
    if kind == "dropout":
        cols = _width(rng) + rng.choice((0, 0, 1, 5))
        return {"kind": kind, "rows": _log_int(rng, 1, min(16384, 8192 * 4096 // (2 * cols))), "cols": cols,
                "dtype": rng.choice(("bf16", "bf16", "f32")), "p": rng.choice((0.0, 0.05, 0.1, 0.3, 0.5)),
                "residual": rng.choice((0, 1))}
    vocab = rng.choice((32000, 32003)) if rng.random() < 0.3 else _log_int(rng, 1000, 131072)
    k = rng.choice((512, 1024, 2048, 4096, 5120)) if rng.random() < 0.5 else 8 * _log_int(rng, 64, 640)
    dw = 0 if kind == "xent_eval" else rng.choice((0, 0, 1))
    cost = (1 if kind == "xent_eval" else 2 + dw) * vocab * k
    return {"kind": kind, "rows": _log_int(rng, 1, min(8192, _MAX_XENT // cost)), "vocab": vocab, "k": k, "dw": dw}


# ---- 8 bits, elementary ----------------------------------------------------
def _scale_bytes(amax):
    """The scale byte for a block's largest magnitude (fp32)."""
    bits = amax.view(I32)
    field = bits >> 23
    s = (field - 8 + ((bits & 0x7FFFFF) > 0x600000)).clamp_min(0)
    return torch.where(field == 255, 255, s)


def _power(e):
    """2^e of whole numbers from -126 to 127, from its bits: exact."""
    return ((e.to(I32) + 127) << 23).view(F32)


def _fp8_blocks(x, block_rows):
    """fp32 [rows, k] -> values over their scales [rows, B, 128] and scale bytes [rows, B], B blocks to a row."""
    rows, k = x.shape
    v = torch.zeros((rows, (k + 127) // 128 * 128), dtype=F32, device=x.device)
    v[:, :k] = x
    v = v.view(rows, -1, 128)
    # the largest as bits: a NaN or an infinity comes out on top
    amax = (v.view(I32) & 0x7FFFFFFF).amax(2)
    if block_rows > 1:
        groups = (rows + block_rows - 1) // block_rows
        padded = torch.zeros((groups * block_rows, amax.shape[1]), dtype=I32, device=x.device)
        padded[:rows] = amax
        amax = padded.view(groups, block_rows, -1).amax(1).repeat_interleave(block_rows, 0)[:rows]
    s = _scale_bytes(amax.contiguous().view(F32))
    y = v * _power(127 - s.clamp_max(253))[:, :, None]
    exponent = ((y.view(I32) >> 23) & 255) - 127
    step = _power(exponent.clamp_min(-6) - 3)
    return torch.round(y / step) * step, s


def _fp8_values(y, s):
    """Values over their scales and scale bytes [.., B] -> the values in fp32 [rows, 128 B]."""
    unit = _power(s.to(I32).clamp(1, 254) - 127) * torch.where(s == 0, 0.5, 1.0)
    unit = torch.where(s == 255, torch.full_like(unit, math.nan), unit)
    return (y * unit[:, :, None]).view(y.shape[0], -1)


def _fp8_quantised(x, block_rows):
    y, s = _fp8_blocks(x, block_rows)
    return _fp8_values(torch.where((s == 255)[:, :, None], 0.0, y), s)[:, :x.shape[1]]


def _weight_values(codes, scales, k):
    """A weight's codes and scales -> fp32 [n, k]."""
    n = codes.shape[0]
    s = scales.view((n + 127) // 128, -1).repeat_interleave(128, 0)[:n]
    return _fp8_values(codes.view(torch.float8_e4m3fn).to(F32).view(n, -1, 128), s)[:, :k]


# ---- the generator, elementary ---------------------------------------------
_M0, _M1 = 0xD2E7470EE14C6C93, 0xCA5A826395121157
_W0, _W1 = 0x9E3779B97F4A7C15, 0xBB67AE8584CAA73B
_MASK64 = (1 << 64) - 1


def _signed(x: int) -> int:
    x &= _MASK64
    return x - (1 << 64) if x >> 63 else x


def _mul(a: int, b):
    """High and low words of a times each of b, 64-bit words held as signed."""
    low = 0xFFFFFFFF
    a0, a1, b0, b1 = a & low, a >> 32, b & low, (b >> 32) & low
    t = a1 * b0 + (((a0 * b0) >> 32) & low)
    u = a0 * b1 + (t & low)
    return a1 * b1 + ((t >> 32) & low) + ((u >> 32) & low), b * _signed(a)


def _draws(seed, offset, count, device):
    """The 16-bit draws of elements 0 .. count - 1 (I64)."""
    t = torch.arange((count + 15) // 16, device=device, dtype=I64)
    c0 = t + _signed(offset)
    # the carry into the counter's second word: the sum, unsigned, below what was added
    c1 = ((c0 ^ -(1 << 63)) < _signed(offset ^ (1 << 63))).to(I64)
    c2, c3 = torch.zeros_like(c0), torch.zeros_like(c0)
    k0, k1 = seed & _MASK64, 0
    for _ in range(10):
        h0, l0 = _mul(_M0, c0)
        h1, l1 = _mul(_M1, c2)
        c0, c1, c2, c3 = h1 ^ c1 ^ _signed(k0), l1, h0 ^ c3 ^ _signed(k1), l0
        k0, k1 = (k0 + _W0) & _MASK64, (k1 + _W1) & _MASK64
    words = torch.stack((c0, c1, c2, c3), 1)
    shift = torch.arange(0, 64, 16, device=device)
    return ((words[:, :, None] >> shift) & 0xFFFF).view(-1)[:count]


def _threshold(p):
    return math.floor((1.0 - float(np.float32(p))) * 65536.0 + 0.5)


# ---- inputs ----------------------------------------------------------------
def _normal(shape, gen, std=1.0):
    return torch.randn(shape, generator=gen, device="cuda", dtype=F32).mul_(std)


def prepare(case: dict, seed: int) -> dict:
    """Inputs on the GPU, and the output buffers that a program keeps."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    st = {"kind": kind}

    def empty(shape, dtype):
        return torch.empty(shape, dtype=dtype, device="cuda")

    if kind == "fp8_roundtrip":
        m, k = case["m"], case["k"]
        gain = torch.where(torch.rand(k, generator=gen, device="cuda") < 0.005, 20.0, 1.0)
        blocks, by = (k + 127) // 128, case["block_rows"]
        x = _normal((m, k), gen) * (gain if by == 1 else k ** -0.5)
        st.update(X=x.to(BF16), by=by, codes=empty((m, 128 * blocks), U8), values=empty((m, k), BF16),
                  scales=empty((m + 63) // 64 * 64 * blocks if by == 1 else (m + 127) // 128 * blocks, U8))
        return st
    if kind.startswith("fp8"):
        m, n, k = case["m"], case["n"], case["k"]
        y, s = _fp8_blocks(_normal((n, k), gen, k ** -0.5).to(BF16).float(), 128)
        st["k"] = k
        st["Wc"] = y.view(n, -1).to(torch.float8_e4m3fn).view(U8)
        st["Ws"] = s[::128].to(U8).contiguous().view(-1)
        if kind == "fp8_fwd":
            # hidden states: a few channels much larger than the others
            gain = torch.where(torch.rand(k, generator=gen, device="cuda") < 0.005, 20.0, 1.0)
            st.update(X=_normal((m, k), gen).mul_(gain).to(BF16), Y=empty((m, n), BF16))
        else:
            # gradients: small, rows of very different size
            size = torch.exp(_normal((m, 1), gen, 1.5)) * 1e-4
            st.update(dY=_normal((m, n), gen).mul_(size).to(BF16), dX=empty((m, k), BF16))
        return st
    if kind == "dropout":
        shape, dtype = (case["rows"], case["cols"]), BF16 if case["dtype"] == "bf16" else F32
        st.update(X=_normal(shape, gen).to(dtype), R=_normal(shape, gen).to(dtype) if case["residual"] else None,
                  Y=empty(shape, dtype), p=float(case["p"]), seed=0x9E3779B97F4A7C15 * (seed + 1) & _MASK64,
                  offset=seed * 1000003)
        return st
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    # an output layer whose logits have a spread of 2.5, and hidden states that know their label more or less
    W = _normal((vocab, k), gen, 2.5 * k ** -0.5).to(BF16)
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=I64)
    sure = torch.rand((rows, 1), generator=gen, device="cuda") * 8 / 2.5
    X = (_normal((rows, k), gen) + sure * W[labels].float()).to(BF16)
    skipped = torch.rand(rows, generator=gen, device="cuda") < 0.05     # positions of the prompt and of padding
    dloss = torch.rand(rows, generator=gen, device="cuda", dtype=F32).add_(0.5).div_(rows)
    st.update(X=X, W=W, labels=torch.where(skipped, -100, labels).to(I32), dloss=dloss, loss=empty(rows, F32))
    if kind == "xent_fwd_bwd":
        st["saved"] = empty((rows, 2), F32)
    if kind != "xent_eval":
        st.update(dX=empty((rows, k), BF16), dW=empty((vocab, k), BF16) if case["dw"] else None)
    return st


# ---- one pass --------------------------------------------------------------
def run(st: dict) -> dict:
    return _run_own(st) if own else _run_plain(st)


def _run_own(st):
    import paper_2403_11366_amd as lora
    kind = st["kind"]

    def workspace(size, *args):
        if "ws" not in st:
            st["ws"] = torch.empty(size(*args), dtype=U8, device="cuda")
        return st["ws"]

    if kind == "fp8_roundtrip":
        lora.lora_fp8_quantize(st["X"], st["codes"], st["scales"], block_rows=st["by"])
        lora.lora_fp8_dequantize(st["codes"], st["scales"], st["values"], block_rows=st["by"])
        return {"values": st["values"]}
    if kind == "fp8_fwd":
        X, Y = st["X"], st["Y"]
        ws = workspace(lora.lora_linear_fp8_fwd_workspace_size, X.shape[0], Y.shape[1], st["k"])
        lora.lora_linear_fp8_fwd(X, st["Wc"], st["Ws"], Y, ws)
        return {"Y": Y}
    if kind == "fp8_bwd":
        dY, dX = st["dY"], st["dX"]
        ws = workspace(lora.lora_linear_fp8_bwd_workspace_size, dY.shape[0], dY.shape[1], st["k"])
        lora.lora_linear_fp8_bwd(dY, st["Wc"], st["Ws"], dX, ws)
        return {"dX": dX}
    if kind == "dropout":
        lora.lora_dropout(st["X"], st["Y"], st["seed"], st["offset"], st["p"], residual=st["R"])
        return {"Y": st["Y"]}
    X, W, labels, loss = st["X"], st["W"], st["labels"], st["loss"]
    dX, dW = st.get("dX"), st.get("dW")
    ws = workspace(lora.lora_linear_xent_workspace_size, X.shape[0], W.shape[0], X.shape[1], dX is not None,
                   dW is not None)
    if kind == "xent_step":
        lora.lora_linear_xent_step(X, W, labels, st["dloss"], loss, dX, dW, ws)
    else:
        lora.lora_linear_xent_fwd(X, W, labels, loss, st.get("saved"), ws)
        if kind == "xent_eval":
            return {"loss": loss}
        lora.lora_linear_xent_bwd(X, W, labels, st["saved"], st["dloss"], dX, dW, ws)
    out = {"loss": loss, "dX": dX}
    if dW is not None:
        out["dW"] = dW
    return out


def _run_plain(st):
    kind = st["kind"]
    if kind == "fp8_roundtrip":
        return {"values": _fp8_quantised(st["X"].float(), st["by"]).to(BF16)}
    if kind == "fp8_fwd":
        w = _weight_values(st["Wc"], st["Ws"], st["k"])
        return {"Y": (_fp8_quantised(st["X"].float(), 1) @ w.t()).to(BF16)}
    if kind == "fp8_bwd":
        w = _weight_values(st["Wc"], st["Ws"], st["k"])
        return {"dX": (_fp8_quantised(st["dY"].float(), 1) @ w).to(BF16)}
    if kind == "dropout":
        X, p = st["X"], st["p"]
        keep = (_draws(st["seed"], st["offset"], X.numel(), X.device) < _threshold(p)).view(X.shape)
        y = torch.where(keep, X.float() * (1.0 / (1.0 - np.float32(p)).item()), 0.0)
        return {"Y": (y if st["R"] is None else y + st["R"].float()).to(X.dtype)}
    X, W, labels = st["X"].float(), st["W"].float(), st["labels"].long()
    z = X @ W.t()
    known = (labels >= 0) & (labels < W.shape[0])
    y = torch.where(known, labels, 0)[:, None]
    d = z - z.amax(1, keepdim=True)
    e = torch.exp(d)
    s = e.sum(1, keepdim=True)
    out = {"loss": torch.where(known, torch.log(s[:, 0]) - d.gather(1, y)[:, 0], 0.0)}
    if kind == "xent_eval":
        return out
    g = e / s
    # the label's own, 1 less: less what the others have in all where that is more than half
    own_p = g.gather(1, y)
    others = torch.where(own_p > 0.5, -(g.scatter(1, y, 0.0)).sum(1, keepdim=True), own_p - 1.0)
    g.scatter_(1, y, others)
    g *= torch.where(known, st["dloss"], 0.0)[:, None]
    out["dX"] = (g @ W).to(BF16)
    if st["dW"] is not None:
        out["dW"] = (g.t() @ X).to(BF16)
    return out


# ---- what a pass cannot do without -----------------------------------------
def work(case: dict) -> dict:
    kind = case["kind"]
    if kind == "fp8_roundtrip":
        m, k = case["m"], case["k"]
        return {"bytes": 4 * m * k + m * k + m * k // (128 * case["block_rows"]), "flops": 2 * m * k}
    if kind.startswith("fp8"):
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": 2 * m * k + n * k + n * k // 16384 + 2 * m * n, "flops": 2 * m * n * k}
    if kind == "dropout":
        count, size = case["rows"] * case["cols"], 2 if case["dtype"] == "bf16" else 4
        return {"bytes": (2 + case["residual"]) * count * size, "flops": 2 * count}
    rows, vocab, k = case["rows"], case["vocab"], case["k"]
    read = 2 * (rows + vocab) * k + 8 * rows          # X, W, the labels, the loss
    if kind == "xent_eval":
        return {"bytes": read, "flops": 2 * rows * vocab * k}
    return {"bytes": read + 4 * rows + 2 * rows * k + 2 * case["dw"] * vocab * k,
            "flops": (4 + 2 * case["dw"]) * rows * vocab * k}


# ---- the same in 64 bits ---------------------------------------------------
def _power64(e):
    return ((e.to(I64) + 1023) << 52).view(F64)


def _quantised64(x, block_rows):
    """fp64 [rows, k] -> the values that 8 bits stand for, block by block of the padded matrix."""
    rows, k = x.shape
    v = torch.nn.functional.pad(x, (0, -k % 128, 0, -rows % block_rows))
    v = v.view(v.shape[0] // block_rows, block_rows, -1, 128)
    amax = v.abs().amax((1, 3), keepdim=True)
    mantissa, exponent = torch.frexp(amax)                            # amax = mantissa 2^exponent, mantissa in [1/2, 1)
    power = exponent.to(F64) - 9.0 + (mantissa > 0.875).to(F64)       # 448 = 0.875 2^9
    unit = _power64(torch.where(amax > 0, power, -127.0).clamp_min(-127.0))
    y = v / unit
    step = _power64(torch.frexp(y.abs().clamp_min(2.0 ** -6))[1] - 4)
    return (torch.round(y / step) * step * unit).view(-1, v.shape[2] * 128)[:rows, :k]


def _weight64(codes, scales, n, k):
    c = codes.to(I64)
    e, f = (c >> 3) & 15, (c & 7).to(F64)
    mag = torch.where(e == 0, f * 2.0 ** -9, (1.0 + f / 8.0) * _power64(e - 7))
    i, b = torch.arange(n, device=codes.device) // 128, torch.arange(k, device=codes.device) // 128
    unit = _power64(scales.to(I64).view((n + 127) // 128, -1) - 127)
    return (torch.where(c < 128, mag, -mag)[:, :k]) * unit[i[:, None], b[None]]


def _keep64(seed, offset, p, count):
    """Philox4x64-10 with 64-bit words of numpy, products by 32-bit halves."""
    blocks = (count + 15) // 16
    with np.errstate(over="ignore"):
        half, lo32 = np.uint64(32), np.uint64(0xFFFFFFFF)

        def high(a, b):
            a0, a1, b0, b1 = a & lo32, a >> half, b & lo32, b >> half
            mid = a1 * b0 + (a0 * b0 >> half)
            return a1 * b1 + (mid >> half) + ((a0 * b1 + (mid & lo32)) >> half)

        x = [np.arange(blocks, dtype=np.uint64) + np.uint64(offset & _MASK64)]
        x.append((x[0] < np.uint64(offset & _MASK64)).astype(np.uint64))
        x += [np.zeros(blocks, np.uint64), np.zeros(blocks, np.uint64)]
        key = [np.uint64(seed & _MASK64), np.uint64(0)]
        m0, m1 = np.uint64(_M0), np.uint64(_M1)
        for _ in range(10):
            x = [high(m1, x[2]) ^ x[1] ^ key[0], m1 * x[2], high(m0, x[0]) ^ x[3] ^ key[1], m0 * x[0]]
            key = [np.add(key[0], np.uint64(_W0)), np.add(key[1], np.uint64(_W1))]
        draws = np.stack(x, 1).astype("<u8").view("<u2").reshape(-1)[:count]
    return draws < _threshold(p)


def exact(case: dict, seed: int):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "fp8_roundtrip":
        return {"values": _quantised64(st["X"].to(F64), case["block_rows"])}
    if kind.startswith("fp8"):
        w = _weight64(st["Wc"], st["Ws"], case["n"], case["k"])
        if kind == "fp8_fwd":
            return {"Y": _quantised64(st["X"].to(F64), 1) @ w.t()}
        return {"dX": _quantised64(st["dY"].to(F64), 1) @ w}
    if kind == "dropout":
        X = st["X"]
        keep = torch.from_numpy(_keep64(st["seed"], st["offset"], st["p"], X.numel())).to(X.device).view(X.shape)
        y = X.to(F64) * keep / (1.0 - float(np.float32(st["p"])))
        return {"Y": y if st["R"] is None else y + st["R"].to(F64)}
    X, W, labels = st["X"].to(F64), st["W"].to(F64), st["labels"].long()
    rows, vocab = X.shape[0], W.shape[0]
    logp = torch.log_softmax(X @ W.t(), 1)
    known = (labels >= 0) & (labels < vocab)
    line, label = torch.arange(rows, device=X.device), labels.clamp(0, vocab - 1)
    out = {"loss": -torch.where(known, logp[line, label], 0.0)}
    if kind == "xent_eval":
        return out
    g = logp.exp_()
    g[line, label] -= 1.0
    g *= (known * st["dloss"].to(F64))[:, None]
    out["dX"] = g @ W
    if case["dw"]:
        out["dW"] = g.t() @ X
    return out
