"""The operators of a fine-tuning step together: examples/fp8_finetune_step.py's step
against float64, on side streams, in captured graphs, two at once, and far ends of what
the calls take."""
import importlib.util
import math
import os

import numpy as np
import pytest

import oracle
from oracle import train_ops as ops

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("fp8_finetune_step", os.path.join(ROOT, "examples", "fp8_finetune_step.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def f64(t):
    return t.double().cpu().numpy()


def test_steps_gradients_match_float64():
    """The step's formulas in float64 on the same weights, every 8-bit operand quantised as
    the definition says from the bf16 values that the step hands on.  An intermediate is
    rounded to bf16 (2^-8 of an element at most, independent ones add as squares), and a
    rounding may move an 8-bit operand by a step (2^-3 of it) where it lay at a border: of the
    elements that a rounding of 2^-9 either way moves across one, at most 2^-8 2^3 / 2 in
    size, their rms error is below (2^-8 x 2^-3 / 12)^(1/2) = 0.007 of the operand.  Six such
    roundings and two quantised operands in a row: 6^(1/2) 2^-8 + 2^(1/2) 0.007 = 0.02."""
    import torch
    ex = example()
    m, k, vocab, r = 200, 264, 1000, 8
    model = ex.Model(m, k, vocab, r, 0.1, 3)
    gen = torch.Generator(device="cuda").manual_seed(4)
    X = torch.randn((m, k), generator=gen, device="cuda").to(torch.bfloat16)
    labels = torch.randint(0, vocab, (m,), generator=gen, device="cuda", dtype=torch.int32)
    labels[::7] = -100
    model.counter = 12345
    loss, dA, dB = model.step(X, labels, 77)

    def q8(x):
        return ops.fp8_decode(*ops.fp8_encode(oracle.f64_to_bf16_bits(x), 1), x.shape[1], 1)
    x, W1, W2, W3 = f64(X), f64(model.up_bf16), f64(model.down.values()), f64(model.head)
    A, B, s = f64(model.A), f64(model.B), model.alpha / r
    kept = ops.dropout_kept(77, 12345, 0.1, (m, k)) / (1 - float(np.float32(0.1)))
    hidden = x + kept * (x @ W1.T + s * (x @ A.T) @ B.T)
    out = q8(hidden) @ W2.T
    y = labels.cpu().numpy()
    d = ((y >= 0) & (y < vocab)) / ((y >= 0) & (y < vocab)).sum()
    want, _, dout, _ = ops.xent(out, W3, y, d)
    dY = kept * (q8(dout) @ W2)
    want_dB, want_dA = s * dY.T @ (x @ A.T), (s * dY @ B).T @ x
    for name, got, ref in (("loss", loss, want), ("dA", dA, want_dA), ("dB", dB, want_dB)):
        assert np.linalg.norm(f64(got) - ref) <= 0.02 * np.linalg.norm(ref), name


def test_example_runs():
    losses = example().train(tokens=96, features=136, vocab=500, rank=4, steps=3)
    assert len(losses) == 3 and all(math.isfinite(x) for x in losses)


class Calls:
    """Every operator's calls on buffers of their own; run() returns what they wrote."""

    def __init__(self, m, n, k, vocab, seed):
        import torch
        import paper_2403_11366_amd as lora
        self.lora, gen = lora, torch.Generator(device="cuda").manual_seed(seed)
        bf = lambda *shape: torch.randn(shape, generator=gen, device="cuda").to(torch.bfloat16)
        u8 = lambda size: torch.full((size,), 0xA5, dtype=torch.uint8, device="cuda")
        self.x, self.dy, self.head = bf(m, k), bf(m, n), bf(vocab, k)
        W = bf(n, k)
        self.wc, self.wsc = u8(lora.lora_fp8_codes_size(n, k)).view(n, -1), u8(lora.lora_fp8_scales_size(n, k))
        lora.lora_fp8_quantize(W, self.wc, self.wsc)
        self.xc, self.xsc = u8(lora.lora_fp8_codes_size(m, k)).view(m, -1), u8(lora.lora_fp8_scales_size(m, k, 1))
        self.labels = torch.randint(-1, vocab, (m,), generator=gen, device="cuda", dtype=torch.int32)
        self.dloss = torch.rand(m, generator=gen, device="cuda")
        self.outs = [torch.zeros_like(self.x) for _ in range(5)] + [torch.zeros_like(self.dy), torch.zeros_like(self.head)]
        self.loss, self.loss2, self.saved = (torch.zeros(s, device="cuda") for s in ((m,), (m,), (m, 2)))
        self.ws = [u8(lora.lora_linear_fp8_fwd_workspace_size(m, n, k)), u8(lora.lora_linear_fp8_bwd_workspace_size(m, n, k)),
                   u8(lora.lora_linear_xent_workspace_size(m, vocab, k, True, True))]

    def run(self, stream=None):
        lora, o = self.lora, self.outs
        lora.lora_fp8_quantize(self.x, self.xc, self.xsc, block_rows=1, stream=stream)
        lora.lora_fp8_dequantize(self.xc, self.xsc, o[0], block_rows=1, stream=stream)
        lora.lora_linear_fp8_fwd(self.x, self.wc, self.wsc, o[5], self.ws[0], stream=stream)
        lora.lora_linear_fp8_bwd(self.dy, self.wc, self.wsc, o[1], self.ws[1], stream=stream)
        lora.lora_dropout(self.x, o[2], 5, 6, 0.3, residual=o[1], stream=stream)
        lora.lora_linear_xent_step(self.x, self.head, self.labels, self.dloss, self.loss, o[3], None, self.ws[2], stream=stream)
        lora.lora_linear_xent_fwd(self.x, self.head, self.labels, self.loss2, self.saved, self.ws[2], stream=stream)
        lora.lora_linear_xent_bwd(self.x, self.head, self.labels, self.saved, self.dloss, o[4], o[6], self.ws[2], stream=stream)

    def values(self):
        return [t.clone() for t in self.outs + [self.loss, self.loss2, self.saved, self.xc, self.xsc]]


SIZES = [(1, 520, 264, 700), (40, 1032, 520, 3000), (300, 2056, 264, 5000), (2100, 4104, 264, 1500)]


@pytest.mark.parametrize("m,n,k,vocab", SIZES)
def test_same_bits_on_streams_in_graphs_and_again(m, n, k, vocab):
    """Every call on a side stream and in a captured graph, replayed with eager work between
    and with inputs changed in place, against the eager calls on the default stream."""
    import torch
    c = Calls(m, n, k, vocab, 1)
    c.run()
    want = c.values()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    c.run(stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(c.values(), want))
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.run(stream=side)
    torch.cuda.synchronize()
    for turn in range(3):
        for t in c.outs:
            t.fill_(float("nan"))
        for w in c.ws:
            w.fill_(0xFF if turn % 2 else 0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(c.values(), want)), turn
        other = Calls(m, n, k, vocab, 50 + turn)      # eager work between replays
        other.run()
    c.x.copy_(other.x)
    c.labels.copy_(other.labels)
    c.run()
    want = c.values()
    for _ in range(2):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(c.values(), want))


def test_two_at_once():
    """Calls of different sizes under way on two streams, each with buffers of its own."""
    import torch
    a, b = Calls(300, 2056, 264, 5000, 1), Calls(40, 1032, 520, 3000, 2)
    a.run()
    b.run()
    want = a.values(), b.values()
    sides = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        a.run(stream=sides[0])
        b.run(stream=sides[1])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(a.values(), want[0]))
    assert all(torch.equal(x, y) for x, y in zip(b.values(), want[1]))


def test_output_weight_past_32_bits():
    """W of 5.4e9 bytes: rows of it past 2^32 bytes are read, and their gradients written."""
    import torch
    import paper_2403_11366_amd as lora
    vocab, k, rows = 2 ** 20, 2560, 5
    gen = torch.Generator(device="cuda").manual_seed(0)
    W = torch.zeros((vocab, k), dtype=torch.bfloat16, device="cuda")
    live = torch.tensor([0, 77, 400000, 838861, 838900, vocab - 1], device="cuda")   # 838860.8 rows are 2^32 bytes
    W[live] = torch.randn((6, k), generator=gen, device="cuda").to(torch.bfloat16)
    X = (torch.randn((rows, k), generator=gen, device="cuda") * 0.1).to(torch.bfloat16)
    X[:] += (0.004 * W[live[1:]].float()).to(torch.bfloat16)
    labels = torch.tensor([vocab - 1, 838861, 5, -1, 400000], dtype=torch.int32, device="cuda")
    dloss = torch.tensor([1.0, 0.5, 2.0, 3.0, -1.0], device="cuda")
    loss, dX, dW = torch.empty(rows, device="cuda"), torch.empty_like(X), torch.full_like(W, float("nan"))
    ws = torch.empty(lora.lora_linear_xent_workspace_size(rows, vocab, k, True, True), dtype=torch.uint8, device="cuda")
    lora.lora_linear_xent_step(X, W, labels, dloss, loss, dX, dW, ws)
    # the definition over the live columns, and the others' exp(0) each
    x, w = f64(X), f64(W[live])
    z = x @ w.T
    top = np.maximum(z.max(axis=1), 0.0)
    total = np.exp(z - top[:, None]).sum(axis=1) + (vocab - 6) * np.exp(-top)
    lab, d = labels.cpu().numpy(), f64(dloss)
    known = lab >= 0
    at = {int(v): i for i, v in enumerate(live.tolist())}
    zy = np.array([z[i, at[int(v)]] if int(v) in at else 0.0 for i, v in enumerate(lab)])
    lse = np.log(total) + top
    # a logit is off by (k + 1) 2^-24 sum |x||w| <= 2561 x 2^-24 x 500, the sum of 2^20 powers by 2^14 roundings at most
    assert (np.abs(f64(loss) - np.where(known, lse - zy, 0.0)) <= 0.08 * 2 + 2.0 ** -10 * lse).all()
    g = np.where(known[:, None], d[:, None] * np.exp(z - lse[:, None]), 0.0)
    for i, v in enumerate(lab):
        if int(v) in at:
            g[i, at[int(v)]] -= d[i]
    want = g @ w
    tol = 0.1 * (np.abs(g) @ np.abs(w)) + 2.0 ** -8 * np.abs(want)
    assert (np.abs(f64(dX) - want) <= tol).all()
    want = g.T @ x
    assert (np.abs(f64(dW[live]) - want) <= 0.1 * (np.abs(g).T @ np.abs(x)) + 2.0 ** -8 * np.abs(want)).all()
    assert torch.isfinite(dW.view(-1)[-10 * k:]).all() and torch.isfinite(dW[838850:838880]).all()


@pytest.mark.parametrize("shift", [-110, -60, 60, 110])
def test_8_bit_layer_on_values_far_from_one(shift):
    """X scaled by a power of two scales Y by it, bit for bit, until the results leave bf16's
    normal numbers."""
    import torch
    import paper_2403_11366_amd as lora
    for m, n, k in ((3, 520, 264), (20, 520, 264), (200, 1032, 520), (2100, 4104, 264)):
        gen = torch.Generator(device="cuda").manual_seed(m)
        x, W = (torch.randn(s, generator=gen, device="cuda").to(torch.bfloat16) for s in ((m, k), (n, k)))
        wc = torch.empty((n, lora.lora_fp8_codes_size(n, k) // n), dtype=torch.uint8, device="cuda")
        wsc = torch.empty(lora.lora_fp8_scales_size(n, k), dtype=torch.uint8, device="cuda")
        lora.lora_fp8_quantize(W, wc, wsc)
        ws = torch.empty(lora.lora_linear_fp8_fwd_workspace_size(m, n, k), dtype=torch.uint8, device="cuda")
        Y, Z = (torch.empty((m, n), dtype=torch.bfloat16, device="cuda") for _ in range(2))
        lora.lora_linear_fp8_fwd(x, wc, wsc, Y, ws)
        lora.lora_linear_fp8_fwd((x.float() * 2.0 ** shift).to(torch.bfloat16), wc, wsc, Z, ws)
        want = Y.double() * 2.0 ** shift
        fine = (want.abs() < 2.0 ** 127) & (want.abs() >= 2.0 ** -126)
        assert fine.double().mean() > 0.9 and torch.equal(Z.double()[fine], want[fine])


def test_tensors_of_another_device_are_refused():
    import torch
    import paper_2403_11366_amd as lora
    if torch.cuda.device_count() < 2:
        class Elsewhere:
            def get_device(self):
                return 1
        with pytest.raises(ValueError):
            lora._same_device(Elsewhere())
        return
    x = torch.zeros(64, device="cuda:1")
    with pytest.raises(ValueError):
        lora.lora_dropout(x, x, 0, 0, 0.5)
