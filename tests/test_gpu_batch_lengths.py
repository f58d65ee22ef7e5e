"""One workspace, sized for the longest batch, under batches of other lengths: the
operators of a fine-tuning step and the example that runs them."""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

# the longest, and shorter ones that need more than it does for itself
LENGTHS = [(700, [700, 300, 257, 256, 129, 128, 64, 17, 16, 1, 700])]


@pytest.mark.parametrize("longest,lengths", LENGTHS)
@pytest.mark.parametrize("n,k", [(4096, 4096), (4096, 11008), (1032, 8192)])
def test_8_bit_layer(longest, lengths, n, k):
    import torch
    import paper_2403_11366_amd as lora
    gen = torch.Generator(device="cuda").manual_seed(0)
    W = torch.randn((n, k), generator=gen, device="cuda").bfloat16()
    codes = torch.empty((n, lora.lora_fp8_codes_size(n, k) // n), dtype=torch.uint8, device="cuda")
    scales = torch.empty(lora.lora_fp8_scales_size(n, k), dtype=torch.uint8, device="cuda")
    lora.lora_fp8_quantize(W, codes, scales)
    for size, call, a, o in ((lora.lora_linear_fp8_fwd_workspace_size, lora.lora_linear_fp8_fwd, k, n),
                             (lora.lora_linear_fp8_bwd_workspace_size, lora.lora_linear_fp8_bwd, n, k)):
        one = torch.full((size(longest, n, k),), 0xFF, dtype=torch.uint8, device="cuda")
        for m in lengths:
            A = torch.randn((m, a), generator=gen, device="cuda").bfloat16()
            got, want = (torch.full((m, o), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
            call(A, codes, scales, got, one)
            call(A, codes, scales, want, torch.full((size(m, n, k),), 0xA5, dtype=torch.uint8, device="cuda"))
            assert torch.isfinite(got).all() and torch.equal(got, want), (call.__name__, m)


@pytest.mark.parametrize("vocab,k,longest,lengths", [(32000, 4096, 1500, [1500, 1024, 512, 37, 1]), (2000, 520, 700, [700, 513, 512, 64, 3])])
@pytest.mark.parametrize("dw", [False, True])
def test_loss(vocab, k, longest, lengths, dw):
    import torch
    import paper_2403_11366_amd as lora
    gen = torch.Generator(device="cuda").manual_seed(0)
    W = torch.randn((vocab, k), generator=gen, device="cuda").bfloat16()
    one = torch.full((lora.lora_linear_xent_workspace_size(longest, vocab, k, True, dw),), 0xFF, dtype=torch.uint8, device="cuda")
    for rows in lengths:
        X = (torch.randn((rows, k), generator=gen, device="cuda") * k ** -0.5).bfloat16()
        labels = torch.randint(-1, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
        dloss = torch.rand(rows, generator=gen, device="cuda")
        out = []
        for ws in (one, torch.full((lora.lora_linear_xent_workspace_size(rows, vocab, k, True, dw),), 0xA5, dtype=torch.uint8, device="cuda")):
            loss, dX, dW = torch.empty(rows, device="cuda"), torch.empty_like(X), torch.empty_like(W) if dw else None
            lora.lora_linear_xent_step(X, W, labels, dloss, loss, dX, dW, ws)
            out.append([loss, dX] + ([dW] if dw else []))
        assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(*out)), rows


def test_examples_shorter_batches():
    """A last batch that is shorter than the others, on the model that the longest made."""
    import torch
    spec = importlib.util.spec_from_file_location("fp8_finetune_step", os.path.join(ROOT, "examples", "fp8_finetune_step.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    model = example.Model(512, 4096, 8000, 8, 0.1, 0)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for m in (512, 300, 77, 1, 512):
        X = torch.randn((m, 4096), generator=gen, device="cuda").to(torch.bfloat16)
        labels = torch.randint(0, 8000, (m,), generator=gen, device="cuda", dtype=torch.int32)
        loss, dA, dB = model.step(X, labels, 3)
        assert loss.shape == (m,) and all(torch.isfinite(t).all() for t in (loss, dA, dB)), m
