"""Workspace sizes of the 8-bit layer and of the loss: one that is asked for the longest
batch serves every shorter one.  Host only."""
import random

import pytest

import paper_2403_11366_amd as lora

ROWS = list(range(1, 140)) + [191, 192, 193, 255, 256, 257, 300, 383, 384, 385, 511, 512, 513, 700, 1000, 1023, 1024, 1025, 1500,
                              2047, 2048, 2049, 4096, 4097, 8192, 30000]


def grows(size, rows=ROWS):
    last = 0
    for m in rows:
        now = size(m)
        assert now >= last > -1 and now > 0, (m, last, now)
        last = now


@pytest.mark.parametrize("n,k", [(8, 8), (4096, 4096), (4096, 11008), (11008, 4096), (1024, 8192), (264, 16384), (16384, 264)])
def test_8_bit_layer(n, k):
    grows(lambda m: lora.lora_linear_fp8_fwd_workspace_size(m, n, k))
    grows(lambda m: lora.lora_linear_fp8_bwd_workspace_size(m, n, k))


@pytest.mark.parametrize("vocab,k", [(1, 8), (700, 64), (2634, 4096), (32000, 4096), (32003, 512), (50021, 2048), (131072, 5120)])
@pytest.mark.parametrize("dx,dw", [(False, False), (True, False), (False, True), (True, True)])
def test_loss(vocab, k, dx, dw):
    grows(lambda rows: lora.lora_linear_xent_workspace_size(rows, vocab, k, dx, dw))


def test_drawn_sizes():
    """Between any two lengths of any sizes, fewer outputs among them."""
    rng = random.Random(1)
    for _ in range(2000):
        few, more = sorted(int(2 ** rng.uniform(0, 13)) for _ in range(2))
        n, k = 8 * int(2 ** rng.uniform(0, 11)), 8 * int(2 ** rng.uniform(0, 11))
        assert lora.lora_linear_fp8_fwd_workspace_size(few, n, k) <= lora.lora_linear_fp8_fwd_workspace_size(more, n, k), (few, more, n, k)
        assert lora.lora_linear_fp8_bwd_workspace_size(few, n, k) <= lora.lora_linear_fp8_bwd_workspace_size(more, n, k), (few, more, n, k)
        vocab = int(2 ** rng.uniform(0, 17))
        size = lora.lora_linear_xent_workspace_size
        for a in (0, 1):
            for b in (0, 1):
                assert size(few, vocab, k, a, b) <= size(more, vocab, k, a, b) <= size(more, vocab, k, 1, 1), (few, more, vocab, k, a, b)


def test_largest_sizes_are_quick():
    """Sizes of the most rows that the calls take, which look at every 64 of them."""
    assert lora.lora_linear_fp8_fwd_workspace_size(1 << 22, 256, 256) >= (1 << 22) * 256
    assert lora.lora_linear_fp8_bwd_workspace_size(1 << 22, 256, 256) >= (1 << 22) * 256
    assert lora.lora_linear_xent_workspace_size(1 << 20, 1 << 20, 1024, True, True) >= (1 << 20) * 1024 * 2
