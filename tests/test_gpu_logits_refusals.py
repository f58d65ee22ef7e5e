"""Shapes that the binding of the operators on logits refuses for device tensors."""
import pytest

pytestmark = pytest.mark.gpu


def test_alternatives_and_lists_of_other_ranks_are_value_errors():
    import torch
    import paper_2403_11366_amd as lora
    z = torch.zeros((4, 64), device="cuda")
    i32, f32 = dict(dtype=torch.int32, device="cuda"), dict(device="cuda")
    entropy, ws = torch.zeros(4, **f32), torch.zeros(1 << 12, dtype=torch.uint8, device="cuda")
    for shape in ((4,), (4, 1, 5), (3, 5), (5,)):
        with pytest.raises(ValueError):
            lora.lora_token_logprobs(z, None, None, entropy, torch.zeros(shape, **i32), torch.zeros(shape, **f32), ws)
        with pytest.raises(ValueError):
            lora.lora_distill_fwd(z, torch.zeros(shape, **i32), torch.zeros(shape, **f32), None, entropy, torch.zeros((4, 4), **f32))
    with pytest.raises(ValueError):
        lora.lora_token_logprobs(z, None, None, entropy, torch.zeros((4, 5), **i32), torch.zeros((4, 6), **f32), ws)
    with pytest.raises(ValueError):
        lora.lora_token_logprobs(z, torch.zeros((4, 1), **i32), torch.zeros(4, **f32), entropy, None, None, ws)
