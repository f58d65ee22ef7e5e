"""Operators of a fine-tuning step on tensors of another device than the current one:
every tensor argument of every entry point is looked at, and nothing is launched.  One
device is enough: each tensor in turn says that it lies elsewhere."""
import pytest

pytestmark = pytest.mark.gpu


def calls():
    """Entry point, tensors by name in the order of its arguments, and a call of them."""
    import torch
    import paper_2403_11366_amd as lora
    m, n, k, vocab = 24, 64, 256, 100
    zeros = lambda *shape, dtype=torch.bfloat16: torch.zeros(shape, dtype=dtype, device="cuda")
    u8, f32 = (lambda size: zeros(size, dtype=torch.uint8)), (lambda *shape: zeros(*shape, dtype=torch.float32))
    weight = {"W_codes": zeros(n, k, dtype=torch.uint8), "W_scales": u8(lora.lora_fp8_scales_size(n, k))}
    loss = {"X": zeros(m, k), "W": zeros(vocab, k), "labels": zeros(m, dtype=torch.int32)}
    ws = u8(lora.lora_linear_xent_workspace_size(m, vocab, k, True, True))
    codes, scales = zeros(m, k, dtype=torch.uint8), u8(lora.lora_fp8_scales_size(m, k, 1))
    return [
        (lora.lora_fp8_quantize, {"X": zeros(m, k), "codes": codes, "scales": scales}, {"block_rows": 1}),
        (lora.lora_fp8_dequantize, {"codes": codes, "scales": scales, "X": zeros(m, k)}, {"block_rows": 1}),
        (lora.lora_linear_fp8_fwd, {"X": zeros(m, k), **weight, "Y": zeros(m, n),
                                    "workspace": u8(lora.lora_linear_fp8_fwd_workspace_size(m, n, k))}, {}),
        (lora.lora_linear_fp8_bwd, {"dY": zeros(m, n), **weight, "dX": zeros(m, k),
                                    "workspace": u8(lora.lora_linear_fp8_bwd_workspace_size(m, n, k))}, {}),
        (lora.lora_dropout, {"X": zeros(m, k), "Y": zeros(m, k), "residual": zeros(m, k)}, {"seed": 0, "offset": 0, "p": 0.5}),
        (lora.lora_linear_xent_fwd, {**loss, "loss": f32(m), "saved": f32(m, 2), "workspace": ws}, {}),
        (lora.lora_linear_xent_bwd, {**loss, "saved": f32(m, 2), "dloss": f32(m), "dX": zeros(m, k), "dW": zeros(vocab, k),
                                     "workspace": ws}, {}),
        (lora.lora_linear_xent_step, {**loss, "dloss": f32(m), "loss": f32(m), "dX": zeros(m, k), "dW": zeros(vocab, k),
                                      "workspace": ws}, {}),
    ]



@pytest.mark.parametrize("at", range(8))
def test_each_tensor_of_each_call(at, monkeypatch):
    import torch
    import paper_2403_11366_amd as lora
    fn, tensors, other = calls()[at]
    fn(**tensors, **other)                                       # the call itself is valid
    torch.cuda.synchronize()
    reached = []

    class Unreached:                                             # the library must not be entered
        def __getattr__(self, name):
            reached.append(name)
            return getattr(lora_library, name)
    lora_library = lora.load_library()
    for name, t in tensors.items():
        class Elsewhere(torch.Tensor):
            def get_device(self):
                return 1
        moved = dict(tensors)
        moved[name] = t.as_subclass(Elsewhere)
        with monkeypatch.context() as patch:
            patch.setattr(lora, "load_library", lambda: Unreached())
            with pytest.raises(ValueError, match="current device"):
                fn(**moved, **other)
        assert not reached, (fn.__name__, name, reached)


@pytest.mark.parametrize("at", range(8))
def test_another_current_device(at, monkeypatch):
    import paper_2403_11366_amd as lora
    fn, tensors, other = calls()[at]
    fn(**tensors, **other)
    monkeypatch.setattr(lora, "_current_device", lambda: 1)
    with pytest.raises(ValueError, match="current device"):
        fn(**tensors, **other)
