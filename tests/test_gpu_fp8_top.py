"""8-bit matrices at the top of bf16's range: scale bytes 246 and 247, and which values come
back as infinity, as include/lora_linear.h says."""
import numpy as np
import pytest

import oracle
from oracle import train_ops as ops
from test_gpu_fp8 import quantise

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("block_rows", [1, 128])
@pytest.mark.parametrize("sign", [0, 0x8000])
def test_top_of_the_range(block_rows, sign):
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import device_to_bits
    tops = np.arange(0x7F40, 0x7F80, dtype=np.uint16)             # 1.5 2^127 to the largest finite value
    x = np.zeros((64 * block_rows, 128), np.uint16)
    x[::block_rows, 5] = tops | sign
    x[::block_rows, 77] = 0x7E80 | sign                           # 2^126, beside each
    codes, scales = quantise(x, block_rows)
    want_c, want_s = ops.fp8_encode(x, block_rows)
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
    assert set(want_s[want_s > 0].tolist()) == {246, 247}
    assert ((ops.fp8_scale_bytes(oracle.bf16_bits_to_f64(x), block_rows)[:, 0] == 247) == (tops > 0x7F60)).all()
    back = torch.zeros(x.shape, dtype=torch.bfloat16, device="cuda")
    lora.lora_fp8_dequantize(codes, scales, back, block_rows=block_rows)
    got = oracle.bf16_bits_to_f64(device_to_bits(back))
    far = np.isinf(got[::block_rows, 5])
    assert (far == (tops >= 0x7F78)).all()                        # 1.9375 2^127: halfway from 1.875 2^127 to 2^128, to even
    value = ops.fp8_decode(want_c, want_s, 128, block_rows)
    assert (np.abs(value[::block_rows, 5][far]) == 2.0 ** 128).all()
    assert np.array_equal(np.where(np.abs(value) < 2.0 ** 128, value, np.inf * np.sign(value)), got)
