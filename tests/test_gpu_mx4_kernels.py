"""The 4-bit forward at sizes that reach each of its kernels with ragged edges:
against the float64 definition, and on another stream with a dirty workspace."""
import numpy as np
import pytest

import test_gpu_mx4 as base
from oracle import output_ops as ops

pytestmark = pytest.mark.gpu

SIZES = [(2, 13000, 4096), (1, 32000, 512), (9, 4096, 8200), (16, 520, 16392), (31, 4104, 8192), (60, 2056, 4096),
         (128, 4096, 4096), (200, 8200, 1032), (700, 4104, 776), (1300, 4104, 1032), (2050, 4104, 776), (4100, 4360, 520)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_rows_and_columns_of_the_definition(m, n, k):
    """Sampled rows (the first and last of each 64 and the ends) over all columns.
    An output is a bf16 rounding of an fp32 sum: 2^-8 of its size, and of the sum
    of its products' sizes 2^-22 k / 128 for the products' own sums of 128."""
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import bits_to_device, device_to_bits
    print(f"mx4 kernels {m} x {n} x {k}", flush=True)
    x = base.hidden(m, k, m + n + k)
    wc, ws = base.random_weight(n, k, m * 7 + k)
    c, s = base.device(wc, ws)
    Y = base.linear(x, c, s, n)
    rows = sorted({i for i in range(m) if i % 64 in (0, 63) or i in (m - 1, m - 2, 1)})[:40]
    rows = sorted(set(rows) | {m - 1, max(0, m - 2)})
    xq = ops.mx4_decode(*ops.mx4_encode(x[rows]), k)
    wq = ops.mx4_decode(wc, ws, k)
    got = base.oracle.bf16_bits_to_f64(device_to_bits(Y))[rows]
    want, size = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -22 * max(1.0, k / 128) * size + 1e-30).all()
    # the same bits on a side stream, with a workspace of other contents
    side = torch.cuda.Stream()
    d, other = bits_to_device(x), torch.empty_like(Y)
    work = torch.full((lora.lora_linear_mx4_fwd_workspace_size(m, n, k),), 0xFF, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    lora.lora_linear_mx4_fwd(d, c, s, other, work, stream=side)
    side.synchronize()
    assert torch.equal(other.view(torch.int16), Y.view(torch.int16))
