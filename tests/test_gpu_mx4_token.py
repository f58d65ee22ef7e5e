"""One-launch 4-bit forward of one to three tokens on wide inputs (down
projections, up to the last width that its LDS holds), features ragged against 16
and 64, in both of its forms.  Tolerances as in test_gpu_mx4.py."""
import numpy as np
import pytest

import test_gpu_mx4 as base
from oracle import output_ops as ops

pytestmark = pytest.mark.gpu

# eight waves to a group of features, then two
SIZES = [(1, 4096, 11008), (2, 4104, 13824), (1, 5120, 13824), (1, 5128, 8448), (1, 5000, 8712), (3, 1040, 10920),
         (1, 72, 18176), (1, 8, 17928), (1, 6144, 16384),
         (1, 6152, 11008), (1, 32008, 13824), (2, 8200, 16384), (1, 13000, 18176), (3, 8208, 10920)]


@pytest.mark.parametrize("m,n,k", SIZES)
def test_wide_inputs_match_the_definition(m, n, k):
    from paper_2403_11366_amd.device_io import device_to_bits
    print(f"mx4 token {m} x {n} x {k}", flush=True)
    x = base.hidden(m, k, m + 3 * n + 7 * k)
    wc, ws = base.random_weight(n, k, n + k)
    Y = base.oracle.bf16_bits_to_f64(device_to_bits(base.linear(x, *base.device(wc, ws), n)))
    xq = ops.mx4_decode(*ops.mx4_encode(x), k)
    for n0 in range(0, n, 4096):            # (in pieces: the definition's weight is fp64)
        rows = slice(n0, min(n, n0 + 4096))
        wq = np.empty((rows.stop - n0, k))
        i = np.arange(n0, rows.stop)
        nibble = np.stack((wc[rows] % 16, wc[rows] // 16), 2).reshape(len(i), -1)[:, :k]
        for b in range(-(-k // 32)):
            unit = 2.0 ** (ws[ops.mx4_scale_place(i, b, n)].astype(np.float64) - 127)
            cols = slice(32 * b, min(k, 32 * b + 32))
            code = nibble[:, cols]
            wq[:, cols] = ops.E2M1[code % 8] * np.where(code < 8, 1.0, -1.0) * unit[:, None]
        want, size = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
        assert (np.abs(Y[:, rows] - want) <= 2.0 ** -8 * np.abs(want) * (1 + 1e-6) + (k + 1) * 2.0 ** -24 * size).all()
