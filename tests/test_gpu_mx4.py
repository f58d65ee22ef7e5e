"""4-bit matrices and their linear layer on the GPU against the float64
definition (oracle/output_ops.py).

Tolerances.  Codes, scales and dequantised values are exact.  The linear
layer's products are exact and its sums fp32, so an output is off by at most
half a bf16 spacing (2^-8 of its size: 8 significant bits) and the sum's error, k 2^-24 of the sum of
the products' magnitudes; where every partial sum is a small whole number the
output is the definition's value rounded to bf16, bit for bit."""
import numpy as np
import pytest

import oracle
from oracle import output_ops as ops

pytestmark = pytest.mark.gpu


def to_bits(x):
    return oracle.f64_to_bf16_bits(x)


def hidden(rows, k, seed):
    """bf16 patterns of normal values, some columns and some rows much larger, one row zero."""
    rng = np.random.default_rng(seed)
    x = rng.normal(size=(rows, k)) * np.where(rng.random(k) < 0.02, 30.0, 1.0) * 2.0 ** rng.integers(-8, 8, (rows, 1))
    if rows > 2:
        x[rows // 2] = 0.0
    return to_bits(x)


def quantise(x):
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import bits_to_device
    rows, k = x.shape
    codes = torch.full((rows, lora.lora_mx4_codes_size(rows, k) // rows), 0xAA, dtype=torch.uint8, device="cuda")
    scales = torch.full((lora.lora_mx4_scales_size(rows, k),), 0xAA, dtype=torch.uint8, device="cuda")
    lora.lora_mx4_quantize(bits_to_device(x), codes, scales)
    return codes, scales


SHAPES = [(1, 8), (1, 256), (3, 40), (17, 264), (64, 512), (65, 4096), (200, 776), (130, 2056)]


@pytest.mark.parametrize("rows,k", SHAPES)
def test_quantise_and_back(rows, k):
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import device_to_bits
    x = hidden(rows, k, rows * 10007 + k)
    codes, scales = quantise(x)
    want_c, want_s = ops.mx4_encode(x)
    assert np.array_equal(codes.cpu().numpy(), want_c) and np.array_equal(scales.cpu().numpy(), want_s)
    back = torch.full((rows, k), 7.0, dtype=torch.bfloat16, device="cuda")
    lora.lora_mx4_dequantize(codes, scales, back)
    assert np.array_equal(oracle.bf16_bits_to_f64(device_to_bits(back)), ops.mx4_decode(want_c, want_s, k))


def test_quantise_every_bf16_value():
    """All 65536 patterns as the lower values of blocks headed by each of a range
    of exponents, and alone: rounding, saturation, subnormals, NaN and infinities."""
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import device_to_bits
    pats = np.arange(65536, dtype=np.uint16)
    for head in (0x0000, 0x0001, 0x007F, 0x0080, 0x0180, 0x0200, 0x3F80, 0x3FFF, 0x40C0, 0x7F00, 0x7F7F):
        x = np.full((1024, 2048), 0, np.uint16)               # 64 patterns a row, each with 31 companions
        blk = x.reshape(1024, 64, 32)
        blk[:, :, 0] = pats.reshape(1024, 64)
        blk[:, :, 7] = head
        blk[:, :, 31] = pats.reshape(1024, 64) ^ 0x8000
        codes, scales = quantise(x)
        want_c, want_s = ops.mx4_encode(x)
        assert np.array_equal(scales.cpu().numpy(), want_s), hex(head)
        assert np.array_equal(codes.cpu().numpy(), want_c), hex(head)
        back = torch.empty((1024, 2048), dtype=torch.bfloat16, device="cuda")
        lora.lora_mx4_dequantize(codes, scales, back)
        got, want = oracle.bf16_bits_to_f64(device_to_bits(back)), ops.mx4_decode(want_c, want_s, 2048)
        assert np.array_equal(got, want, equal_nan=True), hex(head)


def linear(x, codes, scales, n):
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import bits_to_device
    m, k = x.shape
    Y = torch.full((m, n), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.full((lora.lora_linear_mx4_fwd_workspace_size(m, n, k),), 0xFF, dtype=torch.uint8, device="cuda")
    lora.lora_linear_mx4_fwd(bits_to_device(x), codes, scales, Y, ws)
    return Y


def random_weight(n, k, seed, lo=118, hi=128):
    """Random codes and scales of a weight, with the zero padding of the layout."""
    rng = np.random.default_rng(seed)
    slabs = -(-k // 256)
    wide = np.zeros((n, slabs * 256), np.int64)
    wide[:, :k] = rng.integers(0, 16, (n, k))
    codes = (wide[:, 0::2] + 16 * wide[:, 1::2]).astype(np.uint8)
    scales = np.zeros(-(-n // 64) * slabs * 512, np.uint8)
    i, b = np.indices((n, -(-k // 32)))
    scales[ops.mx4_scale_place(i, b, n)] = rng.integers(lo, hi, i.shape)
    return codes, scales


def device(*arrays):
    import torch
    return [torch.from_numpy(a).cuda() for a in arrays]


LINEAR = [(1, 8, 8), (1, 4096, 4096), (2, 24, 40), (3, 520, 264), (4, 1024, 2048), (7, 136, 72), (8, 4104, 512), (15, 64, 4096),
          (16, 256, 1000), (17, 4096, 1024), (24, 11008, 512), (33, 200, 1288), (64, 512, 2048), (65, 72, 256),
          (100, 1032, 520), (128, 128, 4096), (129, 392, 768), (200, 5120, 264), (255, 264, 2056), (256, 256, 256),
          (257, 520, 512), (300, 4096, 1024), (513, 1544, 776), (700, 2048, 2048), (1000, 1000, 1000),
          (1024, 4096, 264), (1531, 4104, 1608), (2048, 4096, 512), (2050, 8200, 256)]


@pytest.mark.parametrize("m,n,k", LINEAR)
def test_linear_matches_the_definition(m, n, k):
    from paper_2403_11366_amd.device_io import device_to_bits
    print(f"mx4 linear {m} x {n} x {k}", flush=True)
    x = hidden(m, k, m + 3 * n + 7 * k)
    wc, ws = random_weight(n, k, n + k)
    Y = oracle.bf16_bits_to_f64(device_to_bits(linear(x, *device(wc, ws), n)))
    xq = ops.mx4_decode(*ops.mx4_encode(x), k)
    wq = ops.mx4_decode(wc, ws, k)
    want, size = xq @ wq.T, np.abs(xq) @ np.abs(wq).T
    assert (np.abs(Y - want) <= 2.0 ** -8 * np.abs(want) * (1 + 1e-6) + (k + 1) * 2.0 ** -24 * size).all()


@pytest.mark.parametrize("m,n,k", [(1, 64, 256), (5, 520, 1000), (40, 4096, 520), (96, 264, 2048), (300, 1288, 776),
                                   (1030, 2056, 512), (2100, 4104, 256)])
def test_linear_of_whole_numbers_is_exact(m, n, k):
    """Values 0, +-1, +-2, +-4 (blocks headed by 4, so X is its own quantisation) and
    scales 1: every partial sum is a small whole number."""
    from paper_2403_11366_amd.device_io import device_to_bits
    rng = np.random.default_rng(m + n + k)
    x = rng.choice([0, 0, 0, 1, -1, 2, -2], (m, k)).astype(np.float64)
    x[:, ::32] = rng.choice([4, -4], x[:, ::32].shape)
    wc, ws = random_weight(n, k, 5, lo=127, hi=128)
    wc &= 0xBB                                     # codes 0..3 and their negatives: at most 1.5
    want = x @ ops.mx4_decode(wc, ws, k).T
    assert np.abs(want).max() * 2 < 2 ** 23
    assert np.array_equal(device_to_bits(linear(to_bits(x), *device(wc, ws), n)) & 0xFFFF, to_bits(want))


def test_nan_blocks_reach_their_outputs_alone():
    from paper_2403_11366_amd.device_io import device_to_bits
    for m, n, k in ((3, 72, 520), (70, 264, 520), (400, 1032, 520)):
        x = hidden(m, k, 9)
        x[1, 300] = 0x7F80                          # an infinity of X
        wc, ws = random_weight(n, k, 11)
        ws[ops.mx4_scale_place(5, 2, n)] = 255      # a NaN block of W
        Y = oracle.bf16_bits_to_f64(device_to_bits(linear(x, *device(wc, ws), n)))
        bad = np.zeros((m, n), bool)
        bad[1], bad[:, 5] = True, True
        assert np.array_equal(np.isnan(Y), bad), (m, n, k)


def test_extreme_scales():
    """The smallest and large scales of W with an X that brings them back."""
    from paper_2403_11366_amd.device_io import device_to_bits
    m, n, k = 20, 40, 512
    x = to_bits(np.random.default_rng(0).choice([1.0, 2.0, -4.0], (m, k)))
    for s, shift in ((0, 100), (3, 100), (240, -100)):
        wc, ws = random_weight(n, k, 3, lo=s, hi=s + 1)
        xs = to_bits(oracle.bf16_bits_to_f64(x) * 2.0 ** shift)
        Y = oracle.bf16_bits_to_f64(device_to_bits(linear(xs, *device(wc, ws), n)))
        want = ops.mx4_linear(xs, wc, ws)
        assert np.abs(Y - want).max() <= 2.0 ** -8 * np.abs(want).max(), s


def test_same_bits_on_streams_and_in_graphs():
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import bits_to_device
    for m, n, k in ((2, 1032, 776), (37, 520, 4096), (600, 1544, 520), (2300, 4096, 512)):
        d = bits_to_device(hidden(m, k, 1))
        other = bits_to_device(hidden(m, k, 2))
        wc, ws = device(*random_weight(n, k, 3))
        Y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
        work = torch.empty(lora.lora_linear_mx4_fwd_workspace_size(m, n, k), dtype=torch.uint8, device="cuda")

        def call(x, out):
            lora.lora_linear_mx4_fwd(x, wc, ws, out, work)
            return out

        eager, eager2 = call(d, Y).clone(), call(other, Y).clone()
        x = d.clone()
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            call(x, Y)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                call(x, Y)
        side.synchronize()
        assert torch.equal(Y, eager), (m, n, k)
        for it in range(4):
            x.copy_(other if it % 2 else d)
            Y.fill_(float("nan"))
            work.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(Y, eager2 if it % 2 else eager), (m, n, k, it)


def test_large_operands():
    """Codes past 2^28 bytes and outputs past 2^29: a tall X whose rows repeat, so that
    the definition needs one period, and a wide W likewise."""
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import bits_to_device, device_to_bits
    period, k = 64, 256
    x = hidden(period, k, 21)
    wc, ws = random_weight(period, k, 22)
    want = ops.mx4_linear(x, wc, ws)
    size = np.abs(ops.mx4_decode(*ops.mx4_encode(x), k)) @ np.abs(ops.mx4_decode(wc, ws, k)).T
    tol = 2.0 ** -8 * np.abs(want) * (1 + 1e-6) + (k + 1) * 2.0 ** -24 * size
    dx, (dc, ds) = bits_to_device(x), device(wc, ws)
    for m, n in (((1 << 22), period), (period, 1 << 22)):
        rx, rw = m // period, n // period
        X = dx.repeat(rx, 1)
        C, S = dc.repeat(rw, 1).contiguous(), ds.repeat(rw).contiguous()     # one slab: cells of 64 rows follow each other
        Y = torch.empty((m, n), dtype=torch.bfloat16, device="cuda")
        work = torch.empty(lora.lora_linear_mx4_fwd_workspace_size(m, n, k), dtype=torch.uint8, device="cuda")
        lora.lora_linear_mx4_fwd(X, C, S, Y, work)
        got = Y.view(rx, period, rw, period)
        assert bool((got == got[:1, :, :1]).all())
        first = oracle.bf16_bits_to_f64(device_to_bits(got[0, :, 0].contiguous()))
        assert (np.abs(first - want) <= tol).all()
