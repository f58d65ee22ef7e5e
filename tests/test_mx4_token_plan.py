"""Sizes of the GPU tests against the one-launch 4-bit forward: both of its forms
up to the last width that its LDS holds.  No GPU is used."""
import os

from test_ops_plan import _run, driver  # noqa: F401


def kinds(driver, sizes):
    text = _run([driver] + [str(x) for s in sizes for x in s], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    return [int(x) for x in text.split()]


def test_gpu_sizes_reach_the_widest_inputs(driver):  # noqa: F811
    import test_gpu_mx4_token as gpu
    of = dict(zip(gpu.SIZES, kinds(driver, gpu.SIZES)))
    assert set(of.values()) == {0, 1}, of                       # this kernel alone
    widths = list(range(8, 1 << 15, 8))
    last = max(k for k, q in zip(widths, kinds(driver, [(1, 72, k) for k in widths])) if q <= 1)
    for kind in (0, 1):
        assert last in [k for (m, n, k), q in of.items() if q == kind]
        assert {m for (m, n, k), q in of.items() if q == kind and k > 8448} >= {1, 2, 3}
    # ragged against the 16 features of a group and the 64 of a cell of scales
    assert any(n % 16 for m, n, k in of) and any(n % 64 and n % 16 == 0 for m, n, k in of)


def test_eight_waves_to_a_group_of_features(driver):  # noqa: F811
    """Up to 512 groups, of more than eight tokens up to 256, at every width (measured on both sides)."""
    for k in (4096, 8192, 8704, 11008, 13824, 16384):
        sizes = [(1, 16 * groups, k) for groups in (1, 256, 320, 384, 448, 512, 513, 1024)]
        assert kinds(driver, sizes) == [0] * 6 + [1] * 2, k
    assert kinds(driver, [(8, 8192, 4096), (8, 8200, 4096), (16, 4096, 2048), (16, 4104, 2048), (16, 5120, 512)]) == [0, 1, 0, 1, 1]
