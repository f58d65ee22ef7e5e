"""The shapes of test_gpu_xent_pieces.py against the launch rules of the loss: with several
pieces of the vocabulary, every tile of dX is met both unshared and shared.  No GPU is
used."""
import os

from test_train_plan import _run, driver  # noqa: F401


def plans(exe, shapes):
    """(tile of dX, several pieces, shared, references of tiles) of each shape."""
    text = _run([exe, "xent"] + [str(x) for shape in shapes for x in shape], env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    out = []
    for line in text.splitlines():
        word = {w.rstrip("-0123456789"): int(w[len(w.rstrip("-0123456789")):]) for w in line.split()}
        out.append((word["grad"], word["pieces"] == 1, word["join"] >= 0, word["local"] >= 0))
    return out


def test_every_tile_of_dX_with_several_pieces(driver):  # noqa: F811
    import test_gpu_xent_pieces as gpu
    got = plans(driver, gpu.SEVERAL)
    assert set(got) == {(tile, True, shared, False) for tile in range(3) for shared in (False, True)}
    assert plans(driver, [(8192, 32000, 1024), (4096, 32000, 4096)]) == [(1, True, False, False), (2, True, False, False)]
    assert plans(driver, gpu.ONE) == [(1, False, True, False)]
