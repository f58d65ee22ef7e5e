"""Refusals of the operators of a fine-tuning step, through the C ABI and the Python
binding, on the CPU: every call below fails validation, which runs before any HIP
call."""
import os

import pytest

import paper_2403_11366_amd as lora

NULL, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE, ALIAS = 1, 2, 3, 4, 5, 6


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(lora.lib_path()):
        from paper_2403_11366_amd import build
        build.build()
    return lora.load_library()


def addr(i, off=0):
    return (1 << 40) + i * (1 << 36) + off


def call(fn, base, **change):
    args = dict(base)
    assert set(change) <= set(args), change
    args.update(change)
    return fn(*args.values())


def nulls(fn, base, names):
    for q in names:
        assert call(fn, base, **{q: None}) == NULL, q


QUANT = dict(X=addr(0), codes=addr(1), scales=addr(2), rows=64, k=64, by=128, stream=None)
BACK = dict(codes=addr(1), scales=addr(2), X=addr(0), rows=64, k=64, by=1, stream=None)
LINEAR = dict(A=addr(0), Wc=addr(1), Ws=addr(2), out=addr(3), ws=addr(4), ws_bytes=1 << 30, m=64, n=64, k=64, stream=None)
DROP = dict(X=addr(0), R=addr(1), Y=addr(2), dtype=0, count=1000, seed=1, offset=2, p=0.5, stream=None)
FWD = dict(X=addr(0), W=addr(1), labels=addr(2), loss=addr(3), saved=addr(4), ws=addr(5), ws_bytes=1 << 40, rows=8,
           vocab=100, k=64, stream=None)
BWD = dict(X=addr(0), W=addr(1), labels=addr(2), saved=addr(3), dloss=addr(4), dX=addr(5), dW=addr(6), ws=addr(7),
           ws_bytes=1 << 40, rows=8, vocab=100, k=64, stream=None)
STEP = dict(X=addr(0), W=addr(1), labels=addr(2), dloss=addr(3), loss=addr(4), dX=addr(5), dW=addr(6), ws=addr(7),
            ws_bytes=1 << 40, rows=8, vocab=100, k=64, stream=None)


@pytest.mark.parametrize("name,base", [("lora_fp8_quantize", QUANT), ("lora_fp8_dequantize", BACK)])
def test_fp8_refusals(lib, name, base):
    fn = getattr(lib, name)
    nulls(fn, base, ("X", "codes", "scales"))
    for rows, k in ((0, 64), (-1, 64), (64, 0), (64, 4), (64, 12), (64, -8)):
        assert call(fn, base, rows=rows, k=k) == SHAPE
    for by in (0, 2, 64, -1, 129):
        assert call(fn, base, by=by) == SHAPE
    for rows, k in ((1 << 23, 8), (8, 1 << 23), (1 << 22, 264), (1 << 62, 1 << 62)):
        assert call(fn, base, rows=rows, k=k) == UNSUPPORTED
    for q in ("X", "codes", "scales"):
        assert call(fn, base, **{q: base[q] + 8}) == ALIGN
    assert call(fn, base, codes=base["X"] + 16) == ALIAS
    assert call(fn, base, scales=base["X"] + 64 * 64 * 2 - 16) == ALIAS
    if name == "lora_fp8_quantize":
        assert call(fn, base, scales=base["codes"]) == ALIAS


def test_fp8_sizes(lib):
    assert lora.lora_fp8_codes_size(3, 136) == 3 * 256 and lora.lora_fp8_scales_size(3, 136) == 2
    assert lora.lora_fp8_scales_size(129, 136) == 4 and lora.lora_fp8_scales_size(65, 136, 1) == 256
    assert lora.lora_fp8_codes_size(0, 8) == lora.lora_fp8_codes_size(8, 12) == lora.lora_fp8_scales_size(8, 8, 7) == 0
    for fn in (lora.lora_linear_fp8_fwd_workspace_size, lora.lora_linear_fp8_bwd_workspace_size):
        assert fn(8, 8, 12) == fn(0, 8, 8) == fn(8, 1 << 23, 8) == 0 and fn(8, 64, 64) > 0


@pytest.mark.parametrize("name", ["lora_linear_fp8_fwd", "lora_linear_fp8_bwd"])
def test_linear_fp8_refusals(lib, name):
    fn = getattr(lib, name)
    nulls(fn, LINEAR, ("A", "Wc", "Ws", "out"))
    for m, n, k in ((0, 64, 64), (64, 0, 64), (64, 12, 64), (64, 64, 12), (64, 64, 0), (-5, 64, 64)):
        assert call(fn, LINEAR, m=m, n=n, k=k) == SHAPE
    for m, n, k in ((1 << 23, 8, 8), (1 << 20, 1 << 20, 8), (1 << 20, 8, 1 << 20), (8, 1 << 20, 1 << 20)):
        assert call(fn, LINEAR, m=m, n=n, k=k) == UNSUPPORTED
    for q in ("A", "Wc", "Ws", "out", "ws"):
        assert call(fn, LINEAR, **{q: LINEAR[q] + 4}) == ALIGN
    assert call(fn, LINEAR, ws=None) == WORKSPACE and call(fn, LINEAR, ws_bytes=100) == WORKSPACE
    for q in ("A", "Wc", "Ws", "ws"):
        assert call(fn, LINEAR, out=LINEAR[q]) == ALIAS
        if q != "ws":
            assert call(fn, LINEAR, ws=LINEAR[q]) == ALIAS


def test_dropout_refusals(lib):
    fn = lib.lora_dropout
    nulls(fn, DROP, ("X", "Y"))
    assert call(fn, DROP, dtype=2) == UNSUPPORTED and call(fn, DROP, dtype=-1) == UNSUPPORTED
    assert call(fn, DROP, count=0) == SHAPE and call(fn, DROP, count=-3) == SHAPE
    assert call(fn, DROP, count=(1 << 35) + 1) == call(fn, DROP, count=(1 << 40) + 1) == UNSUPPORTED
    for p in (1.0, -0.1, float("nan"), float("inf")):
        assert call(fn, DROP, p=p) == SHAPE
    for q in ("X", "R", "Y"):
        assert call(fn, DROP, **{q: DROP[q] + 8}) == ALIGN
    assert call(fn, DROP, Y=DROP["X"] + 16) == ALIAS and call(fn, DROP, Y=DROP["R"] + 1984) == ALIAS
    assert call(fn, DROP, R=DROP["Y"] + 3984, dtype=1) == ALIAS


@pytest.mark.parametrize("name,base,needed", [("lora_linear_xent_fwd", FWD, ("X", "W", "labels", "loss")),
                                              ("lora_linear_xent_bwd", BWD, ("X", "W", "labels", "saved", "dloss")),
                                              ("lora_linear_xent_step", STEP, ("X", "W", "labels", "dloss", "loss"))])
def test_xent_refusals(lib, name, base, needed):
    fn = getattr(lib, name)
    nulls(fn, base, needed)
    if base is not FWD:
        assert call(fn, base, dX=None, dW=None) == NULL
    for rows, vocab, k in ((0, 100, 64), (8, 0, 64), (8, 100, 0), (8, 100, 12), (-1, 100, 64)):
        assert call(fn, base, rows=rows, vocab=vocab, k=k) == SHAPE
    for rows, vocab, k in (((1 << 20) + 1, 100, 8), (8, (1 << 20) + 1, 64), (8, 100, (1 << 16) + 8), (1 << 20, 100, 2048)):
        assert call(fn, base, rows=rows, vocab=vocab, k=k) == UNSUPPORTED
    for q in base:
        if q in ("X", "W", "dX", "dW", "ws"):
            assert call(fn, base, **{q: base[q] + 8}) == ALIGN, q
        elif q in ("labels", "saved", "dloss", "loss"):
            assert call(fn, base, **{q: base[q] + 2}) == ALIGN, q
    assert call(fn, base, ws=None) == WORKSPACE and call(fn, base, ws_bytes=64) == WORKSPACE
    outs = [q for q in base if q in ("dX", "dW", "ws") or (q == "loss") or (q == "saved" and base is FWD)]
    ins = [q for q in base if q in ("X", "W", "labels", "dloss") or (q == "saved" and base is BWD)]
    for o in outs:
        for i in ins + [q for q in outs if q != o]:
            assert call(fn, base, **{o: base[i]}) == ALIAS, (o, i)


def test_xent_workspace_sizes(lib):
    size = lora.lora_linear_xent_workspace_size
    assert size(0, 10, 8) == size(8, 0, 8) == size(8, 10, 12) == size(8, (1 << 20) + 1, 8) == 0
    plain, dx, dw, both = size(300, 5000, 512), size(300, 5000, 512, True), size(300, 5000, 512, False, True), \
        size(300, 5000, 512, True, True)
    assert 0 < plain < dx < both and plain < dw <= both
    # far below the logits themselves where those are large
    assert size(8192, 131072, 4096, True) < 8192 * 131072 * 2 // 3


def test_binding_refuses_host_tensors_and_wrong_shapes(lib):
    import torch
    x, w = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros((8, 64), dtype=torch.bfloat16)
    u8, f, i = torch.zeros(64, dtype=torch.uint8), torch.zeros(4), torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError):
        lora.lora_fp8_quantize(x, u8.view(4, 16), u8)
    with pytest.raises(TypeError):
        lora.lora_fp8_quantize(x.float(), u8, u8)
    with pytest.raises((ValueError, RuntimeError)):
        lora.lora_linear_fp8_fwd(x, u8, u8, x, u8)
    with pytest.raises(ValueError):
        lora.lora_dropout(x, x, 1, 0, 0.5)
    with pytest.raises(TypeError):
        lora.lora_dropout(i, i, 1, 0, 0.5)
    with pytest.raises((TypeError, ValueError)):
        lora.lora_linear_xent_fwd(x, w, i.long(), f, None, u8)
    with pytest.raises(ValueError):
        lora.lora_linear_xent_step(x, w[:, :32], i, f, f, x, None, u8)
