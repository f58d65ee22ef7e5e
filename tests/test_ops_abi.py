"""Refusals of the operators around the layer's output, through the C ABI and the
Python binding, on the CPU: every call below fails validation, which runs before
any HIP call."""
import ctypes
import math
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
    """fn with the named arguments of `base`, some changed."""
    args = dict(base)
    assert set(change) <= set(args), change
    args.update(change)
    return fn(*args.values())


def nulls(fn, base, names):
    for q in names:
        assert call(fn, base, **{q: None}) == NULL, q


QUANT = dict(X=addr(0), codes=addr(1), scales=addr(2), rows=64, k=64, stream=None)
LINEAR = dict(X=addr(0), Wc=addr(1), Ws=addr(2), Y=addr(3), ws=addr(4), ws_bytes=1 << 30, m=64, n=64, k=64, stream=None)
SCORE = dict(z=addr(0), dtype=0, ld=1000, tokens=addr(1), T=1.0, logp=addr(2), entropy=addr(3), ids=addr(4),
             lps=addr(5), ws=addr(6), ws_bytes=1 << 20, rows=8, vocab=1000, top=5, stream=None)
FWD = dict(z=addr(0), dtype=0, ld=1000, ids=addr(1), t=addr(2), labels=addr(3), T=1.0, w=0.5, loss=addr(4),
           saved=addr(5), rows=8, vocab=1000, top=5, stream=None)
BWD = dict(z=addr(0), dtype=0, ld=1000, ids=addr(1), t=addr(2), labels=addr(3), T=1.0, w=0.5, saved=addr(4),
           dloss=addr(5), dz=addr(6), rows=8, vocab=1000, top=5, stream=None)
STEP = dict(z=addr(0), dtype=0, ld=1000, ids=addr(1), t=addr(2), labels=addr(3), T=1.0, w=0.5, dloss=addr(4),
            loss=addr(5), dz=addr(6), rows=8, vocab=1000, top=5, stream=None)


@pytest.mark.parametrize("name", ["lora_mx4_quantize", "lora_mx4_dequantize"])
def test_mx4_refusals(lib, name):
    fn = getattr(lib, name)
    base = QUANT if name.endswith("_quantize") and "de" not in name.split("_")[2][:2] else \
        dict(codes=addr(1), scales=addr(2), X=addr(0), rows=64, k=64, stream=None)
    nulls(fn, base, ("X", "codes", "scales"))
    for rows, k in ((0, 64), (-1, 64), (64, 0), (64, 4), (64, 12), (64, -8)):
        assert call(fn, base, rows=rows, k=k) == SHAPE
    for rows, k in ((1 << 23, 8), (8, 1 << 23), (1 << 22, 264), (1 << 16, 1 << 16)):
        assert call(fn, base, rows=rows, k=k) == UNSUPPORTED
    for q in ("X", "codes", "scales"):
        assert call(fn, base, **{q: base[q] + 8}) == ALIGN
    out = ("X",) if base is not QUANT else ("codes", "scales")
    for q in out:
        for other in {"X", "codes", "scales"} - {q}:
            assert call(fn, base, **{q: base[other] + 16}) == ALIAS, (q, other)


def test_mx4_sizes(lib):
    assert lora.lora_mx4_codes_size(3, 264) == 3 * 256 and lora.lora_mx4_scales_size(65, 264) == 2 * 2 * 512
    for rows, k in ((0, 64), (64, 12), (1 << 23, 64), (1 << 22, 264)):
        assert lora.lora_mx4_codes_size(rows, k) == 0 and lora.lora_mx4_scales_size(rows, k) == 0
    assert lora.lora_linear_mx4_fwd_workspace_size(64, 60, 64) == 0
    assert lora.lora_linear_mx4_fwd_workspace_size(64, 64, 64) >= 64 * 128 + 512


def test_linear_mx4_refusals(lib):
    fn = lib.lora_linear_mx4_fwd
    nulls(fn, LINEAR, ("X", "Wc", "Ws", "Y"))
    assert call(fn, LINEAR, ws=None) == WORKSPACE
    need = lora.lora_linear_mx4_fwd_workspace_size(64, 64, 64)
    assert call(fn, LINEAR, ws_bytes=need - 1) == WORKSPACE
    for m, n, k in ((0, 64, 64), (64, 0, 64), (64, 60, 64), (64, 64, 12), (-5, 64, 64)):
        assert call(fn, LINEAR, m=m, n=n, k=k) == SHAPE
    for m, n, k in ((1 << 23, 8, 8), (1 << 21, 1 << 10, 64), (8, 1 << 22, 512)):
        assert call(fn, LINEAR, m=m, n=n, k=k, ws_bytes=1 << 40) == UNSUPPORTED
    for q in ("X", "Wc", "Ws", "Y", "ws"):
        assert call(fn, LINEAR, **{q: LINEAR[q] + 8}) == ALIGN
    for q in ("Y", "ws"):
        for other in {"X", "Wc", "Ws", "Y", "ws"} - {q}:
            assert call(fn, LINEAR, **{q: LINEAR[other] + 16}) == ALIAS, (q, other)


def test_token_logprobs_refusals(lib):
    fn = lib.lora_token_logprobs
    nulls(fn, SCORE, ("z", "tokens", "logp", "entropy", "ids", "lps"))
    assert call(fn, SCORE, ws=None) == WORKSPACE and call(fn, SCORE, ws_bytes=0) == WORKSPACE
    assert call(fn, SCORE, dtype=2) == UNSUPPORTED and call(fn, SCORE, dtype=-1) == UNSUPPORTED
    for bad in (dict(rows=0), dict(vocab=0), dict(ld=999), dict(top=-1), dict(top=1001, vocab=1000), dict(T=0.0),
                dict(T=-1.0), dict(T=math.inf), dict(T=math.nan)):
        assert call(fn, SCORE, **bad) == SHAPE, bad
    for bad in (dict(top=129), dict(rows=(1 << 21) + 1), dict(vocab=(1 << 20) + 1, ld=1 << 21),
                dict(ld=1 << 34), dict(ld=(1 << 62))):
        assert call(fn, SCORE, **bad) == UNSUPPORTED, bad
    assert call(fn, SCORE, z=addr(0, 1)) == ALIGN and call(fn, SCORE, z=addr(0, 2), dtype=1) == ALIGN
    for q in ("tokens", "logp", "entropy", "ids", "lps"):
        assert call(fn, SCORE, **{q: SCORE[q] + 2}) == ALIGN, q
    assert call(fn, SCORE, ws=addr(6, 8)) == ALIGN
    for q in ("logp", "entropy", "ids", "lps", "ws"):
        for other in {"z", "tokens", "logp", "entropy", "ids", "lps", "ws"} - {q}:
            assert call(fn, SCORE, **{q: SCORE[other] + 16}) == ALIAS, (q, other)
    assert call(fn, SCORE, entropy=addr(0, 2 * (7 * 1000 + 996))) == ALIAS        # the last row's end
    assert lora.lora_token_logprobs_workspace_size(8, 1000, 5) > 0
    assert lora.lora_token_logprobs_workspace_size(0, 1000, 5) == 0
    assert lora.lora_token_logprobs_workspace_size(8, 1000, 1001) == 0


@pytest.mark.parametrize("name,base", [("lora_distill_fwd", FWD), ("lora_distill_bwd", BWD), ("lora_distill_step", STEP)])
def test_distill_refusals(lib, name, base):
    fn = getattr(lib, name)
    pointers = [q for q, v in base.items() if isinstance(v, int) and v >= 1 << 40]
    nulls(fn, base, pointers)                     # (labels too: the soft weight is not 1)
    assert call(fn, base, dtype=2) == UNSUPPORTED
    for bad in (dict(rows=0), dict(vocab=0), dict(ld=999), dict(top=0), dict(top=-1), dict(T=0.0), dict(T=math.nan),
                dict(T=math.inf), dict(w=-0.1), dict(w=1.1), dict(w=math.nan)):
        assert call(fn, base, **bad) == SHAPE, bad
    for bad in (dict(top=129), dict(rows=(1 << 21) + 1), dict(vocab=(1 << 20) + 1, ld=1 << 21), dict(ld=1 << 34)):
        assert call(fn, base, **bad) == UNSUPPORTED, bad
    for q in pointers:
        off = 1 if q in ("z", "dz") else (8 if q == "saved" else 2)
        assert call(fn, base, **{q: base[q] + off}) == ALIGN, q
    outs = {"lora_distill_fwd": ("loss", "saved"), "lora_distill_bwd": ("dz",), "lora_distill_step": ("loss", "dz")}[name]
    for q in outs:
        for other in set(pointers) - {q}:
            assert call(fn, base, **{q: base[other] + 16}) == ALIAS, (q, other)
    if name == "lora_distill_step":               # the loss apart from the logits, also where the gradient is in place
        assert call(fn, base, dz=base["z"], loss=base["z"] + 64) == ALIAS


def test_binding_refuses_host_tensors_and_wrong_shapes(lib):
    import torch
    bf, f32, i32, u8 = torch.bfloat16, torch.float32, torch.int32, torch.uint8
    x = torch.zeros((4, 64), dtype=bf)
    with pytest.raises(ValueError):
        lora.lora_mx4_quantize(x, torch.zeros((4, 128), dtype=u8), torch.zeros(512, dtype=u8))
    with pytest.raises(TypeError):
        lora.lora_mx4_quantize(x.float(), torch.zeros((4, 128), dtype=u8), torch.zeros(512, dtype=u8))
    with pytest.raises(ValueError):
        lora.lora_token_logprobs(torch.zeros((2, 8)), None, None, torch.zeros(2), None, None, torch.zeros(256, dtype=u8))
    with pytest.raises(TypeError):
        lora.lora_token_logprobs(torch.zeros((2, 8), dtype=torch.float16), None, None, torch.zeros(2), None, None,
                                 torch.zeros(256, dtype=u8))
    with pytest.raises(ValueError):
        lora.lora_distill_fwd(torch.zeros((2, 8)), torch.zeros((2, 3), dtype=i32), torch.zeros((2, 3)), None,
                              torch.zeros(2), torch.zeros((2, 4)))
