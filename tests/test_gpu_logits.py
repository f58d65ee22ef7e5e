"""Token log probabilities and distillation on the GPU against the float64
definition (oracle/output_ops.py).

Tolerances.  With y = (z - max z) / T and S = sum exp y: y carries three
roundings, so it is off by at most 3 2^-24 |y|; S by the terms' (at most 3 2^-24 |y|
+ 2^-23, weighted by exp y <= 1) and by the chained sums of at most 160 terms a
thread and 10 across threads, 2^-24 each: below 2e-5 of S, as log S then is in
absolute terms.  A log probability is held to 2e-5 + 2^-21 of its size, the
entropy to 2e-5 (1 + its size), a probability to 5e-5 of its own (its exponent's
error included for the sizes here).  Losses add what they sum; a gradient in
bf16 adds half a spacing, 2^-8 of its size at most."""
import numpy as np
import pytest

import oracle
from oracle import output_ops as ops

pytestmark = pytest.mark.gpu

DTYPES = ["bf16", "f32"]
# widths at the ends of every regime: single elements alone, rows kept in registers of each size, rows read again
VOCABS = [1, 2, 5, 8, 13, 64, 255, 1000, 4097, 8192, 8193, 16391, 32003, 40000, 65541, 131072, 140001, 280003]


def torch_type(dtype):
    import torch
    return torch.bfloat16 if dtype == "bf16" else torch.float32


def as_stored(z, dtype):
    """float64 values as the type holds them."""
    z = np.asarray(z, np.float32)
    if dtype == "f32":
        return z.astype(np.float64)
    import torch
    return torch.from_numpy(z).to(torch.bfloat16).to(torch.float64).numpy()


def on_device(z, dtype, pad=0, offset=0):
    """z [rows, vocab] on the device with row pitch vocab + pad, the first row
    `offset` elements into its buffer; the rest of the buffer holds NaN."""
    import torch
    rows, vocab = z.shape
    ld = vocab + pad
    buf = torch.full((offset + rows * ld,), float("nan"), dtype=torch_type(dtype), device="cuda")
    view = buf[offset:].view(rows, ld)[:, :vocab]
    view.copy_(torch.from_numpy(np.asarray(z, np.float32)))
    return view


def score(z, tokens, top, T=1.0, stream=None):
    import torch
    import paper_2403_11366_amd as lora
    rows, vocab = z.shape
    out = [torch.full(s, v, dtype=t, device="cuda") for s, v, t in
           (((rows,), 7.0, torch.float32), ((rows,), 7.0, torch.float32), ((rows, top), -7, torch.int32),
            ((rows, top), 7.0, torch.float32))]
    ws = torch.full((lora.lora_token_logprobs_workspace_size(rows, vocab, top),), 0xFF, dtype=torch.uint8, device="cuda")
    tok = torch.tensor(np.asarray(tokens), dtype=torch.int32, device="cuda")
    lora.lora_token_logprobs(z, tok, out[0], out[1], out[2] if top else None, out[3] if top else None, ws, temperature=T,
                             stream=stream)
    return [x.cpu().numpy() for x in out]


def close(got, want, rel=2.0 ** -21, tol=2e-5):
    got, want = np.asarray(got, np.float64), np.asarray(want, np.float64)
    with np.errstate(over="ignore"):                # values past the outputs' range are infinite
        want = np.where(np.isinf(want.astype(np.float32)), np.sign(want) * np.inf, want)
    fin = np.isfinite(want)
    assert np.array_equal(got[~fin], want[~fin], equal_nan=True), (got, want)
    assert (np.abs(got - want)[fin] <= tol + rel * np.abs(want[fin])).all(), np.abs(got - want)[fin].max()


def check_scores(z, tokens, top, T, got):
    logp, entropy, ids, lps = ops.token_logprobs(z, tokens, T, top)
    close(got[0], logp)
    close(got[1], entropy, rel=2e-5)
    assert np.array_equal(got[2], ids)
    close(got[3], lps)


def rows_of(vocab, seed, rows=5):
    """Ordinary rows, one banned in part by -inf, one by the lowest value, one of many ties."""
    rng = np.random.default_rng(seed)
    z = rng.normal(size=(rows, vocab)) * 2.5
    z[1, rng.random(vocab) < 0.3] = -np.inf
    z[2, rng.random(vocab) < 0.3] = -3.3895313892515355e38      # bf16's lowest
    z[3] = np.round(z[3])
    z[3, z[3] == 0] = rng.choice([0.0, -0.0])
    tokens = rng.integers(0, vocab, rows)
    tokens[4] = rng.choice([-1, vocab, -100])
    return z, tokens


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_scores_match_the_definition(vocab, dtype):
    print(f"scores {vocab} {dtype}", flush=True)
    z, tokens = rows_of(vocab, vocab)
    z = as_stored(z, dtype)
    for top, T, pad, offset in ((min(vocab, 20), 1.0, 0, 0), (min(vocab, 128), 0.7, 3, 1), (min(vocab, 1), 4.0, 8, 0),
                                (0, 1.0, 5, 3)):
        check_scores(z, tokens, top, T, score(on_device(z, dtype, pad, offset), tokens, top, T))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [9, 300, 5000, 33000, 150001])
def test_scores_of_special_rows(vocab, dtype):
    """Constant rows (every value ties), sorted ones, rows without a value, with NaN
    and infinities, and rows of the type's lowest value."""
    inf, nan = np.inf, np.nan
    rng = np.random.default_rng(vocab)
    low = -3.3895313892515355e38 if dtype == "bf16" else -3.4028234663852886e38
    line = np.arange(vocab, dtype=np.float64)
    z = np.stack([np.zeros(vocab), line / vocab * 8, -line / vocab * 8, np.full(vocab, -inf), np.full(vocab, low),
                  np.where(line == vocab - 1, 3.0, -inf), rng.normal(size=vocab), rng.normal(size=vocab),
                  np.full(vocab, nan), np.where(line % 2 == 0, -inf, nan), np.full(vocab, 1e4), rng.normal(size=vocab) * 1e3,
                  np.where(line < vocab // 2, low, -low), rng.integers(0, 2, vocab).astype(float)])
    z[6, vocab // 2] = nan
    z[7, vocab // 3] = inf
    z = as_stored(z, dtype)
    tokens = np.array([0, 1, 2, 3, 4, vocab - 1, 0, 1, 2, 3, 5, 6, vocab - 1, 1])
    for top in (1, min(vocab, 7), min(vocab, 128)):
        check_scores(z, tokens, top, 1.0, score(on_device(z, dtype, 1, 1), tokens, top, 1.0))


def test_scores_without_tokens():
    import torch
    import paper_2403_11366_amd as lora
    z, _ = rows_of(1000, 1)
    z = as_stored(z, "f32")
    d = on_device(z, "f32")
    entropy = torch.empty(5, device="cuda")
    ws = torch.empty(lora.lora_token_logprobs_workspace_size(5, 1000, 0), dtype=torch.uint8, device="cuda")
    lora.lora_token_logprobs(d, None, None, entropy, None, None, ws)
    close(entropy.cpu().numpy(), ops.token_logprobs(z, [-1] * 5, 1.0, 0)[1], rel=2e-5)


# ---- distillation -------------------------------------------------------------
def lists_of(z, top, seed):
    """Teacher lists: whole, shorter, with one id twice, with ids outside, with -inf
    logits, none; labels listed, unlisted and none."""
    rng = np.random.default_rng(seed)
    rows, vocab = z.shape
    ids = np.full((rows, top), -1)
    for i in range(rows):
        n = min(top, vocab)
        ids[i, :n] = rng.permutation(vocab)[:n]
    t = rng.normal(size=(rows, top)) * 2
    if rows > 1:
        ids[1, top // 2:] = -1
    if rows > 2 and top > 2:
        ids[2, top - 1] = ids[2, 0]
        t[2, 1] = -np.inf
    if rows > 3:
        ids[3, 0] = vocab
        ids[3, -1] = 2 ** 31 - 1
    if rows > 4:
        ids[4] = -1
    labels = rng.integers(0, vocab, rows)
    labels[0] = max(ids[0, 0], 0)
    if rows > 3:
        labels[3] = -100
    return ids, t.astype(np.float32), labels, rng.uniform(0.2, 2.0, rows).astype(np.float32)


def run_distill(d, ids, t, labels, dl, T, w, dtype, pad, offset, stream=None):
    """(loss, gradient) by the two calls and by the one call."""
    import torch
    import paper_2403_11366_amd as lora
    rows, vocab = d.shape
    dev = [torch.tensor(np.asarray(x), dtype=ty, device="cuda") for x, ty in
           ((ids, torch.int32), (t, torch.float32), (dl, torch.float32))]
    lab = None if labels is None else torch.tensor(labels, dtype=torch.int32, device="cuda")
    got = []
    for calls in ("two", "one"):
        loss = torch.full((rows,), 7.0, device="cuda")
        saved = torch.full((rows, 4), 7.0, device="cuda")
        g = on_device(np.full((rows, vocab), 9.0), dtype, pad, offset)
        if calls == "two":
            lora.lora_distill_fwd(d, dev[0], dev[1], lab, loss, saved, temperature=T, soft_weight=w, stream=stream)
            lora.lora_distill_bwd(d, dev[0], dev[1], lab, saved, dev[2], g, temperature=T, soft_weight=w, stream=stream)
        else:
            lora.lora_distill_step(d, dev[0], dev[1], lab, dev[2], loss, g, temperature=T, soft_weight=w, stream=stream)
        whole = g.as_strided((rows, vocab + pad), (vocab + pad, 1)) if rows == 1 or not pad else None
        got.append((loss.cpu().numpy(), g.double().cpu().numpy()))
        if pad and rows > 1:        # the elements between rows are left alone
            between = g.as_strided((rows - 1, pad), (vocab + pad, 1), g.storage_offset() + vocab)
            assert bool(torch.isnan(between).all())
        del whole
    return got


def check_distill(z, ids, t, labels, dl, T, w, got, dtype):
    loss, grad = ops.distill(z, ids, t.astype(np.float64), labels, T, w, dl.astype(np.float64))
    rows, vocab = z.shape
    for l, g in got:
        close(l, loss, rel=2.0 ** -20, tol=4e-5 * (w * T * T + (1 - w) + 1e-3))
        for i in range(rows):
            fin = np.isfinite(grad[i])
            assert np.array_equal(g[i][~fin], grad[i][~fin], equal_nan=True), i
            if not fin.any():
                continue
            q = np.exp(ops.log_softmax(z[i] / T)) if w else np.zeros(vocab)
            h = np.exp(ops.log_softmax(z[i])) if w < 1 else np.zeros(vocab)
            p = ops.teacher_distribution(ids[i], t[i].astype(np.float64), T, vocab) if w else np.zeros(vocab)
            one = np.arange(vocab) == (labels[i] if labels is not None else -1)
            part = dl[i] * (w * T * (q + p) + (1 - w) * (h + one))
            part = np.where(np.isfinite(part), part, 0.0)
            tol = 5e-5 * part + (2.0 ** -8 * np.abs(grad[i]) if dtype == "bf16" else 0.0) + 1e-30
            bad = np.abs(g[i] - grad[i])[fin] > tol[fin]
            assert not bad.any(), (i, np.flatnonzero(bad)[:5], g[i][fin][bad][:5], grad[i][fin][bad][:5])


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", VOCABS)
def test_distillation_matches_the_definition(vocab, dtype):
    print(f"distill {vocab} {dtype}", flush=True)
    rng = np.random.default_rng(vocab)
    z = as_stored(rng.normal(size=(6, vocab)) * 2.5, dtype)
    for top, T, w, pad, offset in ((5, 1.0, 1.0, 0, 0), (32, 2.0, 0.75, 3, 1), (128, 4.0, 0.5, 8, 0), (1, 0.7, 0.25, 1, 2),
                                   (7, 3.0, 0.0, 5, 0)):
        ids, t, labels, dl = lists_of(z, top, vocab + top)
        lab = None if w == 1.0 else labels
        d = on_device(z, dtype, pad, offset)
        check_distill(z, ids, t, lab, dl, T, w, run_distill(d, ids, t, lab, dl, T, w, dtype, pad, offset), dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [9, 300, 33000, 150001])
def test_distillation_of_special_rows(vocab, dtype):
    """Columns at -inf listed and not, rows of -inf alone, NaN, +inf, the lowest
    value, constant rows, large logits, and a list of -inf alone."""
    inf, nan = np.inf, np.nan
    rng = np.random.default_rng(vocab)
    z = rng.normal(size=(11, vocab)) * 2
    ids, t, labels, dl = lists_of(z, 6, 3)
    ids[:] = ids[0]
    t[:] = t[0]
    z[1, [j for j in range(vocab) if j not in ids[1]][: vocab // 2]] = -inf     # unlisted columns banned
    labels[1] = ids[1, 1]
    z[2, ids[2, 0]] = -inf                                                       # a listed one
    z[3] = -inf
    z[4, vocab // 2] = nan
    z[5, vocab // 2] = inf
    z[6] = -3.3895313892515355e38
    z[7] = 0.0
    z[8] = z[8] * 300
    t[9] = -inf
    t[10, 2] = nan
    z = as_stored(z, dtype)
    for T, w in ((2.0, 0.5), (1.0, 1.0), (1.0, 0.0)):
        lab = None if w == 1.0 else labels
        tt, zz = t, z
        if w == 0.0:
            tt, zz = t[:10], z[:10]                     # (no soft term: the list's NaN is not looked at)
        n = len(zz)
        d = on_device(zz, dtype, 1, 1)
        got = run_distill(d, ids[:n], tt, lab if lab is None else lab[:n], dl[:n], T, w, dtype, 1, 1)
        check_distill(zz, ids[:n], tt, lab if lab is None else lab[:n], dl[:n], T, w, got, dtype)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("vocab", [64, 5001, 33000, 150001])
def test_gradient_in_place_and_on_another_alignment(vocab, dtype):
    import torch
    import paper_2403_11366_amd as lora
    rng = np.random.default_rng(vocab)
    z = as_stored(rng.normal(size=(7, vocab)), dtype)
    ids, t, labels, dl = lists_of(z, 9, 4)
    dev = [torch.tensor(x, dtype=ty, device="cuda") for x, ty in
           ((ids, torch.int32), (t, torch.float32), (labels, torch.int32), (dl, torch.float32))]
    how = {"temperature": 2.0, "soft_weight": 0.5}
    loss = torch.empty(7, device="cuda")
    d = on_device(z, dtype, 3, 0)
    want = on_device(z * 0, dtype, 3, 0)
    lora.lora_distill_step(d, *dev, loss, want, **how)
    for offset in (1, 2, 3):
        other = on_device(z * 0, dtype, 3, offset)
        lora.lora_distill_step(d, *dev, loss, other, **how)
        assert torch.equal(other, want), offset
    saved = torch.empty((7, 4), device="cuda")
    lora.lora_distill_fwd(d, *dev[:3], loss, saved, **how)
    two = on_device(z * 0, dtype, 3, 1)
    lora.lora_distill_bwd(d, *dev[:3], saved, dev[3], two, **how)
    here = on_device(z, dtype, 3, 0)
    lora.lora_distill_bwd(here, *dev[:3], saved, dev[3], here, **how)
    assert torch.equal(here, two)
    here = on_device(z, dtype, 3, 0)
    lora.lora_distill_step(here, *dev, loss, here, **how)
    assert torch.equal(here, want)


def test_gradient_against_differences_of_the_loss():
    """Central differences of the GPU's own fp32 loss in directions of each row:
    with steps of 2^-6 their error is about 2^-24 |loss| / 2^-6 and the third
    derivative's 2^-12 / 6."""
    import torch
    import paper_2403_11366_amd as lora
    rng = np.random.default_rng(5)
    z = as_stored(rng.normal(size=(6, 50)), "f32")
    ids, t, labels, dl = lists_of(z, 8, 6)
    dev = [torch.tensor(x, dtype=ty, device="cuda") for x, ty in
           ((ids, torch.int32), (t, torch.float32), (labels, torch.int32), (np.ones(6), torch.float32))]
    for T, w in ((1.0, 1.0), (2.0, 0.5), (1.0, 0.0)):
        how = {"temperature": T, "soft_weight": w}

        def loss_at(x):
            loss, g = torch.empty(6, device="cuda"), torch.empty((6, 50), device="cuda")
            lora.lora_distill_step(on_device(x, "f32"), *dev, loss, g, **how)
            return loss.double().cpu().numpy(), g.double().cpu().numpy()

        grad = loss_at(z)[1]
        for _ in range(4):
            u = rng.normal(size=z.shape)
            u = as_stored(u / np.linalg.norm(u, axis=1, keepdims=True), "f32")
            h = 2.0 ** -6
            num = (loss_at(z + h * u)[0] - loss_at(z - h * u)[0]) / (2 * h)
            assert np.abs(num - (grad * u).sum(1)).max() < 5e-4


def test_same_bits_on_streams_in_graphs_and_again():
    """Every call on a side stream and in a captured graph, replayed with eager work
    between, against the eager call on the default stream."""
    import torch
    import paper_2403_11366_amd as lora
    for rows, vocab, dtype in ((1, 32000, "bf16"), (9, 1003, "f32"), (40, 33001, "bf16"), (3, 140001, "f32")):
        rng = np.random.default_rng(rows)
        zs = [as_stored(rng.normal(size=(rows, vocab)) * 2, dtype) for _ in range(2)]
        ids, t, labels, dl = lists_of(zs[0], 16, 8)
        dev = [torch.tensor(x, dtype=ty, device="cuda") for x, ty in
               ((ids, torch.int32), (t, torch.float32), (labels, torch.int32), (dl, torch.float32))]
        z = on_device(zs[0], dtype, 1, 0)
        o = {"logp": torch.empty(rows, device="cuda"), "entropy": torch.empty(rows, device="cuda"),
             "ids": torch.empty((rows, 16), dtype=torch.int32, device="cuda"), "lps": torch.empty((rows, 16), device="cuda"),
             "loss": torch.empty(rows, device="cuda"), "saved": torch.empty((rows, 4), device="cuda"),
             "g": on_device(zs[0] * 0, dtype, 1, 0), "loss1": torch.empty(rows, device="cuda"),
             "g1": on_device(zs[0] * 0, dtype, 1, 0)}
        ws = torch.empty(lora.lora_token_logprobs_workspace_size(rows, vocab, 16), dtype=torch.uint8, device="cuda")
        how = {"temperature": 2.0, "soft_weight": 0.5}

        def calls():
            lora.lora_token_logprobs(z, dev[2], o["logp"], o["entropy"], o["ids"], o["lps"], ws)
            lora.lora_distill_fwd(z, *dev[:3], o["loss"], o["saved"], **how)
            lora.lora_distill_bwd(z, *dev[:3], o["saved"], dev[3], o["g"], **how)
            lora.lora_distill_step(z, *dev, o["loss1"], o["g1"], **how)

        want = []
        for x in zs:
            z.copy_(torch.from_numpy(x.astype(np.float32)))
            calls()
            want.append({q: v.clone() for q, v in o.items()})
        z.copy_(torch.from_numpy(zs[0].astype(np.float32)))
        torch.cuda.synchronize()
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            calls()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                calls()
        side.synchronize()
        assert all(torch.equal(o[q], want[0][q]) for q in o)
        for it in range(4):
            z.copy_(torch.from_numpy(zs[it % 2].astype(np.float32)))
            for v in o.values():
                v.fill_(3)
            ws.fill_(0xFF)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(o[q], want[it % 2][q]) for q in o), (rows, vocab, it)


def test_logits_past_32_bit_offsets():
    """2.2e9 logits: the last rows of the whole equal the same rows on their own."""
    import torch
    import paper_2403_11366_amd as lora
    rows, vocab, top = 16800, 131072, 4
    z = torch.empty((rows, vocab), dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    few = torch.randn((1200, vocab), generator=gen, device="cuda", dtype=torch.float32).to(torch.bfloat16)
    for i in range(0, rows, 1200):
        z[i:i + 1200] = torch.roll(few, i // 1200, 1)
    del few
    ids = torch.randint(0, vocab, (rows, top), generator=gen, device="cuda", dtype=torch.int32)
    t = torch.randn((rows, top), generator=gen, device="cuda")
    labels, dl = ids[:, 0].contiguous(), torch.rand(rows, generator=gen, device="cuda")

    def calls(a, b):
        n = b - a
        out = [torch.empty(n, device="cuda"), torch.empty(n, device="cuda"), torch.empty((n, top), dtype=torch.int32, device="cuda"),
               torch.empty((n, top), device="cuda")]
        ws = torch.empty(lora.lora_token_logprobs_workspace_size(n, vocab, top), dtype=torch.uint8, device="cuda")
        lora.lora_token_logprobs(z[a:b], labels[a:b], *out, ws)
        loss, saved, g = torch.empty(n, device="cuda"), torch.empty((n, 4), device="cuda"), torch.empty_like(z[a:b])
        args = (ids[a:b], t[a:b], labels[a:b])
        how = {"temperature": 2.0, "soft_weight": 0.5}
        lora.lora_distill_fwd(z[a:b], *args, loss, saved, **how)
        lora.lora_distill_bwd(z[a:b], *args, saved, dl[a:b], g, **how)
        out += [loss, saved[-8:].clone(), g[-8:].clone()]
        lora.lora_distill_step(z[a:b], *args, dl[a:b], loss, g, **how)
        return [x[-8:].clone() for x in out] + [loss[-8:].clone(), g[-8:].clone()]

    whole, last = calls(0, rows), calls(rows - 8, rows)
    for x, y in zip(whole, last):
        assert torch.equal(x, y)
