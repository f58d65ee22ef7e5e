"""Cross entropy without logits on the GPU against the float64 definition
(oracle/train_ops.py).

Tolerances.  A logit is an fp32 sum of k exact products: off by e_iv <= (k + 1) 2^-24
sum |x||w|.  An exponent is formed by one rounding of a number of at most A = 1.5 (|z|
largest + |reference|) + 64 and carries z's error: its power is off by a factor within
rho_i = max_v e_iv + 2^-23 (A + 2).  A row's sum adds up to T = 64 + tiles more roundings
of 2^-24.  So the loss is off by 2 (max_v e_iv + 2^-23 (A + 2)) + T 2^-24 and half a
spacing of itself, and G by a factor within 2 rho_i + T 2^-24 and, as an operand, half a
bf16 spacing (2^-8; the label's own as all others').  dX and dW are fp32 sums of G's
products rounded to bf16: 2^-8 of themselves, and of sum |g||w| (or |g||x|) the factors
above and 2^-24 for each term; and a power, or a G, below 2^-126 may count as 0: 2^-125
of sum |w| (or |x|) and of dX or dW itself."""
import numpy as np
import pytest

import oracle
from oracle import train_ops as ops

pytestmark = pytest.mark.gpu


def to_bits(x):
    return oracle.f64_to_bf16_bits(x)


def f64(bits):
    return oracle.bf16_bits_to_f64(bits)


def case(rows, vocab, k, seed, spread=2.5, sure=8.0):
    """Hidden states that know their label more or less; some rows without one."""
    rng = np.random.default_rng(seed)
    w = rng.normal(size=(vocab, k)) * spread * k ** -0.5
    labels = rng.integers(0, vocab, rows)
    x = rng.normal(size=(rows, k)) + rng.random((rows, 1)) * sure / spread * w[labels]
    none = rng.random(rows) < 0.1
    if rows > 3:
        none[0], none[1] = False, True
    labels = np.where(none, rng.choice([-100, -1, vocab, 2 ** 31 - 1], rows), labels).astype(np.int32)
    return to_bits(x), to_bits(w), labels, (rng.normal(size=rows) / rows).astype(np.float32)


def buffers(rows, vocab, k, dx, dw, fill=0xFF):
    import torch
    import paper_2403_11366_amd as lora
    nan = float("nan")
    return (torch.full((rows,), nan, device="cuda"), torch.full((rows, 2), nan, device="cuda"),
            torch.full((rows, k), nan, dtype=torch.bfloat16, device="cuda") if dx else None,
            torch.full((vocab, k), nan, dtype=torch.bfloat16, device="cuda") if dw else None,
            torch.full((lora.lora_linear_xent_workspace_size(rows, vocab, k, dx, dw),), fill, dtype=torch.uint8, device="cuda"))


def run(x, w, labels, dloss, how, dx=True, dw=False, fill=0xFF):
    """how: "step", or "two" (forward and backward).  Returns loss, dX, dW on the host in float64."""
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import bits_to_device, device_to_bits
    X, W = bits_to_device(x), bits_to_device(w)
    y, d = torch.from_numpy(labels).cuda(), torch.from_numpy(dloss).cuda()
    loss, saved, dX, dW, ws = buffers(*x.shape[:1], w.shape[0], x.shape[1], dx, dw, fill)
    if how == "step":
        lora.lora_linear_xent_step(X, W, y, d, loss, dX, dW, ws)
    else:
        lora.lora_linear_xent_fwd(X, W, y, loss, saved, ws)
        lora.lora_linear_xent_bwd(X, W, y, saved, d, dX, dW, ws)
    out = lambda t: None if t is None else f64(device_to_bits(t))
    return loss.double().cpu().numpy(), out(dX), out(dW)


def bounds(x, w, labels, dloss):
    z, size = x @ w.T, np.abs(x) @ np.abs(w).T
    k = x.shape[1]
    e = (k + 1) * 2.0 ** -24 * size.max(axis=1)
    rho = e + 2.0 ** -23 * (1.5 * 2 * np.abs(z).max(axis=1) + 66)
    terms = 64 + -(-w.shape[0] // 128)
    loss, g, dX, dW = ops.xent(x, w, labels, dloss)
    t_loss = 2 * rho + terms * 2.0 ** -24 + 2.0 ** -24 * np.abs(loss)
    factor = 2.0 ** -8 + 2 * rho + terms * 2.0 ** -24
    ga = np.abs(g) * factor[:, None]
    t_dx = 2.0 ** -8 * np.abs(dX) + ga @ np.abs(w) + (w.shape[0] + 64) * 2.0 ** -24 * (np.abs(g) @ np.abs(w)) + 2.0 ** -125 * (1 + np.abs(w).sum(axis=0))
    t_dw = 2.0 ** -8 * np.abs(dW) + ga.T @ np.abs(x) + (len(x) + 64) * 2.0 ** -24 * (np.abs(g).T @ np.abs(x)) + 2.0 ** -125 * (1 + np.abs(x).sum(axis=0))
    return (loss, dX, dW), (t_loss, t_dx, t_dw)


def close(got, want, tol, label=""):
    for name, a, b, t in zip(("loss", "dX", "dW"), got, want, tol):
        if a is not None:
            bad = ~(np.abs(a - b) <= t * (1 + 1e-6))
            assert not bad.any(), (label, name, np.argwhere(bad)[:5].tolist(), int(bad.sum()))


SIZES = [(1, 1, 8), (1, 2, 64), (1, 32000, 512), (2, 129, 40), (5, 1000, 264), (16, 128, 64), (37, 5001, 520), (63, 127, 72),
         (64, 257, 128), (65, 4000, 256), (100, 333, 1032), (128, 2048, 512), (129, 300, 64), (130, 1023, 200), (200, 10007, 136),
         (256, 256, 64), (257, 257, 328), (300, 5000, 512), (513, 2049, 72), (700, 1500, 264), (1000, 8003, 64), (1500, 769, 512),
         (90, 16000, 2056), (200, 20000, 1024), (250, 9001, 2048), (600, 4000, 1032), (1030, 2000, 72), (2060, 3000, 264), (4100, 1000, 4104), (1000, 15000, 4104), (384, 5000, 4104), (2000, 9000, 1032)]


@pytest.mark.parametrize("rows,vocab,k", SIZES)
def test_matches_the_definition(rows, vocab, k):
    print(f"xent {rows} x {vocab} x {k}", flush=True)
    x, w, labels, d = case(rows, vocab, k, rows + 3 * vocab + 5 * k)
    want, tol = bounds(f64(x), f64(w), labels, d.astype(np.float64))
    for how, dx, dw in (("step", True, False), ("step", True, True), ("step", False, True), ("two", True, False),
                        ("two", False, True), ("two", True, True)):
        got = run(x, w, labels, d, how, dx, dw)
        close(got, want, tol, (how, dx, dw))
        none = (labels < 0) | (labels >= vocab)
        assert (got[0][none] == 0).all() and (not dx or (got[1][none] == 0).all())


def test_several_pieces():
    """Rows and columns that take three pieces, the last one short; splits of a piece."""
    x, w, labels, d = case(4100, 20011, 72, 1)
    want, tol = bounds(f64(x), f64(w), labels, d.astype(np.float64))
    close(run(x, w, labels, d, "step"), want, tol, "step")
    close(run(x, w, labels, d, "two", True, True), want, tol, "two")


@pytest.mark.parametrize("rows,vocab,cols", [(9, 700, 64), (40, 3000, 64), (300, 900, 64), (4097, 20000, 64)])
@pytest.mark.parametrize("size", [60.0, 400.0, 3000.0])
def test_logits_of_any_size(rows, vocab, cols, size):
    """Rows whose logits are large, all far below zero, or grow from piece to piece: the
    reference of the exponentials has to move."""
    rng = np.random.default_rng(int(size) + rows)
    x, w, labels, d = case(rows, vocab, cols, 5, spread=1.0, sure=1.0)
    x, w = f64(x), f64(w)
    w[:, 0] = 1.0                                             # column 0 of x shifts a row's logits
    w[:, 1] = np.linspace(0, 1, vocab)                        # column 1 makes them grow along the vocabulary
    kind = rng.integers(0, 5, rows)
    x[:, 0] = np.choose(kind, [0.0, size, -size, 0.0, -size])
    x[:, 1] = np.choose(kind, [0.0, 0.0, 0.0, size, 2 * size])
    x, w = to_bits(x), to_bits(w)
    want, tol = bounds(f64(x), f64(w), labels, d.astype(np.float64))
    close(run(x, w, labels, d, "step"), want, tol, "step")
    close(run(x, w, labels, d, "two", True, True), want, tol, "two")


def test_sure_rows_keep_their_digits():
    """Labels of probability 1 - 1e-3 .. 1 - 1e-12: the loss and the gradient to a few parts
    in a thousand of themselves, not of 1."""
    rows, vocab, k = 48, 3000, 64
    rng = np.random.default_rng(0)
    w = rng.choice([-1.0, 1.0], (vocab, k)) * 0.5
    labels = rng.permutation(vocab)[:rows].astype(np.int32)
    x = w[labels] * np.linspace(1.0, 3.0, rows)[:, None]      # logits in steps of 0.25: exact in fp32
    x, w = to_bits(x), to_bits(w)
    loss, _, dX, _ = ops.xent(f64(x), f64(w), labels, np.ones(rows))
    for how in ("step", "two"):
        got = run(x, w, labels, np.ones(rows, np.float32), how)
        # the power of a difference D of up to 96 is off by 2^-23 (1.5 D + 66) < 3e-5 of itself, G by 2^-8
        assert (np.abs(got[0] - loss) <= 1e-4 * loss).all(), how
        size = loss[:, None] * np.abs(f64(w)).max() * 2
        assert (np.abs(got[1] - dX) <= (2.0 ** -7 + 1e-3) * size).all(), how


@pytest.mark.parametrize("rows", [6, 300])
def test_not_a_number(rows):
    """A NaN, an infinity and an overflowing product in rows of X: those rows alone; a
    row without a label is 0 whatever its logits."""
    vocab, k = 1000, 64
    x, w, labels, d = case(rows, vocab, k, 11)
    labels[:6] = [1, 2, 3, -1, -1, 5]
    x[0, 3], x[1, 4], x[2, :], x[3, 5], x[4, :] = 0x7FC0, 0x7F80, 0x7F7F, 0x7FC0, 0xFF7F
    for how in ("step", "two"):
        loss, dX, _ = run(x, w, labels, d, how)
        assert np.isnan(loss[:3]).all() and np.isnan(dX[:3]).all(), how
        assert (loss[3:5] == 0).all() and (dX[3:5] == 0).all(), how
        assert np.isfinite(loss[5:]).all() and np.isfinite(dX[5:]).all(), how
    labels[:3] = [-1, vocab, -100]                            # padding may hold anything
    clean = x.copy()
    clean[:5] = 0
    for how in ("step", "two"):
        got, want = run(x, w, labels, d, how, True, True), run(clean, w, labels, d, how, True, True)
        assert all(np.array_equal(a, b) for a, b in zip(got, want)), how


@pytest.mark.parametrize("rows,vocab,k,spread", [(1, 1, 8, 1.0), (1, 500, 64, 0.01), (3, 40000, 264, 0.01), (40, 700, 520, 0.01),
                                                 (2500, 600, 72, 0.01), (5000, 30011, 40, 0.01), (300, 3000, 1032, 2.5)])
def test_labels_rows_of_dW(rows, vocab, k, spread):
    """A label's entry of G enters dW with more than its bf16: where all other entries are
    small, a label's row of dW is off by its own rounding.  Some labels are many rows'."""
    x, w, labels, d = case(rows, vocab, k, rows + vocab, spread=spread, sure=0.0)
    labels[rows // 3:rows // 2] = vocab - 1
    fx, fw, fd = f64(x), f64(w), d.astype(np.float64)
    (_, _, want), (_, _, tol) = bounds(fx, fw, labels, fd)
    got = run(x, w, labels, d, "two", False, True)[2]
    assert (np.abs(got - want) <= tol * (1 + 1e-6)).all()
    _, g, _, _ = ops.xent(fx, fw, labels, fd)
    known = np.flatnonzero((labels >= 0) & (labels < vocab))
    own = np.zeros_like(g)
    own[known, labels[known]] = np.abs(g[known, labels[known]])
    # of the label's entries 2^-8 becomes 2^-16 (the rest, rounded from fp32), everything else as it was
    lesser = tol - (own.T @ np.abs(fx)) * (2.0 ** -8 - 2.0 ** -16)
    assert (np.abs(got - want) <= lesser * (1 + 1e-6)).all()


@pytest.mark.parametrize("rows,vocab,k", [(5, 1000, 4096), (300, 3001, 5000), (70, 2, 1032)])
def test_labels_logit_is_exact(rows, vocab, k):
    """All other logits 0, the label's a sum of k terms that cancel: the loss is off by its
    own rounding and that of the sum of powers alone, not by an fp32 sum over k."""
    x, w, labels, d = case(rows, vocab, k, k, spread=1.0, sure=0.0)
    w = f64(w) * 16
    y = vocab // 2
    w[:y], w[y + 1:] = 0, 0
    w, labels = to_bits(w), np.full(rows, y, np.int32)
    z = f64(x) @ f64(w)[y]
    want = np.where(z > 0, np.log1p((vocab - 1) * np.exp(-z)), np.log(vocab - 1 + np.exp(np.minimum(z, 0))) - z)   # (no cancellation)
    assert want.max() > 16
    # the sum of powers, its rounding and the label's power: 2^-24 of it each (vocab - 1 is exact), a
    # power whose exponent was rounded to 2^-24 of at most 128, and a small loss's quotient
    # and logarithm: 2^-22 of it; the result's rounding
    unlikely = z < 0
    tol = np.where(unlikely, 4 * 2.0 ** -24 + 2.0 ** -24 * want, 2.0 ** -17 * want)
    for how in ("step", "two"):
        loss = run(x, w, labels, d, how)[0]
        assert (np.abs(loss - want) <= tol * (1 + 1e-6)).all(), how


@pytest.mark.parametrize("rows,vocab", [(6, 1000), (300, 1300)])
def test_logits_of_minus_infinity(rows, vocab):
    """They have probability 0; a row with such a label has an infinite loss."""
    k = 64
    x, w, labels, d = case(rows, vocab, k, 12, sure=0.0)
    x = f64(x)
    x[:, 0] = np.abs(x[:, 0]) + 0.125
    x, labels = to_bits(x), np.where(labels < vocab, labels, -1)
    w[7, 0] = w[vocab - 1, 0] = 0xFF80
    labels[2], labels[4] = 7, vocab - 1
    labels = np.where((np.arange(rows) == 2) | (np.arange(rows) == 4), labels, np.where(labels % vocab == 7, 8, labels)).astype(np.int32)
    labels = np.where((np.arange(rows) != 4) & (labels == vocab - 1), 8, labels).astype(np.int32)
    kept = [v for v in range(vocab) if v not in (7, vocab - 1)]
    at = {v: i for i, v in enumerate(kept)}
    rest = np.array([at.get(y, -1) for y in labels], np.int32)
    want, tol = bounds(f64(x), f64(w[kept]), rest, d.astype(np.float64))
    for how in ("step", "two"):
        loss, dX, dW = run(x, w, labels, d, how, True, how == "two")
        assert (loss[[2, 4]] == np.inf).all(), how
        some = np.ones(rows, bool)
        some[[2, 4]] = False
        assert (np.abs(loss - want[0])[some] <= tol[0][some]).all(), how
        # where W is finite, the gradient of those rows is the one without such columns
        assert (np.abs(dX - want[1])[some][:, 1:] <= tol[1][some][:, 1:]).all(), how


def test_more_tiles_than_a_launch_has():
    """2^20 rows and 2^19 columns: a thread for each 128 logits would be 2^32 of them.  The
    loss of some rows against the definition."""
    import torch
    import paper_2403_11366_amd as lora
    rows, vocab, k = 1 << 20, 1 << 19, 8
    g = torch.Generator("cuda").manual_seed(3)
    X = torch.randn(rows, k, device="cuda", generator=g).bfloat16()
    W = torch.randn(vocab, k, device="cuda", generator=g).bfloat16()
    labels = torch.randint(0, vocab, (rows,), device="cuda", dtype=torch.int32, generator=g)
    loss = torch.empty(rows, device="cuda")
    ws = torch.empty(lora.lora_linear_xent_workspace_size(rows, vocab, k), dtype=torch.uint8, device="cuda")
    lora.lora_linear_xent_fwd(X, W, labels, loss, None, ws)
    torch.cuda.synchronize()
    at = [0, 1, 255, 256, 77777, rows // 2 - 1, rows // 2, rows - 257, rows - 1]
    x, w, y, got = X[at].double().cpu(), W.double().cpu(), labels[at].long().cpu(), loss[at].double().cpu()
    z = x @ w.t()
    want = torch.logsumexp(z, 1) - z.gather(1, y[:, None])[:, 0]
    size = (x.abs() @ w.abs().t()).max()   # as above, |z| and the reference at most size log2 e, 2^12 tiles
    tol = 2 * (9 * 2.0 ** -24 * size + 2.0 ** -23 * (1.5 * 2 * 1.45 * size + 66)) + (64 + 4096) * 2.0 ** -24
    assert ((got - want).abs() <= tol + 2.0 ** -24 * want).all()


def test_no_labels_at_all():
    x, w, labels, d = case(150, 500, 64, 2)
    labels[:] = -100
    for how in ("step", "two"):
        loss, dX, dW = run(x, w, labels, d, how, True, True)
        assert (loss == 0).all() and (dX == 0).all() and (dW == 0).all()


def test_columns_far_below():
    """Logits so low that their powers vanish count as probability 0."""
    rows, vocab, k = 70, 400, 64
    x, w, labels, d = case(rows, vocab, k, 4, spread=0.5, sure=0.0)
    x, w = f64(x), f64(w)
    x[:, 0], w[:, 0] = 16.0, np.where(np.arange(vocab) % 3 == 0, 0.0, -512.0)
    labels = np.where(labels >= 0, labels // 3 * 3, labels).astype(np.int32)
    x, w = to_bits(x), to_bits(w)
    want, tol = bounds(f64(x), f64(w), labels, d.astype(np.float64))
    close(run(x, w, labels, d, "step"), want, tol)
    close(run(x, w, labels, d, "two", True, True), want, tol)


@pytest.mark.parametrize("rows,vocab,k", [(5, 1000, 264), (300, 3001, 200)])
def test_repeated_calls_are_bit_identical_and_stay_in_their_buffers(rows, vocab, k):
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import bits_to_device
    x, w, labels, d = case(rows, vocab, k, 8)
    X, W, y, d = bits_to_device(x), bits_to_device(w), torch.from_numpy(labels).cuda(), torch.from_numpy(d).cuda()

    def inner(t, nbytes, dtype, shape):
        return t[256:256 + nbytes].view(dtype).view(shape)
    for dx, dw in ((True, False), (True, True)):
        runs = []
        for fill in (0x00, 0xA5):
            sizes = {"loss": 4 * rows, "saved": 8 * rows, "dX": 2 * rows * k, "dW": 2 * vocab * k,
                     "ws": lora.lora_linear_xent_workspace_size(rows, vocab, k, dx, dw)}
            raw = {q: torch.full((n + 512,), fill, dtype=torch.uint8, device="cuda") for q, n in sizes.items()}
            loss = inner(raw["loss"], sizes["loss"], torch.float32, (rows,))
            saved = inner(raw["saved"], sizes["saved"], torch.float32, (rows, 2))
            dX = inner(raw["dX"], sizes["dX"], torch.bfloat16, (rows, k))
            dW = inner(raw["dW"], sizes["dW"], torch.bfloat16, (vocab, k)) if dw else None
            ws = inner(raw["ws"], sizes["ws"], torch.uint8, (-1,))
            out = []
            lora.lora_linear_xent_step(X, W, y, d, loss, dX, dW, ws)
            out += [loss.clone(), dX.clone()] + ([dW.clone()] if dw else [])
            lora.lora_linear_xent_fwd(X, W, y, loss, saved, ws)
            lora.lora_linear_xent_bwd(X, W, y, saved, d, dX, dW, ws)
            out += [loss.clone(), saved.clone(), dX.clone()] + ([dW.clone()] if dw else [])
            runs.append(out)
            for q, t in raw.items():
                assert (t[:256] == fill).all() and (t[256 + sizes[q]:] == fill).all(), q
        assert all(torch.equal(a, b) for a, b in zip(*runs))


def test_forward_alone_and_without_saved():
    import torch
    import paper_2403_11366_amd as lora
    from paper_2403_11366_amd.device_io import bits_to_device
    x, w, labels, _ = case(40, 600, 64, 3)
    X, W, y = bits_to_device(x), bits_to_device(w), torch.from_numpy(labels).cuda()
    loss, saved, _, _, ws = buffers(40, 600, 64, False, False)
    lora.lora_linear_xent_fwd(X, W, y, loss, saved, ws)
    again = torch.full_like(loss, 5.0)
    lora.lora_linear_xent_fwd(X, W, y, again, None, ws)
    assert torch.equal(loss, again)


def test_gradient_is_the_losses_difference():
    """Along random directions: (loss(x + h v) - loss(x - h v)) / 2h of the definition
    against <dX, v> of the kernels (fp32 sums of bf16 products: 2^-8 of the terms)."""
    x, w, labels, d = case(30, 500, 64, 21)
    _, dX, dW = run(x, w, labels, d, "two", True, True)
    xf, wf, df = f64(x), f64(w), d.astype(np.float64)
    (_, rX, rW), (_, tX, tW) = bounds(xf, wf, labels, df)
    rng = np.random.default_rng(1)
    for _ in range(5):
        v, u, h = rng.normal(size=xf.shape), rng.normal(size=wf.shape), 1e-5
        fx = [(ops.xent(xf + s * h * v, wf, labels, df)[0] * df).sum() for s in (1, -1)]
        fw = [(ops.xent(xf, wf + s * h * u, labels, df)[0] * df).sum() for s in (1, -1)]
        assert abs((fx[0] - fx[1]) / (2 * h) - (dX * v).sum()) <= (tX * np.abs(v)).sum() + 1e-7
        assert abs((fw[0] - fw[1]) / (2 * h) - (dW * u).sum()) <= (tW * np.abs(u)).sum() + 1e-7
