"""Cross entropy without logits over several pieces of the vocabulary, on every tile of dX,
with a piece's part of dX formed by one workgroup alone (the sums that pieces carry are
scaled, joined by the last piece's and by the label's in one kernel) and by several.
Selected rows against the definition in 64 bits, with references that stay, move in a
later piece and move in the last one.  test_xent_pieces_plan.py holds the shapes to
these plans."""
import numpy as np
import pytest

from test_gpu_xent import bounds

pytestmark = pytest.mark.gpu

# rows, vocabulary, k: 128 x 256, 256 x 256 (three) and 64 x 256 tiles of dX, unshared; 64 x
# 256, 128 x 256 and 256 x 256, shared; and one piece, shared, with references for rows alone
SEVERAL = [(8192, 32000, 1024), (4096, 32000, 4096), (8300, 20003, 1032), (16400, 9001, 264), (13777, 3397, 8),
           (261, 72717, 8), (5000, 30011, 40), (4738, 6889, 1024)]
ONE = [(519, 11037, 5120)]


@pytest.mark.parametrize("rows,vocab,k", SEVERAL + ONE)
@pytest.mark.parametrize("grow", [0.0, 400.0, -400.0])
def test_several_pieces(rows, vocab, k, grow):
    import torch
    import paper_2403_11366_amd as lora
    print(f"xent pieces {rows} x {vocab} x {k}, grow {grow}", flush=True)
    gen = torch.Generator(device="cuda").manual_seed(rows + k)
    X = torch.randn((rows, k), generator=gen, device="cuda").bfloat16()
    W = (torch.randn((vocab, k), generator=gen, device="cuda") * 2 * k ** -0.5).bfloat16()
    labels = torch.randint(0, vocab, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    labels[1::11] = -100
    # logits that grow along the vocabulary, in some rows, and in others in the last columns alone
    X[:, :2], W[:, :2] = 0, 0
    W[:, 0] = torch.linspace(0, 1, vocab, device="cuda").bfloat16()
    W[-40:, 1] = 1.0
    X[0::3, 0] = grow
    X[1::3, 1] = grow
    dloss = torch.randn(rows, generator=gen, device="cuda") / rows
    nan = float("nan")
    loss, loss2, dX, dX2 = (torch.full(s, nan, dtype=t, device="cuda") for s, t in
                            (((rows,), torch.float32), ((rows,), torch.float32), ((rows, k), torch.bfloat16), ((rows, k), torch.bfloat16)))
    saved = torch.full((rows, 2), nan, device="cuda")
    ws = torch.full((lora.lora_linear_xent_workspace_size(rows, vocab, k, True),), 0xFF, dtype=torch.uint8, device="cuda")
    lora.lora_linear_xent_step(X, W, labels, dloss, loss, dX, None, ws)
    ws.fill_(0xFF)
    lora.lora_linear_xent_fwd(X, W, labels, loss2, saved, ws)
    lora.lora_linear_xent_bwd(X, W, labels, saved, dloss, dX2, None, ws)
    rng = np.random.default_rng(rows)
    at = sorted({0, 1, 2, 63, 64, 127, 128, 255, 256, 257, rows // 2, rows - 257, rows - 3, rows - 2, rows - 1} |
                set(rng.choice(rows, 60, replace=False).tolist()))
    x, w = X[at].double().cpu().numpy(), W.double().cpu().numpy()
    y, d = labels[at].cpu().numpy(), dloss[at].double().cpu().numpy()
    (want, want_dX, _), (t_loss, t_dX, _) = bounds(x, w, y, d)
    for how, l, g in (("step", loss, dX), ("two", loss2, dX2)):
        assert (np.abs(l[at].double().cpu().numpy() - want) <= t_loss * (1 + 1e-6)).all(), how
        assert (np.abs(g[at].double().cpu().numpy() - want_dX) <= t_dX * (1 + 1e-6)).all(), how
        assert torch.isfinite(l).all() and torch.isfinite(g).all(), how
