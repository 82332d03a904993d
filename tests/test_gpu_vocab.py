"""Token embedding and vocabulary cross entropy on the GPU against their float64 definitions."""
import pytest
import torch

import vocab_ref as ref
from paper_2406_08128_b200 import chela

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"bf16": chela.BF16, "f32": chela.F32}


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def normal(g, *shape, dtype=torch.float32, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def token_ids(g, T, V, left_out=0.0, skew=True, dtype=torch.int64):
    u = torch.rand(T, generator=g, device="cuda", dtype=torch.float64)
    ids = ((V + 1) ** u - 1 if skew else u * V).long().clamp(0, V - 1)
    if left_out:
        out = torch.rand(T, generator=g, device="cuda") < left_out
        ids = torch.where(out, torch.where(ids % 2 == 0, -1 - ids, V + ids), ids)   # on either side of the table
    return ids.to(dtype)


def within(got, true, bound, what):
    got = got.double()
    assert torch.isfinite(got).all(), what
    over = (got - true).abs() - bound
    i = int(over.argmax())
    assert float(over.max()) <= 0, "%s: off by %g at %d, allowed %g, value %g" % (
        what, float((got - true).abs().flatten()[i]), i, float(torch.as_tensor(bound).expand_as(true).flatten()[i]), float(true.flatten()[i]))


# ------------------------------------------------------------------------------------------------ embedding

@pytest.mark.parametrize("T,V,D,wt,ot,left_out,ids", [
    (1, 1, 8, "bf16", "bf16", 0, torch.int64), (3, 7, 16, "f32", "bf16", 0.5, torch.int32), (65, 1000, 264, "bf16", "f32", 0.2, torch.int32),
    (257, 50, 1024, "f32", "f32", 0, torch.int64), (1000, 3000, 520, "bf16", "bf16", 0.9, torch.int64), (4097, 100, 72, "bf16", "bf16", 0, torch.int32)])
def test_embedding(T, V, D, wt, ot, left_out, ids):
    g = gen(T + V)
    w = normal(g, V, D, dtype=DT[wt])
    i = token_ids(g, T, V, left_out, dtype=ids)
    out = chela.embed_fwd(i, w, scale=1.7, out_dtype=CODE[ot])
    true = ref.embed(i, w, 1.7)
    within(out, true, (2.0 ** -23 + ref.HALF[DT[ot]]) * true.abs(), "out")   # the scale as fp32, its product, the output


@pytest.mark.parametrize("T,V,D,it,gt,left_out,skew", [
    (1, 1, 8, "bf16", "f32", 0, True), (2, 300, 8, "f32", "bf16", 0, True), (63, 10, 24, "bf16", "bf16", 0.3, True), (64, 1, 1024, "bf16", "f32", 0, True),
    (65, 1, 264, "f32", "f32", 0, True), (129, 2, 256, "bf16", "f32", 0.1, False), (1000, 511, 520, "bf16", "bf16", 0.5, True),
    (1000, 512, 136, "f32", "f32", 0, True), (4096, 513, 64, "bf16", "f32", 0, True), (4097, 3, 72, "bf16", "f32", 0.2, False),
    (5000, 262143, 8, "bf16", "f32", 0, False), (5000, 262144, 16, "bf16", "bf16", 0.1, True), (20000, 70000, 40, "f32", "f32", 0.6, True),
    (9000, 1, 32, "bf16", "f32", 0, True), (300, 20, 2048, "bf16", "f32", 1.0, True),
    (65536, 700, 8, "f32", "f32", 0, True), (65537, 70000, 8, "bf16", "f32", 0.3, True), (140001, 100, 16, "bf16", "bf16", 0, False),
    (33, 9, 4104, "f32", "f32", 0, True)])
@pytest.mark.parametrize("before", ["none", "other", "same"])
def test_embedding_gradient(T, V, D, it, gt, left_out, skew, before):
    g = gen(T + 3 * V + D)
    d_out = normal(g, T, D, dtype=DT[it])
    ids = token_ids(g, T, V, left_out, skew, torch.int32 if D % 16 else torch.int64)
    d_w_in = None if before == "none" else normal(g, V, D, dtype=DT[gt])
    true = ref.embed_bwd(ids, d_out, V, 0.3, d_w_in)
    mag = ref.embed_bwd(ids, d_out, V, 0.3, d_w_in, mag=True)
    d_w = d_w_in.clone() if before == "same" else None
    got = chela.embed_bwd(ids, d_out, V, scale=0.3, grad_dtype=CODE[gt], d_w_in=d_w if before == "same" else d_w_in, d_w=d_w)
    # at most 16 sums in a block, one a block for an eighth of them, 8 for the eighths; the scale, the product, the last sum
    within(got, true, (28 + T / 128) * 2.0 ** -24 * mag + 1.01 * ref.HALF[DT[gt]] * true.abs(), "d_w")
    again = chela.embed_bwd(ids, d_out, V, scale=0.3, grad_dtype=CODE[gt], d_w_in=d_w_in)
    assert torch.equal(again, got)


# ------------------------------------------------------------------------------------------------ cross entropy

def hidden(g, T, V, D, dtype, targets, lean=4.0):
    w = normal(g, V, D, dtype=dtype, std=1.5 * D ** -0.5)
    kept = ref.kept_of(targets, V)
    toward = w[torch.where(kept, targets.long(), 0)].float() * (lean * torch.rand(T, 1, generator=g, device="cuda"))
    return (normal(g, T, D) + toward).to(dtype), w


LOSSES = [
    # a few tokens: their own kernels, by 4, 8 and (fp32) 16, up to 1024, 2048 and 4096 channels
    (3, 5, 8, "bf16", "f32", 0.3), (4, 3000, 1024, "f32", "f32", 0), (4, 700, 2056, "bf16", "bf16", 0), (4, 50, 4096, "bf16", "f32", 0.5), (8, 9999, 264, "bf16", "bf16", 0),
    (8, 4001, 2048, "bf16", "bf16", 0.2), (7, 333, 1032, "f32", "bf16", 0), (16, 2500, 344, "f32", "f32", 0.1), (16, 1, 16, "f32", "f32", 0), (9, 130, 1024, "f32", "f32", 0),
    (1, 40000, 72, "bf16", "bf16", 0), (5, 600, 520, "f32", "f32", 1.0), (8, 20, 4104, "bf16", "f32", 0), (16, 700, 2048, "f32", "f32", 0), (16, 700, 256, "bf16", "bf16", 0),
    # T, V, D, operands, gradients, left out
    (1, 1, 8, "bf16", "bf16", 0), (1, 2, 8, "f32", "f32", 0), (2, 300, 64, "bf16", "f32", 0), (48, 5000, 1024, "bf16", "bf16", 0),
    (127, 255, 72, "bf16", "bf16", 0.3), (128, 256, 128, "f32", "f32", 0.2), (129, 257, 136, "bf16", "f32", 0), (255, 511, 264, "f32", "bf16", 0.5),
    (256, 513, 256, "bf16", "bf16", 0), (257, 1000, 520, "bf16", "bf16", 0.9), (300, 205, 512, "bf16", "f32", 1.0), (1000, 3001, 200, "f32", "f32", 0.1),
    (2047, 205, 512, "bf16", "bf16", 0), (4097, 40, 64, "bf16", "bf16", 0.02), (700, 12345, 328, "bf16", "bf16", 0.6), (5000, 4999, 96, "bf16", "f32", 0.01)]


@pytest.mark.parametrize("T,V,D,it,gt,left_out", LOSSES)
def test_loss_and_gradients(T, V, D, it, gt, left_out):
    g = gen(7 * T + V + D)
    targets = token_ids(g, T, V, left_out, dtype=torch.int32 if T % 2 else torch.int64)
    h, w = hidden(g, T, V, D, DT[it], targets)
    d_loss = torch.rand(T, generator=g, device="cuda") / T
    d_lse = normal(g, T, std=0.1 / T) if V % 2 else None
    scale = 1.0 if D % 16 == 8 else 0.8
    r = ref.loss(h, w, targets, scale, d_loss, d_lse)
    if left_out:
        h[~ref.kept_of(targets, V)] = float("nan")   # rows that are left out are not read
    loss, lse = chela.vocabloss_fwd(h, w, targets, scale=scale)
    bound = ref.lse_bound(r, D, DT[it])
    within(lse, r["lse"], bound, "lse")
    within(loss, r["loss"], bound + ref.z_bound(r, D, DT[it]), "loss")
    assert (loss[~ref.kept_of(targets, V)] == 0).all() and (lse[~ref.kept_of(targets, V)] == 0).all()
    got = chela.vocabloss_bwd(h, w, targets, lse, d_loss, d_lse, scale=scale, grad_dtype=CODE[gt])
    for name, a, b in zip(("d_h", "d_w"), got, ref.grad_bounds(r, T, V, D, DT[it], DT[gt])):
        within(a, r[name], b, name)
    assert (got.d_h[~ref.kept_of(targets, V)] == 0).all()
    again = chela.vocabloss_bwd(h, w, targets, lse, d_loss, d_lse, scale=scale, grad_dtype=CODE[gt])
    assert torch.equal(again.d_h, got.d_h) and torch.equal(again.d_w, got.d_w)
