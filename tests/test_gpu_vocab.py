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


@pytest.mark.parametrize("wt,ot", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "bf16"), ("f32", "f32")])
def test_rows_left_out_are_zero_whatever_the_scale(wt, ot):
    w = normal(gen(1), 10, 520, dtype=DT[wt])
    ids = torch.tensor([3, -1, 10, 0], device="cuda")
    for scale in (-2.0, float("inf"), float("nan")):
        rows = chela.embed_fwd(ids, w, scale=scale, out_dtype=CODE[ot])[1:3].float()
        assert (rows == 0).all() and not torch.signbit(rows).any()


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


def test_embedding_of_as_many_tokens_as_there_may_be():
    """2^31 - 4096 tokens, forward and backward; d_out is zero but for a few whole numbers, so that all sums are exact."""
    T, V, D, tail = 2 ** 31 - 4096, 5000, 8, 4096
    torch.cuda.empty_cache()
    need = int(chela.lib().chela_embed_bwd_workspace_bytes(T, V, D)) + T * (2 * D + 4)
    if torch.cuda.mem_get_info()[0] < need + (4 << 30):
        pytest.skip("needs %d GB" % (need >> 30))
    g = gen(18)
    some = token_ids(g, tail, V, 0.01, dtype=torch.int32)
    ids = torch.empty(T, dtype=torch.int32, device="cuda")
    ids.view(-1, tail).copy_(some)
    w = normal(g, V, D, dtype=torch.bfloat16)
    out = chela.embed_fwd(ids, w, scale=0.5)
    rows = chela.embed_fwd(some, w, scale=0.5)
    for part in out.view(-1, tail, D).split(16384):
        assert bool((part == rows).all())
    d_out = out.zero_()
    at = torch.cat([torch.randint(0, T, (3000,), generator=g, device="cuda"), torch.arange(T - 500, T, device="cuda"), torch.arange(500, device="cuda")]).unique()
    values = torch.randint(-3, 4, (len(at), D), generator=g, device="cuda")
    d_out[at] = values.to(torch.bfloat16)
    d_w = chela.embed_bwd(ids, d_out, V)
    kept = ref.kept_of(ids[at], V)
    true = torch.zeros(V, D, dtype=torch.int64, device="cuda").index_add_(0, ids[at][kept].long(), values[kept])
    assert int(true.abs().amax()) > 3 and torch.equal(d_w, true.float())
    del ids, out, part, d_out
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------ cross entropy

def hidden(g, T, V, D, dtype, targets, lean=4.0):
    w = normal(g, V, D, dtype=dtype, std=1.5 * D ** -0.5)
    kept = ref.kept_of(targets, V)
    toward = w[torch.where(kept, targets.long(), 0)].float() * (lean * torch.rand(T, 1, generator=g, device="cuda"))
    return (normal(g, T, D) + toward).to(dtype), w


LOSSES = [
    # a few tokens: their own kernels, by 4, 8 and 16, up to 1024, 2048 and 4096 channels
    (3, 5, 8, "bf16", "f32", 0.3), (4, 3000, 1024, "f32", "f32", 0), (4, 700, 2056, "bf16", "bf16", 0), (4, 50, 4096, "bf16", "f32", 0.5), (8, 9999, 264, "bf16", "bf16", 0),
    (8, 4001, 2048, "bf16", "bf16", 0.2), (7, 333, 1032, "f32", "bf16", 0), (16, 2500, 344, "f32", "f32", 0.1), (16, 1, 16, "f32", "f32", 0), (9, 130, 1024, "f32", "f32", 0),
    (1, 40000, 72, "bf16", "bf16", 0), (5, 600, 520, "f32", "f32", 1.0), (8, 20, 4104, "bf16", "f32", 0), (16, 700, 2048, "f32", "f32", 0), (16, 700, 256, "bf16", "bf16", 0), (13, 519, 232, "bf16", "bf16", 0.1), (16, 8200, 512, "bf16", "bf16", 0),
    (4, 2001, 544, "bf16", "bf16", 0.1), (8, 900, 776, "f32", "f32", 0), (16, 400, 1000, "f32", "bf16", 0), (2, 800, 516 + 4, "bf16", "f32", 0),
    (3, 500, 2000, "f32", "f32", 0), (4, 300, 3000, "bf16", "f32", 0), (7, 640, 1536, "bf16", "f32", 0), (6, 77, 40, "f32", "f32", 0),
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


@pytest.mark.parametrize("gt", ["bf16", "f32"])
@pytest.mark.parametrize("T,V,D,it", [(5, 700, 64, "bf16"), (100, 900, 72, "f32"), (300, 4000, 264, "bf16")])
def test_loss_gradient_on_top_of_another(T, V, D, it, gt):
    g = gen(T * V)
    targets = token_ids(g, T, V, 0.1)
    h, w = hidden(g, T, V, D, DT[it], targets)
    d_lse = normal(g, T, std=1.0 / T)
    d_w_in = normal(g, V, D, dtype=DT[gt], std=0.1)
    r = ref.loss(h, w, targets, 1.3, None, d_lse, d_w_in)   # of lse alone
    _, lse = chela.vocabloss_fwd(h, w, targets, scale=1.3)
    bounds = ref.grad_bounds(r, T, V, D, DT[it], DT[gt])
    other = chela.vocabloss_bwd(h, w, targets, lse, None, d_lse, scale=1.3, grad_dtype=CODE[gt], d_w_in=d_w_in)
    buf = d_w_in.clone()
    same = chela.vocabloss_bwd(h, w, targets, lse, None, d_lse, scale=1.3, grad_dtype=CODE[gt], d_w_in=buf, d_w=buf)
    assert same.d_w is buf and torch.equal(buf, other.d_w) and torch.equal(same.d_h, other.d_h)
    for name, a, b in zip(("d_h", "d_w"), other, bounds):
        within(a, r[name], b, name)


@pytest.mark.parametrize("T,V,D,gt", [(65536, 4500, 64, "bf16"), (40000, 3000, 40, "f32")])
def test_loss_of_several_pieces_of_the_vocabulary(T, V, D, gt):
    """More dz than a piece holds: the pieces' sums of d_h go on top of each other."""
    g = gen(T)
    targets = token_ids(g, T, V, 0.05)
    h, w = hidden(g, T, V, D, torch.bfloat16, targets)
    d_loss = torch.rand(T, generator=g, device="cuda") / T
    r = ref.loss(h, w, targets, 1.0, d_loss)
    loss, lse = chela.vocabloss_fwd(h, w, targets)
    within(loss, r["loss"], ref.lse_bound(r, D, torch.bfloat16) + ref.z_bound(r, D, torch.bfloat16), "loss")
    got = chela.vocabloss_bwd(h, w, targets, lse, d_loss, grad_dtype=CODE[gt])
    for name, a, b in zip(("d_h", "d_w"), got, ref.grad_bounds(r, T, V, D, torch.bfloat16, DT[gt])):
        within(a, r[name], b, name)


@pytest.mark.parametrize("T,V,D,it,gt", [
    (65536, 4500, 64, "bf16", "bf16"), (40000, 3000, 40, "bf16", "f32"),     # d_w in slices, added up by a kernel of their own
    (16384, 20000, 1024, "bf16", "bf16"), (9000, 50001, 264, "bf16", "f32"),  # in whole sums, from the products' epilogues
    (300, 90000, 2048, "f32", "bf16"), (24, 90000, 2048, "f32", "f32")])      # the same, and d_h in slices over the pieces
def test_pieces_of_the_vocabulary_on_top_of_another_gradient(T, V, D, it, gt):
    """Every piece finds its rows of the earlier gradient, in a buffer of its own and in place."""
    g = gen(T + D)
    targets = token_ids(g, T, V, 0.05)
    h, w = hidden(g, T, V, D, DT[it], targets)
    d_loss = torch.rand(T, generator=g, device="cuda") / T
    # of a word's own size: rows that are put on top of another word's show
    d_w_in = (normal(g, V, D) * (1e-3 * (1 + torch.arange(V, device="cuda") % 997))[:, None]).to(DT[gt])
    _, lse = chela.vocabloss_fwd(h, w, targets)
    got = chela.vocabloss_bwd(h, w, targets, lse, d_loss, grad_dtype=CODE[gt], d_w_in=d_w_in)
    held = d_w_in.clone()
    same = chela.vocabloss_bwd(h, w, targets, lse, d_loss, grad_dtype=CODE[gt], d_w_in=held, d_w=held)
    assert same.d_w is held and torch.equal(held, got.d_w) and torch.equal(same.d_h, got.d_h)
    r = ref.loss(h, w, targets, 1.0, d_loss, None, d_w_in)
    for name, a, b in zip(("d_h", "d_w"), got, ref.grad_bounds(r, T, V, D, DT[it], DT[gt])):
        within(a, r[name], b, name)


@pytest.mark.parametrize("T,V,D,it,left_out", [(2047, 3000, 264, "bf16", 0.1), (4097, 40, 512, "bf16", 0), (300, 20001, 136, "bf16", 0), (700, 3000, 1032, "bf16", 0.5),
                                               (48, 9000, 256, "bf16", 0), (7, 3000, 256, "bf16", 0), (500, 3000, 200, "f32", 0)])
def test_bf16_gradients_in_the_norm(T, V, D, it, left_out):
    """Errors against the norms: dz's rounding where it has one plane and more than 64 tokens, and the result's.  A rounding error
    is spread over half a step, 2^-8 / sqrt(3) of the value in the quadratic mean at most; those of dz are independent, so that their
    squares add up, weighted by the other factor's."""
    g = gen(T + V + D)
    targets = token_ids(g, T, V, left_out)
    h, w = hidden(g, T, V, D, DT[it], targets)
    d_loss = torch.rand(T, generator=g, device="cuda") / T
    r = ref.loss(h, w, targets, 1.0, d_loss)
    _, lse = chela.vocabloss_fwd(h, w, targets)
    got = chela.vocabloss_bwd(h, w, targets, lse, d_loss, grad_dtype=chela.BF16)
    kept = ref.kept_of(targets, V)
    hd, wd, y = torch.where(kept[:, None], h.double(), 0.0), w.double(), torch.where(kept, targets, 0)[:, None]
    dz = torch.softmax(hd @ wd.t(), 1)
    dz -= torch.zeros_like(dz).scatter_(1, y, 1.0)
    dz *= torch.where(kept, d_loss.double(), 0.0)[:, None]
    one_plane = it == "bf16" and T > 64
    half = 2.0 ** -8 / 3 ** 0.5
    # what is left: logits and exponentials, 2^-15 of a softmax value or less at these widths; 5 of 100 for the mean of few roundings
    for name, a, terms in (("d_h", got.d_h, dz.square() @ wd.square()), ("d_w", got.d_w, dz.square().t() @ hd.square())):
        far, true = float((a.double() - r[name]).norm()), float(r[name].norm())
        allowed = half * ((float(terms.sum()) if one_plane else 0.0) + true ** 2) ** 0.5 * 1.05 + 2.0 ** -13 * true
        assert far <= allowed, (name, far / true, allowed / true)


def test_fp32_weights_of_several_pieces():
    """The weights' parts are laid out a piece at a time: 90000 x 2048 take more than one, forward and backward."""
    T, V, D = 24, 90000, 2048
    g = gen(3)
    targets = token_ids(g, T, V)
    h, w = hidden(g, T, V, D, torch.float32, targets)
    d_loss = torch.rand(T, generator=g, device="cuda")
    r = ref.loss(h, w, targets, 1.0, d_loss)
    loss, lse = chela.vocabloss_fwd(h, w, targets)
    within(lse, r["lse"], ref.lse_bound(r, D, torch.float32), "lse")
    got = chela.vocabloss_bwd(h, w, targets, lse, d_loss)
    for name, a, b in zip(("d_h", "d_w"), got, ref.grad_bounds(r, T, V, D, torch.float32, torch.float32)):
        within(a, r[name], b, name)


def positive(g, rows, D):
    """bf16 values between 1 and 4, larger towards the last columns, so that rounded sums of a column have mantissas of every kind."""
    out, slope = torch.empty(rows, D, dtype=torch.bfloat16, device="cuda"), 1 + torch.arange(D, device="cuda") / D
    for part in out.split(8192):
        part.copy_((1 + torch.rand(part.shape, generator=g, device="cuda")) * slope)
    return out


def relative_mean(got, true):
    """Mean of the signed relative errors, which rounding to nearest leaves near zero and truncation does not."""
    return float(((got.double() - true) / true).mean())


@pytest.mark.parametrize("D", [1024, 1032, 8192, 65536])
@pytest.mark.parametrize("it", ["bf16", "f32"])
def test_logits_of_many_columns(D, it):
    """Products of one sign, so that the truncated sums lose from all of them: no more for many columns than for 1024."""
    T, V = 40, 300
    g = gen(D)
    h, w = positive(g, T, D).to(DT[it]), positive(g, V, D).to(DT[it])
    y = torch.arange(T, device="cuda")
    loss, lse = chela.vocabloss_fwd(h, w, y, scale=1.0 / 64)
    z = torch.cat([part.double() @ w.double().t() for part in h.split(8)]) / 64
    true = torch.logsumexp(z, 1)
    # 64 steps of 2^-23 (fp32: 16 and, for small terms, next to nothing, and what six products leave out, 3 2^-24), as many fp32
    # sums as there are segments, and some roundings
    steps, sums = (64, D / 1024) if it == "bf16" else (17 + 2, D / 256)
    bound = (steps * 2.0 ** -23 + (sums + 8) * 2.0 ** -24) * z.amax(1) + 2.0 ** -20
    within(lse, true, bound, "lse")
    within(loss, true - z[y, y], 2 * bound, "loss")


def test_gradients_of_many_tokens_lose_nothing_to_truncation():
    """d_w in bf16 over 2^18 tokens, all terms of one sign and every dz a bf16 value: half a step, and the truncations of 16384 terms,
    1024 of at most 2^-23, of the mean."""
    T, V, D = 2 ** 18, 1024, 8192
    g = gen(41)
    h, d_lse = positive(g, T, D), positive(g, T, 1)[:, 0].float()
    w, y = torch.zeros(V, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    _, lse = chela.vocabloss_fwd(h, w, y)
    got = chela.vocabloss_bwd(h, w, y, lse, None, d_lse, grad_dtype=chela.BF16).d_w
    true = sum((a.double() * b.double()[:, None]).sum(0) for a, b in zip(h.split(8192), d_lse.split(8192))) / V
    within(got[1], true, (2.0 ** -8 + 2.0 ** -13) * true, "d_w")
    # beside the truncations: the mean of D roundings, each off by at most 2^-8 (0.42 of that in the quadratic mean)
    assert abs(relative_mean(got[1], true)) <= 2.0 ** -13 + 5 * 0.42 * 2.0 ** -8 / D ** 0.5


def test_gradients_over_many_words_lose_nothing_to_truncation():
    """The same of d_h over 2^16 words."""
    T, V, D = 512, 2 ** 16, 16384
    g = gen(42)
    w, d_lse = positive(g, V, D), positive(g, T, 1)[:, 0].float()
    h, y = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    _, lse = chela.vocabloss_fwd(h, w, y)
    got = chela.vocabloss_bwd(h, w, y, lse, None, d_lse, grad_dtype=chela.BF16).d_h
    true = d_lse.double()[:, None] * (sum(part.double().sum(0) for part in w.split(8192)) / V)
    within(got, true, (2.0 ** -8 + 2.0 ** -13) * true, "d_h")
    assert abs(relative_mean(got, true)) <= 2.0 ** -13 + 5 * 0.42 * 2.0 ** -8 / D ** 0.5


@pytest.mark.parametrize("T", [4, 70, 700])
def test_gradients_against_differences_of_the_definition(T):
    V, D, eps = 150, 48, 1e-5
    g = gen(T + 1)
    targets = token_ids(g, T, V, 0.2)
    h, w = hidden(g, T, V, D, torch.float32, targets)
    a, b = torch.rand(T, generator=g, device="cuda"), normal(g, T, std=0.3)
    _, lse = chela.vocabloss_fwd(h, w, targets, scale=0.9)
    got = chela.vocabloss_bwd(h, w, targets, lse, a, b, scale=0.9)
    bounds = ref.grad_bounds(ref.loss(h, w, targets, 0.9, a, b), T, V, D, torch.float32, torch.float32)

    def value(dh, dw):
        r = ref.loss(h.double() + dh, w.double() + dw, targets, 0.9)
        return float((a * r["loss"] + b * r["lse"]).sum())
    for k in range(3):
        u, v = normal(g, T, D).double(), normal(g, V, D).double()
        slope = (value(eps * u, eps * v) - value(-eps * u, -eps * v)) / (2 * eps)
        mine = float((got.d_h.double() * u).sum() + (got.d_w.double() * v).sum())
        allowed = float((bounds[0] * u.abs()).sum() + (bounds[1] * v.abs()).sum())
        # the quotient: third derivatives (eps^2 of at most the cube of the directions' logits) and 2^-52 of the values over eps
        assert abs(slope - mine) <= allowed + 1e-4 * (1 + abs(slope)), (k, slope, mine)


def test_slices_batches_and_scalars():
    """Column slices of wider tensors, tokens by batch and position, ids of any shape, one-dimensional and none."""
    g = gen(11)
    B, L, V, D = 3, 50, 333, 72
    wide_h, wide_w = normal(g, B, L, 200, dtype=torch.bfloat16), normal(g, V, 96, dtype=torch.bfloat16, std=0.1)
    h, w = wide_h[:, :, 64:64 + D], wide_w[:, 16:16 + D]
    targets = token_ids(g, B * L, V, 0.1).view(B, L)
    loss, lse = chela.vocabloss_fwd(h, w, targets)
    dense = chela.vocabloss_fwd(h.contiguous().view(-1, D), w.contiguous(), targets.view(-1))
    assert loss.shape == (B, L) and torch.equal(loss.view(-1), dense[0]) and torch.equal(lse.view(-1), dense[1])
    d_loss = torch.rand(B, L, generator=g, device="cuda")
    got = chela.vocabloss_bwd(h, w, targets, lse, d_loss)
    flat = chela.vocabloss_bwd(h.contiguous().view(-1, D), w.contiguous(), targets.view(-1), lse.view(-1), d_loss.view(-1))
    assert got.d_h.shape == (B, L, D) and torch.equal(got.d_h.view(-1, D), flat.d_h) and torch.equal(got.d_w, flat.d_w)
    rows = chela.embed_fwd(targets, w, scale=2.0)
    assert rows.shape == (B, L, D) and torch.equal(rows, chela.embed_fwd(targets.view(2, 3, 25), w.contiguous(), scale=2.0).view(B, L, D))
    d_w = chela.embed_bwd(targets, h, V)
    assert torch.equal(d_w, chela.embed_bwd(targets.view(-1), h.contiguous().view(-1, D), V))
    one = torch.tensor(7, device="cuda")
    assert torch.equal(chela.embed_fwd(one, w), w[7]) and chela.vocabloss_fwd(h[0, 0].contiguous(), w, one)[0].shape == ()
    few = chela.vocabloss_fwd(h[0, :5], w, targets[0, :5].contiguous())     # the path for a few tokens, with strides
    assert torch.allclose(few[0], loss[0, :5], atol=1e-4)


def test_tables_beyond_32_bits_of_elements():
    V, D, T = 2200000, 1032, 40
    g = gen(5)
    w = torch.empty(V, D, dtype=torch.bfloat16, device="cuda")
    for part in w.split(100000):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * 0.03)
    ids = torch.cat([torch.tensor([V - 1, 0, V, -1, V - 2], device="cuda"), torch.randint(V // 2, V, (T - 5,), generator=g, device="cuda")])
    out = chela.embed_fwd(ids, w)
    assert torch.equal(out, torch.where(ref.kept_of(ids, V)[:, None], w[ids.clamp(0, V - 1)], 0))
    for count in (3, T):
        h, y = out[:count] + 0.5 * normal(g, count, D, dtype=torch.bfloat16), ids[:count]
        loss, lse = chela.vocabloss_fwd(h, w, y)
        z = torch.cat([torch.mm(h.double(), part.double().t()) for part in w.split(100000)], 1)
        kept = ref.kept_of(y, V)
        true = torch.where(kept, torch.logsumexp(z, 1), 0.0)
        m_z = torch.cat([torch.mm(h.double().abs(), part.double().abs().t()).amax(1, keepdim=True) for part in w.split(100000)], 1).amax(1)
        within(lse, true, ref.lse_bound({"m_z": m_z, "lse": true}, D, torch.bfloat16), "lse")
        d_loss = torch.ones(count, device="cuda")
        got = chela.vocabloss_bwd(h, w, y, lse, d_loss, grad_dtype=chela.BF16)
        dz = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
        dz[torch.arange(count, device="cuda"), y.clamp(0, V - 1)] -= 1
        dz = torch.where(kept[:, None], dz, 0.0)
        rows = torch.cat([torch.arange(50, device="cuda"), torch.arange(V - 50, V, device="cuda"), ids[:count].clamp(0, V - 1)])
        true_w = dz[:, rows].t() @ torch.where(kept[:, None], h.double(), 0.0)
        mag = dz[:, rows].abs().t() @ torch.where(kept[:, None], h.double(), 0.0).abs()
        rel = float((2 * ref.z_bound({"m_z": m_z}, D, torch.bfloat16)).amax()) + 2.0 ** -19
        within(got.d_w[rows], true_w, (rel + 2 * 2.0 ** -8) * mag + 2.0 ** -8 * true_w.abs() + 1e-37, "d_w")
        del got, z, dz
    d_w = chela.embed_bwd(ids, out, V, grad_dtype=chela.BF16)
    within(d_w[V - 3:], ref.embed_bwd(torch.where(ids >= V - 3, ids - (V - 3), -1), out, 3, 1.0), 2.0 ** -7 * out.double().abs().amax() * T, "d_w")
    assert float(d_w[:100].float().abs().sum()) == float(out[ids.eq(0)].float().abs().sum())


def test_loss_of_as_many_tokens_as_there_may_be():
    """2^31 - 4096 tokens, all but a few of them kept: 4096 tokens and their losses over and over."""
    T, V, D, tail = 2 ** 31 - 4096, 24, 8, 4096
    torch.cuda.empty_cache()
    need = int(chela.lib().chela_vocabloss_workspace_bytes(T, V, D, chela.BF16)) + T * (2 * D + 4 + 8)
    if torch.cuda.mem_get_info()[0] < need + (4 << 30):
        pytest.skip("needs %d GB" % (need >> 30))
    g = gen(17)
    y = token_ids(g, tail, V, skew=False, dtype=torch.int32)
    some, w = hidden(g, tail, V, D, torch.bfloat16, y)
    true = chela.vocabloss_fwd(some, w, y)
    h, targets = torch.empty(T, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, dtype=torch.int32, device="cuda")
    h.view(-1, tail, D).copy_(some)
    targets.view(-1, tail).copy_(y)
    out = torch.tensor([5, T // 2, T - 2, T - 1], device="cuda")
    targets[out] = -1
    got = chela.vocabloss_fwd(h, w, targets)
    for a, b in zip(got, true):
        assert (a[out] == 0).all()
        for i in out.tolist():
            a[i] = b[i % tail]
        for part in a.view(-1, tail).split(65536):
            assert bool((part == b).all())
    del h, targets, got, a, part
    torch.cuda.empty_cache()


@pytest.mark.parametrize("T", [6, 300])
def test_what_is_not_finite_stays_with_its_token(T):
    V, D = 500, 64
    g = gen(T)
    targets = token_ids(g, T, V)
    h, w = hidden(g, T, V, D, torch.bfloat16, targets)
    clean = chela.vocabloss_fwd(h, w, targets)
    h[1, 3], h[2, 5] = float("nan"), float("inf")
    loss, lse = chela.vocabloss_fwd(h, w, targets)
    bad = torch.zeros(T, dtype=torch.bool, device="cuda")
    bad[1:3] = True
    assert not torch.isfinite(loss[bad]).any() and not torch.isfinite(lse[bad]).any()
    assert torch.equal(loss[~bad], clean[0][~bad]) and torch.equal(lse[~bad], clean[1][~bad])
    got = chela.vocabloss_bwd(h, w, targets, lse, torch.ones(T, device="cuda"))
    assert torch.isfinite(got.d_h[~bad]).all() and torch.isnan(got.d_h[1]).all() and torch.isnan(got.d_w).any(0).all()
    # left out, they reach nothing
    targets[1], targets[2] = -1, V
    got = chela.vocabloss_bwd(h, w, targets, clean[1], torch.full((T,), 1.0, device="cuda"))
    assert torch.isfinite(got.d_h).all() and torch.isfinite(got.d_w).all() and (got.d_h[bad] == 0).all()
    d_w = chela.embed_bwd(targets, h, V)
    assert torch.isfinite(d_w).all()


@pytest.mark.parametrize("it", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 7, 13, 21, 300])
def test_tokens_left_out_take_nothing_from_weights_that_are_not_finite(T, it):
    V, D = 500, 64
    g = gen(T + 40)
    targets = token_ids(g, T, V)
    h, w = hidden(g, T, V, D, DT[it], targets)
    w[3], w[77, 5], w[V - 1, 9] = float("nan"), float("inf"), float("-inf")
    targets[::3] = -1
    left = ~ref.kept_of(targets, V)
    d_w_in = normal(g, V, D)
    for y in (targets, torch.full_like(targets, V)):   # some, and all of them
        loss, lse = chela.vocabloss_fwd(h, w, y)
        got = chela.vocabloss_bwd(h, w, y, lse, torch.ones(T, device="cuda"), d_w_in=d_w_in)
        assert (loss[left] == 0).all() and (lse[left] == 0).all() and (got.d_h[left] == 0).all()
        if y is not targets:
            assert (got.d_h == 0).all() and torch.equal(got.d_w, d_w_in)


@pytest.mark.parametrize("T,it", [(5, "bf16"), (5, "f32"), (11, "f32"), (21, "bf16"), (70, "bf16"), (300, "bf16")])
def test_a_word_that_its_weights_rule_out(T, it):
    """A logit of minus infinity for every token: the word has no probability, and its gradient is zero."""
    V, D, out = 400, 64, 123
    g = gen(T + 50)
    targets = token_ids(g, T, V)
    targets[targets == out] = 0
    h, w = hidden(g, T, V, D, DT[it], targets)
    h = h.abs()
    w[out] = float("-inf")
    _, lse = chela.vocabloss_fwd(h, w, targets)
    some = torch.arange(V, device="cuda") != out
    r = ref.loss(h, w[some], targets - (targets > out).to(targets.dtype), 1.0, torch.ones(T, device="cuda"))
    within(lse, r["lse"], ref.lse_bound(r, D, DT[it]), "lse")
    d_w = chela.vocabloss_bwd(h, w, targets, lse, torch.ones(T, device="cuda")).d_w
    assert (d_w[out] == 0).all()
    within(d_w[some], r["d_w"], ref.grad_bounds(r, T, V, D, DT[it], torch.float32)[1], "d_w")


def test_large_logits_and_a_certain_target():
    """Logits of hundreds, and tokens whose target has all the weight: the loss keeps its digits near zero."""
    T, V, D = 200, 1000, 64
    g = gen(2)
    targets = token_ids(g, T, V, skew=False)
    w = normal(g, V, D, std=3.0)
    h = w[targets] * torch.linspace(0.02, 3.0, T, device="cuda")[:, None]
    r = ref.loss(h, w, targets, 1.0)
    loss, lse = chela.vocabloss_fwd(h, w, targets)
    within(lse, r["lse"], ref.lse_bound(r, D, torch.float32), "lse")
    within(loss, r["loss"], ref.lse_bound(r, D, torch.float32) + ref.z_bound(r, D, torch.float32), "loss")
    # a certain target's loss is the logarithm of an approximate exponential of next to nothing, off by at most 2^-22, its
    # rounding and that of the maximum's difference to the target, which is itself
    certain = r["loss"] < 1e-9
    assert int(certain.sum()) > T // 2 and float(loss[certain].abs().amax()) <= 2.0 ** -21


# ------------------------------------------------------------------------------------------------ streams, graphs, threads

def calls(ids, h, w, d_loss, grads=chela.BF16):
    V = w.shape[0]
    loss, lse = chela.vocabloss_fwd(h, w, ids)
    g = chela.vocabloss_bwd(h, w, ids, lse, d_loss, grad_dtype=grads)
    x = chela.embed_fwd(ids, w, scale=0.5)
    d_w = chela.embed_bwd(ids, g.d_h, V, grad_dtype=grads, d_w_in=g.d_w)
    return loss, lse, g.d_h, g.d_w, x, d_w


@pytest.mark.parametrize("T", [3, 40, 900])
def test_graph_replay_and_side_streams_give_equal_bits(T):
    V, D = 2500, 136
    g = gen(T)
    sets = []
    for _ in range(2):
        ids = token_ids(g, T, V, 0.2)
        h, w = hidden(g, T, V, D, torch.bfloat16, ids)
        sets.append((ids, h, w, torch.rand(T, generator=g, device="cuda")))
    eager = [calls(*s) for s in sets]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for s, e in zip(sets, eager):
            for a, b in zip(calls(*s), e):
                assert torch.equal(a, b)
    torch.cuda.current_stream().wait_stream(side)
    held = tuple(t.clone() for t in sets[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = calls(*held)
    for s, e in list(zip(sets, eager)) * 2:
        for t, v in zip(held, s):
            t.copy_(v)
        graph.replay()
        for a, b in zip(out, e):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    """Calls of different sizes side by side on two streams, each as if it were alone."""
    g = gen(9)
    sizes = [(700, 5000, 256), (30, 9000, 512)]
    data, alone = [], []
    for T, V, D in sizes:
        ids = token_ids(g, T, V)
        h, w = hidden(g, T, V, D, torch.bfloat16, ids)
        data.append((ids, h, w, torch.rand(T, generator=g, device="cuda")))
        alone.append(calls(*data[-1]))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sizes]
    got = [[], []]
    for _ in range(8):
        for k, st in enumerate(streams):
            with torch.cuda.stream(st):
                got[k].append(calls(*data[k]))
    torch.cuda.synchronize()
    for k in range(2):
        for out in got[k]:
            assert all(torch.equal(a, b) for a, b in zip(out, alone[k]))


def test_threads_on_one_stream():
    import threading
    g = gen(13)
    data, alone = [], []
    for T, V, D in [(300, 3000, 128), (5, 700, 64), (4000, 200, 72), (64, 20000, 256)]:
        ids = token_ids(g, T, V)
        h, w = hidden(g, T, V, D, torch.bfloat16, ids)
        data.append((ids, h, w, torch.rand(T, generator=g, device="cuda")))
        alone.append(calls(*data[-1]))
    torch.cuda.synchronize()
    right = []

    def work(k):
        for _ in range(30):
            out = calls(*data[k])
            torch.cuda.current_stream().synchronize()
            if all(torch.equal(a, b) for a, b in zip(out, alone[k])):
                right.append(k)
    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(data))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert sorted(right) == sorted(list(range(len(data))) * 30)   # no call refused, none wrong


@pytest.mark.parametrize("dt", ["bf16", "f32"])
def test_threads_with_rows_of_different_widths(dt):
    """The kernels of a few tokens take shared memory by the width of the rows: threads with narrow and wide ones at once."""
    import threading
    g = gen(19)
    data, alone = [], []
    for D in (64, 512, 1024, 8, 960, 128):
        ids = token_ids(g, 4, 3000)
        h, w = hidden(g, 4, 3000, D, DT[dt], ids)
        data.append((ids, h, w, torch.rand(4, generator=g, device="cuda")))
        alone.append(calls(*data[-1]))
    torch.cuda.synchronize()
    right, refused = [], []

    def work(k):
        for _ in range(300):
            try:
                out = calls(*data[k])
            except chela.ChelaError as e:
                refused.append((k, e))
                return
            if all(torch.equal(a, b) for a, b in zip(out, alone[k])):
                right.append(k)
    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(data))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not refused and sorted(right) == sorted(list(range(len(data))) * 300)


def test_a_wait_that_runs_out_is_reported_and_the_next_call_is_clean():
    g = gen(21)
    T, V, D = 600, 60000, 64   # enough units that the first CTA comes back to the buffer whose hand-back was left out
    ids = token_ids(g, T, V)
    h, w = hidden(g, T, V, D, torch.bfloat16, ids)
    clean = chela.vocabloss_fwd(h, w, ids)
    ws = torch.zeros(int(chela.lib().chela_vocabloss_workspace_bytes(T, V, D, chela.BF16)), dtype=torch.uint8, device="cuda")
    try:
        chela.debug_wait_control(6_000_000, 1)
        chela.vocabloss_fwd(h, w, ids, workspace=ws)
        assert chela.async_status(ws) == chela.ERR_TIMEOUT
    finally:
        chela.debug_wait_control(0, 0)
    got = chela.vocabloss_fwd(h, w, ids, workspace=ws)
    assert chela.async_status(ws) == chela.OK
    assert torch.equal(got[0], clean[0]) and torch.equal(got[1], clean[1])


@pytest.mark.parametrize("T,V,D,it,gt", [(4, 30000, 256, "bf16", "bf16"), (14, 30000, 520, "f32", "f32"),   # a few tokens
                                         (600, 60000, 64, "bf16", "bf16"), (600, 60000, 64, "bf16", "f32")])
def test_waits_that_run_out_forward_and_backward(T, V, D, it, gt):
    """CTA 0 leaves out an arrival: the status says so, later launches of the call end too, and the next call is clean."""
    g = gen(23)
    ids = token_ids(g, T, V)
    h, w = hidden(g, T, V, D, DT[it], ids)
    d_loss = torch.rand(T, generator=g, device="cuda")
    _, lse = clean = chela.vocabloss_fwd(h, w, ids)
    grads = chela.vocabloss_bwd(h, w, ids, lse, d_loss, grad_dtype=CODE[gt])
    lib = chela.lib()
    for call, need, want in (
            (lambda ws: chela.vocabloss_fwd(h, w, ids, workspace=ws), lib.chela_vocabloss_workspace_bytes(T, V, D, CODE[it]), clean),
            (lambda ws: chela.vocabloss_bwd(h, w, ids, lse, d_loss, grad_dtype=CODE[gt], workspace=ws),
             lib.chela_vocabloss_bwd_workspace_bytes(T, V, D, CODE[it], CODE[gt]), grads)):
        ws = torch.zeros(int(need), dtype=torch.uint8, device="cuda")
        try:
            chela.debug_wait_control(6_000_000, 1)
            call(ws)
            assert chela.async_status(ws) == chela.ERR_TIMEOUT
        finally:
            chela.debug_wait_control(0, 0)
        got = call(ws)
        assert chela.async_status(ws) == chela.OK
        assert all(torch.equal(a, b) for a, b in zip(got, want))


# ------------------------------------------------------------------------------------------------ together

def test_a_language_model_with_tied_weights_trains_as_its_definition_says():
    """ids -> embedding -> norm -> short convolution -> residual and norm -> loss against the same table, and back: every gradient
    against automatic differentiation of the same formulas in 64 bits.  Two packed sequences, padding behind them."""
    T, pad, V, D, W, scale, eps = 150, 10, 700, 64, 4, 8.0, 1e-6
    g = gen(31)
    ids = token_ids(g, T + pad, V)
    ids[T:] = -100
    off = torch.tensor([0, 90, T], dtype=torch.int32, device="cuda")
    targets = torch.full_like(ids, -100)
    targets[:T - 1] = ids[1:T]
    targets[89] = -100   # the first sequence's last token has nothing to foretell
    table, taps = normal(g, V, D, std=D ** -0.5), normal(g, D, W, std=0.5)
    w_in, w_out = 1 + 0.1 * normal(g, D), 1 + 0.1 * normal(g, D)
    weight = torch.where(ref.kept_of(targets, V), 1.0, 0.0) / float(ref.kept_of(targets, V).sum())

    x = chela.embed_fwd(ids, table, scale=scale)
    _, o = chela.blocknorm_fwd(x, w_pre=w_in, eps=eps)
    y, _ = chela.shortconv_carry_fwd(o, taps, seq_offsets=off)
    res, top = chela.blocknorm_fwd(x, y=y, norm_post=chela.NORM_NONE, w_pre=w_out, eps=eps)
    loss, lse = chela.vocabloss_fwd(top, table, targets)
    gl = chela.vocabloss_bwd(top, table, targets, lse, weight)
    gt = chela.blocknorm_bwd(res, y=y, d_o=gl.d_h, norm_post=chela.NORM_NONE, w_pre=w_out, eps=eps)
    gc = chela.shortconv_bwd(o, taps, gt.d_y, seq_offsets=off)
    gi = chela.blocknorm_bwd(x, d_o=gc.d_x, d_res_out=gt.d_res, w_pre=w_in, eps=eps)
    d_table = chela.embed_bwd(ids, gi.d_res, V, scale=scale, d_w_in=gl.d_w, d_w=gl.d_w)
    assert d_table is gl.d_w

    leaves = [t.double().requires_grad_() for t in (table, taps, w_in, w_out)]
    tab, tap, wi, wo = leaves

    def norm(v, weights):
        return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + eps) * weights
    kept = ref.kept_of(ids, V)
    e = torch.where(kept[:, None], scale * tab[torch.where(kept, ids, 0)], 0.0)
    n = norm(e, wi)
    parts = []
    for a, b in ((0, 90), (90, T)):
        padded = torch.cat([torch.zeros(W - 1, D, dtype=torch.float64, device="cuda"), n[a:b]])
        u = sum(tap[:, j] * padded[W - 1 - j:W - 1 - j + b - a] for j in range(W))
        parts.append(u * torch.sigmoid(u))
    parts.append(torch.zeros(pad, D, dtype=torch.float64, device="cuda"))
    z = norm(e + torch.cat(parts), wo) @ tab.t()
    rows = torch.where(ref.kept_of(targets, V), torch.logsumexp(z, 1) - z.gather(1, targets.clamp(0)[:, None])[:, 0], 0.0)
    total = (rows * weight.double()).sum()
    total.backward()
    assert abs(float((loss * weight).sum()) - total.item()) <= 1e-5 * total.item()
    # fp32 throughout: each of some ten stages adds up at most a few hundred roundings of 2^-24 of its majorant
    for name, got, leaf in zip(("table", "taps", "w_in", "w_out"), (d_table, gc.d_w, gi.d_w_pre, gt.d_w_pre), leaves):
        far = float((got.double() - leaf.grad).norm() / leaf.grad.norm())
        assert far <= 2e-5, (name, far)
