"""CPU checks of the token embedding and the vocabulary's cross entropy: bad arguments are refused before anything is launched."""
import ctypes

import pytest
import torch

import vocab_ref as ref
from paper_2406_08128_b200 import build, chela

one, two, three, four, odd = (ctypes.c_void_p(v) for v in (256, 512, 768, 1024, 260))   # never dereferenced
null = None
BIG = 1 << 50
bad, no, small = chela.ERR_INVALID_ARG, chela.ERR_UNSUPPORTED, chela.ERR_WORKSPACE


@pytest.fixture(scope="module")
def lib():
    build.build()
    return chela.lib()


def test_embedding_refusals(lib):
    def fwd(ids=one, wide=1, w=two, ws=64, out=three, T=4, V=10, D=64, wt=1, ot=1):
        return lib.chela_embed_fwd(ids, wide, w, ws, out, T, V, D, 1.0, wt, ot, null)
    assert fwd(ids=null) == fwd(w=null) == fwd(out=null) == fwd(out=two) == fwd(out=one) == bad
    assert fwd(ids=ctypes.c_void_p(260)) == fwd(ids=ctypes.c_void_p(258), wide=0) == fwd(w=odd) == fwd(out=odd) == bad
    assert fwd(wide=2) == fwd(wt=2) == fwd(ot=2) == fwd(T=0) == fwd(V=0) == fwd(D=0) == fwd(T=-1) == bad
    assert fwd(ws=56) == fwd(ws=68) == bad
    assert fwd(D=60) == fwd(T=2 ** 31 - 4000) == fwd(V=2 ** 30 + 1) == fwd(D=2 ** 20 + 8, ws=2 ** 20 + 8) == no

    def bwd(ids=one, wide=0, d=two, ds=64, before=null, dw=three, T=4, V=10, D=64, dt=1, gt=0, ws=four, n=BIG):
        return lib.chela_embed_bwd(ids, wide, d, ds, before, dw, T, V, D, 1.0, dt, gt, ws, n, null)
    assert bwd(ids=null) == bwd(d=null) == bwd(dw=null) == bwd(dw=one) == bwd(dw=two) == bwd(before=odd) == bwd(ws=odd) == bad
    assert bwd(ws=one) == bwd(ws=two) == bwd(ws=three) == bwd(before=four) == bad      # the workspace is nobody else's buffer
    assert bwd(dt=2) == bwd(gt=2) == bwd(ds=60) == bwd(T=0) == bwd(V=-3) == bad
    assert bwd(ws=null) == bwd(n=16) == small
    assert bwd(D=12, ds=16) == no
    q = lib.chela_embed_bwd_workspace_bytes
    assert q(0, 10, 64) == q(4, 0, 64) == q(4, 10, 60) == 0 < q(4, 10, 64) < q(100000, 10, 64)


def loss_args(**kw):
    r = chela.VocablossArgs()
    base = dict(h=256, w=512, targets=768, h_stride=64, w_stride=64, T=20, V=10, D=64, wide_ids=1, scale=1.0, in_dtype=1)
    for k, v in (base | kw).items():
        setattr(r, k, v)
    return ctypes.byref(r)


def test_loss_refusals(lib):
    five, six, seven = (ctypes.c_void_p(v) for v in (1280, 1536, 1792))
    fwd = lambda loss=four, lse=five, ws=six, n=BIG, **kw: lib.chela_vocabloss_fwd(loss_args(**kw), loss, lse, ws, n, null)  # noqa: E731
    bwd = lambda lse=four, dl=five, dlse=null, dh=six, before=null, dw=seven, gt=0, ws=ctypes.c_void_p(2048), n=BIG, **kw: \
        lib.chela_vocabloss_bwd(loss_args(**kw), lse, dl, dlse, dh, before, dw, gt, ws, n, null)  # noqa: E731
    assert lib.chela_vocabloss_fwd(null, four, five, six, BIG, null) == lib.chela_vocabloss_bwd(null, four, five, null, six, null, seven, 0, one, BIG, null) == bad
    for call in (fwd, bwd):
        for k in ("h", "w", "targets"):
            assert call(**{k: 0}) == bad
        assert call(h=260) == call(w=264) == call(targets=772) == bad
        assert call(targets=770, wide_ids=0) == call(wide_ids=2) == call(in_dtype=2) == call(T=0) == call(V=0) == call(D=-8) == bad
        assert call(h_stride=56) == call(w_stride=68) == call(h_stride=2 ** 40) == bad
        for scale in (0.0, -1.0, float("inf"), float("nan")):
            assert call(scale=scale) == bad
        assert call(D=60) == call(T=2 ** 31 - 4000) == call(V=2 ** 30 + 1) == no
        assert call(ws=null) == call(n=64) == small
        assert call(T=2 ** 31 - 4097, V=2 ** 24) == no and call(scale=2e30) == bad
        for T in (3, 20):   # both paths
            assert call(T=T, n=64) == call(T=T, in_dtype=0, n=64) == small
    assert fwd(loss=null) == fwd(lse=null) == fwd(lse=four) == fwd(loss=one) == fwd(lse=two) == fwd(loss=ctypes.c_void_p(1025)) == fwd(ws=odd) == fwd(ws=four) == fwd(ws=one) == bad
    assert bwd(lse=null) == bwd(dl=null) == bwd(dh=null) == bwd(dw=null) == bwd(gt=2) == bwd(dh=odd) == bwd(dw=odd) == bwd(before=odd) == bad
    for out in (one, two, three, four, five):
        assert bwd(dh=out) == bwd(dw=out) == bad
    assert bwd(dh=seven) == bwd(before=six) == bwd(ws=six) == bwd(ws=seven) == bwd(dlse=six) == bad
    qf, qb = lib.chela_vocabloss_workspace_bytes, lib.chela_vocabloss_bwd_workspace_bytes
    assert qf(0, 10, 64, 1) == qf(4, 10, 60, 1) == qf(4, 10, 64, 2) == qb(4, 10, 64, 1, 2) == qb(4, 0, 64, 1, 1) == 0
    assert 0 < qf(20, 10, 64, 1) < qf(20, 10, 64, 0) and 0 < qb(300, 10, 64, 1, 1) < qb(300, 10, 64, 1, 0)
    assert qf(2 ** 31 - 4097, 2 ** 24, 64, 1) == 0 < qf(2 ** 31 - 4097, 2 ** 12, 64, 1)
    # dz of a piece is bounded, however large the vocabulary
    assert qb(16384, 2 ** 20, 1024, 1, 1) < 2 << 30


def test_binding_refuses_before_the_library():
    ids, w, h = torch.zeros(4, dtype=torch.int64), torch.zeros(10, 64), torch.zeros(4, 64)
    for call in (lambda: chela.embed_fwd(ids, w), lambda: chela.embed_bwd(ids, h, 10), lambda: chela.vocabloss_fwd(h, w, ids),
                 lambda: chela.embed_fwd(ids.float(), w), lambda: chela.vocabloss_fwd(h, w, ids[::2])):
        with pytest.raises(chela.ChelaError) as e:
            call()
        assert e.value.status == bad


def test_definitions_agree_with_automatic_differentiation():
    torch.manual_seed(0)
    T, V, D = 12, 9, 8
    h, w = torch.randn(T, D, dtype=torch.float64, requires_grad=True), torch.randn(V, D, dtype=torch.float64, requires_grad=True)
    y = torch.randint(0, V, (T,))
    y[3], y[5] = -1, V
    a, b = torch.rand(T), torch.randn(T)
    r = ref.loss(h.detach(), w.detach(), y, 0.7, a, b)
    kept = ref.kept_of(y, V)
    z = 0.7 * h @ w.t()
    lse = torch.logsumexp(z, 1)
    loss = lse - z.gather(1, torch.where(kept, y, 0)[:, None])[:, 0]
    assert torch.allclose(r["loss"], torch.where(kept, loss, 0.0)) and torch.allclose(r["lse"], torch.where(kept, lse, 0.0))
    torch.where(kept, a * loss + b * lse, 0.0).sum().backward()
    assert torch.allclose(r["d_h"], h.grad) and torch.allclose(r["d_w"], w.grad)
    table = torch.randn(V, D, dtype=torch.float64, requires_grad=True)
    out = torch.where(kept[:, None], 1.5 * table[torch.where(kept, y, 0)], 0.0)
    assert torch.allclose(ref.embed(y, table.detach(), 1.5), out)
    out.backward(h.detach())
    assert torch.allclose(ref.embed_bwd(y, h.detach(), V, 1.5), table.grad)
