"""CPU checks of the packed-sequence operators: bad arguments are refused before anything is launched, and the plain
forms the GPU tests compare with agree with each other."""
import ctypes

import numpy as np
import pytest

import block_ref as ref
from paper_2406_08128_b200 import build, chela

one, two, three, odd = (ctypes.c_void_p(v) for v in (256, 512, 768, 260))   # never dereferenced: validation fails first
null = None
BIG = 1 << 50


@pytest.fixture(scope="module")
def lib():
    build.build()
    return chela.lib()


def scan_args(**kw):
    r = chela.SelscanArgs()
    base = dict(x=256, dt=256, b=256, c=256, a=256, x_stride=64, dt_stride=64, b_stride=16, c_stride=16, S=1, T=4, D=64, N=16, G=1,
                softplus=1, in_dtype=1)
    for k, v in (base | kw).items():
        setattr(r, k, v)
    return ctypes.byref(r)


def norm_args(**kw):
    r = chela.BlocknormArgs()
    base = dict(res=256, y=512, res_stride=64, y_stride=64, gate_stride=64, T=4, D=64, norm_post=1, norm_pre=1, eps=1e-6, in_dtype=1, res_dtype=0)
    for k, v in (base | kw).items():
        setattr(r, k, v)
    return ctypes.byref(r)


def test_short_convolution_refusals(lib):
    def fwd(x=one, xs=64, w=one, bias=null, y=two, si=null, so=null, off=null, S=2, T=8, D=64, W=4, act=1, dt=1):
        return lib.chela_shortconv_carry_fwd(x, xs, w, bias, y, si, so, off, S, T, D, W, act, dt, null)
    bad = chela.ERR_INVALID_ARG
    assert fwd(x=null) == fwd(w=null) == fwd(y=null) == fwd(y=one) == bad
    assert fwd(x=odd) == fwd(y=odd) == fwd(si=odd) == fwd(so=odd) == fwd(w=odd) == fwd(bias=odd) == bad
    assert fwd(off=ctypes.c_void_p(258)) == bad
    assert fwd(S=0) == fwd(T=0) == fwd(D=0) == fwd(W=0) == fwd(act=2) == fwd(dt=2) == bad
    assert fwd(T=7) == bad                      # no offsets: T must be a multiple of S
    assert fwd(xs=56) == fwd(xs=68) == bad      # shorter than a row, not a multiple of 8
    assert fwd(D=60) == fwd(W=17) == fwd(S=1, T=2 ** 31 - 4000) == chela.ERR_UNSUPPORTED
    assert lib.chela_shortconv_step(one, 64, one, null, two, null, two, 2, 64, 4, 1, 1, null) == bad
    assert lib.chela_shortconv_step(one, 64, one, null, two, one, null, 2, 64, 4, 1, 1, null) == bad

    def bwd(dy=two, dys=64, dx=three, ws=one, n=BIG, gdt=0, W=4):
        return lib.chela_shortconv_bwd(one, 64, one, null, dy, dys, null, null, dx, null, null, null, null, 2, 8, 64, W, 1, 1, gdt, ws, n, null)
    assert bwd(dy=null) == bwd(dx=null) == bwd(dx=one) == bwd(dx=two) == bwd(dys=8) == bwd(gdt=2) == bwd(ws=odd) == bad
    assert bwd(ws=null) == bwd(n=16) == chela.ERR_WORKSPACE
    assert bwd(W=17) == chela.ERR_UNSUPPORTED
    assert lib.chela_shortconv_bwd_workspace_bytes(0, 64, 4) == lib.chela_shortconv_bwd_workspace_bytes(8, 60, 4) == 0


def test_selective_scan_refusals(lib):
    bad, no = chela.ERR_INVALID_ARG, chela.ERR_UNSUPPORTED
    fwd = lambda y=two, so=null, ck=null, odt=0, ws=one, n=BIG, **kw: lib.chela_selscan_fwd(scan_args(**kw), y, so, ck, odt, ws, n, null)  # noqa: E731
    assert lib.chela_selscan_fwd(null, two, null, null, 0, one, BIG, null) == bad
    for k in ("x", "dt", "a", "b", "c"):
        assert fwd(**{k: 0}) == fwd(**{k: 260}) == bad
    assert fwd(z=512, z_stride=8) == fwd(z=260, z_stride=64) == fwd(state_in=260) == fwd(d_skip=260) == fwd(dt_bias=260) == bad
    assert fwd(x_stride=63) == fwd(x_stride=68) == fwd(b_stride=8) == fwd(c_stride=20) == bad
    assert fwd(S=0) == fwd(T=0) == fwd(S=3) == fwd(G=0) == fwd(in_dtype=2) == fwd(odt=2) == fwd(softplus=2) == bad
    assert fwd(y=null) == fwd(y=odd) == fwd(so=odd) == fwd(ck=odd) == bad
    assert fwd(ws=odd) == bad
    assert fwd(T=4096, ws=null) == fwd(T=4096, n=64) == chela.ERR_WORKSPACE   # two chains of 32 channels: split into segments
    assert lib.chela_selscan_workspace_bytes(4096, 1, 64, 16) > 0 == lib.chela_selscan_workspace_bytes(4096, 64, 1024, 16)
    assert fwd(N=24, b_stride=24, c_stride=24) == fwd(D=60, x_stride=64) == no
    assert fwd(G=4, b_stride=64, c_stride=64) == no   # 16 channels a group
    step = lambda y=two, so=two, odt=0, **kw: lib.chela_selscan_step(scan_args(**({"S": 4, "state_in": 256} | kw)), y, so, odt, null)  # noqa: E731
    assert step(S=2) == step(state_in=0) == step(y=null) == step(so=null) == step(seq_offsets=256) == bad

    def bwd(dy=one, dx=two, ddt=two, da=two, db=two, dc=two, dz=null, ws=one, n=BIG, gdt=0, dys=64, **kw):
        return lib.chela_selscan_bwd(scan_args(**kw), dy, dys, null, null, dx, ddt, da, db, dc, null, dz, null, null, gdt, ws, n, null)
    assert bwd(dy=null) == bwd(dx=null) == bwd(ddt=null) == bwd(da=null) == bwd(db=null) == bwd(dc=null) == bwd(gdt=2) == bwd(dys=12) == bad
    assert bwd(dz=two) == bwd(z=512, z_stride=64) == bwd(ws=odd) == bwd(dx=odd) == bad
    assert bwd(ws=null) == bwd(n=64) == chela.ERR_WORKSPACE
    assert lib.chela_selscan_bwd_workspace_bytes(4, 1, 64, 24, 0) == lib.chela_selscan_checkpoint_bytes(0, 1, 64, 16) == 0
    assert lib.chela_selscan_bwd_workspace_bytes(4, 1, 64, 16, 1) < lib.chela_selscan_bwd_workspace_bytes(4, 1, 64, 16, 0)


def test_block_norm_refusals(lib):
    bad, no = chela.ERR_INVALID_ARG, chela.ERR_UNSUPPORTED
    fwd = lambda ro=three, o=ctypes.c_void_p(1024), odt=0, **kw: lib.chela_blocknorm_fwd(norm_args(**kw), ro, o, odt, null)  # noqa: E731
    assert lib.chela_blocknorm_fwd(null, one, one, 0, null) == bad
    assert fwd(res=0, y=0) == fwd(y=0, gate=256) == fwd(y=0) == bad     # the last: res_out without y
    assert fwd(ro=null, o=null) == fwd(ro=two) == fwd(o=one) == fwd(o=two) == fwd(ro=odd) == fwd(o=odd) == bad
    assert fwd(ro=one, res_stride=128) == bad                            # in place needs equal strides
    assert fwd(T=0) == fwd(D=0) == fwd(norm_post=3) == fwd(norm_pre=-1) == fwd(gate_act=3) == fwd(gate_after=2) == fwd(odt=2) == bad
    assert fwd(eps=-1.0) == fwd(eps=float("nan")) == fwd(in_dtype=2) == fwd(res_dtype=2) == bad
    assert fwd(res=260) == fwd(y=260) == fwd(gate=260) == fwd(w_pre=260) == fwd(scale=260) == bad
    assert fwd(res_stride=56) == fwd(y_stride=60) == fwd(gate=256, gate_stride=63) == bad
    assert fwd(D=60) == fwd(D=8200, res_stride=8200, y_stride=8200) == no

    def bwd(d_o=one, d_r=one, d_res=three, dy=three, dg=null, ws=one, n=BIG, gdt=0, **kw):
        return lib.chela_blocknorm_bwd(norm_args(**kw), d_o, d_r, d_res, dy, dg, null, null, null, null, null, gdt, ws, n, null)
    assert bwd(d_o=null, d_r=null) == bwd(d_res=null) == bwd(dy=null) == bwd(dg=two) == bwd(y=0) == bwd(gdt=2) == bwd(ws=odd) == bad
    assert bwd(res=0) == bad                                             # the pre-norm's gradient needs r'
    assert bwd(ws=null) == bwd(n=16) == chela.ERR_WORKSPACE
    assert lib.chela_blocknorm_bwd_workspace_bytes(4, 60) == 0


def test_outputs_in_operands_and_sizes_past_the_limits_are_refused(lib):
    bad, no, huge = chela.ERR_INVALID_ARG, chela.ERR_UNSUPPORTED, 2 ** 30 + 1
    ptrs = {"x": 4096, "dt": 8192, "b": 12288, "c": 16384, "z": 20480, "z_stride": 64}
    at = ctypes.c_void_p
    for k in ("x", "dt", "b", "c", "z"):
        assert lib.chela_selscan_fwd(scan_args(**ptrs), at(ptrs[k]), null, null, 0, null, 0, null) == bad
        assert lib.chela_selscan_step(scan_args(**ptrs, S=4, state_in=256), at(ptrs[k]), two, 0, null) == bad
    grads = [24576, 28672, 32768, 36864, 40960]   # d_x, d_dt, d_b, d_c, d_z
    dy = 45056

    def bwd(n=16, **kw):
        p = dict(zip(("d_x", "d_dt", "d_b", "d_c", "d_z"), grads)) | kw
        return lib.chela_selscan_bwd(scan_args(**ptrs), at(dy), 64, null, null, at(p["d_x"]), at(p["d_dt"]), one, at(p["d_b"]), at(p["d_c"]),
                                     null, at(p["d_z"]), null, null, 0, one, n, null)
    assert bwd() == chela.ERR_WORKSPACE
    for k in ("d_x", "d_dt", "d_b", "d_c", "d_z"):
        assert bwd(**{k: dy}) == bwd(**{k: ptrs["x"]}) == bwd(**{k: ptrs["c"]}) == bad

    def norm(d_res=three, d_y=at(2048), d_gate=at(2304), d_o=at(2560), d_r=at(2816)):
        return lib.chela_blocknorm_bwd(norm_args(gate=1024), d_o, d_r, d_res, d_y, d_gate, null, null, null, null, null, 0, one, 16, null)
    assert norm() == norm(d_res=at(2816)) == chela.ERR_WORKSPACE   # d_res may be d_res_out
    assert norm(d_res=one) == norm(d_res=at(2560)) == norm(d_y=two) == norm(d_y=at(2816)) == norm(d_gate=at(1024)) == bad

    assert lib.chela_shortconv_carry_fwd(one, 64, one, null, two, null, null, one, huge, 8, 64, 4, 1, 1, null) == no
    assert lib.chela_selscan_fwd(scan_args(S=huge, seq_offsets=256), two, null, null, 0, null, 0, null) == no
    # sizes that pass 32 bits: T / 8 + S checkpoints, of 64 x 64 states and of 32 x 8
    T, S = 2 ** 31 - 4096, 2 ** 30
    assert lib.chela_selscan_checkpoint_bytes(T, S, 64, 64) == (T // 8 + S) * 64 * 64 * 4
    assert lib.chela_selscan_checkpoint_bytes(T, 2 ** 31 - 1, 8, 8) == (T // 8 + 2 ** 31 - 1) * 32 * 8 * 4


def test_the_flag_on_a_switch_leaves_other_values_refused(lib):
    """CHELA_ZERO_REST goes with act and softplus, 0 or 1; nothing else does.  (A null stream of work is never reached: y or the
    workspace is missing.)"""
    bad, flag = chela.ERR_INVALID_ARG, chela.ZERO_REST

    def conv(act):
        return lib.chela_shortconv_bwd(one, 64, one, null, two, 64, null, null, three, null, null, null, null, 2, 8, 64, 4, act, 1, 0, null, 0, null)

    def scan(softplus):
        return lib.chela_selscan_bwd(scan_args(softplus=softplus), one, 64, null, null, two, two, two, two, two, null, null, null, null, 0, null, 0, null)
    for call in (conv, scan):
        assert call(0) == call(1) == call(flag) == call(flag + 1) == chela.ERR_WORKSPACE
        assert call(2) == call(-1) == call(flag + 2) == call(2 * flag) == call(flag + 2 ** 31 - 512) == bad


def at(i):
    """The i-th of some addresses of their own."""
    return ctypes.c_void_p(1 << 20 | i << 12)


CONV = ("x", "w", "bias", "y", "state_in", "state_out", "off")
CONV_BWD = ("x", "w", "bias", "d_y", "state_in", "d_state_out", "off", "d_x", "d_w", "d_bias", "d_state_in")
SCAN_IN = ("x", "dt", "b", "c", "z", "a", "d_skip", "dt_bias", "state_in", "seq_offsets")
SCAN_BWD = ("d_y", "d_state_out", "checkpoints", "d_x", "d_dt", "d_a", "d_b", "d_c", "d_skip_grad", "d_z", "d_dt_bias", "d_state_in")
NORM_IN = ("res", "y", "gate", "w_post", "b_post", "scale", "w_pre", "b_pre")
NORM_BWD = ("d_o", "d_res_out", "d_res", "d_y", "d_gate", "d_w_post", "d_b_post", "d_scale", "d_w_pre", "d_b_pre")


def calls(lib):
    """name: (call on addresses by name, operands, outputs, pairs that the header allows to be one buffer)."""
    def conv(p):
        return lib.chela_shortconv_carry_fwd(p["x"], 64, p["w"], p["bias"], p["y"], p["state_in"], p["state_out"], p["off"], 2, 8, 64, 4, 1, 1, null)

    def conv_step(p):
        return lib.chela_shortconv_step(p["x"], 64, p["w"], p["bias"], p["y"], p["state_in"], p["state_out"], 2, 64, 4, 1, 1, null)

    def conv_bwd(p):
        return lib.chela_shortconv_bwd(p["x"], 64, p["w"], p["bias"], p["d_y"], 64, p["state_in"], p["d_state_out"], p["d_x"], p["d_w"],
                                       p["d_bias"], p["d_state_in"], p["off"], 2, 8, 64, 4, 1, 1, 1, at(60), BIG, null)

    def scan_in(p, **kw):
        return scan_args(**{k: p[k].value for k in SCAN_IN if k in p}, z_stride=64, **kw)

    def scan(p):
        return lib.chela_selscan_fwd(scan_in(p), p["y"], p["state_out"], p["checkpoints"], 1, at(60), BIG, null)

    def scan_step(p):
        return lib.chela_selscan_step(scan_in(p, S=4), p["y"], p["state_out"], 1, null)

    def scan_bwd(p):
        return lib.chela_selscan_bwd(scan_in(p), p["d_y"], 64, *(p[k] for k in SCAN_BWD[1:]), 0, at(60), BIG, null)

    def norm_in(p):
        return norm_args(**{k: p[k].value for k in NORM_IN})

    def norm(p):
        return lib.chela_blocknorm_fwd(norm_in(p), p["res_out"], p["o"], 1, null)

    def norm_bwd(p):
        return lib.chela_blocknorm_bwd(norm_in(p), *(p[k] for k in NORM_BWD), 0, at(60), BIG, null)

    state = {("state_out", "state_in")}
    steps = tuple(k for k in SCAN_IN if k != "seq_offsets")
    return {"conv": (conv, CONV[:3] + ("state_in", "off"), ("y", "state_out"), state),
            "conv_step": (conv_step, CONV[:3] + ("state_in",), ("y", "state_out"), state),
            "conv_bwd": (conv_bwd, CONV_BWD[:7], CONV_BWD[7:], set()),
            "scan": (scan, SCAN_IN, ("y", "state_out", "checkpoints"), state),
            "scan_step": (scan_step, steps, ("y", "state_out"), state),
            "scan_bwd": (scan_bwd, SCAN_IN + SCAN_BWD[:3], SCAN_BWD[3:], set()),
            "norm": (norm, NORM_IN, ("res_out", "o"), {("res_out", "res")}),
            "norm_bwd": (norm_bwd, NORM_IN + NORM_BWD[:2], NORM_BWD[2:], {("d_res", "d_res_out")})}


ENTRY_POINTS = ("conv", "conv_step", "conv_bwd", "scan", "scan_step", "scan_bwd", "norm", "norm_bwd")


@pytest.mark.parametrize("entry", ENTRY_POINTS)
def test_no_output_may_be_an_operand(lib, entry):
    """Every pair of an output and an operand in one buffer is refused, but for those that the header allows."""
    call, operands, outputs, allowed = calls(lib)[entry]
    place = {k: at(i) for i, k in enumerate(operands + outputs)}
    for o in outputs:
        for i in operands:
            if (o, i) not in allowed:
                assert call(place | {o: place[i]}) == chela.ERR_INVALID_ARG, (o, i)


@pytest.mark.parametrize("entry", ENTRY_POINTS)
def test_no_two_outputs_may_be_one_buffer(lib, entry):
    call, operands, outputs, _ = calls(lib)[entry]
    place = {k: at(i) for i, k in enumerate(operands + outputs)}
    for n, o in enumerate(outputs):
        for other in outputs[:n]:
            assert call(place | {o: place[other]}) == chela.ERR_INVALID_ARG, (o, other)


def test_the_binding_refuses_what_does_not_fit(lib):
    import torch
    x = torch.zeros(4, 64)
    for call in (lambda: chela.shortconv_carry_fwd(x, torch.zeros(64, 4)),
                 lambda: chela.selscan_fwd(x, x, torch.zeros(64, 16), torch.zeros(4, 1, 16), torch.zeros(4, 1, 16)),
                 lambda: chela.blocknorm_fwd(x)):
        with pytest.raises(chela.ChelaError, match="no CPU fallback") as e:
            call()
        assert e.value.status == chela.ERR_INVALID_ARG
    many = torch.zeros(1).expand(2 ** 32 + 64, 8)   # 64 tokens if cut to 32 bits
    for call in (lambda: chela.blocknorm_fwd(many), lambda: chela.shortconv_carry_fwd(many.expand(2, -1, -1), torch.zeros(8, 4))):
        with pytest.raises(chela.ChelaError, match="tokens, at most"):
            call()
    where, d, f = "here", -1, torch.float32
    rows = lambda t, lead, inner: chela._rows(t, where, "t", lead, f, d, inner)[1]  # noqa: E731
    assert rows(torch.zeros(4, 128)[:, 64:], (4,), (64,)) == 128
    assert rows(torch.zeros(2, 4, 128)[..., :64], (2, 4), (64,)) == 128
    assert rows(torch.zeros(2, 1, 64)[:, :, :], (2, 1), (64,)) == 64
    assert rows(torch.zeros(1, 64), (1,), (64,)) == 64
    assert rows(torch.zeros(4, 80).as_strided((4, 2, 16), (80, 16, 1)), (4,), (2, 16)) == 80
    for t, lead, inner in ((torch.zeros(64, 4).t(), (4,), (64,)), (torch.zeros(2, 5, 64)[:, :4], (2, 4), (64,)),
                           (torch.zeros(4, 2, 32)[..., :16], (4,), (2, 16)), (torch.zeros(4, 64).double(), (4,), (64,)),
                           (torch.zeros(4, 32), (4,), (64,))):
        with pytest.raises(chela.ChelaError):
            rows(t, lead, inner)
    with pytest.raises(chela.ChelaError):
        chela._flat(torch.zeros(4, 8)[:, :4], where, "t", (4, 4), f, d)


def test_a_workspace_lives_until_the_call_has_returned(lib, monkeypatch):
    """The library's function runs without the interpreter's lock, so the binding holds what it allocated for it."""
    import weakref
    import torch

    class OnDevice(torch.Tensor):   # the checks of a CPU tensor's placement pass; nothing is launched
        is_cuda = property(lambda self: True)

    made, calls = [], []
    empty = torch.empty

    def tracked(*args, **kw):
        t = empty(*args, **kw)
        if kw.get("dtype") is torch.uint8:
            made.append((weakref.ref(t), t.data_ptr()))
        return t

    def run(fn, where, index, *args):
        (alive, address), = made
        assert alive() is not None and address in args, where
        calls.append(where)

    monkeypatch.setattr(torch, "empty", tracked)
    monkeypatch.setattr(chela, "_run", run)
    T, D, N = 4096, 64, 16   # split: the forward scan has a workspace too
    x = torch.zeros(T, D).as_subclass(OnDevice)
    a, bc, w = torch.zeros(D, N), torch.zeros(T, 1, N), torch.zeros(D, 4)
    for call in (lambda: chela.shortconv_bwd(x, w, x), lambda: chela.selscan_fwd(x, x, a, bc, bc), lambda: chela.selscan_bwd(x, x, a, bc, bc, x),
                 lambda: chela.blocknorm_bwd(x, x, d_o=x)):
        made.clear()
        call()
    assert calls == ["chela_shortconv_bwd", "chela_selscan_fwd", "chela_selscan_bwd", "chela_blocknorm_bwd"]


def test_a_step_without_a_state_is_refused_like_any_bad_argument(lib, monkeypatch):
    import torch

    class OnDevice(torch.Tensor):
        is_cuda = property(lambda self: True)

    monkeypatch.setattr(chela, "_run", lambda fn, where, index, *args: chela._check(fn(*args, None), where))
    x = torch.zeros(4, 64).as_subclass(OnDevice)
    for call in (lambda: chela.selscan_step(x, x, torch.zeros(64, 16), torch.zeros(4, 1, 16), torch.zeros(4, 1, 16), None),
                 lambda: chela.shortconv_step(x, torch.zeros(64, 4), None)):
        with pytest.raises(chela.ChelaError) as e:
            call()
        assert e.value.status == chela.ERR_INVALID_ARG


def test_sizes_that_ctypes_would_cut_are_refused(lib, monkeypatch):
    """Channels, sequences, groups and taps past 31 bits: 2^32 + 64 channels would be taken for 64."""
    import torch

    class OnDevice(torch.Tensor):
        is_cuda = property(lambda self: True)

    monkeypatch.setattr(chela, "_run", lambda *a: pytest.fail("the library was called"))
    huge = 2 ** 32 + 64
    on = lambda t: t.as_subclass(OnDevice)  # noqa: E731
    x = on(torch.zeros(4, 64))
    wide = on(torch.zeros(1).expand(4, huge))
    a, bc = torch.zeros(64, 8), torch.zeros(4, 1, 8)
    for call in (lambda: chela.blocknorm_fwd(wide),
                 lambda: chela.shortconv_carry_fwd(wide, torch.zeros(1).expand(huge, 4)),
                 lambda: chela.shortconv_step(x, torch.zeros(1).expand(64, huge), torch.zeros(4, 3, 64)),
                 lambda: chela.shortconv_bwd(x, torch.zeros(64, 0), x),
                 lambda: chela.shortconv_carry_fwd(x, torch.zeros(64)),
                 lambda: chela.shortconv_carry_fwd(x, torch.zeros(64, 4), seq_offsets=torch.zeros(1, dtype=torch.int32).expand(huge)),
                 lambda: chela.selscan_fwd(x, x, a, torch.zeros(1).expand(4, huge, 8), bc)):
        with pytest.raises(chela.ChelaError) as e:
            call()
        assert e.value.status == chela.ERR_INVALID_ARG


def test_plain_forms_agree_with_differences():
    """The float64 gradients of the reference against central differences of its forward forms."""
    rng = np.random.default_rng(0)
    lengths, D, N, G, W = [5, 0, 1, 7], 4, 3, 2, 3
    T = sum(lengths)
    n = rng.standard_normal
    v = {"x": n((T, D)), "dt": n((T, D)), "a": -np.exp(n((D, N))), "b": n((T, G, N)), "c": n((T, G, N)), "d_skip": n(D), "z": n((T, D)),
         "dt_bias": n(D), "state": n((4, D, N))}
    dy, ds = n((T, D)), n((4, D, N))

    def scan_loss(u):
        y, s = ref.scan(u["x"], u["dt"], u["a"], u["b"], u["c"], lengths, u["d_skip"], u["z"], u["dt_bias"], True, u["state"])
        return (y * dy).sum() + (s * ds).sum()

    g = ref.scan_bwd(v["x"], v["dt"], v["a"], v["b"], v["c"], dy, lengths, v["d_skip"], v["z"], v["dt_bias"], True, v["state"], ds)
    names = {"x": "d_x", "dt": "d_dt", "a": "d_a", "b": "d_b", "c": "d_c", "d_skip": "d_skip", "z": "d_z", "dt_bias": "d_dt_bias", "state": "d_state_in"}
    for k, gk in names.items():
        way = n(v[k].shape)
        num = (scan_loss(v | {k: v[k] + 1e-5 * way}) - scan_loss(v | {k: v[k] - 1e-5 * way})) / 2e-5
        assert abs(num - (g[gk] * way).sum()) <= 1e-6 * (1 + abs(num)), k

    c = {"x": n((T, D)), "w": n((D, W)), "bias": n(D), "state": n((4, W - 1, D))}
    dst = n((4, W - 1, D))
    conv_loss = lambda u: (lambda y, s: (y * dy).sum() + (s * dst).sum())(*ref.conv(u["x"], u["w"], u["bias"], lengths, u["state"]))  # noqa: E731
    got = ref.conv_bwd(c["x"], c["w"], c["bias"], dy, lengths, c["state"], dst)
    for k, gk in zip(("x", "w", "bias", "state"), got):
        way = n(c[k].shape)
        num = (conv_loss(c | {k: c[k] + 1e-5 * way}) - conv_loss(c | {k: c[k] - 1e-5 * way})) / 2e-5
        assert abs(num - (gk * way).sum()) <= 1e-6 * (1 + abs(num)), k

    for post, pre, act, after in ((1, 2, 1, False), (2, 1, 2, True), (0, 1, 0, False)):
        w = {"res": n((T, D)), "y": n((T, D)), "gate": n((T, D)), "w_post": n(D), "b_post": n(D), "scale": n(D), "w_pre": n(D), "b_pre": n(D)}
        d_o, d_r = n((T, D)), n((T, D))
        kw = {"norm_post": post, "norm_pre": pre, "gate_act": act, "gate_after": after, "eps": 1e-3}

        def norm_loss(u):
            r, o, _ = ref.junction(**u, **kw)
            return (r * d_r).sum() + (o * d_o).sum()

        r = ref.junction(**w, **kw)[0]
        g = ref.junction_bwd(r, w["y"], w["gate"], d_o, d_r, *(w[k] for k in ("w_post", "b_post")), post, w["scale"], w["w_pre"], w["b_pre"], pre,
                             act, after, 1e-3)
        for k in w:
            way = n(w[k].shape)
            num = (norm_loss(w | {k: w[k] + 1e-5 * way}) - norm_loss(w | {k: w[k] - 1e-5 * way})) / 2e-5
            assert abs(num - (g["d_" + k] * way).sum()) <= 1e-6 * (1 + abs(num)), (k, post, pre)
