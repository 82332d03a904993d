"""GPU parity of the operators over packed sequences (short convolution with carried inputs, selective scan, block norms)
against plain float64 forms.

Tolerances are factors of the sums' majorants (block_ref, ``mag=True``).  A single precision operation is off by at most
2^-24 of its result, the approximate exponential by 2^-22; a recurrence over L tokens multiplies L such decays, each off
by at most 2^-21 (exponential, rounding of the exponent, time step), so states are within (L + 4) 2^-21 of their majorant and
gradients, which chain two recurrences, within twice that.  Sums over T tokens or D channels add at most their count times
2^-24.  bf16 outputs add half a step, 2^-8 of the value.
"""
import numpy as np
import pytest

import block_ref as ref
from paper_2406_08128_b200 import chela, inputs
from util import to_device, to_numpy

pytestmark = pytest.mark.gpu

BF16_HALF = 2.0 ** -8
DT = {"f32": chela.F32, "bf16": chela.BF16}


def f32(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).cuda()


def i32(a):
    import torch
    return torch.from_numpy(np.asarray(a, dtype=np.int32)).cuda()


def dev(a, dtype, extra=0):
    """Device tensor; with ``extra`` a column slice of a wider one, so that its token stride is not its width."""
    import torch
    if a is None:
        return None
    if not extra:
        return to_device(a, dtype)
    flat = a.reshape(a.shape[0], -1)
    wide = np.concatenate([np.full((flat.shape[0], extra), np.nan, np.float32), flat, np.full((flat.shape[0], extra), np.nan, np.float32)], 1)
    t = to_device(np.ascontiguousarray(wide, dtype=np.float32), dtype)[:, extra:extra + flat.shape[1]]
    return t if a.ndim == 2 else t.unflatten(1, a.shape[1:])


def close(got, want, mag, factor, dtype="f32", extra=0.0):
    got = to_numpy(got) if not isinstance(got, np.ndarray) else got
    assert got.shape == want.shape
    tol = factor * mag + (BF16_HALF * np.abs(want) if dtype == "bf16" else 0.0) + extra + 1e-30
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:3], got[bad][:3], want[bad][:3], np.max(np.abs(got - want) / tol))


LENGTHS = [[1], [0, 1, 2, 0], [5, 0, 33, 1, 64], [16, 17, 15], [31, 32, 33], [127, 128, 129, 3], [300]]


# ------------------------------------------------------------------------------------------------ short convolution

def conv_inputs(seed, lengths, D, W, dtype, pad=0):
    rng = np.random.default_rng(seed)
    T = sum(lengths) + pad
    r = lambda *s: inputs.round_storage(rng.standard_normal(s, dtype=np.float32), dtype)  # noqa: E731
    x, dy = r(T, D), r(T, D)
    w = (rng.standard_normal((D, W), dtype=np.float32) / np.sqrt(W)).astype(np.float32)
    bias = rng.standard_normal(D, dtype=np.float32)
    return x, w, bias, r(len(lengths), W - 1, D), dy, r(len(lengths), W - 1, D)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("W,D,act", [(1, 8, True), (2, 40, True), (3, 64, False), (4, 136, True), (7, 24, True), (16, 16, True)])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("carry", [True, False])
def test_conv_forward_backward(dtype, W, D, act, lengths, carry):
    pad = 3
    x, w, bias, state, dy, d_so = conv_inputs(W * 100 + len(lengths), lengths, D, W, dtype, pad)
    n = sum(lengths)
    x[n:] = dy[n:] = np.nan   # no sequence's tokens
    b = bias if D != 24 else None
    st = state if carry else None
    off = i32(ref.offsets(lengths))
    out = dev(np.full((n + pad, D), 7.0, np.float32), dtype)
    extra = 8 if D != 64 else 0
    y, so = chela.shortconv_carry_fwd(dev(x, dtype, extra), f32(w), None if b is None else f32(b), act=act, state_in=dev(st, dtype),
                                      seq_offsets=off, out=out)
    want, want_s = ref.conv(x, w, b, lengths, st, act)
    mag = ref.conv(np.abs(x), np.abs(w), None if b is None else np.abs(b), lengths, None if st is None else np.abs(st), False)[0]
    # W + 1 roundings of the sum, silu with its exponential and reciprocal (slope at most 1.1)
    close(y[:n], want[:n], mag[:n], (W + 8) * 2.0 ** -23, dtype)
    assert np.all(to_numpy(y[n:]) == 7.0)
    assert np.array_equal(to_numpy(so), want_s)

    g = chela.shortconv_bwd(dev(x, dtype, extra), f32(w), dev(dy, dtype, extra), None if b is None else f32(b), act=act,
                            state_in=dev(st, dtype), d_state_out=dev(d_so, dtype) if carry else None, seq_offsets=off,
                            grad_dtype=DT[dtype], want_d_state=True)
    args = (x, w, b, dy, lengths, st, d_so if carry else None, act)
    r, m = ref.conv_bwd(*args), ref.conv_bwd(*args, mag=True)
    sums = (W + 16 + n) * 2.0 ** -23
    close(g.d_x[:n], r[0][:n], m[0][:n], (2 * W + 16) * 2.0 ** -23, dtype)
    close(g.d_w, r[1], m[1], sums)
    close(g.d_bias, r[2], m[2], sums)
    close(g.d_state_in, r[3], m[3], (2 * W + 16) * 2.0 ** -23, dtype)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_conv_steps_continue_a_prompt(dtype):
    """A prompt, then single tokens with the state updated in place, give the longer prompt's rows bit for bit; so does the
    prompt cut into segments whose state is carried in place."""
    import torch
    S, L, D, W = 3, 41, 72, 4
    x, w, bias, *_ = conv_inputs(5, [L] * S, D, W, dtype)
    xd, wd, bd = dev(x, dtype).view(S, L, D), f32(w), f32(bias)
    full, last = chela.shortconv_carry_fwd(xd, wd, bd)
    cut = 30
    y, state = chela.shortconv_carry_fwd(xd[:, :cut].contiguous(), wd, bd)
    assert torch.equal(y, full[:, :cut])
    for t in range(cut, L):
        y = chela.shortconv_step(xd[:, t], wd, state, bd)
        assert torch.equal(y, full[:, t])
    assert torch.equal(state, last)
    state = torch.zeros_like(state)
    at = 0
    for n in (1, 2, 7, 31):
        y, state = chela.shortconv_carry_fwd(xd[:, at:at + n].contiguous(), wd, bd, state_in=state, state_out=state)
        assert torch.equal(y, full[:, at:at + n])
        at += n
    assert torch.equal(state, last)


def test_conv_of_one_tap_ignores_its_states():
    """One buffer given for every state of a width of one, through the C entry points: neither read nor written, nor refused."""
    import torch
    T, D, L = 9, 16, chela.lib()
    x, w, bias, _, dy, _ = conv_inputs(1, [T], D, 1, "f32")
    xd, wd, bd, dyd = f32(x), f32(w), f32(bias), f32(dy)
    y, dx, dw, db, state = (torch.empty(s, device="cuda") for s in ((T, D), (T, D), (D, 1), (D,), (T, D)))
    state.fill_(5.0)
    stream, s = torch.cuda.current_stream().cuda_stream, state.data_ptr()
    need = L.chela_shortconv_bwd_workspace_bytes(T, D, 1)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    assert L.chela_shortconv_carry_fwd(xd.data_ptr(), D, wd.data_ptr(), bd.data_ptr(), y.data_ptr(), s, s, None, 1, T, D, 1, 1, chela.F32,
                                       stream) == chela.OK
    assert L.chela_shortconv_bwd(xd.data_ptr(), D, wd.data_ptr(), bd.data_ptr(), dyd.data_ptr(), D, s, s, dx.data_ptr(), dw.data_ptr(),
                                 db.data_ptr(), s, None, 1, T, D, 1, 1, chela.F32, chela.F32, ws.data_ptr(), need, stream) == chela.OK
    want, g = chela.shortconv_carry_fwd(xd, wd, bd)[0], chela.shortconv_bwd(xd, wd, dyd, bd)
    assert torch.equal(y, want) and torch.equal(dx, g.d_x) and torch.equal(dw, g.d_w) and torch.equal(db, g.d_bias) and (state == 5).all()


@pytest.mark.parametrize("W", [1, 3, 4, 5, 8, 11])
def test_conv_reaches_no_further_than_its_width(W):
    """An infinity or NaN in one token's input or gradient: only the outputs and gradients that the width reaches see it."""
    import torch
    T, D, at = 100, 16, 40
    x, w, bias, _, dy, _ = conv_inputs(W, [T], D, W, "f32")
    wd, bd, off = f32(w), f32(bias), i32([0, T])
    clean, _ = chela.shortconv_carry_fwd(f32(x), wd, bd, seq_offsets=off)
    g = chela.shortconv_bwd(f32(x), wd, f32(dy), bd, seq_offsets=off)
    for value in (np.inf, np.nan):
        u, du = x.copy(), dy.copy()
        u[at] = du[at] = value
        y, _ = chela.shortconv_carry_fwd(f32(u), wd, bd, seq_offsets=off)
        assert torch.equal(y[:at], clean[:at]) and torch.equal(y[at + W:], clean[at + W:])
        gd = chela.shortconv_bwd(f32(x), wd, f32(du), bd, seq_offsets=off)
        assert torch.equal(gd.d_x[:at - W + 1], g.d_x[:at - W + 1]) and torch.equal(gd.d_x[at + 1:], g.d_x[at + 1:])
        gx = chela.shortconv_bwd(f32(u), wd, f32(dy), bd, seq_offsets=off)   # through act' of the outputs at .. at + W - 1
        assert torch.equal(gx.d_x[:at - W + 1], g.d_x[:at - W + 1]) and torch.equal(gx.d_x[at + W:], g.d_x[at + W:])


def test_conv_over_more_work_items_than_warps():
    """The backward pass's warps each walk several work items and its partial sums come from several rows of CTAs; the forward
    pass's threads take a second item (against the sequences one by one: the same bits)."""
    import torch
    for dtype, D, lengths in (("f32", 8, [2000, 1, 0, 1777, 1501]), ("bf16", 1024, [9000, 40, 10977])):
        T = sum(lengths)
        x, w, bias, state, dy, d_so = conv_inputs(D, lengths, D, 4, dtype)
        off = i32(ref.offsets(lengths))
        g = chela.shortconv_bwd(dev(x, dtype), f32(w), dev(dy, dtype), f32(bias), state_in=dev(state, dtype), d_state_out=dev(d_so, dtype),
                                seq_offsets=off, grad_dtype=DT[dtype], want_d_state=True)
        args = (x, w, bias, dy, lengths, state, d_so)
        r, m = ref.conv_bwd(*args), ref.conv_bwd(*args, mag=True)
        sums = (4 + 16 + T) * 2.0 ** -23
        close(g.d_x, r[0], m[0], 24 * 2.0 ** -23, dtype)
        close(g.d_w, r[1], m[1], sums)
        close(g.d_bias, r[2], m[2], sums)
        close(g.d_state_in, r[3], m[3], 24 * 2.0 ** -23, dtype)

    lengths, D = [100003, 0, 99990, 120007], 1024
    assert (sum(lengths) // 32) * (D // 4) > 148 * 64 * 256
    x = torch.randn(sum(lengths), D, device="cuda").bfloat16()
    w, bias = torch.randn(D, 4, device="cuda"), torch.randn(D, device="cuda")
    y, last = chela.shortconv_carry_fwd(x, w, bias, seq_offsets=i32(ref.offsets(lengths)))
    at = 0
    for s, n in enumerate(lengths):
        if n:
            y1, last1 = chela.shortconv_carry_fwd(x[at:at + n], w, bias, seq_offsets=i32([0, n]))
            assert torch.equal(y[at:at + n], y1) and torch.equal(last[s], last1[0])
        at += n


# ------------------------------------------------------------------------------------------------ selective scan

def scan_inputs(seed, lengths, D, N, G, dtype, pad=0):
    rng = np.random.default_rng(seed)
    T, S = sum(lengths) + pad, len(lengths)
    r = lambda *s: inputs.round_storage(rng.standard_normal(s, dtype=np.float32), dtype)  # noqa: E731
    v = {"x": r(T, D), "dt": r(T, D), "b": r(T, G, N), "c": r(T, G, N), "z": r(T, D)}
    v["a"] = (-np.arange(1, N + 1, dtype=np.float32) * np.exp(0.3 * rng.standard_normal((D, N), dtype=np.float32))).astype(np.float32)
    v["d_skip"] = rng.standard_normal(D, dtype=np.float32)
    v["dt_bias"] = (-3.0 + rng.standard_normal(D, dtype=np.float32)).astype(np.float32)
    v["state"] = rng.standard_normal((S, D, N), dtype=np.float32)
    v["d_y"] = r(T, D)
    v["d_state_out"] = rng.standard_normal((S, D, N), dtype=np.float32)
    return v


def scan_call(v, lengths, dtype, form, extra=0, **more):
    z, skip, bias, carry, soft = form
    args = [dev(v["x"], dtype, extra), dev(v["dt"], dtype, extra), f32(v["a"]), dev(v["b"], dtype, extra), dev(v["c"], dtype, extra)]
    kw = {"d_skip": f32(v["d_skip"]) if skip else None, "z": dev(v["z"], dtype, extra) if z else None,
          "dt_bias": f32(v["dt_bias"]) if bias else None, "softplus": soft, "state_in": f32(v["state"]) if carry else None,
          "seq_offsets": i32(ref.offsets(lengths))}
    return args, kw | more


def scan_ref(v, lengths, form, mag=False, bwd=False):
    z, skip, bias, carry, soft = form
    kw = {"d_skip": v["d_skip"] if skip else None, "z": v["z"] if z else None, "dt_bias": v["dt_bias"] if bias else None,
          "soft": soft, "state": v["state"] if carry else None, "mag": mag}
    if bwd:
        return ref.scan_bwd(v["x"], v["dt"], v["a"], v["b"], v["c"], v["d_y"], lengths,
                            d_state_out=v["d_state_out"] if carry else None, **kw)
    return ref.scan(v["x"], v["dt"], v["a"], v["b"], v["c"], lengths, **kw)


FORMS = [(True, True, True, True, True), (False, False, False, False, True), (True, False, True, True, False)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D,G", [(8, 24, 1), (16, 40, 1), (16, 128, 2), (32, 72, 1), (64, 64, 2), (64, 8, 1)])
@pytest.mark.parametrize("lengths", LENGTHS, ids=str)
@pytest.mark.parametrize("form", FORMS, ids=["all", "bare", "rawdt"])
def test_scan_forward_backward(dtype, N, D, G, lengths, form):
    import torch
    pad = 2
    v = scan_inputs(N + D + len(lengths), lengths, D, N, G, dtype, pad)
    if not form[4]:   # time steps as they are
        v["dt"] = inputs.round_storage(np.abs(v["dt"]) * np.float32(0.1), dtype)
        v["dt_bias"] = np.abs(v["dt_bias"]) * np.float32(0.01)
    n = sum(lengths)
    for k in ("x", "dt", "b", "c", "z", "d_y"):
        v[k][n:] = np.nan
    extra = 8 if D != 40 else 0
    out = dev(np.full((n + pad, D), 7.0, np.float32), dtype)
    args, kw = scan_call(v, lengths, dtype, form, extra)
    ckpt = chela.selscan_checkpoints(n + pad, len(lengths), D, N, "cuda")
    y, last = chela.selscan_fwd(*args, **kw, out=out, checkpoints=ckpt)
    want, want_s = scan_ref(v, lengths, form)
    mag, mag_s = scan_ref(v, lengths, form, mag=True)
    L = max(lengths)
    tol = (L + 8) * 2.0 ** -21
    close(y[:n], want[:n], mag[:n], tol, dtype)
    close(last, want_s, mag_s, tol)
    assert np.all(to_numpy(y[n:]) == 7.0)

    d_so = f32(v["d_state_out"]) if form[3] else None
    bw = lambda c: chela.selscan_bwd(*args, dev(v["d_y"], dtype, extra), **kw, checkpoints=c, d_state_out=d_so, grad_dtype=DT[dtype],  # noqa: E731
                                     want_d_state=True)
    g = bw(ckpt)
    r, m = scan_ref(v, lengths, form, bwd=True), scan_ref(v, lengths, form, mag=True, bwd=True)
    tol = 2 * (L + 8) * 2.0 ** -21
    for k, more, dt in (("d_x", 0, dtype), ("d_dt", 0, dtype), ("d_z", 0, dtype), ("d_b", D // G, dtype), ("d_c", D // G, dtype),
                        ("d_a", n, "f32"), ("d_skip", n, "f32"), ("d_dt_bias", n, "f32"), ("d_state_in", 0, "f32")):
        got = getattr(g, k)
        if got is None:
            assert (k == "d_z" and not form[0]) or (k == "d_skip" and not form[1]) or (k == "d_dt_bias" and not form[2])
            continue
        sl = slice(0, n) if k in ("d_x", "d_dt", "d_z", "d_b", "d_c") else slice(None)
        close(got[sl], r[k][sl], m[k][sl], tol + more * 2.0 ** -24, dt)
    again = bw(None)   # checkpoints computed again, sums in the same order
    for p, q in zip(g, again):
        assert p is None or torch.equal(p[:n] if p.shape[0] == n + pad else p, q[:n] if q.shape[0] == n + pad else q)


def test_scan_gradients_against_differences():
    """Central differences of the float64 forward form along random directions."""
    lengths, D, N, G = [37, 5], 16, 16, 1
    form = FORMS[0]
    v = scan_inputs(3, lengths, D, N, G, "f32")
    args, kw = scan_call(v, lengths, "f32", form)
    g = chela.selscan_bwd(*args, f32(v["d_y"]), **kw, d_state_out=f32(v["d_state_out"]), want_d_state=True)
    rng = np.random.default_rng(4)

    def loss(u):
        y, last = scan_ref(u, lengths, form)
        return (y * v["d_y"]).sum() + (last * v["d_state_out"]).sum()

    for name, grad in (("x", g.d_x), ("dt", g.d_dt), ("a", g.d_a), ("b", g.d_b), ("c", g.d_c), ("d_skip", g.d_skip), ("z", g.d_z),
                       ("dt_bias", g.d_dt_bias), ("state", g.d_state_in)):
        way = rng.standard_normal(v[name].shape)
        hi, lo = dict(v), dict(v)
        step = 1e-4
        hi[name], lo[name] = v[name].astype(np.float64) + step * way, v[name].astype(np.float64) - step * way
        want = (loss(hi) - loss(lo)) / (2 * step)
        got = (to_numpy(grad) * way).sum()
        # second-order term of the difference (1e-8 x third derivatives) and single precision gradients
        assert abs(got - want) <= 1e-4 * np.abs(to_numpy(grad) * way).sum(), name


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [8, 16, 32, 64])
def test_scan_step_against_the_formula(dtype, N):
    S, D, G = 5, 64, 2
    form = FORMS[0]
    v = scan_inputs(N, [1] * S, D, N, G, dtype)
    args, kw = scan_call(v, [1] * S, dtype, form, 8)
    kw.pop("seq_offsets")
    state = kw.pop("state_in")
    y = chela.selscan_step(*args, state, **kw, out_dtype=chela.F32)
    want, want_s = scan_ref(v, [1] * S, form)
    mag, mag_s = scan_ref(v, [1] * S, form, mag=True)
    close(y, want, mag, 2.0 ** -18)
    close(state, want_s, mag_s, 2.0 ** -18)


def test_scan_segments_and_steps_continue_a_prompt():
    """Segments with the state carried in place, then single tokens, against one call."""
    S, L, D, N = 2, 150, 40, 16
    form = FORMS[0]
    v = scan_inputs(8, [L] * S, D, N, 1, "f32")
    v["state"][:] = 0
    args, kw = scan_call(v, [L] * S, "f32", form)
    for k in ("seq_offsets", "state_in"):
        kw.pop(k)
    cut3 = lambda t, i, j: t.view(S, L, *t.shape[1:])[:, i:j].contiguous()  # noqa: E731
    full, last = chela.selscan_fwd(*[t if k == 2 else cut3(t, 0, L) for k, t in enumerate(args)],
                                   **{k: (cut3(t, 0, L) if k == "z" else t) for k, t in kw.items()})
    import torch
    state = torch.zeros(S, D, N, device="cuda")
    mag, mag_s = scan_ref(v, [L] * S, form, mag=True)
    mag = mag.reshape(S, L, D)
    at = 0
    for n in (1, 63, 64, 12):
        seg = [t if k == 2 else cut3(t, at, at + n) for k, t in enumerate(args)]
        y, state = chela.selscan_fwd(*seg, **{k: (cut3(t, at, at + n) if k == "z" else t) for k, t in kw.items()}, state_in=state,
                                     state_out=state)
        close(y, to_numpy(full[:, at:at + n]), mag[:, at:at + n], 2 * (L + 8) * 2.0 ** -21)
        at += n
    for t in range(at, L):
        one = [u if k == 2 else u.view(S, L, *u.shape[1:])[:, t] for k, u in enumerate(args)]
        y = chela.selscan_step(*one, state, **{k: (u.view(S, L, D)[:, t] if k == "z" else u) for k, u in kw.items()})
        close(y, to_numpy(full[:, t]), mag[:, t], 2 * (L + 8) * 2.0 ** -21)
    close(state, to_numpy(last), mag_s, 2 * (L + 8) * 2.0 ** -21)


@pytest.mark.parametrize("dtype,N,D,G", [("f32", 16, 40, 1), ("bf16", 8, 24, 1), ("bf16", 64, 64, 2), ("f32", 32, 72, 1)])
@pytest.mark.parametrize("lengths", [[2003], [1500, 0, 701, 1], [640, 640]], ids=str)
def test_scan_of_few_long_sequences_is_split(dtype, N, D, G, lengths):
    """So few chains that the sequences are cut into segments: outputs, states (carried in place), checkpoints."""
    import torch
    T, S = sum(lengths), len(lengths)
    form = FORMS[0]
    v = scan_inputs(T + N, lengths, D, N, G, dtype)
    split = chela.lib().chela_selscan_workspace_bytes(T, S, D, N) > 0
    assert split == (T // S >= 512)
    args, kw = scan_call(v, lengths, dtype, form, 8)
    want, want_s = scan_ref(v, lengths, form)
    mag, mag_s = scan_ref(v, lengths, form, mag=True)
    tol = (max(lengths) + 8) * 2.0 ** -21
    state = kw.pop("state_in")
    given = state.clone()
    ckpt = chela.selscan_checkpoints(T, S, D, N, "cuda")
    y, last = chela.selscan_fwd(*args, **kw, state_in=state, state_out=state, checkpoints=ckpt)
    assert last is state
    close(y, want, mag, tol, dtype)
    close(last, want_s, mag_s, tol)
    dy = dev(v["d_y"], dtype, 8)
    g1 = chela.selscan_bwd(*args, dy, **kw, state_in=given, checkpoints=ckpt, want_d_state=True)
    g2 = chela.selscan_bwd(*args, dy, **kw, state_in=given, want_d_state=True)
    for p, q in zip(g1, g2):
        assert torch.equal(p, q)
    form_v = dict(v, d_state_out=np.zeros_like(v["d_state_out"]))
    r, m = scan_ref(form_v, lengths, form, bwd=True), scan_ref(form_v, lengths, form, mag=True, bwd=True)
    for k, more in (("d_x", 0), ("d_dt", 0), ("d_z", 0), ("d_b", D // G), ("d_c", D // G), ("d_a", T), ("d_skip", T), ("d_dt_bias", T), ("d_state_in", 0)):
        close(getattr(g1, k), r[k], m[k], 2 * tol + more * 2.0 ** -24)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N,D,lengths", [(16, 1024, [40, 0, 33, 5, 64, 17, 1]), (16, 520, [9, 21, 0, 8, 1, 30, 16, 17, 2, 0, 5, 12, 33, 7]),
                                         (32, 1024, [65, 0, 12, 31]), (32, 520, [3, 40, 0, 17, 8, 1, 9])], ids=str)
def test_scan_of_many_chains(dtype, N, D, lengths):
    """So many chains that a lane has two channels of 16 or 32 states in whole sequences: outputs, states carried in place,
    checkpoints, gradients."""
    import torch
    S, T, form = len(lengths), sum(lengths), FORMS[0]
    channels = {16: 32, 32: 16}[N]
    assert S * -(-D // channels) > 222
    v = scan_inputs(N + D, lengths, D, N, 1, dtype)
    args, kw = scan_call(v, lengths, dtype, form, 8)
    state = kw.pop("state_in")
    given = state.clone()
    ckpt = chela.selscan_checkpoints(T, S, D, N, "cuda")
    y, last = chela.selscan_fwd(*args, **kw, state_in=state, state_out=state, checkpoints=ckpt)
    (want, want_s), (mag, mag_s) = scan_ref(v, lengths, form), scan_ref(v, lengths, form, mag=True)
    tol = (max(lengths) + 8) * 2.0 ** -21
    close(y, want, mag, tol, dtype)
    close(last, want_s, mag_s, tol)
    d_so = f32(v["d_state_out"])
    g1, g2 = (chela.selscan_bwd(*args, dev(v["d_y"], dtype, 8), **kw, state_in=given, checkpoints=c, d_state_out=d_so, want_d_state=True)
              for c in (ckpt, None))
    for p, q in zip(g1, g2):
        assert torch.equal(p, q)
    r, m = scan_ref(v, lengths, form, bwd=True), scan_ref(v, lengths, form, mag=True, bwd=True)
    for k, more in (("d_x", 0), ("d_dt", 0), ("d_z", 0), ("d_b", D), ("d_c", D), ("d_a", T), ("d_skip", T), ("d_dt_bias", T), ("d_state_in", 0)):
        close(getattr(g1, k), r[k], m[k], 2 * tol + more * 2.0 ** -24)


def test_scan_gradients_of_b_and_c_over_more_tokens_than_threads():
    """The kernel that adds the channel blocks' shares takes a second turn: the same bits as the sequences one by one."""
    import torch
    lengths, D, N = [30000, 29000], 608, 64
    assert D // 8 * 2 > 148 and sum(lengths) * 2 * N // 4 > 148 * 32 * 256
    T = sum(lengths)
    x, dt, dy = (torch.randn(T, D, device="cuda").bfloat16() for _ in range(3))
    b, c = (torch.randn(T, 1, N, device="cuda").bfloat16() for _ in range(2))
    a = -torch.arange(1, N + 1, device="cuda").float().repeat(D, 1)
    g = chela.selscan_bwd(x, dt, a, b, c, dy, seq_offsets=i32(ref.offsets(lengths)))
    at = 0
    for n in lengths:
        sl = slice(at, at + n)
        one = chela.selscan_bwd(x[sl], dt[sl], a, b[sl], c[sl], dy[sl], seq_offsets=i32([0, n]))
        for k in ("d_x", "d_dt", "d_b", "d_c"):
            assert torch.equal(getattr(g, k)[sl], getattr(one, k)), k
        at += n


def test_scan_of_a_split_sequence_with_growing_states():
    """Rates above zero: a segment's whole growth is infinite in single precision, but there is nothing to grow before the
    last ten tokens."""
    T, D, N = 2003, 16, 16
    form = (False, False, False, False, False)
    v = scan_inputs(1, [T], D, N, 1, "f32")
    v["a"] = np.abs(v["a"]) * np.float32(0.1)
    v["dt"] = np.abs(v["dt"])
    v["x"][:-10] = 0.0
    args, kw = scan_call(v, [T], "f32", form)
    assert chela.lib().chela_selscan_workspace_bytes(T, 1, D, N) > 0
    y, s = chela.selscan_fwd(*args, **kw)
    (want, want_s), (mag, mag_s) = scan_ref(v, [T], form), scan_ref(v, [T], form, mag=True)
    # ten decays exp(u), u up to 1.6 x 4 x 4: the exponent's rounding is u 2^-24 of the result, so 10 (2 + 26) 2^-24 in all
    close(y, want, mag, 512 * 2.0 ** -24)
    close(s, want_s, mag_s, 512 * 2.0 ** -24)


def test_scan_of_a_split_sequence_as_long_as_there_may_be():
    """One sequence of nearly 2^31 tokens beside two of one token: its last segment ends past 2^31 if it is not cut off first.
    The states forget what is more than a few hundred tokens back, so the last tokens alone give the same state."""
    import ctypes
    import torch
    T, D, N, tail = 2 ** 31 - 4096, 8, 8, 4096
    pattern = torch.randn(tail, D, device="cuda").bfloat16()
    x = torch.empty(T, D, dtype=torch.bfloat16, device="cuda")   # 34 GB: all four operands
    assert T % tail == 0
    x.view(-1, tail, D).copy_(pattern)
    a = -torch.arange(1, N + 1, device="cuda").float().repeat(D, 1)

    def last_states(t, lengths):
        S, out = len(lengths), torch.zeros(len(lengths), D, N, device="cuda")
        p, off = t.data_ptr(), i32(ref.offsets(lengths))
        r = chela.SelscanArgs(p, p, p, p, None, D, D, N, N, 0, a.data_ptr(), None, None, None, off.data_ptr(), S, t.shape[0], D, N, 1, 1,
                              chela.BF16)
        need = chela.lib().chela_selscan_workspace_bytes(t.shape[0], S, D, N)
        ws = torch.empty(max(need, 16), dtype=torch.uint8, device="cuda")
        assert chela.lib().chela_selscan_fwd(ctypes.byref(r), None, out.data_ptr(), None, chela.F32, ws.data_ptr(), need,
                                             torch.cuda.current_stream().cuda_stream) == chela.OK
        torch.cuda.synchronize()
        return need, out

    need, got = last_states(x, [T - 2, 1, 1])
    assert need > 0
    _, want = last_states(pattern, [tail - 2, 1, 1])
    # the decays of the first 64 tokens of the tail alone (time steps of 0.8 on average) leave nothing of what was before them;
    # both runs then apply the same operations to the same operands and what an older rounding left has decayed too
    assert torch.isfinite(got).all() and (got - want).abs().max().item() <= 2.0 ** -20 * want.abs().max().item()


def test_scan_keeps_what_is_not_finite_where_it_is():
    """NaN and infinities of one sequence stay in it; an infinitely fast decay forgets the state and nothing else."""
    lengths, D, N = [20, 33, 9], 16, 16
    form = FORMS[0]
    v = scan_inputs(11, lengths, D, N, 1, "f32")
    v["a"][3, 2] = -np.inf
    clean_args, kw = scan_call(v, lengths, "f32", form)
    clean, clean_s = chela.selscan_fwd(*clean_args, **kw)
    fast = dict(v)
    fast["a"] = v["a"].copy()
    fast["a"][3, 2] = -1e30
    want, want_s = scan_ref(fast, lengths, form)
    mag, mag_s = scan_ref(fast, lengths, form, mag=True)
    close(clean, want, mag, 50 * 2.0 ** -21)
    close(clean_s, want_s, mag_s, 50 * 2.0 ** -21)
    import torch
    for value in (np.nan, np.inf):
        u = {k: a.copy() for k, a in v.items()}
        u["x"][25, 5] = value
        u["b"][30] = value
        args, kw = scan_call(u, lengths, "f32", form)
        y, s = chela.selscan_fwd(*args, **kw)
        assert torch.equal(y[:25], clean[:25]) and torch.equal(y[53:], clean[53:])
        assert torch.equal(s[0], clean_s[0]) and torch.equal(s[2], clean_s[2])
        assert torch.equal(y[25:30, :5], clean[25:30, :5]) and not torch.isfinite(y[31:53]).any()


@pytest.mark.parametrize("N", [8, 16, 64])
def test_slow_states_over_a_long_sequence(N):
    """16384 decays 2^x with x between -2^-8 and -2^-19 multiplied up, forwards (state_in to state_out) and backwards
    (d_state_out to d_state_in).  One decay is off by up to a step of 2^-24 or so, but the mean over the tokens may not be: the
    library claims at most 0.06 of a step for these exponents, and a tenth is allowed here (backwards less is done: a tile's
    decay comes from its time).  What is left is not one-sided: a rounding of the decay and one of the product or two, of at
    most a step each, over L independent arguments, so 6 L^(1/2) for six standard deviations of one element, and the mean over
    the 256 elements or more of an octave within that over 16.  A correction that fits x below -2^-8 only is off by 0.12 to
    0.22 of a step here, the product of a tile's decays by 0.16 at 2^-14."""
    import torch
    S, L, octaves, each = 8, 16384, 11, 32
    D, step, G = octaves * each, 2.0 ** -24, 1   # enough chains that no sequence is split
    T = S * L
    assert chela.lib().chela_selscan_workspace_bytes(T, S, D, N) == 0
    gen = torch.Generator(device="cuda")
    gen.manual_seed(N)
    scale = 2.0 ** -torch.arange(9, 9 + octaves, device="cuda", dtype=torch.float32).repeat_interleave(each)
    dt = (1 + torch.rand(T, D, generator=gen, device="cuda")) * scale       # |x| in 2^-(k+1) .. 2^-k with the rates below
    a = -0.6931 * (0.98 + 0.02 * torch.rand(D, N, generator=gen, device="cuda"))
    zero, bc = torch.zeros(T, D, device="cuda"), torch.zeros(T, G, N, device="cuda")
    one = torch.ones(S, D, N, device="cuda")
    _, last = chela.selscan_fwd(zero, dt, a, bc, bc, softplus=False, state_in=one, seq_offsets=i32(np.arange(S + 1) * L))
    g = chela.selscan_bwd(zero, dt, a, bc, bc, zero, softplus=False, state_in=one, d_state_out=one, want_d_state=True,
                          seq_offsets=i32(np.arange(S + 1) * L))
    total = dt.view(S, L, D).double().sum(1)
    want = torch.exp(total[:, :, None] * a.double())
    for got in (last, g.d_state_in):
        off = ((got.double() / want - 1) / step).view(S, octaves, each, N)
        most, mean = off.abs().max().item(), off.mean((0, 2, 3)).abs().max().item()
        assert most <= 0.1 * L + 6 * L ** 0.5 and mean <= 0.1 * L + 6 * L ** 0.5 / 16


@pytest.mark.parametrize("N,D,S", [(8, 24, 3), (16, 40, 3), (16, 1024, 7), (64, 16, 3)])
def test_scan_rates_and_time_steps_of_either_sign(N, D, S):
    """Growing, constant and decaying states side by side in a lane, time steps below zero: exponents of up to a few units either
    way, so that the decays' errors stay at 2^-21 and nothing overflows in 40 tokens."""
    lengths = [40, 1, 17, 33, 5, 29, 40][:S]
    form = (True, True, False, True, False)
    v = scan_inputs(N + D, lengths, D, N, 1, "f32")
    rng = np.random.default_rng(D)
    v["a"] = rng.uniform(-1.0, 1.0, (D, N)).astype(np.float32)
    v["a"][:, ::5] = 0.0
    v["dt"] = (0.3 * v["dt"]).astype(np.float32)
    args, kw = scan_call(v, lengths, "f32", form)
    (want, want_s), (mag, mag_s) = scan_ref(v, lengths, form), scan_ref(v, lengths, form, mag=True)
    tol = (max(lengths) + 8) * 2.0 ** -21
    y, last = chela.selscan_fwd(*args, **kw)
    close(y, want, mag, tol)
    close(last, want_s, mag_s, tol)
    g = chela.selscan_bwd(*args, f32(v["d_y"]), **kw, d_state_out=f32(v["d_state_out"]), want_d_state=True)
    r, m = scan_ref(v, lengths, form, bwd=True), scan_ref(v, lengths, form, mag=True, bwd=True)
    n = sum(lengths)
    for k, more in (("d_x", 0), ("d_dt", 0), ("d_z", 0), ("d_b", D), ("d_c", D), ("d_a", n), ("d_skip", n), ("d_state_in", 0)):
        close(getattr(g, k), r[k], m[k], 2 * tol + more * 2.0 ** -24)


def test_scan_time_steps_down_to_tiny_ones():
    """softplus far below and above zero keeps its relative precision: one token from a zero state gives dt x b."""
    raw = np.array([-40.0, -20.0, -12.0, -7.0, -2.0, -0.5, 0.0, 0.5, 3.0, 19.0, 30.0, 88.0, -80.0, 1e-3, -1e-3, 100.0], dtype=np.float32)
    D = raw.size
    x = np.ones((1, D), np.float32)
    a = -np.ones((D, 8), np.float32)
    bc = np.ones((1, 1, 8), np.float32)
    _, s = chela.selscan_fwd(f32(x), f32(raw[None]), f32(a), f32(bc), f32(bc))
    want = np.repeat(ref.softplus(raw.astype(np.float64))[None, :, None], 8, 2)
    assert np.max(np.abs(to_numpy(s) / want - 1)) <= 2.0 ** -21


def test_many_sequences_and_offsets_beyond_32_bits_of_elements():
    """70000 sequences (more than a grid's second axis could hold), and token strides that put the last rows more than 2^31
    elements behind the first."""
    import torch
    S, D, N = 70000, 8, 8
    rng = np.random.default_rng(2)
    lengths = rng.integers(0, 3, S)
    v = scan_inputs(6, [int(lengths.sum())], D, N, 1, "f32")
    off = i32(ref.offsets(lengths))
    args, kw = scan_call(v, [1], "f32", (False, True, True, False, True))
    kw["seq_offsets"] = off
    y, s = chela.selscan_fwd(*args, **kw)
    want, want_s = ref.scan(v["x"], v["dt"], v["a"], v["b"], v["c"], lengths, d_skip=v["d_skip"], dt_bias=v["dt_bias"])
    mag, mag_s = ref.scan(v["x"], v["dt"], v["a"], v["b"], v["c"], lengths, d_skip=v["d_skip"], dt_bias=v["dt_bias"], mag=True)
    close(y, want, mag, 2.0 ** -18)
    close(s, want_s, mag_s, 2.0 ** -18)

    T, stride = 1100, 1 << 21   # 1100 rows x 2^21 elements = 4.6 GB of bf16
    wide = torch.empty(T * stride, dtype=torch.bfloat16, device="cuda")
    x = wide.as_strided((T, 64), (stride, 1))
    x.copy_(torch.randn(T, 64, device="cuda"))
    w = torch.randn(64, 4, device="cuda")
    y, st = chela.shortconv_carry_fwd(x, w, seq_offsets=i32([0, T]))
    y2, st2 = chela.shortconv_carry_fwd(x.contiguous(), w, seq_offsets=i32([0, T]))
    assert torch.equal(y, y2) and torch.equal(st, st2)
    bc = torch.randn(T, 1, 16, device="cuda").bfloat16()
    a = -torch.rand(64, 16, device="cuda")
    r1 = chela.selscan_fwd(x, x, a, bc, bc, z=x, seq_offsets=i32([0, 500, T]))
    r2 = chela.selscan_fwd(x.contiguous(), x.contiguous(), a, bc, bc, z=x.contiguous(), seq_offsets=i32([0, 500, T]))
    assert torch.equal(r1[0], r2[0]) and torch.equal(r1[1], r2[1])
    n1 = chela.blocknorm_fwd(x, x)
    n2 = chela.blocknorm_fwd(x.contiguous(), x.contiguous())
    assert torch.equal(n1[0], n2[0]) and torch.equal(n1[1], n2[1])


# ------------------------------------------------------------------------------------------------ block norms

def norm_inputs(seed, T, D, dtype, res_dtype):
    rng = np.random.default_rng(seed)
    r = lambda dt, *s: inputs.round_storage(rng.standard_normal(s, dtype=np.float32), dt)  # noqa: E731
    v = {"res": r(res_dtype, T, D), "y": r(dtype, T, D), "gate": r(dtype, T, D), "d_o": r(dtype, T, D), "d_r": r(res_dtype, T, D)}
    for k in ("w_post", "b_post", "scale", "w_pre", "b_pre"):
        v[k] = (1.0 + 0.3 * rng.standard_normal(D, dtype=np.float32)).astype(np.float32)
    return v


@pytest.mark.parametrize("dtype,res_dtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("T,D", [(1, 8), (3, 40), (7, 256), (5, 264), (9, 512), (33, 1000), (4, 1032), (5, 2048), (3, 4104), (2, 8192)])
@pytest.mark.parametrize("post,pre", [(1, 1), (2, 2), (1, 2), (0, 1), (2, 0)])
@pytest.mark.parametrize("gate_act,after", [(None, False), (1, False), (2, True), (0, True)])
def test_block_norms(dtype, res_dtype, T, D, post, pre, gate_act, after):
    v = norm_inputs(T + D + post, T, D, dtype, res_dtype)
    eps = 1e-6
    gate = None if gate_act is None else v["gate"]
    kw = {"w_post": v["w_post"], "b_post": v["b_post"] if post == 2 else None, "norm_post": post, "scale": v["scale"],
          "w_pre": v["w_pre"], "b_pre": v["b_pre"] if pre == 2 else None, "norm_pre": pre, "gate_act": gate_act or 0, "gate_after": after,
          "eps": eps}
    dkw = {k: (f32(a) if isinstance(a, np.ndarray) else a) for k, a in kw.items()}
    r, o = chela.blocknorm_fwd(dev(v["res"], res_dtype, 8), dev(v["y"], dtype, 8), dev(gate, dtype, 16), **dkw)
    want_r, want_o, keep = ref.junction(v["res"], v["y"], gate, **kw)
    # row sums of D squares: D/32 roundings a lane and a tree; every factor a few roundings; terms at most a few units large
    tol = (D / 32 + 64) * 2.0 ** -24
    size_r = np.abs(v["res"]) + np.abs(v["scale"]) * (np.abs(keep["m"]) + np.abs(keep["ga"]) * 4)
    close(r, want_r, size_r, tol, res_dtype)
    _, inv = ref.normalised(want_r, pre, eps)
    close(o, want_o, np.abs(want_o) + np.abs(v["w_pre"]) * (size_r * inv + 1) + np.abs(v["b_pre"]), 2 * tol, dtype)

    rb = inputs.round_storage(want_r.astype(np.float32), res_dtype)   # r' as it is stored
    g = chela.blocknorm_bwd(dev(rb, res_dtype), dev(v["y"], dtype, 8), dev(gate, dtype, 16), dev(v["d_o"], dtype), dev(v["d_r"], res_dtype),
                            **dkw, grad_dtype=DT[dtype])
    w = ref.junction_bwd(rb, v["y"], gate, v["d_o"], v["d_r"], **kw)
    _, inv2 = ref.normalised(rb.astype(np.float64), pre, eps)
    hat2 = np.abs(ref.normalised(rb.astype(np.float64), pre, eps)[0])
    # majorants: |d| plus its projections on the row, whose means are at most the row's largest terms
    top = lambda a: np.abs(a).max(1, keepdims=True)  # noqa: E731
    do = np.abs(v["d_o"] * v["w_pre"])
    size = np.abs(v["d_r"]) + inv2 * (do + (hat2 * top(hat2) + 1) * top(do))
    close(g.d_res, w["d_res"], size, 4 * tol, res_dtype)
    ga, hat, inv1 = np.abs(keep["ga"]), np.abs(keep["hat"]), keep["inv"]
    dm = size * np.abs(v["scale"])
    dn = dm * (ga if after else 1) * np.abs(v["w_post"])
    dv = inv1 * (dn + (hat * top(hat) + 1) * top(dn))
    close(g.d_y, w["d_y"], dv * (1 if after else ga), 8 * tol, dtype)
    n_abs = hat * np.abs(v["w_post"]) + np.abs(v["b_post"])
    if gate is not None:
        slope = 1.0 + np.abs(v["gate"])
        close(g.d_gate, w["d_gate"], (dm * n_abs if after else dv * np.abs(v["y"])) * slope, 8 * tol, dtype)
    many = 8 * tol + T * 2.0 ** -24
    close(g.d_w_pre, w["d_w_pre"], (np.abs(v["d_o"]) * (hat2 + 1)).sum(0), many)
    close(g.d_scale, w["d_scale"], (size * n_abs * (ga if after else 1) + size).sum(0), many)
    close(g.d_w_post, w["d_w_post"], (dm * (ga if after else 1) * (hat + 1)).sum(0), many)
    if pre == 2:
        close(g.d_b_pre, w["d_b_pre"], np.abs(v["d_o"]).sum(0), many)
    if post == 2:
        close(g.d_b_post, w["d_b_post"], (dm * (ga if after else 1)).sum(0), many)


@pytest.mark.parametrize("dtype,res_dtype", [("f32", "f32"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("T,D", [(8003, 40), (4001, 264), (2003, 1000), (1301, 2048), (1001, 4104), (901, 8192)])
@pytest.mark.parametrize("post,pre,gate_act,after", [(2, 2, 2, True), (1, 1, 1, False)])
def test_block_norms_of_several_rows_a_warp(dtype, res_dtype, T, D, post, pre, gate_act, after):
    """More rows than three CTAs an SM hold at once: rows fetched ahead, both stages, sums over rows and CTAs."""
    warps = next(w for w in (1, 2, 4, 8, 16, 32) if w * 256 >= D)
    assert T > 148 * 3 * max(8 // warps, 1)
    test_block_norms(dtype, res_dtype, T, D, post, pre, gate_act, after)


def test_block_norm_gradient_in_place_over_several_rows_a_warp():
    """d_res in d_res_out's buffer, which the C entry point allows, with the next row's operands fetched ahead."""
    import ctypes
    import torch
    for T, D in ((8003, 40), (2003, 1000), (901, 4104)):
        res, y, gate, d_r = (torch.randn(T, D, device="cuda") for _ in range(4))
        d_o = torch.randn(T, D, device="cuda")
        want = chela.blocknorm_bwd(res, y, gate, d_o, d_r, norm_post=chela.NORM_LAYER, norm_pre=chela.NORM_LAYER)
        r = chela.BlocknormArgs(res.data_ptr(), y.data_ptr(), gate.data_ptr(), D, D, D, None, None, None, None, None, T, D, 1, 0, 2, 2, 1e-6,
                                chela.F32, chela.F32)
        d_y, d_gate = torch.empty_like(y), torch.empty_like(y)
        need = chela.lib().chela_blocknorm_bwd_workspace_bytes(T, D)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        assert chela.lib().chela_blocknorm_bwd(ctypes.byref(r), d_o.data_ptr(), d_r.data_ptr(), d_r.data_ptr(), d_y.data_ptr(), d_gate.data_ptr(),
                                               None, None, None, None, None, chela.F32, ws.data_ptr(), need,
                                               torch.cuda.current_stream().cuda_stream) == chela.OK
        assert torch.equal(d_r, want.d_res) and torch.equal(d_y, want.d_y) and torch.equal(d_gate, want.d_gate)


def test_block_norm_parts_alone():
    """The norm before a first block, the norm behind a last one, no residual, one gradient missing, weights left out."""
    T, D, eps = 6, 48, 1e-5
    v = norm_inputs(2, T, D, "f32", "f32")
    none = {"w_post": None, "b_post": None, "norm_post": 1, "scale": None, "w_pre": None, "b_pre": None, "norm_pre": 1, "gate_act": 1,
            "gate_after": False, "eps": eps}
    res, y = f32(v["res"]), f32(v["y"])
    r, o = chela.blocknorm_fwd(res, eps=eps)
    assert r is res
    close(o, ref.junction(v["res"], None, None, **none)[1], 1.0, 1e-5)
    r, o = chela.blocknorm_fwd(res, y, eps=eps, pre=False)
    assert o is None
    close(r, ref.junction(v["res"], v["y"], None, **none)[0], 1.0, 1e-5)
    r, o = chela.blocknorm_fwd(None, y, f32(v["gate"]), eps=eps, pre=False)
    close(r, ref.junction(None, v["y"], v["gate"], **none)[0], 1.0, 1e-5)
    for d_o, d_r in ((v["d_o"], None), (None, v["d_r"])):
        g = chela.blocknorm_bwd(res, y, None, None if d_o is None else f32(d_o), None if d_r is None else f32(d_r), eps=eps)
        w = ref.junction_bwd(v["res"], v["y"], None, d_o, d_r, **none)
        close(g.d_res, w["d_res"], 1.0, 1e-4)
        close(g.d_y, w["d_y"], 1.0, 1e-4)
    g = chela.blocknorm_bwd(res, d_o=f32(v["d_o"]), w_pre=f32(v["w_pre"]), eps=eps)
    w = ref.junction_bwd(v["res"], None, None, v["d_o"], None, **{**none, "w_pre": v["w_pre"]})
    close(g.d_res, w["d_res"], 1.0, 1e-4)
    close(g.d_w_pre, w["d_w_pre"], 1.0, 1e-4)
    assert g.d_y is None and g.d_scale is None


def test_block_norm_in_place_constant_and_extreme_rows():
    """res_out = res; rows of zeros and of one value, a large mean (its square alone would lose the deviation), a NaN row."""
    import torch
    D = 64
    rows = np.zeros((5, D), np.float32)
    rows[1] = 3.0
    rows[2] = 4096.0 + np.arange(D) % 3
    rows[3, 7] = np.nan
    rows[4] = np.arange(D)
    for kind in (1, 2):
        _, o = chela.blocknorm_fwd(f32(rows), norm_pre=kind)
        want = ref.junction(rows, None, None, None, None, 0, None, None, None, kind, 0, False, 1e-6)[1]
        got = to_numpy(o)
        assert np.isnan(got[3]).all()
        ok = [0, 1, 2, 4]
        # one part in 2^-24 of the largest value over the deviation (0.8 where the mean is 4097)
        assert np.all(np.abs(got[ok] - want[ok]) <= 4097 * 2.0 ** -22)
    res, y = torch.randn(9, D, device="cuda"), torch.randn(9, D, device="cuda")
    want, o1 = chela.blocknorm_fwd(res, y)
    got, o2 = chela.blocknorm_fwd(res, y, res_out=res)
    assert got is res and torch.equal(got, want) and torch.equal(o1, o2)


@pytest.mark.parametrize("D", [40, 1000, 4104])
def test_block_norm_of_tensors_between_sectors(D):
    """fp32 tensors 16 bytes behind a 32-byte boundary: the same bits as on one."""
    import torch
    T = 5
    off = lambda t: torch.empty(t.numel() + 12, device="cuda", dtype=t.dtype)[4:4 + t.numel()].view(t.shape).copy_(t)  # noqa: E731
    res, y, gate, d_o, d_r = (torch.randn(T, D, device="cuda") for _ in range(5))
    r1, o1 = chela.blocknorm_fwd(res, y, gate)
    empty = lambda: off(torch.zeros(T, D, device="cuda"))  # noqa: E731
    r2, o2 = chela.blocknorm_fwd(off(res), off(y), off(gate), res_out=empty(), out=empty())
    assert res.data_ptr() % 32 == 0 and r2.data_ptr() % 32 == 16 and torch.equal(r1, r2) and torch.equal(o1, o2)
    r3, o3 = chela.blocknorm_fwd(res, y, gate, out=empty())
    assert torch.equal(r1, r3) and torch.equal(o1, o3)
    for p, q in zip(chela.blocknorm_bwd(r1, y, gate, d_o, d_r), chela.blocknorm_bwd(off(r1), off(y), off(gate), off(d_o), off(d_r))):
        assert p is None or torch.equal(p, q)


# ------------------------------------------------------------------------------------------------ types

OTHER = {"f32": "bf16", "bf16": "f32"}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_outputs_and_gradients_of_another_type_than_the_operands(dtype):
    """bf16 results of fp32 operands and fp32 results of bf16 ones against the reference: one rounding, or none."""
    to = OTHER[dtype]
    lengths, D, N, G, W = [37, 0, 70, 1], 64, 16, 2, 4
    off, n, L = i32(ref.offsets(lengths)), sum(lengths), max(lengths)
    x, w, bias, state, dy, d_so = conv_inputs(31, lengths, D, W, dtype)
    g = chela.shortconv_bwd(dev(x, dtype), f32(w), dev(dy, dtype), f32(bias), state_in=dev(state, dtype), d_state_out=dev(d_so, dtype),
                            seq_offsets=off, grad_dtype=DT[to], want_d_state=True)
    args = (x, w, bias, dy, lengths, state, d_so)
    r, m = ref.conv_bwd(*args), ref.conv_bwd(*args, mag=True)
    close(g.d_x, r[0], m[0], (2 * W + 16) * 2.0 ** -23, to)
    close(g.d_w, r[1], m[1], (W + 16 + n) * 2.0 ** -23)
    close(g.d_state_in, r[3], m[3], (2 * W + 16) * 2.0 ** -23, to)

    form = FORMS[0]
    v = scan_inputs(32, lengths, D, N, G, dtype)
    args, kw = scan_call(v, lengths, dtype, form)
    tol = (L + 8) * 2.0 ** -21
    (want, _), (mag, _) = scan_ref(v, lengths, form), scan_ref(v, lengths, form, mag=True)
    y, _ = chela.selscan_fwd(*args, **kw, out_dtype=DT[to])
    close(y, want, mag, tol, to)
    g = chela.selscan_bwd(*args, dev(v["d_y"], dtype), **kw, d_state_out=f32(v["d_state_out"]), grad_dtype=DT[to], want_d_state=True)
    r, m = scan_ref(v, lengths, form, bwd=True), scan_ref(v, lengths, form, mag=True, bwd=True)
    for k, more in (("d_x", 0), ("d_dt", 0), ("d_z", 0), ("d_b", D // G), ("d_c", D // G)):
        close(getattr(g, k), r[k], m[k], 2 * tol + more * 2.0 ** -24, to)
    one = [1] * 5
    v = scan_inputs(33, one, D, N, G, dtype)
    args, kw = scan_call(v, one, dtype, form)
    kw.pop("seq_offsets")
    y = chela.selscan_step(*args, kw.pop("state_in"), **kw, out_dtype=DT[to])
    close(y, scan_ref(v, one, form)[0], scan_ref(v, one, form, mag=True)[0], 2.0 ** -18, to)


@pytest.mark.parametrize("dtype,res_dtype", [("f32", "f32"), ("f32", "bf16"), ("bf16", "f32"), ("bf16", "bf16")])
@pytest.mark.parametrize("D", [40, 1000, 4104])
def test_block_norm_results_of_every_type(dtype, res_dtype, D):
    """o and the gradients of y and gate in fp32 and bf16, whatever the operands' types."""
    T, eps = 5, 1e-6
    v = norm_inputs(41 + D, T, D, dtype, res_dtype)
    kw = {"w_post": v["w_post"], "b_post": v["b_post"], "norm_post": 2, "scale": v["scale"], "w_pre": v["w_pre"], "b_pre": v["b_pre"],
          "norm_pre": 1, "gate_act": 1, "gate_after": False, "eps": eps}
    dkw = {k: (f32(a) if isinstance(a, np.ndarray) else a) for k, a in kw.items()}
    want_r, want_o, keep = ref.junction(v["res"], v["y"], v["gate"], **kw)
    rb = inputs.round_storage(want_r.astype(np.float32), res_dtype)
    w = ref.junction_bwd(rb, v["y"], v["gate"], v["d_o"], v["d_r"], **kw)
    # the tolerances of test_block_norms
    tol = (D / 32 + 64) * 2.0 ** -24
    size_r = np.abs(v["res"]) + np.abs(v["scale"]) * (np.abs(keep["m"]) + np.abs(keep["ga"]) * 4)
    inv = ref.normalised(want_r, 1, eps)[1]
    hat2, inv2 = ref.normalised(rb.astype(np.float64), 1, eps)
    hat2, top = np.abs(hat2), lambda a: np.abs(a).max(1, keepdims=True)
    do = np.abs(v["d_o"] * v["w_pre"])
    size = np.abs(v["d_r"]) + inv2 * (do + (hat2 * top(hat2) + 1) * top(do))
    ga, hat, dn = np.abs(keep["ga"]), np.abs(keep["hat"]), size * np.abs(v["scale"]) * np.abs(v["w_post"])
    dv = keep["inv"] * (dn + (hat * top(hat) + 1) * top(dn))
    for to in ("f32", "bf16"):
        r, o = chela.blocknorm_fwd(dev(v["res"], res_dtype), dev(v["y"], dtype), dev(v["gate"], dtype), **dkw, out_dtype=DT[to])
        close(r, want_r, size_r, tol, res_dtype)
        close(o, want_o, np.abs(want_o) + np.abs(v["w_pre"]) * (size_r * inv + 1) + np.abs(v["b_pre"]), 2 * tol, to)
        g = chela.blocknorm_bwd(dev(rb, res_dtype), dev(v["y"], dtype), dev(v["gate"], dtype), dev(v["d_o"], dtype), dev(v["d_r"], res_dtype),
                                **dkw, grad_dtype=DT[to])
        close(g.d_res, w["d_res"], size, 4 * tol, res_dtype)
        close(g.d_y, w["d_y"], dv * ga, 8 * tol, to)
        close(g.d_gate, w["d_gate"], dv * np.abs(v["y"]) * (1.0 + np.abs(v["gate"])), 8 * tol, to)


# ------------------------------------------------------------------------------------------------ calls

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lengths,pad", [([5, 0, 33], 7), ([0, 0], 4), ([64], 1), ([70, 3], 1000), ([12, 9], 0)], ids=str)
def test_rows_of_no_sequence_are_zero_in_what_a_call_allocates(dtype, lengths, pad):
    """Outputs and gradients of a padded batch go on into sums over all rows.  The allocator hands back blocks of NaN here."""
    import torch
    n, D, N, G = sum(lengths), 64, 16, 2
    T = n + pad
    v = scan_inputs(5, lengths, D, N, G, dtype, pad)
    args, kw = scan_call(v, lengths, dtype, FORMS[0])
    x, w, bias, state, dy, _ = conv_inputs(6, lengths, D, 4, dtype, pad)
    conv = (dev(x, dtype), f32(w))
    off = kw["seq_offsets"]

    def stale(like):
        held = [torch.full(s, float("nan"), dtype=t, device="cuda") for s in ((T, D), (T, G, N)) for t in (torch.float32, torch.bfloat16)
                for _ in range(6)]
        del held
        return like()

    y, _ = stale(lambda: chela.shortconv_carry_fwd(*conv, f32(bias), state_in=dev(state, dtype), seq_offsets=off))
    rows = [y]
    for kind in (chela.F32, chela.BF16):
        rows.append(stale(lambda: chela.shortconv_bwd(*conv, dev(dy, dtype), seq_offsets=off, grad_dtype=kind)).d_x)
        rows.append(stale(lambda: chela.selscan_fwd(*args, **kw, out_dtype=kind))[0])
        g = stale(lambda: chela.selscan_bwd(*args, dev(v["d_y"], dtype), **kw, grad_dtype=kind))
        rows += [g.d_x, g.d_dt, g.d_b, g.d_c, g.d_z]
    for t in rows:
        assert t.shape[0] == T and torch.isfinite(t[:n].float()).all() and not t[n:].float().ne(0).any()
    given = torch.full((T, D), 7.0, device="cuda")
    chela.selscan_fwd(*args, **kw, out_dtype=chela.F32, out=given)
    assert (given[n:] == 7).all()

def test_graph_replay_streams_and_repeated_calls_give_equal_bits():
    import torch
    lengths, D, N = [40, 0, 25, 90], 64, 16
    v = scan_inputs(21, lengths, D, N, 1, "bf16")
    args, kw = scan_call(v, lengths, "bf16", FORMS[0])
    dy = dev(v["d_y"], "bf16")
    xs, w, bias, cst, cdy, _ = (dev(a, "bf16") if i in (0, 3, 4) else f32(a) if i in (1, 2) else None
                                for i, a in enumerate(conv_inputs(3, lengths, D, 4, "bf16")))
    nv = norm_inputs(4, sum(lengths), D, "bf16", "f32")
    res, ny, ngate, nd_o, nd_r = f32(nv["res"]), dev(nv["y"], "bf16"), dev(nv["gate"], "bf16"), dev(nv["d_o"], "bf16"), f32(nv["d_r"])
    wp = f32(nv["w_pre"])

    def run():
        y, s = chela.selscan_fwd(*args, **kw)
        g = chela.selscan_bwd(*args, dy, **kw, want_d_state=True)
        cy, cs = chela.shortconv_carry_fwd(xs, w, bias, state_in=cst, seq_offsets=kw["seq_offsets"])
        cg = chela.shortconv_bwd(xs, w, cdy, bias, state_in=cst, seq_offsets=kw["seq_offsets"])
        r, o = chela.blocknorm_fwd(res, ny, ngate, w_pre=wp)
        ng = chela.blocknorm_bwd(r, ny, ngate, nd_o, nd_r, w_pre=wp)
        return [t for t in (y, s, *g, cy, cs, *cg, r, o, *ng) if t is not None]

    first = [t.clone() for t in run()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = run()
    torch.cuda.current_stream().wait_stream(side)
    for p, q in zip(first, second):
        assert torch.equal(p, q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = run()
    for t in held:
        t.fill_(3.0)
    graph.replay()
    torch.cuda.synchronize()
    for p, q in zip(first, held):
        assert torch.equal(p, q)
    # the graph reads its inputs when it runs
    args[0].zero_()
    graph.replay()
    want = chela.selscan_fwd(*args, **kw)[0]
    assert torch.equal(held[0], want) and not torch.equal(held[0], first[0])


def test_threads_on_one_stream_do_not_share_workspaces():
    """Three threads queue calls that need a workspace on the same stream at the same time; each gets what it gets alone."""
    import threading
    import torch
    jobs = []
    for k in range(3):
        lengths, D, N = [700 + 40 * k, 900 - 100 * k], 40, 16   # split forward: a workspace there too
        v = scan_inputs(60 + k, lengths, D, N, 1, "f32")
        args, kw = scan_call(v, lengths, "f32", FORMS[0])
        dy = f32(v["d_y"])
        c = [f32(t) for t in conv_inputs(70 + k, lengths, D, 4, "f32")]
        nv = {n: f32(t) for n, t in norm_inputs(80 + k, 333 + k, D, "f32", "f32").items()}
        assert chela.lib().chela_selscan_workspace_bytes(sum(lengths), 2, D, N) > 0

        def job(args=args, kw=kw, dy=dy, c=c, nv=nv):
            off = kw["seq_offsets"]
            y, s = chela.selscan_fwd(*args, **kw)
            cg = chela.shortconv_bwd(c[0], c[1], c[4], c[2], seq_offsets=off)
            g = chela.selscan_bwd(*args, dy, **kw)
            ng = chela.blocknorm_bwd(nv["res"], nv["y"], nv["gate"], nv["d_o"], nv["d_r"], w_pre=nv["w_pre"], w_post=nv["w_post"])
            return [t for t in (y, s, *cg, *g, *ng) if t is not None]
        jobs.append((job, [t.clone() for t in job()]))
    wrong, start = [], threading.Barrier(len(jobs))

    def work(job, want):
        start.wait()
        for _ in range(40):
            if not all(torch.equal(p, q) for p, q in zip(job(), want)):
                wrong.append(job)
                return
    threads = [threading.Thread(target=work, args=j) for j in jobs]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong


def test_a_selective_block_decodes_what_its_prompt_computed():
    """norm -> projection -> short convolution -> x and dt projections -> scan -> projection -> junction with the next
    block's norm, over a prompt with the states carried and then token by token, against one longer prompt."""
    import torch
    torch.manual_seed(0)
    S, L, cut, D, inner, N, rank = 3, 40, 33, 128, 256, 16, 32
    p = lambda *s, scale=1.0: torch.randn(*s, device="cuda") * scale  # noqa: E731
    w_in, w_x, w_dt, w_out = p(D, 2 * inner, scale=D ** -0.5), p(inner, rank + 2 * N, scale=inner ** -0.5), p(rank, inner, scale=rank ** -0.5), \
        p(inner, D, scale=inner ** -0.5)
    conv_w, conv_b, a = p(inner, 4, scale=0.5), p(inner, scale=0.1), -torch.arange(1, N + 1, device="cuda").float().repeat(inner, 1)
    bias, skip, n1, n2, s1 = p(inner) - 4.0, p(inner), 1 + p(D, scale=0.1), 1 + p(D, scale=0.1), torch.full((D,), 0.5, device="cuda")
    x = p(S, L, D)
    dense = lambda t, w: chela.dense_fwd(t.reshape(-1, t.shape[-1]), w, y_dtype=chela.F32).view(*t.shape[:-1], w.shape[1])  # noqa: E731

    def block(res, conv_state, scan_state, step):
        _, h = chela.blocknorm_fwd(res, w_pre=n1)
        xz = dense(h, w_in)
        u, z = xz[..., :inner], xz[..., inner:]
        if step:
            u = chela.shortconv_step(u, conv_w, conv_state, conv_b)
        else:
            u, conv_state = chela.shortconv_carry_fwd(u, conv_w, conv_b, state_in=conv_state)
        proj = dense(u, w_x)
        dt = dense(proj[..., :rank].contiguous(), w_dt)
        b, c = (proj[..., k:k + N].unflatten(-1, (1, N)) for k in (rank, rank + N))
        if step:
            y = chela.selscan_step(u, dt, a, b, c, scan_state, d_skip=skip, z=z, dt_bias=bias)
        else:
            y, scan_state = chela.selscan_fwd(u, dt, a, b, c, d_skip=skip, z=z, dt_bias=bias, state_in=scan_state)
        r, o = chela.blocknorm_fwd(res, dense(y, w_out), w_post=n2, scale=s1, w_pre=n1)
        return r, o, conv_state, scan_state

    full_r, full_o, *_ = block(x, None, None, False)
    r, o, cs, ss = block(x[:, :cut].contiguous(), None, None, False)
    bound = 2e-5 * full_o.abs().max().item()   # single precision projections of 256 terms summed in other orders
    assert (o - full_o[:, :cut]).abs().max().item() <= bound
    for t in range(cut, L):
        r, o, cs, ss = block(x[:, t].contiguous(), cs, ss, True)
        assert (r - full_r[:, t]).abs().max().item() <= bound and (o - full_o[:, t]).abs().max().item() <= bound
