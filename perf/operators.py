"""Timed cases of the selective-scan block's operators.

Three operators and the directions they are used in:

  conv    short causal depthwise convolution with the last width - 1 inputs carried between calls
          (prompt, single token, backward)
  scan    selective state space scan: h_t = exp(dt_t A) h_(t-1) + dt_t B_t x_t, y_t = <C_t, h_t> + D x_t, gated
          (prompt, single token, forward + backward)
  norm    the junction of two blocks: gate, norm and scale of one block's output, residual, norm before the next
          (prompt, single token, forward + backward)

Sequences of different lengths are packed along one token axis with their offsets in an int32 tensor.  ``own`` chooses
between the plain torch form and this repository's kernels.
"""
import random

import torch

own = False

EPS = 1e-6
WIDTH = 4
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # prompts of four 16K sequences through a layer with a doubled inner width of 512; x is half of the in-projection
        {"name": "conv_prompt", "op": "conv", "kind": "prompt", "S": 4, "T": 65536, "D": 1024, "width": 4, "act": True,
         "dtype": "bf16", "ragged": False, "carry": False},
        # next segment of 23 documents packed together, state of the previous segment carried in
        {"name": "conv_train_packed", "op": "conv", "kind": "train", "S": 23, "T": 32749, "D": 1024, "width": 4, "act": True,
         "dtype": "bf16", "ragged": True, "carry": True},
        # one decoding step of 64 sequences
        {"name": "conv_step", "op": "conv", "kind": "step", "S": 64, "T": 64, "D": 2048, "width": 4, "act": True,
         "dtype": "bf16", "ragged": False, "carry": True},
        # batch of eight 8K prompts, the layer of the larger mixer configuration
        {"name": "scan_prompt_batch", "op": "scan", "kind": "prompt", "S": 8, "T": 65536, "D": 1024, "N": 16, "G": 1,
         "dtype": "bf16", "ragged": False, "carry": False},
        # one long document alone: parallelism has to come from the time axis
        {"name": "scan_prompt_long", "op": "scan", "kind": "prompt", "S": 1, "T": 32768, "D": 512, "N": 16, "G": 1,
         "dtype": "bf16", "ragged": False, "carry": False},
        # chunked prefill of 29 requests, odd lengths from 0 upwards, states of 64, two groups, single precision
        {"name": "scan_prompt_packed", "op": "scan", "kind": "prompt", "S": 29, "T": 8191, "D": 512, "N": 64, "G": 2,
         "dtype": "f32", "ragged": True, "carry": True},
        # one decoding step of 64 sequences
        {"name": "scan_step", "op": "scan", "kind": "step", "S": 64, "T": 64, "D": 2048, "N": 16, "G": 1,
         "dtype": "bf16", "ragged": False, "carry": True},
        # training step of one layer, four sequences of 4K
        {"name": "scan_train_batch", "op": "scan", "kind": "train", "S": 4, "T": 16384, "D": 1024, "N": 16, "G": 1,
         "dtype": "bf16", "ragged": False, "carry": False},
        # training on packed documents of odd lengths in single precision, channel count not a multiple of 32
        {"name": "scan_train_packed", "op": "scan", "kind": "train", "S": 11, "T": 5003, "D": 520, "N": 16, "G": 1,
         "dtype": "f32", "ragged": True, "carry": False},
        # prompt tokens between two blocks: single-precision residual stream, bf16 block output and gate
        {"name": "norm_prompt", "op": "norm", "kind": "prompt", "T": 65536, "D": 1024, "norm": "rms", "gate": "silu",
         "after": False, "dtype": "bf16"},
        # the same between two blocks of one decoding step
        {"name": "norm_step", "op": "norm", "kind": "step", "T": 64, "D": 1024, "norm": "rms", "gate": "silu",
         "after": False, "dtype": "bf16"},
        # training: layer norm, sigmoid gate behind the norm, gradients of all inputs and weights, odd row count
        {"name": "norm_train", "op": "norm", "kind": "train", "T": 32749, "D": 1024, "norm": "layer", "gate": "sigmoid",
         "after": True, "dtype": "bf16"},
    ]


def _size(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["conv", "scan", "scan", "norm"])
    kind = rng.choice(["prompt", "train", "step"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    D = 8 * _size(rng, 8, 256)
    if op == "norm":
        T = _size(rng, 1, 256) if kind == "step" else _size(rng, 100, (32000 if kind == "train" else 65000) * 1024 // max(D, 1024))
        return {"op": op, "kind": kind, "T": T, "D": D, "norm": rng.choice(["rms", "layer"]),
                "gate": rng.choice(["none", "silu", "sigmoid"]), "after": rng.random() < 0.5, "dtype": dtype}
    case = {"op": op, "kind": kind, "dtype": dtype, "carry": kind == "step" or rng.random() < 0.5}
    if op == "conv":
        case |= {"D": D, "width": rng.choice([2, 3, 4, 4, 7]), "act": rng.random() < 0.8}
        most = 32000 * 1024 // max(D, 512)
    else:
        N = rng.choice([8, 16, 16, 32, 64])
        if rng.random() < 0.3:
            D, G = 64 * max(1, D // 64), 2
        else:
            G = 1
        case |= {"D": D, "N": N, "G": G}
        most = (1 << 26 if kind == "train" else 1 << 28) // (D * N)
    if kind == "step":
        S = T = _size(rng, 1, 128)
        ragged = False
    else:
        S, ragged = _size(rng, 1, 40), rng.random() < 0.6
        T = max(S, _size(rng, 50, min(most, 30000)))
        if not ragged:
            T = T // S * S
    return case | {"S": S, "T": T, "ragged": ragged}


def work(case):
    T, D = case["T"], case["D"]
    es = DTYPES[case["dtype"]].itemsize
    train, step = case["kind"] == "train", case["kind"] == "step"
    if case["op"] == "conv":
        W, S = case["width"], case["S"]
        state = S * D * (W - 1) * es * (2 if case["carry"] else 1)
        if train:  # x, dy in; dx out, and the taps' gradients
            return {"bytes": 3 * T * D * es + D * (W + 1) * 8 + (S * D * (W - 1) * es if case["carry"] else 0),
                    "flops": T * D * (6 * W + 10)}
        return {"bytes": 2 * T * D * es + state + D * (W + 1) * 4, "flops": T * D * (2 * W + 4)}
    if case["op"] == "scan":
        S, N, G = case["S"], case["N"], case["G"]
        weights = D * (N + 2) * 4
        state = S * D * N * 4 * (2 if case["carry"] else 1)
        if train:  # x, dt, z, dy, B, C in; y, dx, ddt, dz, dB, dC out
            return {"bytes": 8 * T * D * es + 4 * T * G * N * es + 2 * weights + state, "flops": T * D * (28 * N + 60)}
        return {"bytes": 4 * T * D * es + 2 * T * G * N * es + weights + state, "flops": T * D * (7 * N + 20)}
    gated = case["gate"] != "none"
    if train:  # residual, y, gate, two gradients in; new residual, output and three gradients out
        return {"bytes": T * D * (4 * 4 + es * (4 + (2 if gated else 0))) + 10 * D * 4, "flops": T * D * 50}
    return {"bytes": T * D * (8 + es * (2 + gated)) + 3 * D * 4, "flops": T * D * 20}


# ------------------------------------------------------------------------------------------------ inputs

def _lengths(case, seed):
    """Lengths of the packed sequences: very different ones, an empty one and one of a single token among them."""
    S, T = case["S"], case["T"]
    if not case["ragged"]:
        return [T // S] * S
    rng = random.Random(1000003 * seed + 31 * T + S)
    weights = [rng.lognormvariate(0.0, 1.2) for _ in range(S)]
    few = set(rng.sample(range(S), 2)) if S >= 4 else set()
    total = sum(w for i, w in enumerate(weights) if i not in few)
    lengths = [0 if i in few else int((T - 1) * w / total) for i, w in enumerate(weights)]
    if few:
        lengths[min(few)] = 1
    big = max(range(S), key=lambda i: lengths[i])
    lengths[big] += T - sum(lengths)
    return lengths


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    T, D = case["T"], case["D"]

    def normal(*shape, dtype=torch.float32, std=1.0):
        return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    st = {"case": case}
    if case["op"] == "norm":
        st["res"] = normal(T, D, std=2.0)
        st["y"] = normal(T, D, dtype=dt) * (0.5 + uniform(T, 1)).to(dt)
        st["gate"] = None if case["gate"] == "none" else normal(T, D, dtype=dt)
        st["w_post"], st["w_pre"] = 1 + 0.2 * normal(D), 1 + 0.2 * normal(D)
        layer = case["norm"] == "layer"
        st["b_post"], st["b_pre"] = (0.1 * normal(D), 0.1 * normal(D)) if layer else (None, None)
        st["scale"] = 0.1 + 0.3 * uniform(D)
        if case["kind"] == "train":
            st["d_o"], st["d_res"] = normal(T, D, dtype=dt), normal(T, D)
        if case["kind"] == "step":
            st["res_out"], st["out"] = torch.empty_like(st["res"]), torch.empty_like(st["y"])
        return st

    S = case["S"]
    lengths = _lengths(case, seed)
    st["longest"] = max(lengths)
    ends = [0]
    for n in lengths:
        ends.append(ends[-1] + n)
    st["offsets"] = torch.tensor(ends, dtype=torch.int32, device="cuda")
    # x and the gate z are the two halves of one projection's output
    xz = normal(T, 2 * D, dtype=dt)
    st["x"], st["z"] = xz[:, :D], xz[:, D:]
    if case["op"] == "conv":
        W = case["width"]
        st["w"], st["bias"] = normal(D, W, std=W ** -0.5), 0.1 * normal(D)
        st["state"] = normal(S, W - 1, D, dtype=dt) if case["carry"] else None
        if case["kind"] == "train":
            st["d_y"] = normal(T, D, dtype=dt)
        if case["kind"] == "step":
            st["state_out"], st["out"] = torch.empty_like(st["state"]), torch.empty(T, D, dtype=dt, device="cuda")
        return st
    N, G = case["N"], case["G"]
    rank = 8 * max(1, D // 128)
    proj = normal(T, rank + 2 * G * N, dtype=dt)
    st["b"] = proj[:, rank:rank + G * N].unflatten(1, (G, N))
    st["c"] = proj[:, rank + G * N:].unflatten(1, (G, N))
    st["a"] = -torch.arange(1, N + 1, device="cuda", dtype=torch.float32) * torch.exp(0.2 * normal(D, N))
    # softplus(dt + bias) is spread over 1e-3 .. 1e-1, as such models are initialised, and moves with the token
    step = torch.exp(uniform(D) * (torch.log(torch.tensor(0.1)) - torch.log(torch.tensor(0.001))).item()) * 0.001
    st["dt_bias"] = step + torch.log(-torch.expm1(-step))
    st["dt"] = normal(T, D, dtype=dt, std=0.7)
    st["d_skip"] = 1 + 0.1 * normal(D)
    st["state"] = normal(S, D, N, std=0.3) if case["carry"] else None
    if case["kind"] == "train":
        st["d_y"] = normal(T, D, dtype=dt)
    if case["kind"] == "step":
        st["state_out"], st["out"] = torch.empty_like(st["state"]), torch.empty(T, D, dtype=dt, device="cuda")
    return st


# ------------------------------------------------------------------------------------------------ plain forms

def _sequences(offsets, T):
    """For every token: its sequence, its position in it, and how many tokens of the sequence follow."""
    off = offsets.long()
    t = torch.arange(T, device=off.device)
    seq = (t[:, None] >= off[None, 1:]).sum(1)
    return seq, t - off[seq], off[seq + 1] - 1 - t


def _silu(u):
    return u / (1 + torch.exp(-u))


def _d_silu(u):
    s = 1 / (1 + torch.exp(-u))
    return s * (1 + u * (1 - s))


def _back(x, pos, j, state, seq):
    """x[t - j] within t's own sequence; rows before its start come from the carried state, or are zero."""
    if j == 0:
        return x
    T = x.shape[0]
    rows = x[(torch.arange(T, device=x.device) - j).clamp(min=0)]
    before = (pos < j)[:, None]
    if state is None:
        return torch.where(before, torch.zeros_like(rows), rows)
    held = state[seq, (pos - j + state.shape[1]).clamp(0, state.shape[1] - 1)]
    return torch.where(before, held, rows)


def _conv_state(x, offsets, state, W):
    """The last W - 1 inputs of every sequence, the carried ones first where it is shorter."""
    off = offsets.long()
    r = torch.arange(W - 1, device=x.device)
    t = off[1:, None] - (W - 1) + r[None, :]
    inside = t >= off[:-1, None]
    rows = x[t.clamp(0, max(x.shape[0] - 1, 0))]
    if state is None:
        return torch.where(inside[..., None], rows, torch.zeros_like(rows))
    held_at = ((off[1:] - off[:-1])[:, None] + r[None, :]).clamp(max=W - 2)
    held = torch.gather(state, 1, held_at[..., None].expand(-1, -1, x.shape[1]))
    return torch.where(inside[..., None], rows, held)


def _plain_conv(st):
    case = st["case"]
    W, dt = case["width"], st["x"].dtype
    x, w = st["x"].float(), st["w"]
    state = None if st["state"] is None else st["state"].float()
    seq, pos, left = _sequences(st["offsets"], x.shape[0])
    u = st["bias"] + sum(w[:, j] * _back(x, pos, j, state, seq) for j in range(W))
    if case["kind"] != "train":
        y = _silu(u) if case["act"] else u
        return y.to(dt), _conv_state(x, st["offsets"], state, W).to(dt)
    d_u = st["d_y"].float() * (_d_silu(u) if case["act"] else 1.0)
    T = x.shape[0]
    t = torch.arange(T, device=x.device)
    ahead = [torch.where((left >= j)[:, None], d_u[(t + j).clamp(max=T - 1)], torch.zeros_like(d_u)) for j in range(W)]
    d_x = sum(w[:, j] * ahead[j] for j in range(W))
    d_w = torch.stack([(d_u * _back(x, pos, j, state, seq)).sum(0) for j in range(W)], 1)
    return d_x.to(dt), d_w, d_u.sum(0)


def _shifted(v, k, keep):
    """v[t - k] where keep[t], zero elsewhere."""
    moved = torch.zeros_like(v)
    moved[k:] = torch.where(keep[k:, None, None], v[:-k], torch.zeros((), device=v.device))
    return moved


def _scan(decay, add, pos, longest):
    """h_t = decay_t h_(t-1) + add_t in every sequence from zero, by doubling; also the decay since its start."""
    k = 1
    while k < longest:
        inside = pos >= k
        add = add + decay * _shifted(add, k, inside)
        decay = torch.where(inside[:, None, None], decay * torch.roll(decay, k, 0), decay)
        k *= 2
    return add, decay


def _per_channel(v, D):
    """[T, G, N] -> [T, D, N]: channel d belongs to group d // (D / G)."""
    return v if v.shape[1] == D else v.repeat_interleave(D // v.shape[1], 1)


def _softplus(v):
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-v.abs()))


def _plain_scan(st):
    case = st["case"]
    out = st["x"].dtype
    x, z, b, c = (st[k].float() for k in ("x", "z", "b", "c"))
    raw = st["dt"].float() + st["dt_bias"]
    dt = _softplus(raw)
    T, D = x.shape
    seq, pos, left = _sequences(st["offsets"], T)
    if case["kind"] == "step":
        h = torch.exp(dt[..., None] * st["a"]) * st["state"] + (dt * x)[..., None] * _per_channel(b, D)
        y = (h * _per_channel(c, D)).sum(-1) + st["d_skip"] * x
        return (y * _silu(z)).to(out), h
    decay = torch.exp(dt[..., None] * st["a"])
    h, since = _scan(decay, (dt * x)[..., None] * _per_channel(b, D), pos, st["longest"])
    if st["state"] is not None:
        h = h + since * st["state"][seq]
    del since
    y = (h * _per_channel(c, D)).sum(-1) + st["d_skip"] * x
    off = st["offsets"].long()
    first = torch.zeros(case["S"], D, case["N"], device=x.device) if st["state"] is None else st["state"]
    last = torch.where((off[1:] > off[:-1])[:, None, None], h[(off[1:] - 1).clamp(min=0)], first)
    if case["kind"] == "prompt":
        return (y * _silu(z)).to(out), last
    # backward
    d_y = st["d_y"].float()
    d_z = d_y * y * _d_silu(z)
    d_in = d_y * _silu(z)
    prev = _shifted(h, 1, pos >= 1)
    if st["state"] is not None:
        prev = torch.where((pos == 0)[:, None, None], st["state"][seq], prev)
    d_c = (d_in[..., None] * h).unflatten(1, (case["G"], -1)).sum(2)
    del h
    ahead = torch.roll(decay, -1, 0)   # a_(t+1); where t is the last token nothing comes from behind it
    g = _scan(ahead.flip(0), (d_in[..., None] * _per_channel(c, D)).flip(0), left.flip(0), st["longest"])[0].flip(0)
    del ahead
    g_b = (g * _per_channel(b, D)).sum(-1)
    d_b = (g * (dt * x)[..., None]).unflatten(1, (case["G"], -1)).sum(2)
    through = g * decay * prev
    d_dt = (through * st["a"]).sum(-1) + x * g_b
    d_a = (through * dt[..., None]).sum(0)
    d_x = dt * g_b + st["d_skip"] * d_in
    d_raw = d_dt / (1 + torch.exp(-raw))
    return ((y * _silu(z)).to(out), last, d_x.to(out), d_raw.to(out), d_a, d_b.to(out), d_c.to(out), (d_in * x).sum(0),
            d_z.to(out), d_raw.sum(0))


def _normalised(v, norm):
    """(v normalised, 1 / its deviation) by rows."""
    if norm == "layer":
        v = v - v.mean(-1, keepdim=True)
    inv = torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * inv, inv


def _norm_back(d, hat, inv, norm):
    """Gradient of the input of _normalised from that of its output."""
    d_v = d - hat * (d * hat).mean(-1, keepdim=True)
    return inv * (d_v - d.mean(-1, keepdim=True) if norm == "layer" else d_v)


def _plain_norm(st):
    case = st["case"]
    norm, after = case["norm"], case["after"]
    out = st["y"].dtype
    y = st["y"].float()
    gate = None if st["gate"] is None else st["gate"].float()
    act = 1.0 if gate is None else _silu(gate) if case["gate"] == "silu" else 1 / (1 + torch.exp(-gate))
    hat, inv = _normalised(y if after else y * act, norm)
    n = hat * st["w_post"] + (0.0 if st["b_post"] is None else st["b_post"])
    m = n * act if after else n
    res = st["res"] + st["scale"] * m
    hat2, inv2 = _normalised(res, norm)
    o = hat2 * st["w_pre"] + (0.0 if st["b_pre"] is None else st["b_pre"])
    if case["kind"] != "train":
        return res, o.to(out)
    d_o = st["d_o"].float()
    d_w_pre, d_b_pre = (d_o * hat2).sum(0), d_o.sum(0)
    d_r = st["d_res"] + _norm_back(d_o * st["w_pre"], hat2, inv2, norm)
    d_scale = (d_r * m).sum(0)
    d_m = d_r * st["scale"]
    d_n = d_m * act if after else d_m
    d_w_post, d_b_post = (d_n * hat).sum(0), d_n.sum(0)
    d_v = _norm_back(d_n * st["w_post"], hat, inv, norm)
    grads = [d_r, (d_v if after else d_v * act).to(out)]
    if gate is not None:
        slope = _d_silu(gate) if case["gate"] == "silu" else act * (1 - act)
        grads.append(((d_m * n if after else d_v * y) * slope).to(out))
    grads += [d_w_post, d_scale, d_w_pre]
    if norm == "layer":
        grads += [d_b_post, d_b_pre]
    return (res, o.to(out), *grads)


# ------------------------------------------------------------------------------------------------ the library's calls

def _own_conv(st):
    from paper_2406_08128_b200 import chela
    case = st["case"]
    if case["kind"] == "step":
        y = chela.shortconv_step(st["x"], st["w"], st["state"], bias=st["bias"], act=case["act"], state_out=st["state_out"],
                                 out=st["out"])
        return y, st["state_out"]
    if case["kind"] == "prompt":
        return chela.shortconv_carry_fwd(st["x"], st["w"], bias=st["bias"], act=case["act"], state_in=st["state"],
                                         seq_offsets=st["offsets"])
    g = chela.shortconv_bwd(st["x"], st["w"], st["d_y"], bias=st["bias"], act=case["act"], state_in=st["state"],
                            seq_offsets=st["offsets"], grad_dtype=chela.BF16 if case["dtype"] == "bf16" else chela.F32)
    return g.d_x, g.d_w, g.d_bias


def _own_scan(st):
    from paper_2406_08128_b200 import chela
    case = st["case"]
    args = (st["x"], st["dt"], st["a"], st["b"], st["c"])
    more = {"d_skip": st["d_skip"], "z": st["z"], "dt_bias": st["dt_bias"], "softplus": True}
    if case["kind"] == "step":
        y = chela.selscan_step(*args, st["state"], **more, state_out=st["state_out"], out=st["out"])
        return y, st["state_out"]
    more |= {"state_in": st["state"], "seq_offsets": st["offsets"]}
    if case["kind"] == "prompt":
        return chela.selscan_fwd(*args, **more)
    ckpt = chela.selscan_checkpoints(case["T"], case["S"], case["D"], case["N"], st["x"].device)
    y, last = chela.selscan_fwd(*args, **more, checkpoints=ckpt)
    g = chela.selscan_bwd(*args, st["d_y"], **more, checkpoints=ckpt,
                          grad_dtype=chela.BF16 if case["dtype"] == "bf16" else chela.F32)
    return y, last, g.d_x, g.d_dt, g.d_a, g.d_b, g.d_c, g.d_skip, g.d_z, g.d_dt_bias


def _own_norm(st):
    from paper_2406_08128_b200 import chela
    case = st["case"]
    norm = chela.NORM_LAYER if case["norm"] == "layer" else chela.NORM_RMS
    more = {"w_post": st["w_post"], "b_post": st["b_post"], "norm_post": norm, "scale": st["scale"], "w_pre": st["w_pre"],
            "b_pre": st["b_pre"], "norm_pre": norm, "gate_act": {"none": 0, "silu": 1, "sigmoid": 2}[case["gate"]],
            "gate_after": case["after"], "eps": EPS}
    if case["kind"] == "step":
        return chela.blocknorm_fwd(st["res"], st["y"], st["gate"], **more, res_out=st["res_out"], out=st["out"])
    res, o = chela.blocknorm_fwd(st["res"], st["y"], st["gate"], **more)
    if case["kind"] == "prompt":
        return res, o
    g = chela.blocknorm_bwd(res, st["y"], st["gate"], st["d_o"], st["d_res"], **more,
                            grad_dtype=chela.BF16 if case["dtype"] == "bf16" else chela.F32)
    grads = [g.d_res, g.d_y] + ([] if st["gate"] is None else [g.d_gate]) + [g.d_w_post, g.d_scale, g.d_w_pre]
    if case["norm"] == "layer":
        grads += [g.d_b_post, g.d_b_pre]
    return (res, o, *grads)


def run(state):
    op = state["case"]["op"]
    if own:
        return {"conv": _own_conv, "scan": _own_scan, "norm": _own_norm}[op](state)
    return {"conv": _plain_conv, "scan": _plain_scan, "norm": _plain_norm}[op](state)


# ------------------------------------------------------------------------------------------------ 64-bit definitions

def _exact_conv(case, st, lengths):
    """Every sequence on its own: the carried rows stand before its inputs, and autograd differentiates the sum of taps."""
    W = case["width"]
    train = case["kind"] == "train"
    w = st["w"].double().requires_grad_(train)
    bias = st["bias"].double().requires_grad_(train)
    ys, states, d_xs = [], [], []
    at = 0
    for s, n in enumerate(lengths):
        x = st["x"][at:at + n].double().requires_grad_(train)
        head = torch.zeros(W - 1, case["D"], dtype=torch.float64, device=x.device) if st["state"] is None else st["state"][s].double()
        ext = torch.cat([head, x])
        u = bias + sum(ext[W - 1 - j:W - 1 - j + n] * w[:, j] for j in range(W))
        y = u * torch.sigmoid(u) if case["act"] else u
        if train:
            if n:
                y.backward(st["d_y"][at:at + n].double())
            d_xs.append(x.grad if n else x.detach())
        else:
            ys.append(y)
            states.append(ext[n:])
        at += n
    if train:
        return torch.cat(d_xs), w.grad, bias.grad
    return torch.cat(ys), torch.stack(states)


def _exact_scan(case, st, lengths):
    """The recurrence token by token over all sequences side by side; autograd over it gives the gradients."""
    T, D, N, G, S = case["T"], case["D"], case["N"], case["G"], case["S"]
    train = case["kind"] == "train"
    L = max(lengths)
    names = ["x", "dt", "b", "c", "z", "a", "d_skip", "dt_bias"]
    v = {k: st[k].double().detach().clone().requires_grad_(train) for k in names}
    dev = v["x"].device
    starts = [sum(lengths[:s]) for s in range(S)]
    at = torch.tensor([[starts[s] + min(t, max(lengths[s] - 1, 0)) for s in range(S)] for t in range(L)], device=dev).clamp(max=T - 1)
    live = torch.tensor([[t < n for n in lengths] for t in range(L)], device=dev)
    delta = torch.nn.functional.softplus(v["dt"] + v["dt_bias"])
    h = torch.zeros(S, D, N, dtype=torch.float64, device=dev) if st["state"] is None else st["state"].double()
    ys = []
    whole = all(n == L for n in lengths)
    for t in range(L):
        i = at[t]
        d = delta[i]
        b = v["b"][i][:, :, None, :].expand(S, G, D // G, N).reshape(S, D, N)
        c = v["c"][i][:, :, None, :].expand(S, G, D // G, N).reshape(S, D, N)
        new = torch.exp(d[:, :, None] * v["a"]) * h + (d * v["x"][i])[:, :, None] * b
        h = new if whole else torch.where(live[t][:, None, None], new, h)
        ys.append(torch.einsum("sdn,sdn->sd", h, c))
    rows = torch.stack(ys)                                   # [L, S, D]
    place = torch.tensor([t * S + s for s in range(S) for t in range(lengths[s])], device=dev)
    y = (rows.reshape(L * S, D)[place] + v["d_skip"] * v["x"]) * torch.nn.functional.silu(v["z"])
    if not train:
        return y, h
    y.backward(st["d_y"].double())
    return (y.detach(), h.detach(), v["x"].grad, v["dt"].grad, v["a"].grad, v["b"].grad, v["c"].grad, v["d_skip"].grad,
            v["z"].grad, v["dt_bias"].grad)


def _exact_norm(case, st):
    train = case["kind"] == "train"
    names = [k for k in ("res", "y", "gate", "w_post", "scale", "w_pre", "b_post", "b_pre") if st[k] is not None]
    v = {k: st[k].double().detach().clone().requires_grad_(train) for k in names}

    def norm(u):
        if case["norm"] == "layer":
            return torch.nn.functional.layer_norm(u, (case["D"],), eps=EPS)
        return u / torch.sqrt(torch.mean(u ** 2, -1, keepdim=True) + EPS)

    gate = 1.0
    if "gate" in v:
        gate = torch.nn.functional.silu(v["gate"]) if case["gate"] == "silu" else torch.sigmoid(v["gate"])
    n = norm(v["y"] if case["after"] else v["y"] * gate) * v["w_post"] + v.get("b_post", 0.0)
    res = v["res"] + v["scale"] * (n * gate if case["after"] else n)
    o = norm(res) * v["w_pre"] + v.get("b_pre", 0.0)
    if not train:
        return res, o
    torch.autograd.backward([res, o], [st["d_res"].double(), st["d_o"].double()])
    return (res.detach(), o.detach(), *[v[k].grad for k in names])


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "norm":
        return _exact_norm(case, st)
    lengths = _lengths(case, seed)
    if case["op"] == "conv":
        return _exact_conv(case, st, lengths)
    if case["kind"] == "train" and max(lengths) * case["S"] > 65536:
        return None   # the recorded recurrence would not fit
    return _exact_scan(case, st, lengths)
