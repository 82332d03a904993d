"""Timed cases of the operators at the two ends of a language model, on either side of its token-mixing layers.

  embed   lookup of token embeddings with a scale: out[t] = scale * w[ids[t]]; ids outside the table give a row of zeros
          (prompt, single token), and the gradient of the table from the tokens' gradients, alone or on top of another
          (train, tied)
  loss    softmax cross entropy of hidden rows against a vocabulary's weight rows, without the logits in memory:
          lse[t] = log sum_v exp(scale <h[t], w[v]>), loss[t] = lse[t] - scale <h[t], w[target[t]]>; rows whose target
          lies outside the vocabulary are left out (score), and forward with the gradients of h and w (train)

``own`` chooses between the plain torch form and this repository's kernels.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases

def listed():
    return [
        # one decoding step of 64 sequences
        {"name": "embed_step", "op": "embed", "kind": "step", "T": 64, "V": 50000, "D": 1024, "dtype": "bf16", "ids": "i64",
         "left_out": 0.0},
        # prompts of 64K tokens over a word-level vocabulary
        {"name": "embed_prompt", "op": "embed", "kind": "prompt", "T": 65536, "V": 260000, "D": 1024, "dtype": "bf16", "ids": "i64",
         "left_out": 0.0},
        # the table's gradient in a training step of 16K tokens: every row of the gradient is written
        {"name": "embed_train", "op": "embed", "kind": "train", "T": 16384, "V": 50000, "D": 1024, "dtype": "bf16", "ids": "i64",
         "left_out": 0.0},
        # tied weights: the table's gradient is the one that the loss has given (kept, as between micro-batches) and the
        # tokens' on top; a third is padding
        {"name": "embed_train_tied", "op": "embed", "kind": "tied", "T": 32749, "V": 260000, "D": 512, "dtype": "bf16", "ids": "i32",
         "left_out": 0.33},
        # scoring a handful of next tokens: the weights are read once
        {"name": "loss_score_few", "op": "loss", "kind": "score", "T": 48, "V": 50000, "D": 1024, "dtype": "bf16", "ids": "i64",
         "left_out": 0.0},
        # scoring prompts (perplexity)
        {"name": "loss_score", "op": "loss", "kind": "score", "T": 16384, "V": 50000, "D": 1024, "dtype": "bf16", "ids": "i64",
         "left_out": 0.0},
        # training step of 16K tokens
        {"name": "loss_train", "op": "loss", "kind": "train", "T": 16384, "V": 50000, "D": 1024, "dtype": "bf16", "ids": "i64",
         "left_out": 0.0},
        # word-level vocabulary, odd number of tokens
        {"name": "loss_train_words", "op": "loss", "kind": "train", "T": 4093, "V": 260000, "D": 1024, "dtype": "bf16", "ids": "i64",
         "left_out": 0.0},
        # a vocabulary of bytes: few columns, many rows
        {"name": "loss_train_bytes", "op": "loss", "kind": "train", "T": 65536, "V": 205, "D": 512, "dtype": "bf16", "ids": "i32",
         "left_out": 0.0},
        # training on answers only: two thirds of the tokens are prompts or padding
        {"name": "loss_train_answers", "op": "loss", "kind": "train", "T": 16001, "V": 32003, "D": 1024, "dtype": "bf16", "ids": "i64",
         "left_out": 0.66},
        # single precision, odd sizes
        {"name": "loss_train_f32", "op": "loss", "kind": "train", "T": 2047, "V": 10007, "D": 520, "dtype": "f32", "ids": "i64",
         "left_out": 0.1},
    ]


def _size(rng, lo, hi):
    """A whole number between lo and hi, spread over its logarithm."""
    return max(lo, min(hi, round(lo * (hi / lo) ** rng.random())))


def draw(rng):
    op = rng.choice(["embed", "loss", "loss"])
    kind = rng.choice(["step", "prompt", "train", "tied"] if op == "embed" else ["score", "train", "train"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    case = {"op": op, "kind": kind, "dtype": dtype, "ids": rng.choice(["i32", "i64"]), "left_out": rng.choice([0.0, 0.0, 0.1, 0.5, 0.9])}
    D = 8 * _size(rng, 8, 256)
    V = _size(rng, 100, 260000 * 1024 // max(D, 1024))
    if op == "embed":
        return case | {"T": _size(rng, 1, 256 if kind == "step" else 65536), "V": V, "D": D}
    # single precision and the gradients in it cost a multiple
    most = (1 << 39) // (8 if dtype == "f32" else 1)
    T = _size(rng, 1, max(1, min(16384, most // (V * D), (1 << 30) // V)))
    return case | {"T": T, "V": V, "D": D}


def work(case):
    T, V, D = case["T"], case["V"], case["D"]
    es, ids = DTYPES[case["dtype"]].itemsize, 8 if case["ids"] == "i64" else 4
    kept = max(1, round(T * (1 - case["left_out"])))
    if case["op"] == "embed":
        touched = min(kept, V)
        if case["kind"] == "train":   # a fresh gradient has all its rows
            return {"bytes": T * ids + kept * D * es + V * D * 4, "flops": kept * D}
        if case["kind"] == "tied":
            return {"bytes": T * ids + kept * D * es + V * D * 8, "flops": 2 * kept * D}
        return {"bytes": T * ids + touched * D * es + T * D * es, "flops": kept * D}
    product = 2 * kept * V * D
    if case["kind"] == "score":
        return {"bytes": (kept + V) * D * es + T * (ids + 8), "flops": product + 3 * kept * V}
    return {"bytes": 2 * (kept + V) * D * es + T * (ids + 12), "flops": 3 * product + 6 * kept * V}


# ------------------------------------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = DTYPES[case["dtype"]]
    T, V, D = case["T"], case["V"], case["D"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda")

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device="cuda")

    # token frequencies fall like one over the rank
    ids = (torch.exp(uniform(T).double() * math.log(V + 1)) - 1).long().clamp(0, V - 1)
    st = {"case": case}
    kept = torch.ones(T, dtype=torch.bool, device="cuda")
    if case["left_out"] > 0:
        # a padded tail and single tokens before it
        kept &= torch.arange(T, device="cuda") < max(1, round(T * (1 - case["left_out"] / 2)))
        kept &= uniform(T) >= case["left_out"] / 2
        ids = torch.where(kept, ids, torch.full_like(ids, -100))
    st["ids"] = ids if case["ids"] == "i64" else ids.int()
    if case["op"] == "embed":
        st["scale"] = math.sqrt(D)
        if case["kind"] in ("step", "prompt"):
            st["w"] = (normal(V, D) * D ** -0.5).to(dt)
        else:
            st["d_out"] = (normal(T, D) * 0.1 * (0.2 + uniform(T, 1))).to(dt)
        if case["kind"] == "tied":
            st["d_w"] = normal(V, D) * 0.01
        return st
    st["scale"] = 1.0
    w = (normal(V, D) * (1.5 * D ** -0.5)).to(dt)
    # hidden rows lean towards their target's weights, some hardly and some so far that the loss is next to nothing
    lean = 6 * uniform(T, 1) ** 2
    st["h"] = (normal(T, D) + lean * w[ids.clamp(min=0)].float()).to(dt)
    st["w"] = w
    if case["kind"] == "train":
        # a mean over the tokens with a weight for each
        weight = torch.where(kept, 0.5 + uniform(T), torch.zeros((), device="cuda"))
        st["d_loss"] = weight / kept.sum().clamp(min=1)
    return st


# ------------------------------------------------------------------------------------------------ plain forms

def _plain_embed(st):
    case, ids = st["case"], st["ids"].long()
    V, D = case["V"], case["D"]
    kept = (ids >= 0) & (ids < V)
    at = torch.where(kept, ids, torch.zeros_like(ids))
    if case["kind"] in ("step", "prompt"):
        rows = st["w"][at].float() * st["scale"]
        return torch.where(kept[:, None], rows, torch.zeros((), device=rows.device)).to(st["w"].dtype)
    add = torch.where(kept[:, None], st["d_out"].float() * st["scale"], torch.zeros((), device=at.device))
    d_w = torch.zeros(V, D, device=at.device) if case["kind"] == "train" else st["d_w"].clone()
    return d_w.index_add_(0, at, add)


def _plain_loss(st):
    case, ids, dt = st["case"], st["ids"].long(), st["h"].dtype
    kept = (ids >= 0) & (ids < case["V"])
    at = torch.where(kept, ids, torch.zeros_like(ids))[:, None]
    nothing = torch.zeros((), device=at.device)
    h, w = torch.where(kept[:, None], st["h"].float(), nothing), st["w"].float()
    z = h @ w.T
    z *= st["scale"]
    most = z.max(1, keepdim=True).values
    lse = (most + torch.log(torch.exp(z - most).sum(1, keepdim=True)))
    loss = torch.where(kept, (lse - z.gather(1, at))[:, 0], nothing)
    if case["kind"] == "score":
        return loss, torch.where(kept, lse[:, 0], nothing)
    z -= lse
    d_z = torch.exp_(z)
    d_z.scatter_add_(1, at, torch.full_like(lse, -1.0))
    d_z *= torch.where(kept, st["d_loss"] * st["scale"], nothing)[:, None]
    return loss, torch.where(kept, lse[:, 0], nothing), (d_z @ w).to(dt), (d_z.T @ h).to(dt)


# ------------------------------------------------------------------------------------------------ the library's calls

def _own_embed(st):
    from paper_2406_08128_b200 import chela
    case = st["case"]
    if case["kind"] in ("step", "prompt"):
        return chela.embed_fwd(st["ids"], st["w"], scale=st["scale"])
    if case["kind"] == "train":
        return chela.embed_bwd(st["ids"], st["d_out"], case["V"], scale=st["scale"], grad_dtype=chela.F32)
    return chela.embed_bwd(st["ids"], st["d_out"], case["V"], scale=st["scale"], grad_dtype=chela.F32, d_w_in=st["d_w"])


def _own_loss(st):
    from paper_2406_08128_b200 import chela
    case = st["case"]
    loss, lse = chela.vocabloss_fwd(st["h"], st["w"], st["ids"], scale=st["scale"])
    if case["kind"] == "score":
        return loss, lse
    g = chela.vocabloss_bwd(st["h"], st["w"], st["ids"], lse, st["d_loss"], scale=st["scale"],
                            grad_dtype=chela.BF16 if case["dtype"] == "bf16" else chela.F32)
    return loss, lse, g.d_h, g.d_w


def run(st):
    if own:
        return _own_embed(st) if st["case"]["op"] == "embed" else _own_loss(st)
    return _plain_embed(st) if st["case"]["op"] == "embed" else _plain_loss(st)


# ------------------------------------------------------------------------------------------------ 64 bits

def exact(case, seed):
    """The outputs from the definitions in 64 bits, a slice of tokens after another."""
    st = prepare(case, seed)
    T, V, D = case["T"], case["V"], case["D"]
    ids = st["ids"].long()
    valid = ((ids >= 0) & (ids < V)).nonzero()[:, 0]
    if case["op"] == "embed":
        if case["kind"] in ("step", "prompt"):
            out = torch.zeros(T, D, dtype=torch.float64, device="cuda")
            out[valid] = st["scale"] * st["w"][ids[valid]].double()
            return out
        d_w = st["d_w"].double() if case["kind"] == "tied" else torch.zeros(V, D, dtype=torch.float64, device="cuda")
        for part in valid.split(8192):
            d_w.index_put_((ids[part],), st["scale"] * st["d_out"][part].double(), accumulate=True)
        return d_w
    w = st["w"].double()
    loss, lse = (torch.zeros(T, dtype=torch.float64, device="cuda") for _ in range(2))
    train = case["kind"] == "train"
    if train:
        d_h, d_w = torch.zeros(T, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda")
    for part in valid.split(max(1, (1 << 28) // V)):
        h, y = st["h"][part].double(), ids[part]
        z = st["scale"] * torch.mm(h, w.t())
        lse[part] = torch.logsumexp(z, 1)
        loss[part] = lse[part] - z[torch.arange(len(part), device="cuda"), y]
        if train:
            p = torch.softmax(z, 1)
            p[torch.arange(len(part), device="cuda"), y] -= 1
            p *= (st["scale"] * st["d_loss"][part].double())[:, None]
            d_h[part] = torch.mm(p, w)
            d_w.addmm_(p.t(), h)
    return (loss, lse, d_h, d_w) if train else (loss, lse)
