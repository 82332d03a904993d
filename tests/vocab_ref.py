"""Plain float64 forms of the token embedding and the vocabulary's cross entropy, from their definitions, and bounds on how
far the kernels may be from them.  Tensors stay on the device that they are on.

Bounds count roundings against majorants (the same sums over absolute values).  A rounding to nearest is off by half a step:
2^-8 of the value for bf16, 2^-24 for fp32.  The tensor cores may cut an accumulator at every 16 terms: up to a step, 2^-23 of
what the sum's absolute values reach.
"""
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def kept_of(ids, V):
    ids = ids.long()
    return (ids >= 0) & (ids < V)


def embed(ids, w, scale):
    kept = kept_of(ids, w.shape[0])
    rows = scale * w[torch.where(kept, ids.long(), 0)].double()
    return torch.where(kept[..., None], rows, 0.0)


def embed_bwd(ids, d_out, V, scale, d_w_in=None, mag=False):
    """d_w, or its majorant and the largest number of tokens of a row."""
    kept = kept_of(ids, V)
    at = ids[kept].long()
    rows = scale * d_out[kept].double()
    d_w = torch.zeros(V, d_out.shape[-1], dtype=torch.float64, device=d_out.device) if d_w_in is None else d_w_in.double().clone()
    if mag:
        d_w, rows = d_w.abs(), rows.abs()
    return d_w.index_add_(0, at, rows)


def loss(h, w, targets, scale, d_loss=None, d_lse=None, d_w_in=None):
    """{loss, lse, d_h, d_w} and under the same names with a leading m the majorants: of a row's logits for m_z, of the sums for
    m_d_h and m_d_w."""
    T, V = h.shape[0], w.shape[0]
    kept = kept_of(targets, V)
    y = torch.where(kept, targets.long(), 0)[:, None]
    hd = torch.where(kept[:, None], h.double(), 0.0)
    wd = w.double()
    z = scale * torch.mm(hd, wd.t())
    lse = torch.logsumexp(z, 1)
    out = {"lse": torch.where(kept, lse, 0.0), "loss": torch.where(kept, lse - z.gather(1, y)[:, 0], 0.0),
           "m_z": scale * torch.mm(hd.abs(), wd.abs().t()).amax(1)}
    if d_loss is not None or d_lse is not None:
        g0 = torch.zeros(T, dtype=torch.float64, device=h.device) if d_loss is None else d_loss.double()
        g = g0 + (0.0 if d_lse is None else d_lse.double())
        p = torch.exp(z - lse[:, None])
        hot = torch.zeros_like(p).scatter_(1, y, 1.0)
        dz = torch.where(kept[:, None], scale * (g[:, None] * p - g0[:, None] * hot), 0.0)
        out["d_h"], out["d_w"] = torch.mm(dz, wd), torch.mm(dz.t(), hd)
        m = torch.where(kept[:, None], scale * (g.abs()[:, None] * p), 0.0)   # an error of p moves dz by this
        out["m_p_h"], out["m_p_w"] = torch.mm(m, wd.abs()), torch.mm(m.t(), hd.abs())
        out["m_d_h"], out["m_d_w"] = torch.mm(dz.abs(), wd.abs()), torch.mm(dz.abs().t(), hd.abs())
        if d_w_in is not None:
            out["d_w"] = out["d_w"] + d_w_in.double()
            out["m_d_w"] = out["m_d_w"] + d_w_in.double().abs()
    return out


def z_bound(r, D, in_dtype):
    """Of a logit: the accumulation (bf16: one step for 16 columns; fp32: the same within 256 columns, in registers beyond, and
    what six products of parts leave out, 3 2^-24), and the product with the scale."""
    steps = D / 16 + 2 if in_dtype is torch.bfloat16 else 6 * 16 + D / 256 + 4
    return (steps * 2.0 ** -23 + 4 * 2.0 ** -24) * r["m_z"]


def lse_bound(r, D, in_dtype):
    """A logit's bound, the approximate exponential and the sum of non-negative terms (2^-21 each at most), the logarithm and its
    last rounding."""
    return z_bound(r, D, in_dtype) + 2.0 ** -20 + 4 * 2.0 ** -24 * r["lse"].abs()


def grad_bounds(r, T, V, D, in_dtype, grad_dtype):
    """(of d_h, of d_w)"""
    rel = (z_bound(r, D, in_dtype) + lse_bound(r, D, in_dtype)).amax() + 2.0 ** -20   # of a softmax value
    half = HALF[grad_dtype]
    bounds = []
    for n, m_p, m, true in ((V, r["m_p_h"], r["m_d_h"], r["d_h"]), (T, r["m_p_w"], r["m_d_w"], r["d_w"])):
        if grad_dtype is torch.bfloat16:   # dz to bf16, and fp32 operands to two parts
            steps, parts = (n / 16 + 2) * 2.0 ** -23, half + 2.0 ** -16
        else:
            steps, parts = (6 * 16 + n / 256 + 64) * 2.0 ** -23, 4 * 2.0 ** -24
        bounds.append(rel * m_p + (steps + parts) * m + half * 1.01 * true.abs() + 1e-37)
    return bounds
