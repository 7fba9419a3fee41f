"""The chunk attention with the kernel's operand roundings restated on the CPU, and what its other roundings may add to that.

Keys, values and queries are rounded to fp16 here as the kernel rounds them (dequantized elements once, c s + z); products, softmax and sums are in 64
bits.  What is left between this and the kernel is small enough that one key too many or too few shows.
"""
import numpy as np
import torch

import chunk_util as CU
from paper_2512_19206_b200 import workloads as W

HALF_STEP = 2.0 ** -11            # of fp16
TILE = 128


def fp16(x):
    """Rounded once to fp16, from 64 bits (torch would round to 32 bits first)."""
    return torch.from_numpy(np.asarray(x, np.float64).astype(np.float16).astype(np.float64))


def operands(st, kn, vn, qn):
    """Keys [T + n, 128], values, queries [g, n, 128] of one stream as the products take them."""
    K = torch.cat([fp16(st.keys()), fp16(kn.double().numpy())])
    V = torch.cat([fp16(st.values()), fp16(vn.double().numpy())])
    return K, V, fp16(qn.double().numpy())


def visible(held, n):
    return torch.arange(held + n)[None] <= held + torch.arange(n)[:, None]


def attend(K, V, q, scale, sees):
    s = (q @ K.T) * scale
    p = torch.softmax(s.masked_fill(~sees, float("-inf")), -1)
    return p, p @ V, s


def allowed(p, s, K, V, q, scale, deepest=516):
    """What the kernel's roundings may add, per output element.

    Probabilities are fp16, each rounded by at most HALF_STEP of itself, independently, in the product and in the denominator alike: six standard
    deviations of HALF_STEP / sqrt(3) of the root of sum (p (v - o))^2; below 2^-19 of the row's reference by 2^-30 of the reference instead, which is no
    more than the row's denominator: 2^-30 sum |v - o|.
    Sums in the tensor core lose at most a unit of 2^-23 for each of a tile's eight steps and one more for its products, over 512 tiles at most (then they
    are set aside).  A logit is such a sum (one tile
    deep), scaled and subtracted in fp32, and its exponential is good to 2^-21; a relative error d of the probabilities moves the output by at most
    d sum p |v - o|, here d sum p |v| twice.  Merging and dividing: 2^-20.  Equal logits give equal powers of two, which fp16 holds."""
    V1, flat = V.abs(), (q == 0).all(-1, keepdim=True)
    pv, o, p2 = p @ V1, p @ V, p * p
    apart = (p2 @ (V * V) - 2 * o * (p2 @ V) + o * o * p2.sum(-1, keepdim=True)).clamp_min(0)
    rounding = 6 / 3 ** 0.5 * HALF_STEP * apart.sqrt() + 2.0 ** -30 * (V1.sum(0) + V.shape[0] * o.abs())
    depth = ((q.abs() @ K.abs().T).amax(-1, keepdim=True)) * scale
    logit = 9 * 2.0 ** -23 * depth + 4 * 2.0 ** -23 * s.abs().amax(-1, keepdim=True) + 2.0 ** -21
    tiles = min(K.shape[0] / TILE + 4, deepest)
    return torch.where(flat, torch.zeros_like(pv), rounding + 2 * logit * pv) + (9 * tiles * 2.0 ** -23 + 2.0 ** -20) * pv


def reference(st, kn, vn, qn, scale):
    K, V, q = operands(st, kn, vn, qn)
    p, out, s = attend(K, V, q, scale, visible(K.shape[0] - kn.shape[0], kn.shape[0]))
    return out, allowed(p, s, K, V, q, scale)


def worst(out, ref, tol, step=0.0):
    """Largest error as a share of what is allowed; `step`: half a step of the output's type."""
    return float(((out - ref).abs() / (tol + step * ref.abs() + 2.0 ** -130)).max())


def check(w, out, sts, kn, vn, qn, counts, scale, only=None):
    """out [B, Hq, n, 128] against every stream; rows behind a count are the caller's affair."""
    step = 0.0 if out.dtype == torch.float32 else torch.finfo(out.dtype).eps / 2
    out, most = out.double().cpu(), 0.0
    for (b, hk), st in sts.items():
        m, hs = counts[b], slice(hk * w.g, (hk + 1) * w.g)
        if m == 0 or (only and (b, hk) not in only):
            continue
        assert torch.isfinite(out[b, hs, :m]).all(), f"stream {(b, hk)}: not finite"
        ref, tol = reference(st, kn[b, hk, :m], vn[b, hk, :m], qn[b, hs, :m], scale)
        share = worst(out[b, hs, :m], ref, tol, step)
        most = max(most, share)
        assert share <= 1.0, f"stream {(b, hk)}: {share:.2f} of what is allowed"
    return most


def simulated(K, V, q, scale, sees, lag=10.0, shift=5.0):
    """The kernel's arithmetic for one row after another: tiles of 128 keys in order, a reference that lags, fp16 probabilities, sums in 32 bits."""
    out = torch.empty(q.shape[0], q.shape[1], V.shape[1], dtype=torch.float64)
    c = np.float32(scale * np.log2(np.e))
    for h in range(q.shape[0]):
        for r in range(q.shape[1]):
            x = np.where(sees[r].numpy(), (q[h, r] @ K.T).numpy().astype(np.float32) * c, np.float32(-np.inf)).astype(np.float32)
            m, l, o = np.float32(-np.inf), np.float32(0), np.zeros(V.shape[1], np.float32)
            for t in range(0, len(x), TILE):
                mx = x[t:t + TILE].max()
                if mx > m + lag:
                    a = np.float32(np.exp2(m - mx))
                    m, l, o = mx, l * a, o * a
                p = np.exp2(x[t:t + TILE] - (m if np.isfinite(m) else 0) + np.float32(shift)).astype(np.float32)
                p = p.astype(np.float16)
                l += p.astype(np.float32).sum(dtype=np.float32)
                o += (p.astype(np.float64) @ V[t:t + TILE].numpy()).astype(np.float32)
            out[h, r] = torch.from_numpy(o / l).double()
    return out



def offset_keys(n4, tokens=330, n=6, R=64):
    """A stream whose keys' groups lie 3 to 18 scales below zero, n4 channels of it UINT4: there c_lo s + z has more bits than fp16 holds, while the
    element itself has not.  Returns (stream, new keys, values [n, 128], queries [2, n, 128] on the UINT4 channels)."""
    w = W.small(W.CONFIGS["tiny"], n_layers=1, n_q_heads=2, tokens=tokens, residual_len=R)
    gen = torch.Generator().manual_seed(n4)
    k = (-3 - 15 * torch.rand((1, 1, tokens, 128), generator=gen)).to(torch.bfloat16)
    v = torch.randn((1, 1, tokens, 128), generator=gen).to(torch.bfloat16)
    q = torch.randn((1, 2, tokens, 128), generator=gen)
    q[..., torch.randperm(128, generator=gen)[:n4]] *= 8          # the same channels in every window
    q = q.to(torch.bfloat16)
    st = CU.streams(w, [tokens], k, v, q, budget_u4=n4)[(0, 0)]
    st.source = (w, k, v, q)
    qn = (2 * torch.randn((2, n, 128), generator=gen) * torch.from_numpy(st.blocks[0].tiers == 1)).to(torch.bfloat16)
    kn, vn = k[0, 0, :n].clone(), v[0, 0, :n].clone()
    return st, kn, vn, qn
