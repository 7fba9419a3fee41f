"""Plain 64-bit chunk attention over what the oracle's streams hold, and the error that the kernel's roundings allow."""
import numpy as np
import torch

import gpu_util as U
from oracle import mixkvq_oracle as O
from paper_2512_19206_b200 import workloads as W

HALF_STEP = 2.0 ** -11            # of fp16: dequantized keys and values and the probabilities are rounded to it


def streams(w, lens, k, v, q, **kw):
    """{(b, hk): OracleStream} after the first lens[b] tokens of k, v, q (CPU bf16 tensors)."""
    out = {}
    for b, t in enumerate(lens):
        for hk in range(w.n_kv_heads):
            st = U.oracle_stream(w, **kw)
            if t:
                st.append_many(U.f32(k[b, hk, :t]), U.f32(v[b, hk, :t]), U.f32(q[b, hk * w.g:(hk + 1) * w.g, :t]))
            out[(b, hk)] = st
    return out


def reference(st, kn, vn, qn, scale):
    """One stream: new keys and values [n, 128], queries [g, n, 128] (bf16) -> (output [g, n, 128], allowed error [g, n, 1]) in 64 bits."""
    K = torch.cat([torch.from_numpy(st.keys()), kn.double()])
    V = torch.cat([torch.from_numpy(st.values()), vn.double()])
    held, n = K.shape[0] - kn.shape[0], kn.shape[0]
    q = qn.double()
    s = (q @ K.T) * scale
    s.masked_fill_(torch.arange(held + n)[None] > held + torch.arange(n)[:, None], float("-inf"))
    p = torch.softmax(s, -1)
    return p @ V, allowed(p, q, K, V, scale)


def allowed(p, q, K, V, scale):
    """A logit is a sum of 128 products whose key was rounded by at most HALF_STEP each, independently: a deviation of at most HALF_STEP scale
    sqrt(sum (q k)^2).  The output moves by sum_t p_t d_t (v_t - o), and by the roundings of p_t and v_t: at most that deviation + 2 HALF_STEP
    times |p|_2 max |v - o| or max |v|.  Eight of these, and what fp32 sums of unit weights lose (the tensor core's accumulation truncates: half a unit of
    2^-23 for each of the 8 products of a tile, twice for the two sums)."""
    dev = HALF_STEP * scale * torch.sqrt(((q * q) @ (K * K).T).amax(-1, keepdim=True))
    big = float(V.abs().max())
    tiles = K.shape[0] / 128 + 4
    return 8 * (2 * dev + 2 * HALF_STEP) * p.square().sum(-1, keepdim=True).sqrt() * big + 16 * tiles * 2.0 ** -23 * big


def check(w, out, sts, kn, vn, qn, counts, scale=None, only=None):
    """Compares out [B, Hq, n, 128] with the oracle's streams; rows behind a count are the caller's affair."""
    scale = scale or W.softmax_scale()
    step = {torch.bfloat16: 2.0 ** -8}.get(out.dtype, 0.0)
    out = out.double().cpu()
    for (b, hk), st in sts.items():
        m = counts[b]
        if m == 0 or (only and (b, hk) not in only):
            continue
        hs = slice(hk * w.g, (hk + 1) * w.g)
        ref, tol = reference(st, kn[b, hk, :m], vn[b, hk, :m], qn[b, hs, :m], scale)
        err = (out[b, hs, :m] - ref).abs()
        assert torch.isfinite(out[b, hs, :m]).all(), f"stream {(b, hk)}: not finite"
        worst = (err / (tol + step * ref.abs())).max()
        assert worst <= 1.0, f"stream {(b, hk)}: {float(worst):.2f} of the allowed error (max abs {float(err.max()):.2e})"
