"""The paged 4-bit cache in plain form: what a pool's bytes have to be, attention over it in 64 bits, and the error that the kernels' roundings allow."""
import numpy as np
import torch

from oracle import mixkvq_oracle as O

D = 128


def f32(t):
    return t.detach().float().cpu().numpy()


def rotate(x, cos, sin, positions, interleaved=False):
    """x [B, H, n, 128] bf16 (CPU), tables float32 numpy, positions [B, n] numpy -> bf16: single fp32 operations, one rounding."""
    y, half = f32(x).copy(), cos.shape[1]
    c, s = cos[positions][:, None], sin[positions][:, None]
    a = (slice(0, 2 * half, 2) if interleaved else slice(0, half))
    b = (slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half))
    u, w = y[..., a].copy(), y[..., b].copy()
    y[..., a] = (u * c).astype(np.float32) - (w * s).astype(np.float32)
    y[..., b] = (w * c).astype(np.float32) + (u * s).astype(np.float32)
    return torch.from_numpy(y).to(torch.bfloat16)


def quantized(x, G):
    """Rows [..., 128] bf16 -> codes uint8 [..., 128], s, z float32 [..., 128 / G]."""
    c, s, z = O.quantize_groups(f32(x).reshape(*x.shape[:-1], D // G, G), 4)
    return c.reshape(*x.shape[:-1], D), s, z


def values(c, s, z):
    g = s.shape[-1]
    return (c.reshape(*c.shape[:-1], g, D // g).astype(np.float64) * s[..., None].astype(np.float64) + z[..., None].astype(np.float64)).reshape(c.shape)


def token_bytes(x, G, values_of, row):
    """The 64 bytes of codes and the scale words of one token's row x [128] (bf16) in slot `row` of its tile."""
    c, s, z = quantized(x, G)
    out = np.zeros(64, np.uint8)
    for ch in range(D):
        j = ch // 32
        if values_of:
            at = (8 * (ch % 32 // 4) + 2 * j + ch % 4 // 2) ^ (32 if row & 4 else 0)
        else:
            at = 16 * (ch // 8 % 4) + 4 * j + ch % 8 // 2
        out[at] |= c[ch] << (4 * (ch % 2))
    meta = np.stack([O.bf16_to_u16(z), O.bf16_to_u16(s)], -1).astype("<u2").tobytes()
    return out.tobytes(), meta


def place(cfg, layer, page, head, slot):
    """Byte offsets (from the start of the pool) of a token: K codes, V codes, K scales, V scales."""
    meta = 512 // cfg.group_size
    tile = 2048 + 32 * meta
    piece = tile * cfg.page_tokens // 16
    at = 256 + ((layer * cfg.n_pages + page) * cfg.n_kv_heads + head) * piece + slot // 16 * tile
    row = slot % 16
    return at + 64 * row, at + 1024 + 64 * row, at + 2048 + meta * row, at + 2048 + meta * (16 + row)


def pages_for(lens, page_tokens, seed, spare=3, extra=0):
    """A page table int32 [B, P] (CPU) with the pages in any order, -1 behind a sequence's last (`extra` columns of that beyond the longest), and the number of pages."""
    each = [-(-t // page_tokens) for t in lens]
    n = sum(each) + spare
    order = torch.randperm(n, generator=torch.Generator().manual_seed(seed))
    table = torch.full((len(lens), max(1, max(each)) + extra), -1, dtype=torch.int32)
    at = 0
    for b, m in enumerate(each):
        table[b, :m] = order[at:at + m].to(torch.int32)
        at += m
    return table, n


def draw(B, Hq, Hkv, n, seed, outliers=True):
    """q [B,Hq,n,128], k, v [B,Hkv,n,128] bf16 (CPU)."""
    gen = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn((B, h, n, D), generator=gen) for h in (Hq, Hkv, Hkv))
    if outliers:
        k[..., torch.randperm(D, generator=gen)[:4]] *= 20.0
    return tuple(t.to(torch.bfloat16) for t in (q, k, v))


HALF_STEP = 2.0 ** -11        # of fp16: the weights of the values are rounded to it, once per token and group


def unpacked(p, qd, K, V, scale):
    """What rounding the elements of keys and values to fp16 once, independently, may add: a logit is a sum of 128 products, its deviation d at most HALF_STEP scale
    sqrt(sum (q k)^2) by size of a standard deviation; the output moves by sum_t p_t d_t (v_t - o), and by the roundings of p_t and v_t: at most 2 d + 2 HALF_STEP times |p|_2
    max |v|.  Eight of these, and the truncation of the tensor core's sums: half a unit of 2^-23 for each of the 8 products of a tile of 128 tokens, twice for the two sums."""
    dev = HALF_STEP * scale * torch.sqrt(((qd * qd) @ (K * K).T).amax(-1, keepdim=True))
    big = float(V.abs().max()) if V.numel() else 0.0
    return 8 * (2 * dev + 2 * HALF_STEP) * p.square().sum(-1, keepdim=True).sqrt() * big + 16 * (K.shape[0] / 128 + 4) * 2.0 ** -23 * big


def reference(q, k, v, G, scale, sees, rounded=False):
    """One KV head: q [g, m, 128], k, v [T, 128] (bf16 rows as appended), sees [m]: the tokens that each row sees -> (output [g, m, 128], allowed error) in 64 bits.

    Logits: keys' codes and queries enter exactly; sums of 128 products in fp32 and of the groups' parts lose at most 2^-19 of the sum of the magnitudes |q| (15 s + |z|)
    (fewer than 16 roundings or truncations of 2^-23 each); a deviation d of all logits moves the output by at most 2 d max |v - o|.
    Weights: p s is rounded to fp16 once per token and group, times a power of two that brings the group's largest s to 2^5 at least: by 2^-11 of itself, so the output
    by 2^-11 sum p 15 s; where that is below 2^-14 by 2^-25, 2^-30 of the largest s, so by 2^-26 of it per token and code (the reference is never above a row's largest
    logit, its denominator at least 1).  Sums in fp32: 2^-18 of sum p (15 s + |z|)."""
    kc, ks, kz = quantized(k, G)
    vc, vs, vz = quantized(v, G)
    K, V = torch.from_numpy(values(kc, ks, kz)), torch.from_numpy(values(vc, vs, vz))
    reach = lambda s, z: torch.from_numpy(np.repeat(15.0 * s.astype(np.float64) + np.abs(z.astype(np.float64)), G, -1))         # noqa: E731
    qd = q.double()
    logits = (qd @ K.T) * scale
    T = K.shape[0]
    hidden = torch.arange(T)[None] >= torch.as_tensor(sees)[:, None]
    logits.masked_fill_(hidden, float("-inf"))
    p = torch.softmax(logits, -1)
    p = torch.where(hidden.all(-1)[:, None].expand_as(p), 0.0, p)
    # values beyond the type's range (a group whose range overflows) reach the rows that see them and no others
    lost = (~hidden).double() @ (~torch.isfinite(V)).double() > 0
    V = torch.where(torch.isfinite(V), V, 0.0)
    out = torch.where(lost, float("nan"), p @ V)
    d = 2.0 ** -19 * scale * (qd.abs() @ reach(ks, kz).T).masked_fill(hidden, 0.0).amax(-1, keepdim=True)
    s15 = torch.from_numpy(np.repeat(15.0 * vs.astype(np.float64), G, -1))
    s15 = torch.where(torch.isfinite(s15), s15, 0.0)
    biggest = float(s15.max()) if T else 0.0
    tol = 2 * d * (V.abs().max() if T else 0.0) + HALF_STEP * (p @ s15) + 2.0 ** -26 * biggest * T + 2.0 ** -18 * (p @ torch.nan_to_num(reach(vs, vz), 0.0, 0.0, 0.0))
    if rounded:
        tol = tol + unpacked(p, qd, K, V, scale)
    return out, tol


def check(out, q, k, v, G, scale, lens, counts, rounded=False):
    """out [B,Hq,n,128] (any device) against rows q [B,Hq,n,128] over the first lens[b] tokens of k, v [B,Hkv,T,128] (CPU, as appended).
    rounded: by the kernel that unpacks keys and values to fp16 (PagedCache.last_attention)."""
    step = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}[out.dtype]
    out = out.double().cpu()
    g = q.shape[1] // k.shape[1]
    for b, (t, m) in enumerate(zip(lens, counts)):
        for h in range(k.shape[1]):
            if m == 0:
                continue
            hs = slice(h * g, h * g + g)
            sees = [max(0, t - m + i + 1) for i in range(m)]
            ref, tol = reference(q[b, hs, :m], k[b, h, :t], v[b, h, :t], G, scale, sees, rounded)
            got = out[b, hs, :m]
            fine = torch.isfinite(ref)
            assert torch.equal(torch.isfinite(got), fine), f"sequence {b}, head {h}: not finite"
            worst = ((got - ref).abs() / (tol + step * ref.abs() + 1e-37))[fine].max() if fine.any() else 0.0
            assert worst <= 1.0, f"sequence {b}, head {h}: {float(worst):.2f} of the allowed error (max abs {float((got - ref).abs().max()):.2e})"
