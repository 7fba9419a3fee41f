"""Timed cases of the operators for tokens that arrive at a cache which already holds some.

  chunk   `Cache.chunk_attention`: n new tokens per sequence attend to everything the layer holds (sink, packed blocks,
          residual window) and, causally, to themselves; nothing is appended.  Chunks of a long prompt, and drafted tokens
          whose acceptance is decided afterwards.
  rope    `Cache.rope_axes`: rotary positions with one coordinate per axis (time, height, width), from the fused projection's
          output [B, n, Hq + 2 Hkv, 128] or from head-major tensors into the head-major q, k, v that the cache's calls take.

Shapes are those of the model shapes in `workloads.CONFIGS`, inputs follow its recipe (N(0,1) in bf16, four outlier key channels
per KV head scaled by 10 to 30, query gains log-uniform in [0.5, 4]), drawn on the GPU from the seed.  The plain form holds what the cache
holds: codes, scales, zero-points and full-precision rows.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
# Query and KV heads of the model shapes.
SHAPES = {"tiny": (1, 1), "qwen7b": (28, 4), "llama8b": (32, 8), "qwen32b": (40, 8)}
# (tau_bf16, tau_u4, score_bits), and the BF16 and UINT4 channels per block that they give on these inputs
PRESETS = {"P24": ((6.5, 1e30, 2), 4, 0), "P27": ((6.5, 3.8, 2), 4, 22), "P4BASE": ((1.3, -1.0, 4), 4, 124)}
SECTIONS = {"split": (16, 24, 24), "interleaved": (24, 20, 20), "one": (64,)}


def _chunk(**kw):
    c = dict(op="chunk", model="qwen7b", lens="32768", counts="1", preset="P24", R=128, G=32, v_bits=2, sink=0)
    c.update(kw)
    return c


def _rope(**kw):
    c = dict(op="rope", model="qwen7b", batch=1, n=1, axes="split", layout="projection", image=1024)
    c.update(kw)
    return c


def listed():
    return [
        # four drafted tokens behind one short sequence on the smallest configuration: launches and latency
        _chunk(name="draft-tiny", model="tiny", lens="1024", counts="4"),
        # drafted tokens of a serving batch: the 7B shape at 32K tokens, five tokens per sequence
        _chunk(name="draft-7b", lens=",".join(["32768"] * 8), counts=",".join(["5"] * 8)),
        # drafts of unequal number behind sequences of unequal length, one of them without any
        _chunk(name="draft-ragged", lens="32768,29000,23500,17000,12345,9000,4097,640", counts="8,3,5,1,0,7,2,8", preset="P27"),
        # one token for one very long sequence, as decode does it
        _chunk(name="single-long", model="llama8b", lens="120000", counts="1"),
        # the first chunk of a prompt: the cache is empty
        _chunk(name="chunk-first", model="llama8b", lens="0", counts="2000"),
        # a later chunk of a long prompt: the most work
        _chunk(name="chunk-7b", lens="32768", counts="2048"),
        # chunks of a few prompts at odd lengths with the optional settings: 4-bit values, a sink, short windows
        _chunk(name="chunk-options", model="llama8b", lens="6001,4500,777", counts="333,256,512", preset="P4BASE", R=64, G=64, v_bits=4, sink=32),
        # the large model's shape, whole key groups of 128 tokens
        _chunk(name="chunk-32b", model="qwen32b", lens="9000,9000", counts="512,512", G=128),
        # the new token of every sequence of a decode batch
        _rope(name="rope-step", batch=8),
        # an odd number of tokens of a few prompts with interleaved axes, already head-major
        _rope(name="rope-prompts", model="llama8b", batch=4, n=777, axes="interleaved", layout="heads"),
        # a picture in a prompt
        _rope(name="rope-image", n=4000, image=2000),
        # a video: most of the prompt is frames
        _rope(name="rope-video", model="qwen32b", batch=2, n=16384, image=15000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    if rng.random() < 0.35:
        n = _log_int(rng, 1, 16384)
        return _rope(model=rng.choice(["qwen7b", "llama8b", "qwen32b"]), batch=max(1, min(_log_int(rng, 1, 64), 32768 // n)), n=n,
                     axes=rng.choice(list(SECTIONS)), layout=rng.choice(["projection", "heads"]), image=_log_int(rng, 1, 16384))
    model = rng.choice(["qwen7b", "llama8b", "qwen32b", "tiny"])
    hq, hkv = SHAPES[model]
    G = rng.choice([32, 32, 64, 128])
    R = max(G, rng.choice([128, 128, 32, 64, 256]))
    opts = dict(model=model, R=R, G=G, preset=rng.choice(["P24", "P24", "P27", "P4BASE"]), v_bits=rng.choice([2, 2, 4]), sink=rng.choice([0, 0, 32]))
    batch = rng.choice([1, 1, 2, 3, 5, 8])
    n = rng.choice([_log_int(rng, 1, 16), _log_int(rng, 1, 2048)])
    # neither more cached tokens nor more products than the largest listed cases
    most = min(120000, 262144 * 4 // (batch * hkv), 33000 * 2048 * 28 // (n * hq * batch))
    longest = _log_int(rng, 1, max(2, most))
    if rng.random() < 0.1:
        longest = 0
    ragged = batch > 1 and rng.random() < 0.5
    lens = [rng.randint(0, longest) if ragged else longest for _ in range(batch)]
    counts = [rng.randint(0, n) if ragged else n for _ in range(batch)]
    counts[0] = n
    return _chunk(lens=",".join(map(str, lens)), counts=",".join(map(str, counts)), **opts)


def _ints(text):
    return [int(x) for x in text.split(",")]


# ------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _chunk_inputs(case, seed):
    """History k, v, q of the longest length and the chunk's k, v, q, head-major."""
    hq, hkv = SHAPES[case["model"]]
    lens, counts = _ints(case["lens"]), _ints(case["counts"])
    B, T, n = len(lens), max(lens), max(counts)
    gen, host = _generator(seed), torch.Generator()
    host.manual_seed(seed)
    gk = torch.ones(hkv, 1, D)
    for h in range(hkv):
        gk[h, 0, torch.randperm(D, generator=host)[:4]] = 10.0 + 20.0 * torch.rand(4, generator=host)
    gq = (0.5 * torch.pow(8.0, torch.rand(hkv, 1, D, generator=host))).repeat_interleave(hq // hkv, 0)
    gq = gq * (0.8 + 0.45 * torch.rand(hq, 1, 1, generator=host))
    gk, gq = gk.cuda().bfloat16(), gq.cuda().bfloat16()

    def tokens(m):
        return _normal(gen, B, hkv, m, D).mul_(gk), _normal(gen, B, hkv, m, D), _normal(gen, B, hq, m, D).mul_(gq)
    return tokens(T), tokens(n)


def _fill(case, length):
    """(sink, packed, residual) tokens of a sequence of `length` tokens: full windows are packed when the next token comes."""
    sink = min(length, case["sink"])
    res = (length - sink - 1) % case["R"] + 1 if length > sink else 0
    return sink, length - sink - res, res


def _over(x, number):
    """x / number, divided: by a host number it would be multiplied with a rounded reciprocal."""
    return x / torch.full((), number, dtype=x.dtype, device=x.device)


def _groups(x, bits):
    """Codes, scales and zero-points of groups along the last dimension: z the minimum, s the range over the levels rounded up to bf16."""
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s = _over(hi - lo, 2 ** bits - 1)
    down = (s.view(torch.int32) & -65536)
    s = torch.where(down == s.view(torch.int32), down, down + 65536).view(torch.float32)
    c = ((x - lo) / torch.where(s == 0, torch.ones_like(s), s)).round().clamp(0, 2 ** bits - 1)
    return c, s, lo


def _held(case, k, v, q):
    """What a cache holds after these tokens: per sequence its sink, packed and residual rows, each padded to the longest of the batch."""
    hq, hkv = SHAPES[case["model"]]
    R, G, g = case["R"], case["G"], hq // hkv
    (tau16, tau4, score_bits), fills = PRESETS[case["preset"]][0], [_fill(case, t) for t in _ints(case["lens"])]
    B, sink, packed = len(fills), max(f[0] for f in fills), max(f[1] for f in fills)
    nb = packed // R
    kp, vp = (x[:, :, sink:sink + packed].float() for x in (k, v))
    s = {"sink": sink, "packed": packed, "fills": torch.tensor(fills, device="cuda")}
    # the channels' tiers: mean |q| over the window and the group's heads times the keys' range over the window's levels
    mags = torch.stack([x[:, sink:sink + packed].reshape(hkv, g, nb, R, D).abs().sum((1, 3), dtype=torch.float64) for x in q])
    win = kp.view(B, hkv, nb, R, D)
    sal = _over(mags, g * R) * _over(win.amax(3).double() - win.amin(3).double(), 2 ** score_bits - 1)
    f32 = lambda t: float(torch.tensor(t, dtype=torch.float32))                   # noqa: E731
    exactly, four = sal > f32(tau16), (sal > f32(tau4)) & ~(sal > f32(tau16))
    keys = kp.view(B, hkv, nb, R // G, G, D).transpose(-1, -2).contiguous()       # groups of G tokens of a channel
    two, more = _groups(keys, 2), _groups(keys, 4)
    pick = four[:, :, :, None, :, None]
    s["kc"], s["ks"], s["kz"] = (torch.where(pick, b, a) for a, b in zip(two, more))
    s["kc"] = s["kc"].to(torch.uint8)
    s["k_exact"] = exactly
    s["k16"] = k[:, :, sink:sink + packed].contiguous()
    s["vc"], s["vs"], s["vz"] = _groups(vp.view(B, hkv, packed, D // G, G), case["v_bits"])
    s["vc"] = s["vc"].to(torch.uint8)
    # the unquantized rows: sink, then the window, wherever it lies in each sequence
    rows = torch.zeros(B, sink + R, dtype=torch.long, device="cuda")
    rows[:, :sink] = torch.arange(sink, device="cuda")
    for b, (sk, pk, _) in enumerate(fills):
        rows[b, sink:] = sk + pk + torch.arange(R, device="cuda")
    if k.shape[2]:
        at = rows.clamp(max=k.shape[2] - 1)[:, None, :, None].expand(B, hkv, sink + R, D)
        s["kr"], s["vr"] = k.gather(2, at), v.gather(2, at)
    else:
        s["kr"], s["vr"] = (x.new_zeros(B, hkv, sink + R, D) for x in (k, v))
    return s


def _rope_inputs(case, seed):
    hq, hkv = SHAPES[case["model"]]
    B, n, sections = case["batch"], case["n"], SECTIONS[case["axes"]]
    gen, host = _generator(seed), torch.Generator()
    host.manual_seed(seed)
    x = _normal(gen, B, n, hq + 2 * hkv, D)
    if case["layout"] == "heads":
        q, k, _ = (t.transpose(1, 2).contiguous() for t in x.split((hq, hkv, hkv), 2))
        v = None                                             # it is where it belongs
    else:
        q, k, v = (t.transpose(1, 2) for t in x.split((hq, hkv, hkv), 2))
    # text up to the picture, then frames of w by h patches at one time each, then text again
    start = torch.randint(0, 4096, (B, 1), generator=host)
    image = min(case["image"], n)
    w = max(1, int(math.sqrt(min(image, 1024))))
    t0 = (n - image) // 2
    i = torch.arange(n)
    inside = (i >= t0) & (i < t0 + image)
    j = (i - t0).clamp(0, max(image - 1, 0))
    after = torch.where(i < t0, i, i - image + w + 1)
    coords = [t0 + j // (w * w), t0 + (j % (w * w)) // w, t0 + j % w]
    pos = torch.stack([torch.where(inside, c, after)[None] + start for c in coords[:len(sections)]]).to(torch.int32)
    n_pos = int(pos.max()) + 1
    angle = torch.arange(n_pos, device="cuda", dtype=torch.float64)[:, None] * torch.pow(1e6, -torch.arange(64, device="cuda", dtype=torch.float64) / 64)
    if case["axes"] == "interleaved":
        pairs, left = [], list(sections)
        while len(pairs) < 64:
            for a in range(len(left)):
                if left[a] and len(pairs) < 64:
                    pairs.append(a)
                    left[a] -= 1
    else:
        pairs = [a for a, m in enumerate(sections) for _ in range(m)]
    return dict(q=q, k=k, v=v, positions=pos.cuda(), cos=angle.cos().float(), sin=angle.sin().float(), pairs=pairs)


def _make_cache(case, batch, max_tokens):
    from paper_2512_19206_b200 import binding
    hq, hkv = SHAPES[case["model"]]
    tau16, tau4, score_bits = PRESETS[case.get("preset", "P24")][0]
    R = case.get("R", 128)
    budget = (max_tokens // R + 3) * 64 * R if case.get("preset") == "P4BASE" else 0      # a dense high plane per block
    return binding.Cache(binding.make_config(1, batch, hq, hkv, max(max_tokens, 1), residual_len=R, group_size=case.get("G", 32), tau_bf16=tau16,
                                             tau_u4=tau4, score_bits=score_bits, v_bits=case.get("v_bits", 2), sink_len=case.get("sink", 0),
                                             extras_budget_bytes=budget))


def prepare(case, seed):
    if case["op"] == "rope":
        s = _rope_inputs(case, seed)
        s["case"] = case
        hq, hkv = SHAPES[case["model"]]
        s["out"] = tuple(torch.empty(case["batch"], h, case["n"], D, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
        if s["v"] is None:
            s["out"] = (*s["out"][:2], None)
        s["axis_of"] = torch.tensor(s["pairs"], device="cuda")
        if own:
            s["cache"] = _make_cache(case, case["batch"], 1)
        return s
    hq, _ = SHAPES[case["model"]]
    lens, counts = _ints(case["lens"]), _ints(case["counts"])
    (k, v, q), new = _chunk_inputs(case, seed)
    s = {"case": case, "new": new, "counts": counts, "out": torch.zeros_like(new[2])}
    if own:
        cache = s["cache"] = _make_cache(case, len(lens), max(lens))
        if max(lens):
            cache.quantize_append_ragged(0, k, v, q, lens)
        s["scratch"] = torch.empty(cache.chunk_scratch_bytes(max(counts)), dtype=torch.uint8, device="cuda")
    else:
        s["held"] = _held(case, k, v, q)
        s["n"] = torch.tensor(counts, device="cuda")
    return s


# ------------------------------------------------------------------------------------------------------- plain forms
def _plain_rope(s):
    def rows(table):
        p = s["positions"].long()[s["axis_of"]]                                    # [64, B, n]
        return table[p, torch.arange(64, device="cuda")[:, None, None]].permute(1, 2, 0)[:, None]
    c, n = rows(s["cos"]), rows(s["sin"])

    def rotated(x):
        a, b = x.float().split(64, -1)
        return torch.cat([a * c - b * n, b * c + a * n], -1).to(torch.bfloat16)
    return rotated(s["q"]), rotated(s["k"]), None if s["v"] is None else s["v"].contiguous()


def _plain_chunk(s):
    case, h, (kn, vn, q) = s["case"], s["held"], s["new"]
    B, hkv, n, _ = kn.shape
    sink, packed, R = h["sink"], h["packed"], case["R"]
    keys = (h["kc"].float() * h["ks"] + h["kz"]).transpose(-1, -2).reshape(B, hkv, packed, D)
    keys = torch.where(h["k_exact"].repeat_interleave(R, 2), h["k16"].float(), keys)
    vals = (h["vc"].float() * h["vs"] + h["vz"]).view(B, hkv, packed, D)
    keys, vals = torch.cat([h["kr"].float(), keys, kn.float()], 2), torch.cat([h["vr"].float(), vals, vn.float()], 2)
    f, i = h["fills"], torch.arange(max(sink, R, packed, n), device="cuda")
    there = torch.cat([i[:sink] < f[:, :1], i[:R] < f[:, 2:], i[:packed] < f[:, 1:2]], 1)                # [B, cached rows]
    sees = torch.cat([there[:, None].expand(B, n, -1), (i[None, :n] <= i[:n, None]).expand(B, n, n)], 2)      # [B, n, rows]
    logits = (q.float().view(B, hkv, -1, D) @ keys.transpose(-1, -2)).view(B, hkv, -1, n, keys.shape[2]).mul_(SCALE)
    logits.masked_fill_(~sees[:, None, None], float("-inf"))
    p = logits.sub_(logits.amax(-1, keepdim=True)).exp_()
    p.div_(p.sum(-1, keepdim=True))
    out = (p.view(B, hkv, -1, p.shape[-1]) @ vals).view(q.shape).to(torch.bfloat16)
    return torch.where((i[:n] < s["n"][:, None])[:, None, :, None], out, s["out"])        # rows past a sequence's count stay as they were


def run(state):
    s = state
    if s["case"]["op"] == "rope":
        if not own:
            return _plain_rope(s)
        return s["cache"].rope_axes(s["q"], s["k"], s["v"], s["cos"], s["sin"], s["positions"], s["pairs"], out=s["out"])
    if not own:
        return _plain_chunk(s)
    k, v, q = s["new"]
    return s["cache"].chunk_attention(0, k, v, q, SCALE, counts=s["counts"], out=s["out"], scratch=s["scratch"])


# ------------------------------------------------------------------------------------------------------- the definition in 64 bits
def _exact_group(x, bits):
    """Dequantized values (64 bits) of the rows of x [..., group], from the definition: codes are the rounded single-precision quotient."""
    top = 2 ** bits - 1
    z = x.min(dim=-1, keepdim=True).values
    step = (x.max(dim=-1, keepdim=True).values - z).div(torch.tensor(float(top), device="cuda"))
    frac, e = torch.frexp(step.double())                         # round up to 8 significant bits
    step = torch.ldexp(torch.ceil(frac * 256), e - 8).float()
    code = torch.where(step > 0, ((x - z) / step.clamp_min(1e-38)).round(), torch.zeros_like(x)).clamp(0, top)
    return code.double() * step.double() + z.double()


def _exact_cache(case, length, k, v, q):
    """Keys and values [length, 128] that a stream of `length` tokens answers with; q [g, length, 128]."""
    (tau16, tau4, score_bits), _, _ = PRESETS[case["preset"]]
    R, G = case["R"], case["G"]
    sink, packed, _ = _fill(case, length)
    keys, vals = k[:length].double(), v[:length].double()
    tau16, tau4 = (torch.tensor(t, dtype=torch.float32, device="cuda").double() for t in (tau16, tau4))
    nb = packed // R
    if nb == 0:
        return keys, vals
    body = slice(sink, sink + packed)
    win = k[body].float().reshape(nb, R, D)
    spread = win.double().max(1).values - win.double().min(1).values
    use = q[:, body].double().abs().reshape(-1, nb, R, D).sum(2).sum(0).div(torch.tensor(q.shape[0] * R, device="cuda"))
    gain = use * spread.div(torch.tensor(2 ** score_bits - 1, device="cuda"))        # [nb, 128]
    cols = win.reshape(nb, R // G, G, D).permute(0, 1, 3, 2)
    low, high = _exact_group(cols, 2), _exact_group(cols, 4)
    gain = gain[:, None, :, None]
    mixed = torch.where(gain > tau16, cols.double(), torch.where(gain > tau4, high, low))
    keys[body] = mixed.permute(0, 1, 3, 2).reshape(packed, D)
    vals[body] = _exact_group(v[body].float().reshape(packed, D // G, G), case["v_bits"]).reshape(packed, D)
    return keys, vals


def exact(case, seed):
    hq, hkv = SHAPES[case["model"]]
    g = hq // hkv
    if case["op"] == "rope":
        s = _rope_inputs(case, seed)
        idx = torch.arange(64, device="cuda")
        pos = torch.stack([s["positions"][a] for a in s["pairs"]], -1).long()        # [B, n, 64]
        unit = torch.complex(s["cos"][pos, idx].double(), s["sin"][pos, idx].double())[:, None]

        def turn(x):
            z = torch.complex(x[..., :64].double(), x[..., 64:].double()) * unit
            return torch.cat((z.real, z.imag), -1)
        return turn(s["q"]), turn(s["k"]), None if s["v"] is None else s["v"].double()
    lens, counts = _ints(case["lens"]), _ints(case["counts"])
    (k, v, q), (kn, vn, qn) = _chunk_inputs(case, seed)
    out = torch.zeros(qn.shape, dtype=torch.float64, device="cuda")
    for b, (length, m) in enumerate(zip(lens, counts)):
        for h in range(hkv):
            heads = slice(h * g, h * g + g)
            ck, cv = _exact_cache(case, length, k[b, h], v[b, h], q[b, heads])
            kk, vv = torch.cat([ck, kn[b, h, :m].double()]), torch.cat([cv, vn[b, h, :m].double()])
            hidden = torch.arange(length + m, device="cuda")[None] > length + torch.arange(m, device="cuda")[:, None]
            for a in range(g if m else 0):
                s = (qn[b, h * g + a, :m].double() @ kk.T) * SCALE
                out[b, h * g + a, :m] = torch.softmax(s.masked_fill(hidden, -math.inf), -1) @ vv
    return out


# ------------------------------------------------------------------------------------------------------- work
def _packed_token_bytes(case):
    """Bytes of one packed token of one KV head: key codes at their tiers, value codes, scales and zero-points."""
    _, n16, n4 = PRESETS[case["preset"]]
    G, n2 = case["G"], D - n16 - n4
    return (2 * n16 + n4 / 2 + n2 / 4 + 4 * (n4 + n2) / G) + (D * case["v_bits"] / 8 + 4 * D / G)


def work(case):
    hq, hkv = SHAPES[case["model"]]
    if case["op"] == "rope":
        B, n = case["batch"], case["n"]
        rows = B * n * (hq + (2 if case["layout"] == "projection" else 1) * hkv)
        return {"bytes": 2 * 2.0 * D * rows + 4.0 * len(SECTIONS[case["axes"]]) * B * n, "flops": 3.0 * D * B * n * (hq + hkv)}
    nbytes = flops = 0.0
    for t, m in zip(_ints(case["lens"]), _ints(case["counts"])):
        if m:
            sink, packed, res = _fill(case, t)
            nbytes += hkv * (packed * _packed_token_bytes(case) + (sink + res) * 512.0) + 512.0 * m * (hkv + hq)
            flops += 4.0 * D * hq * (m * t + m * (m + 1) / 2)
    return {"bytes": nbytes, "flops": flops}
