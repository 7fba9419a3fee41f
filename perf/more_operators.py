"""Timed cases of a key/value cache that is held in 4 bits in pages, and of the rotary positions in front of it.

  tables  `rope_tables`: cosines and sines of a range of positions, the frequencies scaled for contexts longer than those of training.
  rope    `Cache.rope_partial`: rotation of a part of the head, pairs in halves or interleaved, from the fused projection's output
          [B, n, Hq + 2 Hkv, 128] or from head-major tensors into the head-major q, k, v that the cache's calls take.
  append  `PagedCache.append`: new tokens are rotated, quantized (16 levels per token and group of channels) and stored in the pages of their
          sequences; `PagedCache.read` then gives the values that the stored codes stand for.
  attend  `PagedCache.attention`: the newest tokens of every sequence (one: a decode step) attend to all tokens in its pages, causally among themselves.

Shapes are those of the model shapes in `workloads.CONFIGS`, inputs follow its recipe (N(0,1) in bf16, four outlier key channels per KV head scaled
by 10 to 30, query gains log-uniform in [0.5, 4]), drawn on the GPU from the seed.  The plain form holds what the pages hold, one code per byte.
"""
from __future__ import annotations

import math

import torch

own = False

D = 128
SCALE = 1.0 / math.sqrt(D)
# Query and KV heads of the model shapes.
SHAPES = {"tiny": (1, 1), "qwen7b": (28, 4), "llama8b": (32, 8), "qwen32b": (40, 8)}
# How the frequencies are scaled: factor, and what the kind needs beside it
SCALINGS = {"none": dict(factor=1.0), "linear": dict(factor=4.0), "ntk": dict(factor=8.0),
            "bands": dict(factor=8.0, original=8192, low=1.0, high=4.0), "yarn": dict(factor=4.0, original=32768, fast=32.0, slow=1.0)}


def _tables(**kw):
    c = dict(op="tables", n=4096, start=0, rotary=128, base=1e6, scaling="none")
    c.update(kw)
    return c


def _rope(**kw):
    c = dict(op="rope", model="qwen7b", batch=1, n=1, rotary=128, pairs="halves", layout="projection")
    c.update(kw)
    return c


def _append(**kw):
    c = dict(op="append", model="qwen7b", lens="0", counts="1", page=64, G=32, rotary=128, pairs="halves")
    c.update(kw)
    return c


def _attend(**kw):
    c = dict(op="attend", model="qwen7b", lens="1024", counts="1", page=64, G=32)
    c.update(kw)
    return c


def listed():
    return [
        # a context grows beyond the tables it has: the next 256 positions
        _tables(name="tables-grow", n=256, start=32768, scaling="yarn"),
        # the tables of a long context, once
        _tables(name="tables-long", n=131072, base=5e5, scaling="bands"),
        # the new token of every sequence of a decode batch, half of the head turned, neighbouring channels paired
        _rope(name="rope-step", batch=8, rotary=64, pairs="interleaved"),
        # prompts of a batch as the projection leaves them
        _rope(name="rope-prompts", model="qwen32b", batch=4, n=4001),
        # one token of each sequence of a decode batch enters its page
        _append(name="append-step", lens="8191,4096,3000,1777,1024,640,63,0", counts="1,1,1,1,1,1,1,1"),
        # pieces of prompts of unequal length, small pages, a part of the head turned; one sequence has nothing to add
        _append(name="append-ragged", model="llama8b", lens="5000,100,0,777", counts="512,333,0,401", page=16, G=64, rotary=96, pairs="interleaved"),
        # a long prompt
        _append(name="append-prompt", model="llama8b", lens="0", counts="16384"),
        # one short sequence on the smallest configuration: launches and latency
        _attend(name="attend-tiny", model="tiny", lens="300"),
        # a decode step of a serving batch
        _attend(name="attend-batch", lens=",".join(["32768"] * 8), counts=",".join(["1"] * 8)),
        # one token for one very long sequence in small pages
        _attend(name="attend-long", model="llama8b", lens="120001", page=16),
        # drafted tokens of unequal number behind sequences of unequal length, wide groups
        _attend(name="attend-drafts", model="qwen32b", lens="32768,20011,9000,4097,640,5,31", counts="8,3,5,1,7,4,0", G=128, page=128),
        # a later chunk of a long prompt
        _attend(name="attend-chunk", lens="34816", counts="2048"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.random()
    rotary = rng.choice([128, 128, 64, 32, 96, 16])
    if kind < 0.12:
        return _tables(n=_log_int(rng, 1, 131072), start=rng.choice([0, rng.randint(1, 500000)]), rotary=rotary, base=rng.choice([1e4, 5e5, 1e6]),
                       scaling=rng.choice(list(SCALINGS)))
    pairs = rng.choice(["halves", "interleaved"])
    model = rng.choice(["qwen7b", "llama8b", "qwen32b", "tiny"])
    if kind < 0.3:
        n = _log_int(rng, 1, 16384)
        return _rope(model=model, batch=max(1, min(_log_int(rng, 1, 64), 16384 // n)), n=n, rotary=rotary, pairs=pairs, layout=rng.choice(["projection", "heads"]))
    page, G, batch = rng.choice([16, 32, 64, 128, 256]), rng.choice([32, 32, 64, 128]), rng.choice([1, 1, 2, 3, 5, 8])
    ragged = batch > 1 and rng.random() < 0.5
    hq, hkv = SHAPES[model]
    if kind < 0.55:
        n = _log_int(rng, 1, 16384 // batch)
        lens = [_log_int(rng, 1, 20000) - 1 for _ in range(batch)]
        counts = [rng.randint(0, n) if ragged else n for _ in range(batch)]
        counts[0] = n
        return _append(model=model, lens=",".join(map(str, lens)), counts=",".join(map(str, counts)), page=page, G=G, rotary=rotary, pairs=pairs)
    n = rng.choice([1, 1, _log_int(rng, 1, 16), _log_int(rng, 1, 2048)])
    # neither more tokens nor more products than the largest listed cases
    most = min(120000, 262144 * 4 // (batch * hkv), 33000 * 2048 * 28 // (n * hq * batch))
    longest = max(n, _log_int(rng, 1, max(2, most)))
    lens = [rng.randint(1, longest) if ragged else longest for _ in range(batch)]
    lens[0] = longest
    counts = [min(rng.randint(0, n) if ragged else n, t) for t in lens]
    counts[0] = n
    return _attend(model=model, lens=",".join(map(str, lens)), counts=",".join(map(str, counts)), page=page, G=G)


def _ints(text):
    return [int(x) for x in text.split(",")]


# ------------------------------------------------------------------------------------------------------- inputs
def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _normal(gen, *shape):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _gains(case, seed):
    """Gains of the key channels [Hkv, 128] and of the query channels [Hq, 128]."""
    hq, hkv = SHAPES[case["model"]]
    host = torch.Generator()
    host.manual_seed(seed)
    gk = torch.ones(hkv, D)
    for h in range(hkv):
        gk[h, torch.randperm(D, generator=host)[:4]] = 10.0 + 20.0 * torch.rand(4, generator=host)
    gq = (0.5 * torch.pow(8.0, torch.rand(hkv, D, generator=host))).repeat_interleave(hq // hkv, 0)
    gq = gq * (0.8 + 0.45 * torch.rand(hq, 1, generator=host))
    return gk.cuda().bfloat16(), gq.cuda().bfloat16(), host


def _page_table(case, host):
    """Pages of every sequence in any order, int32 [B, most pages of a sequence], and the number of pages of the pool."""
    held = [t + (n if case["op"] == "append" else 0) for t, n in zip(_ints(case["lens"]), _ints(case["counts"]))]
    each = max(1, max(-(-t // case["page"]) for t in held))
    pages = len(held) * each + 7
    return torch.randperm(pages, generator=host)[:len(held) * each].view(len(held), each).to(torch.int32).cuda(), pages


def _angles(n, rotary, start=0):
    """Tables of the plain frequencies as a model's configuration gives them, float32 [n, rotary / 2]."""
    a = torch.arange(start, start + n, device="cuda", dtype=torch.float64)[:, None] * torch.pow(1e6, -torch.arange(rotary // 2, device="cuda", dtype=torch.float64) * 2 / rotary)
    return a.cos().float(), a.sin().float()


def _projection(case, seed, batch, n):
    hq, hkv = SHAPES[case["model"]]
    gk, gq, host = _gains(case, seed)
    x = _normal(_generator(seed), batch, n, hq + 2 * hkv, D)
    x[:, :, :hq] *= gq
    x[:, :, hq:hq + hkv] *= gk
    q, k, v = (t.transpose(1, 2) for t in x.split((hq, hkv, hkv), 2))
    return q, k, v, host


def _rope_inputs(case, seed):
    q, k, v, host = _projection(case, seed, case["batch"], case["n"])
    if case["layout"] == "heads":
        q, k, v = (t.contiguous() for t in (q, k, v))
    start = torch.randint(0, 4096, (case["batch"], 1), generator=host)
    pos = (start + torch.arange(case["n"])).to(torch.int32).cuda()
    cos, sin = _angles(case["n"] + 4096, case["rotary"])
    return dict(q=q, k=k, v=v, positions=pos, cos=cos, sin=sin)


def _append_inputs(case, seed):
    lens, counts = _ints(case["lens"]), _ints(case["counts"])
    q, k, v, host = _projection(case, seed, len(lens), max(counts))
    pages, n_pages = _page_table(case, host)
    cos, sin = _angles(max(lens) + max(counts), case["rotary"])
    as_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")                                    # noqa: E731
    return dict(q=q, k=k, v=v, cos=cos, sin=sin, pages=pages, n_pages=n_pages, lens=as_int(lens), counts=as_int(counts))


def _attend_inputs(case, seed):
    hq, hkv = SHAPES[case["model"]]
    lens, counts = _ints(case["lens"]), _ints(case["counts"])
    gk, gq, host = _gains(case, seed)
    gen = _generator(seed)
    pages, n_pages = _page_table(case, host)
    k, v = (_normal(gen, len(lens), hkv, max(lens), D) for _ in range(2))
    q = _normal(gen, len(lens), hq, max(counts), D) * gq[:, None]
    as_int = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")                                    # noqa: E731
    return dict(q=q, k=k.mul_(gk[:, None]), v=v, pages=pages, n_pages=n_pages, lens=as_int(lens), counts=as_int(counts))


def _over(x, number):
    """x / number, divided: by a host number it would be multiplied with a rounded reciprocal."""
    return x / torch.full((), number, dtype=x.dtype, device=x.device)


def _groups(x, G):
    """Codes [..., 128], scales and zero-points [..., 128 / G] of rows x [..., 128] in bf16: per group z the minimum, s the range over the levels rounded
    up to bf16, codes of 16 levels."""
    x = x.float().unflatten(-1, (D // G, G))
    lo, hi = x.amin(-1, keepdim=True), x.amax(-1, keepdim=True)
    s = _over(hi - lo, 15)
    down = s.view(torch.int32) & -65536
    s = torch.where(down == s.view(torch.int32), down, down + 65536).view(torch.float32)
    c = ((x - lo) / torch.where(s == 0, torch.ones_like(s), s)).round().clamp(0, 15)
    return c.to(torch.uint8).flatten(-2), s[..., 0], lo[..., 0]


def _values(c, s, z):
    """What codes [..., 128] with scales and zero-points [..., groups] stand for, float32."""
    return (c.unflatten(-1, (s.shape[-1], -1)).float() * s[..., None] + z[..., None]).flatten(-2)


def _places(s, case, start, n):
    """Page and slot of tokens start[b] .. start[b] + n - 1 of every sequence, [B, n] each; tokens behind a sequence's last are put on a page behind the pool's."""
    i = start[:, None].long() + torch.arange(n, device="cuda")
    live = i < (s["lens"] + (s["counts"] if case["op"] == "append" else 0))[:, None]
    page = s["pages"].long().gather(1, (i // case["page"]).clamp(max=s["pages"].shape[1] - 1))
    return torch.where(live, page, s["n_pages"]), i % case["page"], live


def _pool(s, case):
    hkv = SHAPES[case["model"]][1]
    shape = (s["n_pages"] + 1, hkv, case["page"])
    new = lambda last, dtype: torch.zeros((*shape, last), dtype=dtype, device="cuda")                       # noqa: E731
    groups = D // case["G"]
    return [(new(D, torch.uint8), new(groups, torch.float32), new(groups, torch.float32)) for _ in range(2)]


def _store(pool, x, page, slot, G):
    """Rows x [B, Hkv, n, 128] into their places of one of the two pools."""
    for held, new in zip(pool, _groups(x, G)):
        held[page, :, slot] = new.transpose(1, 2)


def _make_paged(case, n_pages):
    from paper_2512_19206_b200 import binding
    hq, hkv = SHAPES[case["model"]]
    return binding.PagedCache(binding.make_paged_config(1, hq, hkv, n_pages, page_tokens=case["page"], group_size=case["G"]))


def prepare(case, seed):
    if case["op"] == "tables":
        n, half = case["n"], case["rotary"] // 2
        gen = torch.Generator()
        gen.manual_seed(seed)
        # a program goes through positions: another seed, another stretch of them
        start = case["start"] + int(torch.randint(0, 65536, (), generator=gen))
        return {"case": case, "start": start, "out": tuple(torch.empty((n, half), device="cuda") for _ in range(2))}
    if case["op"] == "rope":
        s = _rope_inputs(case, seed)
        s["case"] = case
        hq, hkv = SHAPES[case["model"]]
        s["out"] = tuple(torch.empty(case["batch"], h, case["n"], D, dtype=torch.bfloat16, device="cuda") for h in (hq, hkv, hkv))
        if own:
            from paper_2512_19206_b200 import binding
            s["cache"] = binding.Cache(binding.make_config(1, case["batch"], hq, hkv, 1))
        return s
    if case["op"] == "append":
        s = _append_inputs(case, seed)
        s["case"] = case
        s["q_out"] = torch.zeros(s["q"].shape, dtype=torch.bfloat16, device="cuda")
        s["values"] = tuple(torch.zeros(s["k"].shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        if own:
            s["cache"] = _make_paged(case, s["n_pages"])
        else:
            s["pool"] = _pool(s, case)
        return s
    s = _attend_inputs(case, seed)
    s["case"] = case
    s["out"] = torch.zeros_like(s["q"])
    k, v = s.pop("k"), s.pop("v")
    start = torch.zeros_like(s["lens"])
    if own:
        s["cache"] = _make_paged(case, s["n_pages"])
        s["cache"].append(0, k, v, s["pages"], start, counts=s["lens"])
    else:
        s["pool"] = _pool(s, case)
        page, slot, _ = _places(s, case, start, k.shape[2])
        _store(s["pool"][0], k, page, slot, case["G"])
        _store(s["pool"][1], v, page, slot, case["G"])
    return s


# ------------------------------------------------------------------------------------------------------- plain forms
def _plain_tables(s):
    case, d = s["case"], s["case"]["rotary"]
    how, sc = case["scaling"], SCALINGS[case["scaling"]]
    i = torch.arange(d // 2, device="cuda", dtype=torch.float64)
    base, m = case["base"], 1.0
    if how == "ntk":
        base = base * sc["factor"] ** (d / (d - 2))
    f = torch.pow(base, -2 * i / d)
    if how == "linear":
        f = f / sc["factor"]
    elif how == "bands":
        turns = sc["original"] * f / (2 * math.pi)
        keep = ((turns - sc["low"]) / (sc["high"] - sc["low"])).clamp(0, 1)
        f = f * keep + f / sc["factor"] * (1 - keep)
    elif how == "yarn":
        dim = lambda turns: d * math.log(sc["original"] / (turns * 2 * math.pi)) / (2 * math.log(base))    # noqa: E731
        lo, hi = max(math.floor(dim(sc["fast"])), 0), min(math.ceil(dim(sc["slow"])), d - 1)
        ramp = ((i - lo) / max(hi - lo, 1e-3)).clamp(0, 1)
        f = f * (1 - ramp) + f / sc["factor"] * ramp
        m = 0.1 * math.log(sc["factor"]) + 1
    a = torch.arange(s["start"], s["start"] + case["n"], device="cuda", dtype=torch.float64)[:, None] * f
    return (a.cos() * m).float(), (a.sin() * m).float()


def _turned(x, cos, sin, positions, case):
    """x [B, H, n, 128] with its first channels rotated, bf16."""
    d = case["rotary"]
    c, n = (t[positions.long()][:, None] for t in (cos, sin))
    part = x[..., :d].float()
    if case["pairs"] == "halves":
        a, b = part.split(d // 2, -1)
        part = torch.cat([a * c - b * n, b * c + a * n], -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        part = torch.stack([a * c - b * n, b * c + a * n], -1).flatten(-2)
    return torch.cat([part.to(torch.bfloat16), x[..., d:]], -1)


def _plain_rope(s):
    turn = lambda x: _turned(x, s["cos"], s["sin"], s["positions"], s["case"])                             # noqa: E731
    return turn(s["q"]), turn(s["k"]), s["v"].contiguous()


def _plain_append(s):
    case, n = s["case"], s["q"].shape[2]
    page, slot, live = _places(s, case, s["lens"], n)
    pos = torch.where(live, s["lens"][:, None] + torch.arange(n, device="cuda"), 0)
    keep = live[:, None, :, None]
    q = torch.where(keep, _turned(s["q"], s["cos"], s["sin"], pos, case), s["q_out"])
    _store(s["pool"][0], _turned(s["k"], s["cos"], s["sin"], pos, case), page, slot, case["G"])
    _store(s["pool"][1], s["v"], page, slot, case["G"])
    back = [_values(*(t[page, :, slot] for t in held)).transpose(1, 2).to(torch.bfloat16) for held in s["pool"]]
    return [q] + [torch.where(keep, x, old) for x, old in zip(back, s["values"])]


def _plain_attend(s):
    case, q = s["case"], s["q"]
    B, hq, n, _ = q.shape
    hkv = SHAPES[case["model"]][1]
    keys, vals = (_values(*(t[s["pages"].long()] for t in held)).transpose(1, 2).reshape(B, hkv, -1, D) for held in s["pool"])
    i, j = torch.arange(n, device="cuda"), torch.arange(keys.shape[2], device="cuda")
    sees = j < (s["lens"] - s["counts"])[:, None, None] + i[:, None] + 1                                   # [B, n, tokens]
    logits = (q.float().view(B, hkv, -1, D) @ keys.transpose(-1, -2)).view(B, hkv, -1, n, keys.shape[2]).mul_(SCALE)
    logits.masked_fill_(~sees[:, None, None], float("-inf"))
    p = logits.sub_(logits.amax(-1, keepdim=True)).exp_()
    p.div_(p.sum(-1, keepdim=True))
    out = (p.view(B, hkv, -1, p.shape[-1]) @ vals).view(q.shape).to(torch.bfloat16)
    return torch.where((i < s["counts"][:, None])[:, None, :, None], out, s["out"])      # rows past a sequence's count stay as they were


def run(state):
    s, case = state, state["case"]
    if case["op"] == "tables":
        if not own:
            return _plain_tables(s)
        from paper_2512_19206_b200 import binding
        return binding.rope_tables(case["n"], case["rotary"], case["base"], case["scaling"], start=s["start"], out=s["out"], **SCALINGS[case["scaling"]])
    if case["op"] == "rope":
        if not own:
            return _plain_rope(s)
        return s["cache"].rope_partial(s["q"], s["k"], s["v"], s["cos"], s["sin"], s["positions"], interleaved=case["pairs"] == "interleaved", out=s["out"])
    if case["op"] == "append":
        if not own:
            return _plain_append(s)
        q = s["cache"].append(0, s["k"], s["v"], s["pages"], s["lens"], counts=s["counts"], q=s["q"], cos=s["cos"], sin=s["sin"],
                              interleaved=case["pairs"] == "interleaved", q_out=s["q_out"])
        return [q, *s["cache"].read(0, s["pages"], s["lens"], q.shape[2], counts=s["counts"], out=s["values"])]
    if not own:
        return _plain_attend(s)
    return s["cache"].attention(0, s["q"], s["pages"], s["lens"], SCALE, counts=s["counts"], out=s["out"])


# ------------------------------------------------------------------------------------------------------- the definition in 64 bits
def _exact_turn(x, cos, sin, positions, case):
    """The rotation as a product of complex numbers, 64 bits."""
    d, y = case["rotary"], x.double()
    unit = torch.complex(cos.double(), sin.double())[positions.long()][:, None]
    if case["pairs"] == "halves":
        z = torch.complex(y[..., :d // 2].contiguous(), y[..., d // 2:d].contiguous()) * unit
        part = torch.cat((z.real, z.imag), -1)
    else:
        z = torch.view_as_complex(y[..., :d].reshape(*y.shape[:-1], d // 2, 2)) * unit
        part = torch.view_as_real(z).flatten(-2)
    return torch.cat((part, y[..., d:]), -1)


def _exact_values(x, G):
    """What rows x [..., 128] of bf16 numbers are kept as, 64 bits: codes are the rounded single-precision quotient."""
    x = x.float().reshape(*x.shape[:-1], D // G, G)
    z = x.min(dim=-1, keepdim=True).values
    step = (x.max(dim=-1, keepdim=True).values - z).div(torch.tensor(15.0, device="cuda"))
    frac, e = torch.frexp(step.double())                         # round up to 8 significant bits
    step = torch.ldexp(torch.ceil(frac * 256), e - 8).float()
    code = torch.where(step > 0, ((x - z) / step.clamp_min(1e-38)).round(), torch.zeros_like(x)).clamp(0, 15)
    return (code.double() * step.double() + z.double()).flatten(-2)


def _exact_tables(case, seed):
    gen = torch.Generator()
    gen.manual_seed(seed)
    start, d = case["start"] + int(torch.randint(0, 65536, (), generator=gen)), case["rotary"]
    how, sc, m, freq = case["scaling"], SCALINGS[case["scaling"]], 1.0, []
    for i in range(d // 2):
        f = math.exp(-2.0 * i / d * math.log(case["base"]))
        if how == "linear":
            f /= sc["factor"]
        elif how == "ntk":                                       # the lowest frequency falls by the factor, the highest stays
            f *= sc["factor"] ** (-2.0 * i / (d - 2))
        elif how == "bands":
            wave = 2 * math.pi / f
            if wave > sc["original"] / sc["low"]:
                f /= sc["factor"]
            elif wave > sc["original"] / sc["high"]:
                t = (sc["original"] / wave - sc["low"]) / (sc["high"] - sc["low"])
                f = (1 - t) * f / sc["factor"] + t * f
        elif how == "yarn":
            lo, hi = (d * math.log(sc["original"] / (2 * math.pi * sc[k])) / (2 * math.log(case["base"])) for k in ("fast", "slow"))
            lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), d - 1)
            t = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            f = f * (1 - t) + f / sc["factor"] * t
            m = 1 + 0.1 * math.log(sc["factor"])
        freq.append(f)
    p = torch.arange(start, start + case["n"], device="cuda", dtype=torch.float64)
    a = torch.remainder(p[:, None] * torch.tensor(freq, device="cuda", dtype=torch.float64), 2 * math.pi)
    z = torch.polar(torch.full_like(a, m), a)
    return z.real, z.imag


def exact(case, seed):
    if case["op"] == "tables":
        return _exact_tables(case, seed)
    if case["op"] == "rope":
        s = _rope_inputs(case, seed)
        return *(_exact_turn(s[x], s["cos"], s["sin"], s["positions"], case) for x in "qk"), s["v"].double()
    if case["op"] == "append":
        s = _append_inputs(case, seed)
        q, k, v = (torch.zeros(s[x].shape, dtype=torch.float64, device="cuda") for x in "qkv")
        for b, (t, m) in enumerate(zip(_ints(case["lens"]), _ints(case["counts"]))):
            at = torch.arange(t, t + m, device="cuda")[None]
            one = slice(b, b + 1)
            q[one, :, :m], turned = (_exact_turn(s[x][one, :, :m], s["cos"], s["sin"], at, case) for x in "qk")
            k[one, :, :m] = _exact_values(turned.to(torch.bfloat16), case["G"])
            v[one, :, :m] = _exact_values(s["v"][one, :, :m], case["G"])
        return [q, k, v]
    s = _attend_inputs(case, seed)
    hq, hkv = SHAPES[case["model"]]
    g, out = hq // hkv, torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    for b, (t, m) in enumerate(zip(_ints(case["lens"]), _ints(case["counts"]))):
        hidden = torch.arange(t, device="cuda")[None] > t - m + torch.arange(m, device="cuda")[:, None]
        for h in range(hkv if m else 0):
            kk, vv = (_exact_values(s[x][b, h, :t], case["G"]) for x in "kv")
            for a in range(h * g, h * g + g):
                logits = (s["q"][b, a, :m].double() @ kk.T) * SCALE
                out[b, a, :m] = torch.softmax(logits.masked_fill(hidden, -math.inf), -1) @ vv
    return out


# ------------------------------------------------------------------------------------------------------- work
def work(case):
    if case["op"] == "tables":
        angles = case["n"] * case["rotary"] / 2
        return {"bytes": 8.0 * angles, "flops": 8.0 * angles}
    hq, hkv = SHAPES[case["model"]]
    if case["op"] == "rope":
        B, n = case["batch"], case["n"]
        return {"bytes": B * n * (4.0 * D * (hq + 2 * hkv) + 4.0) + 4.0 * case["rotary"] * min(B * n, n + 4096), "flops": 3.0 * case["rotary"] * B * n * (hq + hkv)}
    held = 2 * (D / 2 + 4.0 * D / case["G"])                     # bytes of a token of a KV head
    lens, counts = _ints(case["lens"]), _ints(case["counts"])
    if case["op"] == "append":
        n = sum(counts)
        # k, v and q in, q and the pages out; the pages in and the values out; the tables' rows
        nbytes = n * (hkv * (512.0 + held) + 512.0 * hq + hkv * (held + 512.0) + 4.0 * case["rotary"])
        return {"bytes": nbytes, "flops": n * (3.0 * case["rotary"] * (hq + hkv) + hkv * 2 * D * 6.0)}
    nbytes = flops = 0.0
    for t, m in zip(lens, counts):
        if m:
            nbytes += hkv * t * held + 512.0 * m * hq
            flops += 4.0 * D * hq * (m * (t - m) + m * (m + 1) / 2)
    return {"bytes": nbytes, "flops": flops}
