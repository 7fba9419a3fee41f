"""GPU tests of the rotation with several axes: the bits of the oracle's rotation with every pair's own table row, in every layout, and what follows it."""
import numpy as np
import pytest
import torch

import chunk_util as CU
import gpu_util as U
from oracle import mixkvq_oracle as O
from paper_2512_19206_b200 import workloads as W

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19206_b200 import build
    build.build()
    from paper_2512_19206_b200 import binding as b
    b.lib()
    return b


def tables(n_pos):
    ang = np.arange(n_pos, dtype=np.float64)[:, None] * 1e6 ** (-np.arange(64, dtype=np.float64) / 64)[None]
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def draw(B, Hq, Hkv, n, n_axes, n_pos, seed):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn((B, n, Hq + 2 * Hkv, 128), generator=gen).to(torch.bfloat16)
    return x, torch.randint(0, n_pos, (n_axes, B, n), generator=gen, dtype=torch.int32)


def expected(x, cos, sin, positions, axes):
    """x [B, H, n, 128] with the oracle's rotation; the table row of pair i is the coordinate of its axis."""
    p = positions.numpy()[np.asarray(axes)]                          # [64, B, n]
    i = np.arange(64)[:, None, None]
    c, s = (np.moveaxis(t[np.clip(p, 0, len(t) - 1), i], 0, -1) for t in (cos, sin))
    return torch.stack([torch.from_numpy(O.rope(U.f32(x[b]), c[b], s[b])) for b in range(x.shape[0])]).to(torch.bfloat16)


@pytest.mark.parametrize("sections,interleaved", [((64,), False), ((16, 24, 24), False), ((24, 20, 20), True), ((1, 2, 30, 31), True), ((0, 64), False)])
@pytest.mark.parametrize("B,Hq,Hkv,n", [(1, 1, 1, 1), (3, 28, 4, 1), (2, 8, 2, 17), (1, 32, 8, 333), (5, 7, 1, 64)])
@pytest.mark.parametrize("layout", ["projection", "heads", "gaps"])
def test_bits_of_the_rotation(binding, sections, interleaved, B, Hq, Hkv, n, layout):
    axes = binding.axis_sections(sections, interleaved)
    assert [axes.count(a) for a in range(len(sections))] == list(sections)
    cos, sin = tables(900)
    x, pos = draw(B, Hq, Hkv, n, len(sections), 900, B + n)
    parts = x.split((Hq, Hkv, Hkv), 2)
    if layout == "projection":
        xd = x.cuda()
        ins = [t.transpose(1, 2) for t in xd.split((Hq, Hkv, Hkv), 2)]
    elif layout == "heads":
        ins = [t.transpose(1, 2).contiguous().cuda() for t in parts]
    else:                                                            # rows 160 elements apart, heads with a gap behind them
        ins = []
        for t in parts:
            h = t.shape[2]
            room = torch.zeros((B, h, n + 3, 160), dtype=torch.bfloat16, device="cuda")
            room[:, :, :n, :128] = t.transpose(1, 2).cuda()
            ins.append(room[:, :, :n, :128])
    cache = binding.Cache(binding.make_config(1, B, Hq, Hkv, 1))
    cd, sd = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    q, k, v = cache.rope_axes(*ins, cd, sd, pos.cuda(), axes)
    assert cache.status() == 0
    want = [t.transpose(1, 2).contiguous() for t in parts]
    assert torch.equal(q.cpu(), expected(want[0], cos, sin, pos, axes))
    assert torch.equal(k.cpu(), expected(want[1], cos, sin, pos, axes))
    assert torch.equal(v.cpu(), want[2])
    if layout == "heads":                                            # in place, and without the values
        q2, k2, v2 = cache.rope_axes(ins[0], ins[1], None, cd, sd, pos.cuda(), axes, out=(ins[0], ins[1], None))
        assert v2 is None and q2 is ins[0]
        assert torch.equal(ins[0], q) and torch.equal(ins[1], k)


def test_padding_and_bad_positions(binding):
    B, Hq, Hkv, n = 2, 4, 2, 40
    axes = binding.axis_sections((32, 32))
    cos, sin = tables(50)
    cd, sd = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    x, pos = draw(B, Hq, Hkv, n, 3, 50, 3)
    pos[0, 1, 25:] = -1                                              # sequence 1 has 25 tokens
    pos[2] = 2 ** 31 - 1                                             # an axis that no pair uses is not looked at
    ins = [t.transpose(1, 2).contiguous().cuda() for t in x.split((Hq, Hkv, Hkv), 2)]
    cache = binding.Cache(binding.make_config(1, B, Hq, Hkv, 1))
    out = [torch.full_like(t, 3.0) for t in ins]
    cache.rope_axes(*ins, cd, sd, pos.cuda(), axes, out=tuple(out))
    assert cache.status() == 0
    for t, o, turned in zip(ins, out, (True, True, False)):
        ref = expected(t.cpu(), cos, sin, pos, axes) if turned else t.cpu()
        assert torch.equal(o[0].cpu(), ref[0]) and torch.equal(o[1, :, :25].cpu(), ref[1, :, :25])
        assert (o[1, :, 25:] == 3.0).all()
    pos[1, 0, 7] = 50                                                # beyond the tables: that token alone is left, and the status says so
    out2 = [torch.full_like(t, 3.0) for t in ins]
    cache.rope_axes(*ins, cd, sd, pos.cuda(), axes, out=tuple(out2))
    assert cache.status() == binding.DEV_BAD_POSITION
    for o, o2 in zip(out, out2):
        assert (o2[0, :, 7] == 3.0).all()
        o2[0, :, 7] = o[0, :, 7]
        assert torch.equal(o, o2)


def test_one_axis_is_the_plain_rotation(binding):
    """append and decode step with one axis and consecutive positions leave what rope_append and rope_decode_step leave."""
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=2, tokens=300, **W.P24)
    k, v, q = (t.cuda() for t in W.tokens(w, 0, 0, 301))
    cos, sin = (torch.from_numpy(t).cuda() for t in tables(400))
    axes = [0] * 64
    a, b = U.make_cache(binding, w), U.make_cache(binding, w)
    for cache in (a, b):
        cache.mem.zero_()
        cache.reset()
    parts = [[t[:, :, s].contiguous() for t in (k, v, q)] for s in (slice(0, 300), slice(300, 301))]
    pa, pb = [[t.clone() for t in p] for p in parts], [[t.clone() for t in p] for p in parts]
    pos = torch.arange(5, 305, dtype=torch.int32, device="cuda").expand(1, 2, 300).contiguous()
    a.rope_append(0, *pa[0], cos, sin, 5)
    b.rope_axes_append(0, *pb[0], cos, sin, pos, axes)
    oa = a.rope_decode_step(0, *pa[1], cos, sin, 305, W.softmax_scale())
    ob = b.rope_axes_decode_step(0, *pb[1], cos, sin, torch.full((1, 2, 1), 305, dtype=torch.int32, device="cuda"), axes, W.softmax_scale())
    assert torch.equal(oa, ob) and torch.equal(a.mem, b.mem)
    for x, y in zip(pa[0] + pa[1], pb[0] + pb[1]):
        assert torch.equal(x, y)


def test_projection_to_cache(binding):
    """A prompt with a picture in two chunks, as a server runs it: the projection's output rotated and laid out, attended over what is there, appended."""
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=2, tokens=400, **W.P27)
    Hq, Hkv, n, T = w.n_q_heads, w.n_kv_heads, 200, 400
    x, _ = draw(2, Hq, Hkv, T, 3, 1, 11)
    i = torch.arange(T)
    grid = torch.stack([torch.where((i >= 100) & (i < 200), p, i) for p in (torch.full_like(i, 100), 100 + (i - 100) // 10, 100 + (i - 100) % 10)])
    pos = grid[:, None].expand(3, 2, T).to(torch.int32).contiguous()
    cos, sin = tables(T)
    axes = binding.axis_sections((16, 24, 24))
    cache = U.make_cache(binding, w)
    xd, got = x.cuda(), []
    for c in range(2):
        s = slice(c * n, c * n + n)
        ins = [t.transpose(1, 2) for t in xd[:, s].split((Hq, Hkv, Hkv), 2)]
        q, k, v = cache.rope_axes(*ins, torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), pos[:, :, s].contiguous().cuda(), axes)
        got.append(cache.chunk_step(0, k, v, q, W.softmax_scale()))
    assert cache.status() == 0
    qr, kr, vr = [t.transpose(1, 2).contiguous() for t in x.split((Hq, Hkv, Hkv), 2)]
    qr, kr = expected(qr, cos, sin, pos, axes), expected(kr, cos, sin, pos, axes)
    for c in range(2):
        sts = CU.streams(w, [c * n] * 2, kr, vr, qr)
        new = [t[:, :, c * n:c * n + n].contiguous() for t in (kr, vr, qr)]
        CU.check(w, got[c], sts, *new, [n, n], only=[(0, 0), (1, Hkv - 1)])
    U.compare_regions(cache, 0, w, U.oracle_streams(w, 0, kr, vr, qr, streams=[(0, 0), (1, Hkv - 1)]))


def test_refusals(binding):
    B, Hq, Hkv, n = 2, 4, 2, 8
    cache = binding.Cache(binding.make_config(1, B, Hq, Hkv, 64))
    cos, sin = (torch.from_numpy(t).cuda() for t in tables(20))
    pos = torch.zeros((2, B, n), dtype=torch.int32, device="cuda")
    q, k, v = (torch.zeros((B, h, n, 128), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    axes = binding.axis_sections((32, 32))
    before = cache.launch_count()
    for bad in (dict(cos=cos.double()), dict(cos=cos[:, :32]), dict(positions=pos.long()), dict(positions=pos[:, :1]), dict(axes=axes[:63]), dict(q=q.float()),
                dict(q=q[:, :3]), dict(k=k.cpu()), dict(v=v.transpose(2, 3)), dict(out=(q, k, None)), dict(out=(q.transpose(1, 2), k, v))):
        args = dict(q=q, k=k, v=v, cos=cos, sin=sin, positions=pos, axes=axes)
        with pytest.raises(ValueError):
            cache.rope_axes(**{**args, **bad})
    wide = torch.zeros((B, Hq, n, 128 + 4), dtype=torch.bfloat16, device="cuda")
    for bad, code in ((dict(axes=[2] * 64), -1), (dict(q=wide[..., :128]), -3), (dict(out=(q, k, k)), -1)):
        args = dict(q=q, k=k, v=v, cos=cos, sin=sin, positions=pos, axes=axes)
        with pytest.raises(binding.MixKVQError) as e:
            cache.rope_axes(**{**args, **bad})
        assert e.value.code == code
    strided = torch.zeros((B, n, Hq, 128), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(binding.MixKVQError) as e:                     # an output over its own input in another layout
        cache.rope_axes(strided.transpose(1, 2), k, v, cos, sin, pos, axes, out=(strided.view(B, Hq, n, 128), torch.zeros_like(k), torch.zeros_like(v)))
    assert e.value.code == -1
    with pytest.raises(binding.MixKVQError) as e:
        big = torch.zeros((2, B, 65), dtype=torch.int32, device="cuda")
        cache.rope_axes_append(0, *(torch.zeros((B, h, 65, 128), dtype=torch.bfloat16, device="cuda") for h in (Hkv, Hkv, Hq)), cos, sin, big, axes)
    assert e.value.code == -5
    assert cache.launch_count() == before and cache.status() == 0
