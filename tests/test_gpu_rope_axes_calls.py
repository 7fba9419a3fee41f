"""GPU tests of the calls that rotate with several axes and then append or decode: what they refuse, and that a refused call has changed nothing."""
import numpy as np
import pytest
import torch

import gpu_util as U
from paper_2512_19206_b200 import workloads as W

pytestmark = pytest.mark.gpu
SCALE = W.softmax_scale()


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
    return [torch.from_numpy(f(ang).astype(np.float32)).cuda() for f in (np.cos, np.sin)]


def refused(binding, code, call, *args, **kw):
    with pytest.raises(binding.MixKVQError) as e:
        call(*args, **kw)
    assert e.value.code == code


def bf16_at(memory, byte, shape):
    """A bf16 tensor over the memory of another one, from a byte offset on."""
    n = 2 * int(np.prod(shape))
    flat = memory.view(torch.uint8).view(-1)
    assert 0 <= byte <= flat.numel() - n
    return flat[byte:byte + n].view(torch.bfloat16).view(shape)


@pytest.mark.parametrize("which,end", [(w, e) for w in ("cos", "sin", "positions") for e in ("first", "last", "all")] + [("cache", "last"), ("cache", "all")])
def test_outputs_over_what_the_rotation_reads(binding, which, end):
    """An output over a part of the tables, the positions or the cache's memory is refused (thread blocks read angles while others store rows); directly
    behind them it is not."""
    B, Hq, Hkv, n = 2, 4, 2, 32
    axes = binding.axis_sections((32, 32))
    cache = binding.Cache(binding.make_config(1, B, Hq, Hkv, 64))
    size = 2 * B * Hq * n * 128                                   # bytes of q: 65536
    before = cache.launch_count()
    q, k, v = (torch.randn((B, h, n, 128), device="cuda").bfloat16() for h in (Hq, Hkv, Hkv))
    room = torch.zeros(4 * size, dtype=torch.uint8, device="cuda")
    cos, sin = tables(256)                                        # 65536 bytes each
    pos = torch.zeros((2, B, n), dtype=torch.int32, device="cuda")  # 512 bytes
    target = {"cos": cos, "sin": sin, "positions": pos, "cache": None}[which]
    if which == "cache":
        memory, stop = cache.mem, cache.mem.numel()
        at = {"last": stop - size, "all": 256}[end]
    else:
        start, stop = size, size + target.numel() * 4
        held = room[start:stop].view(target.dtype).view(target.shape)
        held.copy_(target)
        cos, sin, pos = (held if t is target else t for t in (cos, sin, pos))
        memory, at = room, {"first": start + 16 - size, "last": stop - 16, "all": start}[end]
    k2, v2 = torch.empty_like(k), torch.empty_like(v)
    over = bf16_at(memory, at, q.shape)
    refused(binding, -1, cache.rope_axes, q, k, v, cos, sin, pos, axes, out=(over, k2, v2))
    refused(binding, -1, cache.rope_axes, over, k, v, cos, sin, pos, axes, out=(over, k2, v2))        # in place too
    assert cache.launch_count() == before
    if which != "cache":
        beside = bf16_at(room, {"first": start - size, "last": stop, "all": stop}[end], q.shape)
        cache.rope_axes(q, k, v, cos, sin, pos, axes, out=(beside, k2, v2))
        assert torch.equal(beside, q) and cache.status() == 0     # (position 0)


@pytest.mark.parametrize("of", ["k", "q"])
def test_values_over_what_is_rotated(binding, of):
    """Values inside the keys or queries that are rotated in place are refused, by the append and by the decode step."""
    B, Hq, Hkv = 2, 4, 2
    axes = binding.axis_sections((32, 32))
    cache = binding.Cache(binding.make_config(1, B, Hq, Hkv, 64))
    cos, sin = tables(16)
    before = cache.launch_count()
    for n in (5, 1):
        pos = torch.ones((2, B, n), dtype=torch.int32, device="cuda")
        kq = [torch.randn((B, h, n, 128), device="cuda").bfloat16() for h in (Hkv, Hq)]
        was = [t.clone() for t in kq]
        k, q = kq
        v = k if of == "k" else bf16_at(q, 2 * B * Hkv * n * 128, k.shape)
        if n > 1:
            refused(binding, -1, cache.rope_axes_append, 0, k, v, q, cos, sin, pos, axes)
        else:
            refused(binding, -1, cache.rope_axes_decode_step, 0, k, v, q, cos, sin, pos, axes, SCALE)
        torch.cuda.synchronize()
        assert torch.equal(k, was[0]) and torch.equal(q, was[1])
    assert cache.launch_count() == before and cache.sequence_fill(0, 0) == (0, 0, 0)


@pytest.mark.parametrize("why", ["batch", "tile", "kernel", "kernel and sink"])
@pytest.mark.parametrize("call", ["axes", "rope", "plain"])
def test_a_step_that_is_not_supported_changes_nothing(binding, why, call):
    """A diverged batch that decode attention does not take: the step's tensors and the cache are as they were, so that a retry on another path rotates
    and appends once."""
    B, Hq, Hkv = 130 if why == "batch" else 3, 4, 2
    more = {"tile": dict(block_layout=1), "kernel and sink": dict(sink_len=32)}.get(why, {})
    cache = binding.Cache(binding.make_config(1, B, Hq, Hkv, 300, **more))
    new = lambda n: [torch.randn((B, h, n, 128), device="cuda").bfloat16() for h in (Hkv, Hkv, Hq)]        # noqa: E731
    counts = [20] * B
    counts[1] = 7
    cache.quantize_append_ragged(0, *new(20), counts)
    if why.startswith("kernel"):
        cache.set_attention_kernel(1)
    cos, sin = tables(16)
    pos = torch.ones((2, B, 1), dtype=torch.int32, device="cuda")
    kvq = new(1)
    was, memory = [t.clone() for t in kvq], cache.mem.clone()
    fill = [cache.sequence_fill(0, b) for b in range(B)]
    before = cache.launch_count()
    if call == "axes":
        refused(binding, -2, cache.rope_axes_decode_step, 0, *kvq, cos, sin, pos, binding.axis_sections((32, 32)), SCALE)
    elif call == "rope":
        refused(binding, -2, cache.rope_decode_step, 0, *kvq, cos, sin, 1, SCALE)
    else:
        refused(binding, -2, cache.decode_step, 0, *kvq, SCALE)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(kvq, was)) and torch.equal(cache.mem, memory)
    assert [cache.sequence_fill(0, b) for b in range(B)] == fill and cache.launch_count() == before


def test_rows_without_a_coordinate_are_appended_as_they_are(binding):
    """The append and the step store every row of the call, those that the rotation leaves alone (no token, beyond the tables) unrotated."""
    B, Hq, Hkv, n = 2, 4, 2, 9
    axes = binding.axis_sections((32, 32))
    cos, sin = tables(16)
    k, v, q = (torch.randn((B, h, n, 128), device="cuda").bfloat16() for h in (Hkv, Hkv, Hq))
    pos = torch.randint(1, 16, (2, B, n), device="cuda", dtype=torch.int32)
    pos[1, 1, 5:], pos[0, 0, 3] = -1, 16
    a, b = (binding.Cache(binding.make_config(1, B, Hq, Hkv, 64)) for _ in range(2))
    for c in (a, b):
        c.mem.zero_()
        c.reset()
    was_k, was_q = k.clone(), q.clone()
    qr, kr = q.clone(), k.clone()
    b.rope_axes(q, k, None, cos, sin, pos, axes, out=(qr, kr, None))
    b.quantize_append(0, kr, v, qr)
    a.rope_axes_append(0, k, v, q, cos, sin, pos, axes)
    assert a.status() == b.status() == binding.DEV_BAD_POSITION
    assert torch.equal(a.mem, b.mem) and a.sequence_fill(0, 1) == (0, 9, 0)
    for t, was in ((k, was_k), (q, was_q)):
        assert torch.equal(t[1, :, 5:], was[1, :, 5:]) and torch.equal(t[0, :, 3], was[0, :, 3])
        assert not torch.equal(t[0, :, 4], was[0, :, 4])
    step = [torch.randn((B, h, 1, 128), device="cuda").bfloat16() for h in (Hkv, Hkv, Hq)]
    none = torch.full((2, B, 1), -1, device="cuda", dtype=torch.int32)
    oa = a.rope_axes_decode_step(0, *[t.clone() for t in step], cos, sin, none, axes, SCALE)
    assert torch.equal(oa, b.decode_step(0, *step, SCALE)) and torch.equal(a.mem, b.mem)


@pytest.mark.parametrize("sections,interleaved", [((16, 24, 24), False), ((24, 20, 20), True), ((8, 24, 16, 16), True)])
@pytest.mark.parametrize("kind,sink", [(0, 0), (0, 32), (1, 0)])
def test_several_axes_into_the_cache(binding, sections, interleaved, kind, sink):
    """A prompt and the steps behind it, every sequence at positions of its own: the append and the step leave the cache, the rotated rows and the outputs
    that rope_axes, then quantize_append or decode_step leave."""
    B, Hq, Hkv, n = 2, 14, 2, 205
    axes, n_axes = binding.axis_sections(sections, interleaved), len(sections)
    cos, sin = tables(500)
    gen = torch.Generator().manual_seed(n_axes)
    new = lambda m: [torch.randn((B, h, m, 128), generator=gen).bfloat16().cuda() for h in (Hkv, Hkv, Hq)]        # noqa: E731
    where = lambda m: torch.randint(0, 500, (n_axes, B, m), generator=gen, dtype=torch.int32).cuda()              # noqa: E731
    a, b = (binding.Cache(binding.make_config(1, B, Hq, Hkv, 256, residual_len=64, sink_len=sink, **W.P27)) for _ in range(2))
    for c in (a, b):
        c.mem.zero_()
        c.reset()
        c.set_attention_kernel(kind)
    k, v, q = new(n)
    pos = where(n)
    qr, kr, _ = b.rope_axes(q, k, None, cos, sin, pos, axes, out=(torch.empty_like(q), torch.empty_like(k), None))
    b.quantize_append(0, kr, v, qr)
    a.rope_axes_append(0, k, v, q, cos, sin, pos, axes)
    assert torch.equal(k, kr) and torch.equal(q, qr)
    for _ in range(40):                                   # (over the end of a window)
        k, v, q = new(1)
        pos = where(1)
        qr, kr, _ = b.rope_axes(q, k, None, cos, sin, pos, axes, out=(torch.empty_like(q), torch.empty_like(k), None))
        ob = b.decode_step(0, kr, v, qr, SCALE)
        oa = a.rope_axes_decode_step(0, k, v, q, cos, sin, pos, axes, SCALE)
        assert torch.equal(oa, ob) and torch.equal(k, kr) and torch.equal(q, qr)
    assert a.status() == b.status() == 0 and torch.equal(a.mem, b.mem)
