"""GPU tests of the chunk attention's edges: values that are no numbers, raised maxima, other streams, captured graphs, chunks behind appends, refusals."""
import pytest
import torch

import chunk_util as CU
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


def plain_cache(binding, B, Hq, Hkv, tokens, seed, extra=0, **kw):
    """A cache of `tokens` N(0, 1) tokens per sequence and a fresh generator."""
    gen = torch.Generator().manual_seed(seed)
    cache = binding.Cache(binding.make_config(1, B, Hq, Hkv, tokens + extra + 1, **{**W.P24, **kw}))
    k, v, q = (torch.randn((B, h, tokens, 128), generator=gen).to(torch.bfloat16) for h in (Hkv, Hkv, Hq))
    if tokens:
        cache.quantize_append(0, k.cuda(), v.cuda(), q.cuda())
    return cache, (k, v, q), gen


def chunk(gen, B, Hq, Hkv, n):
    return [torch.randn((B, h, n, 128), generator=gen).to(torch.bfloat16) for h in (Hkv, Hkv, Hq)]


def causal(k, v, q):
    """The definition in 64 bits for an empty cache, elements that are no numbers included: a masked key takes no part."""
    g = q.shape[1] // k.shape[1]
    K, V = (t.double().repeat_interleave(g, 1) for t in (k, v))
    s = (q.double() @ K.transpose(-1, -2)) * SCALE
    out = torch.empty_like(q, dtype=torch.float64)
    for j in range(q.shape[2]):
        out[:, :, j] = (torch.softmax(s[:, :, j, :j + 1], -1)[..., None] * V[:, :, :j + 1]).sum(2)
    return out


@pytest.mark.parametrize("g,n", [(1, 200), (4, 150), (7, 9)])
def test_elements_that_are_no_numbers(binding, g, n):
    """A NaN or an infinity in a new token's value reaches the rows that see the token, in its channel alone; in its key the rows that see it; in a
    query that row."""
    cache, _, gen = plain_cache(binding, 1, 2 * g, 2, 0, 5, extra=n)
    k, v, q = chunk(gen, 1, 2 * g, 2, n)
    inf, nan = float("inf"), float("nan")
    v[0, 0, n // 2, 3], v[0, 0, n // 3, 70], v[0, 0, n - 1, 71], v[0, 1, n // 2, 9], v[0, 1, n - 1, 9] = nan, inf, -inf, inf, -inf
    k[0, 1, 2 * n // 3, 5] = nan
    q[0, 0, 1, 7] = inf
    out = cache.chunk_attention(0, *(t.cuda() for t in (k, v, q)), SCALE).double().cpu()
    assert cache.status() == 0
    ref = causal(k, v, q)
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    for s in (inf, -inf):
        assert torch.equal(out == s, ref == s)
    fine = torch.isfinite(ref)
    assert float((out - ref)[fine].abs().max()) <= 4e-3
    # and nothing of it stays behind for the next call
    k, v, q = chunk(gen, 1, 2 * g, 2, n)
    out = cache.chunk_attention(0, *(t.cuda() for t in (k, v, q)), SCALE).double().cpu()
    assert float((out - causal(k, v, q)).abs().max()) <= 4e-3


def test_elements_of_the_window_that_are_no_numbers(binding):
    """Held tokens are seen by every row, whichever thread block has them."""
    gen = torch.Generator().manual_seed(8)
    cache = binding.Cache(binding.make_config(1, 1, 4, 2, 800, **W.P24))
    held, new = chunk(gen, 1, 4, 2, 10), chunk(gen, 1, 4, 2, 400)
    held[1][0, 0, 4, 17], held[1][0, 0, 6, 18] = float("inf"), float("nan")
    cache.quantize_append(0, *(t.cuda() for t in held))
    out = cache.chunk_attention(0, *(t.cuda() for t in new), SCALE).double().cpu()
    ref = causal(*(torch.cat(t, 2) for t in zip(held, new)))[:, :, 10:]
    assert cache.status() == 0
    assert torch.equal(torch.isnan(out), torch.isnan(ref)) and torch.equal(torch.isposinf(out), torch.isposinf(ref))
    fine = torch.isfinite(ref)
    assert float((out - ref)[fine].abs().max()) <= 4e-3


@pytest.mark.parametrize("tokens,n", [(0, 300), (1500, 5), (1500, 200)])
def test_maxima_that_rise(binding, tokens, n):
    """Logits that grow along the keys by far more than the kernel lets a maximum rise without rescaling."""
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=1, n_kv_heads=1, n_q_heads=7, tokens=max(tokens, 1), **W.P24)
    gen = torch.Generator().manual_seed(tokens + n)
    k, v, q = (torch.randn((1, h, tokens + n, 128), generator=gen) for h in (1, 1, 7))
    k = k * 0.1 + torch.linspace(-1, 1, tokens + n)[None, None, :, None] * 3
    q = q * 0.1 + 1.5
    k, v, q = (t.to(torch.bfloat16) for t in (k, v, q))
    cache = U.make_cache(binding, w, max_tokens=tokens + n)
    if tokens:
        cache.quantize_append(0, *(t[:, :, :tokens].contiguous().cuda() for t in (k, v, q)))
    new = [t[:, :, tokens:].contiguous() for t in (k, v, q)]
    out = cache.chunk_attention(0, *(t.cuda() for t in new), SCALE)
    assert cache.status() == 0
    sts = CU.streams(w, [tokens], *(t[:, :, :max(tokens, 1)] for t in (k, v, q)))
    CU.check(w, out, sts, *new, [n])


def test_steps_append_as_the_append_does(binding):
    """A prompt in chunks leaves the cache that appends of the same pieces leave, byte for byte; the first chunk's attention is the prompt's."""
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=2, tokens=700, **W.P27)
    k, v, q = W.tokens(w, 0, 0, 700)
    a, b, c = (U.make_cache(binding, w) for _ in range(3))
    for cache in (a, b):
        cache.mem.zero_()                          # (window rows that no append has written yet are compared too)
        cache.reset()
    whole = c.prefill(0, k.cuda(), v.cuda(), q.cuda(), SCALE)
    scratch = torch.empty(b.chunk_scratch_bytes(300), dtype=torch.uint8, device="cuda")
    first = None
    for t0, t1 in ((0, 300), (300, 301), (301, 600), (600, 700)):
        part = [t[:, :, t0:t1].contiguous().cuda() for t in (k, v, q)]
        a.quantize_append(0, *part)
        out = b.chunk_step(0, *part, SCALE, scratch=scratch)
        first = out if first is None else first
    assert a.status() == b.status() == c.status() == 0
    assert torch.equal(a.mem, b.mem)
    assert float((first - whole[:, :, :300]).abs().max()) <= 2e-3


def test_drafts_then_accepted_tokens(binding):
    """Drafted tokens are attended without being appended; the accepted ones go in from the same tensors, and the next draft sees them."""
    w = W.small(W.CONFIGS["llama8b"], n_layers=1, batch=3, n_kv_heads=2, n_q_heads=8, tokens=400, **W.P24)
    k, v, q = W.tokens(w, 0, 0, 400)
    cache = U.make_cache(binding, w)
    lens, accepted = [400, 250, 399], [2, 0, 4]
    cache.quantize_append_ragged(0, k.cuda(), v.cuda(), q.cuda(), lens)
    sts = CU.streams(w, lens, k, v, q)
    gen = torch.Generator().manual_seed(1)
    for _ in range(3):
        new = chunk(gen, 3, 8, 2, 4)
        fill = [cache.sequence_fill(0, b) for b in range(3)]
        out = cache.chunk_attention(0, *(t.cuda() for t in new), SCALE)
        assert [cache.sequence_fill(0, b) for b in range(3)] == fill
        CU.check(w, out, sts, *new, [4, 4, 4])
        cache.quantize_append_ragged(0, *(t.cuda() for t in new), accepted)
        for (b, hk), st in sts.items():
            m = accepted[b]
            if m:
                st.append_many(U.f32(new[0][b, hk, :m]), U.f32(new[1][b, hk, :m]), U.f32(new[2][b, hk * 4:hk * 4 + 4, :m]))
    assert cache.status() == 0
    U.compare_regions(cache, 0, w, sts)


def test_decode_step_behind_a_chunk(binding):
    """The kernels of a decode step that start early find the chunk's window rows."""
    w = W.small(W.CONFIGS["qwen7b"], n_layers=2, batch=2, tokens=300, **W.P24)
    outs = []
    for sync in (True, False):
        cache = U.make_cache(binding, w, max_tokens=900)
        for layer in (0, 1):
            k, v, q = (t.cuda() for t in W.tokens(w, layer, 0, 520))
            cut = lambda a, b: [t[:, :, a:b].contiguous() for t in (k, v, q)]       # noqa: E731
            got = [cache.chunk_step(layer, *cut(0, 260), SCALE)]
            for t in range(260, 266):
                got.append(cache.decode_step(layer, *cut(t, t + 1), SCALE))
                got.append(cache.chunk_step(layer, *cut(266 + 40 * (t - 260), 306 + 40 * (t - 260)), SCALE))
                if sync:
                    torch.cuda.synchronize()
            outs.append(got)
        assert cache.status() == 0
    for a, b in zip(outs[0] + outs[1], outs[2] + outs[3]):
        assert torch.equal(a, b)


def test_scratch_and_padding_of_any_content(binding):
    """What lies in the scratch, in the rows behind the counts and in the output before the call has no effect, and those rows stay."""
    cache, _, gen = plain_cache(binding, 3, 8, 2, 1700, 6, extra=200)
    new = [t.cuda() for t in chunk(gen, 3, 8, 2, 200)]
    counts = [200, 7, 0]
    want = cache.chunk_attention(0, *new, SCALE, counts=counts, dtype=torch.bfloat16)
    for t in new:
        for b, c in enumerate(counts):
            t[b, :, c:] = float("nan")
    scratch = torch.full((cache.chunk_scratch_bytes(200),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full_like(new[2], float("inf"))
    cache.chunk_attention(0, *new, SCALE, counts=counts, out=out, scratch=scratch)
    assert cache.status() == 0
    for b, c in enumerate(counts):
        assert torch.equal(out[b, :, :c], want[b, :, :c]) and torch.isposinf(out[b, :, c:]).all()


@pytest.mark.parametrize("magnitude", [1e-3, 30.0])
def test_large_and_small_values(binding, magnitude):
    """The output follows the values' size; what the chunk adds to the tolerance is relative to it (fp16 keeps 2^-12 of 2^-14 and more: 1e-3 N(0, 1) values,
    and their scales of a third of a group's range, lose at most half of 2^-24 each, 3e-8 of values whose tolerance is above 1e-6)."""
    w = W.small(W.CONFIGS["llama8b"], n_layers=1, batch=1, n_kv_heads=1, n_q_heads=4, tokens=600, **W.P24)
    k, v, q = W.tokens(w, 0, 0, 600)
    v = (v.float() * magnitude).to(torch.bfloat16)
    cache = U.make_cache(binding, w)
    cache.quantize_append(0, *(t[:, :, :560].contiguous().cuda() for t in (k, v, q)))
    new = [t[:, :, 560:].contiguous() for t in (k, v, q)]
    out = cache.chunk_attention(0, *(t.cuda() for t in new), SCALE)
    assert cache.status() == 0
    CU.check(w, out, CU.streams(w, [560], k, v, q), *new, [40])


def test_one_token_is_a_decode_step(binding):
    """A single new token's chunk and the decode step see the same keys; both stay within the decode's tolerance."""
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=2, tokens=601, **W.P27)
    k, v, q = W.tokens(w, 0, 0, 601)
    a = U.make_cache(binding, w)
    a.quantize_append(0, *(t[:, :, :600].contiguous().cuda() for t in (k, v, q)))
    new = [t[:, :, 600:].contiguous().cuda() for t in (k, v, q)]
    out = a.chunk_attention(0, *new, SCALE)
    step = a.decode_step(0, *new, SCALE)
    assert a.status() == 0
    assert float((out[:, :, 0] - step).abs().max()) <= 2e-3 + 2e-3        # (each within 2e-3 of the definition)


def test_streams_beyond_four_gigabytes(binding):
    """A cache whose last streams start beyond 2^32 bytes gives what a small one gives."""
    gen = torch.Generator().manual_seed(3)
    k, v, q = chunk(gen, 2, 16, 8, 700)
    outs = []
    for max_tokens in (800, 4_000_000):
        cache = binding.Cache(binding.make_config(1, 2, 16, 8, max_tokens, **W.P27))
        cache.quantize_append(0, *(t[:, :, :600].contiguous().cuda() for t in (k, v, q)))
        outs.append(cache.chunk_attention(0, *(t[:, :, 600:].contiguous().cuda() for t in (k, v, q)), SCALE))
        assert cache.status() == 0
        big = cache.describe(0)
        last = big.base_off + 15 * big.base_stride
        del cache
    assert last > 1 << 32 and torch.equal(*outs)


def test_another_stream_and_two_scratches(binding):
    cache, _, gen = plain_cache(binding, 2, 8, 2, 900, 3, extra=64)
    new = [[t.cuda() for t in chunk(gen, 2, 8, 2, n)] for n in (3, 64)]
    want = [cache.chunk_attention(0, *t, SCALE) for t in new]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    scratch = [torch.empty(cache.chunk_scratch_bytes(64), dtype=torch.uint8, device="cuda") for _ in range(2)]
    got = [[], []]
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(cache.chunk_attention(0, *new[i], SCALE, scratch=scratch[i]))
    torch.cuda.synchronize()
    assert cache.status() == 0
    for i in range(2):
        assert all(torch.equal(g, want[i]) for g in got[i])


def test_captured_and_replayed(binding):
    """A drafts' pass in a graph: replayed on new inputs and on the same ones it gives what the call gives."""
    cache, _, gen = plain_cache(binding, 2, 8, 2, 500, 9, extra=8)
    new = [t.cuda() for t in chunk(gen, 2, 8, 2, 5)]
    out = torch.empty_like(new[2])
    scratch = torch.empty(cache.chunk_scratch_bytes(5), dtype=torch.uint8, device="cuda")
    want = cache.chunk_attention(0, *new, SCALE, dtype=torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.chunk_attention(0, *new, SCALE, counts=[5, 3], out=out, scratch=scratch)
    for _ in range(3):
        out.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0], want[0]) and torch.equal(out[1, :, :3], want[1, :, :3]) and (out[1, :, 3:] == 5.0).all()
    other = [t.cuda() for t in chunk(gen, 2, 8, 2, 5)]
    for t, o in zip(new, other):
        t.copy_(o)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[0], cache.chunk_attention(0, *other, SCALE, dtype=torch.bfloat16)[0])
    assert cache.status() == 0


def test_more_sequences_than_a_launch_takes(binding):
    B = 131
    cache, hist, gen = plain_cache(binding, B, 2, 1, 40, 2, extra=3, residual_len=32)
    new = chunk(gen, B, 2, 1, 3)
    counts = [(b * 7) % 4 for b in range(B)]
    out = cache.chunk_attention(0, *(t.cuda() for t in new), SCALE, counts=counts)
    assert cache.status() == 0
    w = W.small(W.CONFIGS["tiny"], n_layers=1, batch=B, n_kv_heads=1, n_q_heads=2, tokens=40, residual_len=32, **W.P24)
    keep = [0, 5, 127, 128, 129, 130]
    sts = {k: s for k, s in CU.streams(w, [40] * B, *hist).items() if k[0] in keep}
    CU.check(w, out, sts, *new, counts)


def test_no_new_tokens(binding):
    cache, _, gen = plain_cache(binding, 2, 4, 2, 100, 1, extra=4)
    new = [t.cuda() for t in chunk(gen, 2, 4, 2, 4)]
    out = torch.full_like(new[2], 7.0)
    before = cache.launch_count()
    cache.chunk_step(0, *new, SCALE, counts=[0, 0], out=out)
    assert cache.launch_count() == before and (out == 7.0).all() and cache.sequence_fill(0, 0) == (0, 100, 0)


def test_a_wait_that_runs_out(binding):
    """The first key tile is never announced: the call returns, the status says so, and the next call is as usual."""
    cache, _, gen = plain_cache(binding, 1, 8, 1, 700, 4, extra=50)
    new = [t.cuda() for t in chunk(gen, 1, 8, 1, 50)]
    want = cache.chunk_attention(0, *new, SCALE)
    cache.test_arm_copy_timeout(16, 200)
    cache.chunk_attention(0, *new, SCALE)
    assert cache.status() == binding.DEV_COPY_TIMEOUT
    cache.test_arm_copy_timeout(0, 0)
    assert torch.equal(cache.chunk_attention(0, *new, SCALE), want)


def test_refusals(binding):
    cache, _, gen = plain_cache(binding, 2, 4, 2, 60, 1, extra=8)
    k, v, q = (t.cuda() for t in chunk(gen, 2, 4, 2, 8))
    before = cache.launch_count()
    for bad in (dict(k=k.float()), dict(k=k[:1]), dict(v=v[:, :, :4]), dict(q=q.transpose(1, 2)), dict(q=q.cpu()), dict(counts=[1]), dict(out=q.half()),
                dict(out=q[:, :2]), dict(scratch=torch.empty(1 << 20, device="cuda")), dict(dtype=torch.float16)):
        with pytest.raises(ValueError):
            cache.chunk_attention(0, **{**dict(k=k, v=v, q=q, scale=SCALE), **bad})
    small = torch.empty(cache.chunk_scratch_bytes(8) - 16, dtype=torch.uint8, device="cuda")
    over = torch.empty(cache.chunk_scratch_bytes(8) + v.numel() * 2, dtype=torch.uint8, device="cuda")
    inside = over[-v.numel() * 2 - 16:-16].view(torch.bfloat16).view(v.shape)
    odd = torch.empty(cache.chunk_scratch_bytes(8) + 16, dtype=torch.uint8, device="cuda")[1:]
    for bad, code in ((dict(counts=[9, 1]), -1), (dict(counts=[-1, 1]), -1), (dict(scale=0.0), -1), (dict(scale=float("nan")), -1), (dict(layer=1), -1),
                      (dict(scratch=small), -4), (dict(scratch=odd), -3), (dict(out=q), -1),
                      (dict(v=inside, scratch=over), -1)):
        with pytest.raises(binding.MixKVQError) as e:
            cache.chunk_attention(**{**dict(layer=0, k=k, v=v, q=q, scale=SCALE), **bad})
        assert e.value.code == code
    with pytest.raises(binding.MixKVQError) as e:                     # 60 + 10 of 69 tokens: nothing is enqueued
        cache.chunk_step(0, *(t.cuda() for t in chunk(gen, 2, 4, 2, 10)), SCALE)
    assert e.value.code == -5
    tile = binding.Cache(binding.make_config(1, 2, 4, 2, 256, block_layout=1))
    with pytest.raises(binding.MixKVQError) as e:
        tile.chunk_attention(0, k, v, q, SCALE)
    assert e.value.code == -2
    assert cache.launch_count() == before and cache.status() == 0 and cache.sequence_fill(0, 0) == (0, 60, 0)
