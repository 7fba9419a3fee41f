"""GPU tests of what the chunk attention's calls refuse and report beside those of their edges."""
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


def test_output_and_scratch_over_the_cache(binding):
    """Refused, by both calls, with nothing enqueued or changed; beside the cache's memory they are taken."""
    B, Hq, Hkv, n = 2, 4, 2, 8
    cfg = binding.make_config(1, B, Hq, Hkv, 100000)
    cache = binding.Cache(cfg)
    k, v, q = (torch.randn((B, h, n, 128), device="cuda").bfloat16() for h in (Hkv, Hkv, Hq))
    cache.quantize_append(0, k, v, q)
    size, before, was = 2 * q.numel(), cache.launch_count(), cache.mem.clone()
    scratch = cache.chunk_scratch_bytes(n)
    assert scratch < cache.mem.numel() - 256
    for at in (256, cache.mem.numel() - size):
        out = cache.mem[at:at + size].view(torch.bfloat16).view(q.shape)
        for call in (cache.chunk_attention, cache.chunk_step):
            with pytest.raises(binding.MixKVQError) as e:
                call(0, k, v, q, SCALE, out=out)
            assert e.value.code == -1
    for call in (cache.chunk_attention, cache.chunk_step):
        with pytest.raises(binding.MixKVQError) as e:
            call(0, k, v, q, SCALE, scratch=cache.mem[256:256 + scratch])
        assert e.value.code == -1
    torch.cuda.synchronize()
    assert cache.launch_count() == before and torch.equal(cache.mem, was) and cache.sequence_fill(0, 0) == (0, n, 0)


@pytest.mark.parametrize("preset", ["P24", "P27", "P4BASE"])
@pytest.mark.parametrize("n", [1, 30])
def test_behind_a_full_arena(binding, preset, n):
    """Blocks that found no room for their promoted channels: the status says so, and the chunk reads them as the decode kernels do (the plain one, in 32
    bits).  A token that all rows see decides nothing here: the last of the chunk's rows is the decode step's."""
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=2, tokens=700, **getattr(W, preset))
    cache = U.make_cache(binding, w, extras_budget_bytes=2048 if preset == "P24" else 8192)
    full = U.make_cache(binding, w, extras_budget_bytes=10 * 320 * 128)
    part = [t.cuda() for t in W.tokens(w, 0, 0, 600)]
    new = [t[:, :, :n].contiguous() for t in (x.cuda() for x in W.tokens(w, 0, 600, n))]
    for c in (cache, full):
        c.quantize_append(0, *part)
    assert cache.status() == binding.DEV_EXTRAS_FULL and full.status() == 0
    out = cache.chunk_attention(0, *new, SCALE)
    assert not torch.equal(out, full.chunk_attention(0, *new, SCALE))
    cache.quantize_append(0, *new)
    cache.set_attention_kernel(1)
    ref = cache.decode_attention(0, new[2][:, :, -1].contiguous(), SCALE)
    assert cache.status() == binding.DEV_EXTRAS_FULL
    # keys, values and probabilities in fp16: each moves the output by 2^-11 / sqrt(3) of its own root mean square, the keys' through logits of about 2
    d = (out[:, :, -1] - ref).double()
    assert float(d.norm() / ref.double().norm()) <= 8e-4
