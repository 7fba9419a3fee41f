"""GPU tests of what the chunk attention's calls refuse and report beside those of their edges."""
import pytest
import torch

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
