"""GPU tests of the chunk attention: every kind of stored token, ragged batches, row and key tiles that end anywhere, both output types."""
import pytest
import torch

import chunk_util as CU
import gpu_util as U
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


def fresh(w, n, seed):
    gen = torch.Generator().manual_seed(seed)
    _, _, qgain = W.layer_gains(w, 0)
    k, v = (torch.randn((w.batch, w.n_kv_heads, n, 128), generator=gen).to(torch.bfloat16) for _ in range(2))
    return k, v, (torch.randn((w.batch, w.n_q_heads, n, 128), generator=gen) * qgain[None, :, None]).to(torch.bfloat16)


def run(binding, w, lens, counts, seed=1, dtype=torch.float32, stride=None, **kw):
    """A cache of sequences of `lens` tokens, a chunk of `counts` new ones each; returns (cache, out, the pieces of the check)."""
    k, v, q = W.tokens(w, 0, 0, max(max(lens), 1))
    n = stride or max(counts)
    kn, vn, qn = fresh(w, n, seed)
    cache = U.make_cache(binding, w, max_tokens=max(lens) + n + 1, extras_budget_bytes=(max(lens) // w.residual_len + 3) * 64 * w.residual_len, **kw)
    if max(lens):
        cache.quantize_append_ragged(0, k.cuda(), v.cuda(), q.cuda(), lens)
    sts = CU.streams(w, lens, k, v, q, **kw)
    out = torch.full((w.batch, w.n_q_heads, n, 128), 7.0, device="cuda", dtype=dtype)
    cache.chunk_attention(0, kn.cuda(), vn.cuda(), qn.cuda(), W.softmax_scale(), counts=counts, out=out)
    assert cache.status() == 0
    for b, m in enumerate(counts):
        assert (out[b, :, m:] == 7.0).all()              # rows behind the count are left as they were
    return cache, out, (sts, kn, vn, qn, counts)


@pytest.mark.parametrize("preset", ["P24", "P27", "P4BASE"])
@pytest.mark.parametrize("R,G", [(128, 32), (32, 32), (64, 64), (256, 128), (96, 32)])
def test_presets_and_block_sizes(binding, preset, R, G):
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=1, tokens=700, residual_len=R, group_size=G, **getattr(W, preset))
    cache, out, pieces = run(binding, w, [700], [9])
    CU.check(w, out, *pieces)


@pytest.mark.parametrize("v_bits,sink,preset", [(4, 0, "P24"), (4, 32, "P4BASE"), (2, 64, "P27")])
@pytest.mark.parametrize("tokens", [1, 31, 200, 901])
def test_values_and_sinks(binding, v_bits, sink, preset, tokens):
    w = W.small(W.CONFIGS["llama8b"], n_layers=1, batch=1, n_kv_heads=2, n_q_heads=8, tokens=tokens, **getattr(W, preset))
    cache, out, pieces = run(binding, w, [tokens], [5], v_bits=v_bits, sink_len=sink)
    CU.check(w, out, *pieces)


@pytest.mark.parametrize("g", [1, 2, 3, 5, 7, 8])
@pytest.mark.parametrize("n", [1, 16, 17, 37, 130])
def test_rows_of_every_group_size(binding, g, n):
    """Items of at most 128 rows (both slots share them), of more, and the last one of a stream."""
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=2, n_kv_heads=2, n_q_heads=2 * g, tokens=300, **W.P24)
    cache, out, pieces = run(binding, w, [300, 300], [n, n], seed=g + n)
    CU.check(w, out, *pieces)


@pytest.mark.parametrize("tokens", [0, 1, 127, 128, 129, 256, 257, 384, 512, 513])
@pytest.mark.parametrize("n", [1, 127, 128, 129])
def test_key_tiles_that_end_anywhere(binding, tokens, n):
    w = W.small(W.CONFIGS["tiny"], n_layers=1, tokens=max(tokens, 1), residual_len=32, **W.P24)
    cache, out, pieces = run(binding, w, [tokens], [n], seed=tokens + n)
    CU.check(w, out, *pieces)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ragged_batch(binding, dtype):
    lens, counts = [1000, 0, 129, 640, 77, 300], [3, 40, 0, 300, 1, 20]
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=6, n_kv_heads=2, n_q_heads=14, tokens=1000, **W.P27)
    cache, out, pieces = run(binding, w, lens, counts, dtype=dtype, stride=310, sink_len=32)
    CU.check(w, out, *pieces)


@pytest.mark.parametrize("tokens,n", [(0, 1000), (2500, 700)])
def test_long_chunks(binding, tokens, n):
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=1, tokens=max(tokens, 1), **W.P24)
    cache, out, pieces = run(binding, w, [tokens], [n])
    CU.check(w, out, *pieces, only=[(0, 0), (0, 3)])
