"""GPU tests of the chunk attention against its operand roundings restated on the CPU: what is left is small enough for one key too many or too few to
show, with the model's queries and with queries of zero, for which every key weighs the same."""
import pytest
import torch

import chunk_rounding as CR
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


def both(binding, w, lens, counts, seed=1, dtype=torch.float32, only=None, **kw):
    """Chunks of `counts` new tokens behind sequences of `lens`, with the model's queries and with queries of zero."""
    k, v, q = W.tokens(w, 0, 0, max(max(lens), 1))
    gen, n = torch.Generator().manual_seed(seed), max(counts)
    kn, vn = (torch.randn((w.batch, w.n_kv_heads, n, 128), generator=gen).to(torch.bfloat16) for _ in range(2))
    qn = (torch.randn((w.batch, w.n_q_heads, n, 128), generator=gen) * W.layer_gains(w, 0)[2][None, :, None]).to(torch.bfloat16)
    cache = U.make_cache(binding, w, max_tokens=max(lens) + 1, extras_budget_bytes=(max(lens) // w.residual_len + 3) * 320 * w.residual_len, **kw)
    if max(lens):
        cache.quantize_append_ragged(0, k.cuda(), v.cuda(), q.cuda(), lens)
    sts = CU.streams(w, lens, k, v, q, **kw)
    for queries in (qn, torch.zeros_like(qn)):
        out = torch.full(qn.shape, 7.0, device="cuda", dtype=dtype)
        cache.chunk_attention(0, kn.cuda(), vn.cuda(), queries.cuda(), SCALE, counts=counts, out=out)
        assert cache.status() == 0
        CR.check(w, out, sts, kn, vn, queries, counts, SCALE, only)
        for b, m in enumerate(counts):
            assert (out[b, :, m:] == 7.0).all()
    return sts


@pytest.mark.parametrize("preset", ["P24", "P27", "P4BASE"])
@pytest.mark.parametrize("R,G", [(128, 32), (32, 32), (64, 64), (256, 128), (96, 32)])
def test_presets_and_block_sizes(binding, preset, R, G):
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=1, tokens=700, residual_len=R, group_size=G, **getattr(W, preset))
    both(binding, w, [700], [9])


@pytest.mark.parametrize("preset,v_bits", [("P24", 4), ("P27", 2), ("P4BASE", 2)])
@pytest.mark.parametrize("R,G", [(160, 32), (192, 64), (224, 32)])
def test_blocks_whose_units_divide_no_tile(binding, preset, v_bits, R, G):
    """Five, six and seven units a block: tiles begin anywhere in a block, and a thread block's share anywhere in the sequence."""
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=1, n_kv_heads=2, n_q_heads=6, tokens=2900, residual_len=R, group_size=G, **getattr(W, preset))
    both(binding, w, [2900], [7], v_bits=v_bits)


@pytest.mark.parametrize("v_bits,sink,preset", [(4, 0, "P24"), (4, 32, "P4BASE"), (2, 64, "P27")])
@pytest.mark.parametrize("tokens", [1, 31, 200, 901])
def test_values_and_sinks(binding, v_bits, sink, preset, tokens):
    w = W.small(W.CONFIGS["llama8b"], n_layers=1, batch=1, n_kv_heads=2, n_q_heads=8, tokens=tokens, **getattr(W, preset))
    both(binding, w, [tokens], [5], v_bits=v_bits, sink_len=sink)


@pytest.mark.parametrize("g", [1, 2, 3, 5, 7, 8])
@pytest.mark.parametrize("n", [1, 16, 17, 37, 130])
def test_rows_of_every_group_size(binding, g, n):
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=2, n_kv_heads=2, n_q_heads=2 * g, tokens=300, **W.P24)
    both(binding, w, [300, 300], [n, n], seed=g + n)


@pytest.mark.parametrize("tokens", [0, 1, 127, 128, 129, 256, 257, 384, 512, 513])
@pytest.mark.parametrize("n", [1, 127, 128, 129])
def test_key_tiles_that_end_anywhere(binding, tokens, n):
    w = W.small(W.CONFIGS["tiny"], n_layers=1, tokens=max(tokens, 1), residual_len=32, **W.P24)
    both(binding, w, [tokens], [n], seed=tokens + n)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_ragged_batch(binding, dtype):
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=6, n_kv_heads=2, n_q_heads=14, tokens=1000, **W.P27)
    both(binding, w, [1000, 0, 129, 640, 77, 300], [3, 40, 0, 300, 1, 20], dtype=dtype, sink_len=32)


@pytest.mark.parametrize("tokens,n", [(0, 1000), (2500, 700)])
def test_long_chunks(binding, tokens, n):
    w = W.small(W.CONFIGS["qwen7b"], n_layers=1, batch=1, tokens=max(tokens, 1), **W.P24)
    both(binding, w, [tokens], [n], only=[(0, 0), (0, 3)])


@pytest.mark.parametrize("n16,n4", [(40, 0), (0, 70), (33, 95), (64, 64), (1, 1), (128, 0), (0, 128), (31, 65), (5, 3)])
@pytest.mark.parametrize("n", [3, 40])
def test_fixed_budgets(binding, n16, n4, n):
    """Lists of promoted channels longer than a warp: more than 32 BF16 channels, more than 32 pairs of UINT4 channels; odd numbers of both."""
    w = W.small(W.CONFIGS["llama8b"], n_layers=1, batch=1, n_kv_heads=2, n_q_heads=8, tokens=330, residual_len=64)
    sts = both(binding, w, [330], [n], budget_bf16=n16, budget_u4=n4)
    tiers = next(iter(sts.values())).blocks[0].tiers
    assert ((tiers == 2).sum(), (tiers == 1).sum()) == (n16, n4)


@pytest.mark.parametrize("n4", [64, 37])
def test_four_bit_keys_are_rounded_once(binding, n4):
    st, kn, vn, qn = CR.offset_keys(n4)
    w, k, v, q = st.source
    cache = U.make_cache(binding, w, extras_budget_bytes=8 * 320 * w.residual_len, budget_u4=n4)
    cache.quantize_append(0, k.cuda(), v.cuda(), q.cuda())
    out = cache.chunk_attention(0, kn[None, None].cuda(), vn[None, None].cuda(), qn[None].cuda(), SCALE)
    assert cache.status() == 0
    CR.check(w, out, {(0, 0): st}, kn[None, None], vn[None, None], qn[None], [len(kn)], SCALE)
