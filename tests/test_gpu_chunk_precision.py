"""GPU tests of the chunk attention's precision over long segments: weights far below a row's largest one, sums over many tiles."""
import math

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


def test_a_flat_tail_below_one_key(binding):
    """One key 15 to 21 nats above 16384 others that are equal among themselves, in channels where its value is zero: the others' share of the output is
    there, although each of their weights is below what fp16 holds beside the largest one.  152 items, so that most of an item's keys are one thread
    block's."""
    T, n, Hkv, g = 16384, 1200, 8, 4
    cache = binding.Cache(binding.make_config(1, 1, Hkv * g, Hkv, T))
    k, v = (torch.full((1, Hkv, T, 128), x, device="cuda", dtype=torch.bfloat16) for x in (0.0, 1.0))
    k[:, :, 0, 0], v[:, :, 0] = 24.0, 0.0                     # the group's other keys are 0 and its scale 8: exact, as are values without a range
    cache.quantize_append(0, k, v, torch.ones((1, Hkv * g, T, 128), device="cuda", dtype=torch.bfloat16))
    q = torch.zeros((1, Hkv * g, n, 128), device="cuda", dtype=torch.bfloat16)
    q[..., 0] = torch.linspace(15, 21, n, device="cuda") / (24 * SCALE)
    kn, vn = (torch.full((1, Hkv, n, 128), x, device="cuda", dtype=torch.bfloat16) for x in (0.0, 1.0))
    out = cache.chunk_attention(0, kn, vn, q, SCALE).double()
    assert cache.status() == 0
    tail = (T + torch.arange(n, device="cuda").double()[None, None, :, None]) * torch.exp(-q[..., :1].double() * 24 * SCALE)
    ref = tail / (tail + 1)
    # A weight is rounded by 2^-11 of itself or by 2^-30 of the largest one.  Sums in the tensor core lose up to a unit of 2^-23 for each of a tile's
    # eight steps and one for its products; a logit of 21 in fp32 and its exponential 2^-18.
    tol = (T + n) * 2.0 ** -30 + tail * (2.0 ** -11 + 2.0 ** -18 + 9 * 2.0 ** -23 * ((T + n) / 128 + 4))
    assert bool(((out - ref).abs() <= tol).all()), float(((out - ref).abs() / tol).max())


def test_a_long_flat_sum(binding):
    """524288 keys of equal weight, values with a mean: what the tensor core's truncated sums lose does not grow with the context.  148 items of all keys."""
    T, n, g = 524288, 4736, 8
    gen = torch.Generator(device="cuda").manual_seed(1)
    cache = binding.Cache(binding.make_config(1, 1, g, 1, T))
    total, part = torch.zeros(128, dtype=torch.float64, device="cuda"), 65536
    for _ in range(T // part):
        v = (1 + torch.rand((1, 1, part, 4, 1), generator=gen, device="cuda")).bfloat16().expand(1, 1, part, 4, 32).reshape(1, 1, part, 128)    # exact when packed
        cache.quantize_append(0, torch.zeros_like(v), v, torch.zeros((1, g, part, 128), device="cuda", dtype=torch.bfloat16))
        total += v.double().sum((0, 1, 2))
    vn = (1 + torch.rand((1, 1, n, 128), generator=gen, device="cuda")).bfloat16()
    out = cache.chunk_attention(0, torch.zeros_like(vn), vn, torch.zeros((1, g, n, 128), device="cuda", dtype=torch.bfloat16), SCALE).double()
    assert cache.status() == 0
    ref = (total + vn.double().cumsum(2)) / (T + 1 + torch.arange(n, device="cuda").double()[:, None])
    # equal weights are powers of two; 9 * 2^-23 for each of at most 512 tiles and the few that join them
    tol = (9 * 516 * 2.0 ** -23 + 2.0 ** -20) * ref
    assert bool(((out - ref).abs() <= tol).all()), float(((out - ref).abs() / tol).max())


@pytest.mark.parametrize("trend", [0.0, 1.0, -1.0])
@pytest.mark.parametrize("g,n", [(1, 1), (1, 100), (2, 130)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_segments_in_pieces(binding, trend, g, n, dtype):
    """An item of more than 512 key tiles is summed in pieces, whichever of them has the larger logits; 148 items, so that each is one thread block's.
    Keys are the same over 32 tokens and values over 32 channels: packed, they are exact."""
    B, Hkv, T = 37, 4, 70000
    gen = torch.Generator(device="cuda").manual_seed(n)
    cache = binding.Cache(binding.make_config(1, B, Hkv * g, Hkv, T))
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")            # noqa: E731
    keep, held = [(0, 0), (20, 1), (36, 3)], {}
    for t in range(0, T, 3500):
        k = (rand(B, Hkv, 111, 1, 128) * (0.3 + trend * (t / T - 0.5) * 0.5)).bfloat16().expand(-1, -1, -1, 32, -1).reshape(B, Hkv, 3552, 128)[:, :, t % 32:][:, :, :3500]
        v = (rand(B, Hkv, 3500, 4, 1) + 0.5).bfloat16().expand(-1, -1, -1, -1, 32).reshape(B, Hkv, 3500, 128)
        cache.quantize_append(0, k.contiguous(), v.contiguous(), torch.zeros((B, Hkv * g, 3500, 128), device="cuda", dtype=torch.bfloat16))
        for b, h in keep:
            held.setdefault((b, h), []).append((k[b, h].clone(), v[b, h].clone()))
    kn, vn, q = rand(B, Hkv, n, 128).bfloat16(), rand(B, Hkv, n, 128).bfloat16(), (1.5 * rand(B, Hkv * g, n, 128)).bfloat16()
    out = cache.chunk_attention(0, kn, vn, q, SCALE, dtype=dtype)
    assert cache.status() == 0
    sees = CR.visible(T, n).cuda()
    for b, h in keep:
        K, V = (torch.cat([*(x[i] for x in held[(b, h)]), new[b, h]]).half().double() for i, new in ((0, kn), (1, vn)))
        hs = slice(h * g, h * g + g)
        qq = q[b, hs].half().double()
        p, ref, s = CR.attend(K, V, qq, SCALE, sees)
        step = 0.0 if dtype == torch.float32 else torch.finfo(dtype).eps / 2
        share = CR.worst(out[b, hs].double(), ref, CR.allowed(p, s, K, V, qq, SCALE), step)
        assert share <= 1.0, (b, h, share)


def test_no_number_in_an_earlier_piece(binding):
    """An infinity and a NaN among 70000 new tokens reach the rows behind them through the later pieces of their segments."""
    n = 70000
    gen = torch.Generator(device="cuda").manual_seed(7)
    k, v, q = (torch.randn((1, 1, n, 128), generator=gen, device="cuda").bfloat16() for _ in range(3))
    cache = binding.Cache(binding.make_config(1, 1, 1, 1, 128))
    want = cache.chunk_attention(0, k, v, q, SCALE)
    v2 = v.clone()
    v2[0, 0, 10, 3], v2[0, 0, 300, 4], v2[0, 0, 69000, 5] = float("nan"), float("inf"), float("-inf")
    out = cache.chunk_attention(0, k, v2, q, SCALE)
    assert cache.status() == 0
    rows = torch.arange(n, device="cuda")
    assert torch.equal(torch.isnan(out[0, 0, :, 3]), rows >= 10)
    assert torch.equal(torch.isposinf(out[0, 0, :, 4]), rows >= 300) and torch.equal(torch.isneginf(out[0, 0, :, 5]), rows >= 69000)
    fine = torch.isfinite(out)
    assert int((~fine).sum()) == (n - 10) + (n - 300) + (n - 69000)
    same = fine.clone()
    same[..., 3:6] = False
    assert torch.equal(out[same], want[same])


@pytest.mark.parametrize("name,batch,tokens,preset,v_bits", [("qwen7b", 4, 8000, "P24", 2), ("qwen7b", 4, 8000, "P27", 2), ("llama8b", 2, 8000, "P4BASE", 4),
                                                              ("qwen7b", 1, 32700, "P24", 2), ("llama8b", 1, 32700, "P27", 2), ("llama8b", 1, 65400, "P24", 4)])
def test_relative_error_of_long_caches(binding, name, batch, tokens, preset, v_bits):
    """One new token's chunk against the plain decode kernel, 32 bits throughout, on the same cache with the token appended."""
    w = W.small(W.CONFIGS[name], n_layers=1, batch=batch, tokens=tokens + 1, **getattr(W, preset))
    cache = U.make_cache(binding, w, v_bits=v_bits, extras_budget_bytes=(tokens // 128 + 3) * 64 * 128)
    for t in range(0, tokens, 4096):
        cache.quantize_append(0, *W.tokens(w, 0, t, min(4096, tokens - t), device="cuda"))
    new = W.tokens(w, 0, tokens, 1, device="cuda")
    out = cache.chunk_attention(0, *new, SCALE)[:, :, 0].double()
    fill = cache.sequence_fill(0, 0)
    cache.quantize_append(0, *new)
    assert cache.sequence_fill(0, 0) == (fill[0], fill[1] + 1, 0)                     # (no window was packed in between)
    cache.set_attention_kernel(1)
    ref = cache.decode_attention(0, new[2][:, :, 0].contiguous(), SCALE).double()
    assert cache.status() == 0
    # Elements of keys and values and probabilities are rounded to fp16, by at most 2^-11 / sqrt(3) = 2.8e-4 in the root mean square, which would be 6.7e-4 of
    # an output that is a sum of many.  Here one key dominates most rows: what its probability's rounding does is in the denominator too, and its
    # value is a bf16 one or of few bits.  Half way between what that gives, 2.4e-5 to 5.6e-5, and what a denominator of unrounded probabilities
    # gives with a reference that does not make the largest one a power of two, 17.6e-5 to 23.4e-5.
    assert float((out - ref).norm() / ref.norm()) <= 12e-5


@pytest.mark.parametrize("v_bits,preset", [(2, "P24"), (4, "P4BASE")])
@pytest.mark.parametrize("size", [2.0 ** -14, 2.0 ** -17, 2.0 ** -20])
def test_tiny_values(binding, v_bits, preset, size):
    """Values whose groups' scales are below what a quarter of them needs in fp16."""
    w = W.small(W.CONFIGS["llama8b"], n_layers=1, batch=1, n_kv_heads=2, n_q_heads=8, tokens=800, **getattr(W, preset))
    k, v, q = W.tokens(w, 0, 0, 806)
    v = (v.float() * size).bfloat16()
    held, new = [t[:, :, :800].contiguous() for t in (k, v, q)], [t[:, :, 800:].contiguous() for t in (k, v, q)]
    cache = U.make_cache(binding, w, v_bits=v_bits, extras_budget_bytes=10 * 320 * 128)
    cache.quantize_append(0, *(t.cuda() for t in held))
    out = cache.chunk_attention(0, *(t.cuda() for t in new), SCALE).double().cpu()
    assert cache.status() == 0
    for (b, hk), st in CU.streams(w, [800], *held, v_bits=v_bits).items():
        K = torch.cat([CR.fp16(st.keys()), new[0][b, hk].double()])
        V = torch.cat([torch.from_numpy(st.values()), new[1][b, hk].double()])
        qq = new[2][b, hk * 4:hk * 4 + 4].double()
        p, ref, s = CR.attend(K, V, qq, SCALE, CR.visible(800, 6))
        # scale and a quarter of it, zero-point and element each rounded by half a step of fp16 (2^-25 among the subnormals): 5 c + 2 of them for a
        # code c, and the new tokens' one
        tiny = (5 * (2 ** v_bits - 1) + 2) * 2.0 ** -25
        tol = CR.allowed(p, s, K, V, qq, SCALE) + tiny + CR.HALF_STEP * (p @ V.abs())
        assert CR.worst(out[b, hk * 4:hk * 4 + 4], ref, tol) <= 1.0


def test_rows_beside_one_whose_maximum_rises(binding):
    """A weight is rounded once where another row of the same 32 needs its sums rescaled: by 2^-11 of itself, not by that of three roundings.  The first
    quarter of a tile's keys has values of one, the rest of zero; half a tile later every 32nd row's maximum rises by e^22, the others' by e^0.3 to e^2."""
    Hkv, n = 8, 70
    cache = binding.Cache(binding.make_config(1, 1, Hkv, Hkv, 256))
    k, v = (torch.zeros((1, Hkv, 129, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[:, :, :32, 1], k[:, :, 64:128, 1], k[:, :, 64:128, 0], v[:, :, :32] = -1.0, 1.0, 16.0, 1.0            # (groups without a range: exact)
    gen = torch.Generator(device="cuda").manual_seed(2)
    q = torch.zeros((1, Hkv, n, 128), dtype=torch.bfloat16, device="cuda")
    q[..., 1] = (0.3 + 1.7 * torch.rand((1, Hkv, n), generator=gen, device="cuda")) / SCALE
    q[:, :, ::32, 1], q[:, :, ::32, 0] = 0.0, 16.0
    cache.quantize_append(0, k, v, torch.ones_like(k))
    assert cache.sequence_fill(0, 0) == (1, 1, 0)
    zero = torch.zeros((1, Hkv, n, 128), dtype=torch.bfloat16, device="cuda")
    out = cache.chunk_attention(0, zero, zero, q, SCALE).double()
    assert cache.status() == 0
    x = q.double() @ k.double().transpose(-1, -2) * SCALE                            # the new tokens' logits are 0, as the 129th's
    w = x.exp()
    ref = (w[..., :32].sum(-1) / (w.sum(-1) + 1 + torch.arange(n, device="cuda")))[..., None].expand_as(out)
    # One rounding of equal weights: 2^-11 of the first quarter's in the product, 2^-11 of all in the denominator.  In fp32 logits of up to 2 and their
    # exponentials 2^-20, two tiles' sums 2^-18.
    share = ((out - ref).abs() / (ref * (2.0 ** -10 + 2.0 ** -17) + 2.0 ** -40))
    share[:, :, ::32] = 0                                                            # (there the weights are e^-22 of the others)
    assert float(share.max()) <= 1.0, float(share.max())


def test_denominator_of_many_equal_weights(binding):
    """65000 keys of one weight that is no power of two, beside 32 of twice that: every fourth key's value is one, so that the tensor core's sums stay within 24
    bits and only the denominator can be off.  148 items of all keys and 256 rows."""
    B, Hkv, T, n, part = 37, 4, 65000, 256, 3250
    cache = binding.Cache(binding.make_config(1, B, Hkv, Hkv, T))
    v = torch.zeros((B, Hkv, T, 128), device="cuda", dtype=torch.bfloat16)
    v[:, :, ::4] = 1.0
    for t in range(0, T, part):
        k = torch.zeros((B, Hkv, part, 128), device="cuda", dtype=torch.bfloat16)
        if t == 0:
            k[:, :, :32, 0] = 1.0                            # (a group without a range: exact)
        cache.quantize_append(0, k, v[:, :, t:t + part].contiguous(), torch.ones_like(k))
    q, new = (torch.zeros((B, Hkv, n, 128), device="cuda", dtype=torch.bfloat16) for _ in range(2))
    q[..., 0] = 7.8125                                       # e^-0.6905 of the largest: 16.042 in units of its 32nd part, 16.047 in fp16
    out = cache.chunk_attention(0, new, new, q, SCALE).double()
    assert cache.status() == 0
    w = torch.full((T,), 1.0, dtype=torch.float64, device="cuda")
    w[:32] = torch.tensor(7.8125 * SCALE, dtype=torch.float64).exp()
    ref = (w[::4].sum() / (w.sum() + 1 + torch.arange(n, device="cuda")))[:, None].expand_as(out)
    # the rounding of the weights, 3e-4, is in the sum and in the denominator; 64 of 65000 weights are not the others'.  fp32: 2^-18
    share = ((out - ref).abs() / (ref * (2.0 ** -11 * 64 / 16000 + 2.0 ** -18))).max()
    assert float(share) <= 1.0, float(share)


@pytest.mark.parametrize("g,n", [(1, 140), (1, 70), (3, 90)])
def test_weights_of_a_tile_whose_second_half_is_far_above(binding, g, n):
    """A first half whose logits are 9 to 10 (in powers of two) above the ones before, which raises nothing, and a second half 11 to 12 above that: the first half's
    probabilities are scaled by 2^-20 to 2^-22.  Only its keys have values.  148 items and more, so that a thread block has all their tiles."""
    B, Hkv, T = 37, 4, 513
    cache = binding.Cache(binding.make_config(1, B, Hkv * g, Hkv, T))
    k, v = (torch.zeros((B, Hkv, T, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for tile in (1, 2):                                       # (slots of few rows take turns at the tiles)
        k[:, :, 128 * tile:128 * tile + 32, 1], k[:, :, 128 * tile + 64:128 * tile + 96, 1], v[:, :, 128 * tile:128 * tile + 32] = 0.90625, 2.0, 1.0
    cache.quantize_append(0, k, v, torch.ones((B, Hkv * g, T, 128), dtype=torch.bfloat16, device="cuda"))
    gen = torch.Generator(device="cuda").manual_seed(n)
    q = torch.zeros((B, Hkv * g, n, 128), dtype=torch.bfloat16, device="cuda")
    q[..., 1] = (10 + torch.rand((B, Hkv * g, n), generator=gen, device="cuda")) / (SCALE * math.log2(math.e))
    zero = torch.zeros((B, Hkv, n, 128), dtype=torch.bfloat16, device="cuda")
    out = cache.chunk_attention(0, zero, zero, q, SCALE).double()
    assert cache.status() == 0
    x = q.double() @ k.double().repeat_interleave(g, 1).transpose(-1, -2) * SCALE
    w = (x - x.amax(-1, keepdim=True)).exp()
    new = (1 + torch.arange(n, device="cuda")) * (-x.amax(-1)).exp()
    ref = ((w * v.double()[:, :, :, 0].repeat_interleave(g, 1)[:, :, None]).sum(-1) / (w.sum(-1) + new))[..., None].expand_as(out)
    # two roundings of the weight, one more of all in the denominator; logits of 15 in fp32 2^-19, sums 2^-18
    share = ((out - ref).abs() / (ref * (3 * 2.0 ** -11 + 2.0 ** -17))).max()
    assert float(share) <= 1.0, float(share)
