"""GPU tests of the chunk attention's joined partial results: what is no number survives a weight that rounds to zero."""
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


def definition(st, kn, vn, qn):
    """Eq. 1 row by row over the keys that the row sees."""
    K, V = torch.cat([torch.from_numpy(st.keys()), kn.double()]), torch.cat([torch.from_numpy(st.values()), vn.double()])
    held = K.shape[0] - kn.shape[0]
    out = torch.empty(qn.shape, dtype=torch.float64)
    for h in range(qn.shape[0]):
        for j in range(qn.shape[1]):
            m = held + j + 1
            out[h, j] = (torch.softmax((K[:m] @ qn[h, j].double()) * SCALE, 0)[:, None] * V[:m]).sum(0)
    return out


@pytest.mark.parametrize("tokens,n", [(65, 5), (65, 70), (1500, 5), (1500, 40), (1500, 300), (3000, 1)])
@pytest.mark.parametrize("what", ["value nan", "value inf", "value -inf", "values inf and -inf", "key nan", "held value inf"])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_far_below_the_packed_keys(binding, tokens, n, what, dtype):
    """The packed keys' logits lie 226 above those of the window and the new tokens: e^-226 is zero in 32 bits, and infinity or NaN times it is not.
    (65 tokens: one thread block, whose two slots are joined.  1500: the window and the new tokens in another thread block than the packed ones.)"""
    w = W.small(W.CONFIGS["tiny"], n_layers=1, n_q_heads=2, tokens=tokens, residual_len=64)
    gen = torch.Generator().manual_seed(tokens + n)
    k, v, q = (torch.randn((1, h, tokens, 128), generator=gen).to(torch.bfloat16) for h in (1, 1, 2))
    kn, vn, qn = (torch.randn((1, h, n, 128), generator=gen).to(torch.bfloat16) for h in (1, 1, 2))
    packed = (tokens - 1) // 64 * 64
    k[..., 0] = 0.0
    k[:, :, :packed, 0] = 40.0                               # a group without a range: stored exactly
    kn[..., 0], qn[..., 0] = 0.0, 64.0
    inf, nan, at = float("inf"), float("nan"), n // 2
    if what == "value nan":
        vn[0, 0, at, 5] = nan
    elif what == "value inf":
        vn[0, 0, at, 5] = inf
    elif what == "value -inf":
        vn[0, 0, at, 5] = -inf
    elif what == "values inf and -inf":
        vn[0, 0, 0, 5], vn[0, 0, at, 6], vn[0, 0, n - 1, 5], vn[0, 0, n - 1, 7] = inf, inf, -inf, -inf
    elif what == "key nan":
        kn[0, 0, at, 9] = nan
    else:
        v[0, 0, packed, 5] = inf                             # the window's first row
    cache = U.make_cache(binding, w)
    cache.quantize_append(0, k.cuda(), v.cuda(), q.cuda())
    assert cache.sequence_fill(0, 0) == (packed // 64, tokens - packed, 0)
    out = cache.chunk_attention(0, kn.cuda(), vn.cuda(), qn.cuda(), SCALE, dtype=dtype).double().cpu()[0]
    assert cache.status() == 0
    ref = definition(CU.streams(w, [tokens], k, v, q)[(0, 0)], kn[0, 0], vn[0, 0], qn[0])
    assert not torch.isfinite(ref).all()
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    for s in (inf, -inf):
        assert torch.equal(out == s, ref == s)
    fine = torch.isfinite(ref)
    # a logit of 226 in fp32: 2^-16 of it, less than 2^-11 of a probability; keys and probabilities in fp16; bf16 outputs by half a step
    tol = 4e-3 + (2.0 ** -8 * ref[fine].abs() if dtype == torch.bfloat16 else 0.0)
    assert not fine.any() or bool(((out - ref)[fine].abs() <= tol).all())
