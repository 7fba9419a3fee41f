"""GPU tests of the chunk attention's precision over long segments: weights far below a row's largest one, sums over many tiles."""
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
