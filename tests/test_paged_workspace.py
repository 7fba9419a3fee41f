"""The workspace of the paged attention, without a GPU: it never falls as a call grows."""
import ctypes as C

import pytest

from paper_2512_19206_b200 import binding


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2512_19206_b200 import build
    build.build()


def size(cfg, batch, n, pages):
    return binding.lib().mixkvq_paged_workspace_bytes(C.byref(cfg), batch, n, pages)


@pytest.mark.parametrize("Hq,Hkv,page", [(64, 8, 256), (32, 8, 64), (28, 4, 16), (1, 1, 128), (40, 40, 32)])
def test_larger_calls_never_need_less(Hq, Hkv, page):
    cfg = binding.make_paged_config(1, Hq, Hkv, 4, page_tokens=page)
    most = min((1 << 28) // page, 1 << 17)
    pages = sorted({p for e in range(18) for p in ((1 << e) - 1, 1 << e, (1 << e) + 1, 3 << e) if 1 <= p <= most})
    batches, tokens = [1, 2, 3, 7, 8, 9, 33, 500, 4096], [1, 2, 8, 9, 10, 25, 73, 100, 1000, 5000]
    sizes = {(b, n, p): size(cfg, b, n, p) for b in batches for n in tokens for p in pages}
    assert all(s > 0 and s % 16 == 0 for s in sizes.values())
    for axis, steps in enumerate((batches, tokens, pages)):
        for key in sizes:
            at = steps.index(key[axis])
            if at + 1 < len(steps):
                larger = key[:axis] + (steps[at + 1],) + key[axis + 1:]
                assert sizes[key] <= sizes[larger], (key, larger)


def test_the_largest_is_bounded():
    cfg = binding.make_paged_config(1, 64, 8, 4, page_tokens=256)
    assert size(cfg, 4096, 16384, 1 << 20) < 1 << 30
