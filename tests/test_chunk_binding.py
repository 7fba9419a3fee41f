"""The chunk's and the several axes' calls without a GPU: what the binding refuses, what it passes on, null handles, sizes."""
import ctypes as C

import pytest
import torch

from paper_2512_19206_b200 import binding

B, HQ, HKV, N = 2, 8, 2, 5


class Recorder:
    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2512_19206_b200 import build
    build.build()


@pytest.fixture
def cache(monkeypatch):
    native = Recorder()
    native.calls = []
    monkeypatch.setattr(binding, "_native", native)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    import contextlib
    monkeypatch.setattr(binding, "_device_of", lambda dev: contextlib.nullcontext())
    c = object.__new__(binding.Cache)
    c.handle = C.c_void_p(None)
    c.cfg = binding.make_config(1, B, HQ, HKV, 256)
    c.mem = torch.empty(1, dtype=torch.uint8)
    c.native = native
    return c


def tensors(n=N):
    return [torch.zeros((B, h, n, 128), dtype=torch.bfloat16) for h in (HKV, HKV, HQ)]


def test_chunk_arguments_are_passed_on(cache):
    k, v, q = tensors()
    out = cache.chunk_attention(0, k, v, q, 0.1)
    assert out.dtype == torch.float32 and out.shape == q.shape
    out = cache.chunk_step(0, k, v, q, 0.1, counts=[5, 0], dtype=torch.bfloat16)
    assert out.dtype == torch.bfloat16 and not out.any()
    (n0, a0), (n1, a1) = cache.native.calls
    assert n0 == n1 == "chunk" and (a0[0], a1[0]) == (0, 1) and (a0[7], a1[7]) == (None, [5, 0]) and (a0[9], a1[9]) == (0, 1)
    assert a0[12] == a0[11].numel() == cache.chunk_scratch_bytes(N)


@pytest.mark.parametrize("bad", ["dtype", "batch", "heads", "tokens", "strided", "flat", "out shape", "out dtype", "out type", "scratch", "counts"])
def test_chunk_refusals(cache, bad):
    k, v, q = tensors()
    args = dict(layer=0, k=k, v=v, q=q, scale=0.1)
    args.update({"dtype": dict(k=k.float()), "batch": dict(v=v[:1]), "heads": dict(k=q), "tokens": dict(q=q[:, :, :4].contiguous()),
                 "strided": dict(q=torch.zeros((B, N, HQ, 128), dtype=torch.bfloat16).transpose(1, 2)), "flat": dict(k=k[0]), "out shape": dict(out=k),
                 "out dtype": dict(out=q.half()), "out type": dict(dtype=torch.float16), "scratch": dict(scratch=torch.zeros(1 << 24)),
                 "counts": dict(counts=[1, 2, 3])}[bad])
    for call in (cache.chunk_attention, cache.chunk_step):
        with pytest.raises(ValueError):
            call(**args)
    assert not cache.native.calls


def test_native_chunk_and_rotation_check_their_arguments():
    n = binding._calls()
    k, v, q = tensors()
    chunk = [0, None, 0, None, None, None, 1, None, None, 0, 0.1, None, 0, 0]
    assert n.chunk(*chunk) == -1
    with pytest.raises(TypeError):
        n.chunk(*chunk[:-1])
    with pytest.raises(AssertionError):                     # a CPU tensor
        n.chunk(*chunk[:3], k, *chunk[4:])
    for counts, error in ((3, TypeError), (["a"], TypeError), ([1 << 40], OverflowError), ([1 << 80], OverflowError)):
        with pytest.raises(error):
            n.chunk(*chunk[:7], counts, *chunk[8:])
    rope = [None, None, None, None, [0] * 9, 1, None, None, 1, None, 1, bytes(64), None, None, None, 0]
    assert n.rope_axes(*rope) == -1
    for i, bad, error in ((4, [0] * 8, ValueError), (11, bytes(63), ValueError), (11, [0] * 64, TypeError), (4, None, TypeError)):
        with pytest.raises(error):
            n.rope_axes(*rope[:i], bad, *rope[i + 1:])


def test_null_handles_and_sizes():
    lib = binding.lib()
    assert lib.mixkvq_chunk_attention(None, 0, None, None, None, 1, None, None, 0, 1.0, None, 0, None) == -1
    assert lib.mixkvq_chunk_step(None, 0, None, None, None, 1, None, None, 0, 1.0, None, 0, None) == -1
    assert lib.mixkvq_rope_axes(None, None, None, None, None, 1, None, None, 1, None, 1, None, None, None, None, None) == -1
    assert lib.mixkvq_rope_axes_append(None, 0, None, None, None, None, None, 1, None, 1, None, 1, None) == -1
    assert lib.mixkvq_rope_axes_decode_step(None, 0, None, None, None, None, None, 1, None, 1, None, None, 1.0, None, 0, None) == -1
    cfg = binding.make_config(1, B, HQ, HKV, 256)
    size = lambda n: int(lib.mixkvq_chunk_scratch_bytes(C.byref(cfg), n))                          # noqa: E731
    assert size(1) > 0 and size(0) == size(-3) == 0 and int(lib.mixkvq_chunk_scratch_bytes(None, 4)) == 0
    sizes = [size(n) for n in (1, 2, 7, 63, 64, 4096, 1 << 24)]
    assert sizes == sorted(sizes) and sizes[-1] == sizes[-2] == sizes[-3] < 1 << 26                  # (an item has 256 rows at most)
    assert all(s % 16 == 0 for s in sizes)


def test_sections_of_the_axes():
    assert binding.axis_sections((64,)) == [0] * 64
    assert binding.axis_sections((16, 24, 24)) == [0] * 16 + [1] * 24 + [2] * 24
    for bad in ((16, 24), (64, 1), (-1, 65), (13,) * 5):
        with pytest.raises(ValueError):
            binding.axis_sections(bad)


@pytest.mark.parametrize("bad", ["tables", "table type", "positions type", "positions shape", "axes", "q", "out", "v alone", "last dimension"])
def test_rotation_refusals(cache, bad):
    k, v, q = tensors()
    cos = torch.zeros((7, 64))
    pos = torch.zeros((2, B, N), dtype=torch.int32)
    args = dict(q=q, k=k, v=v, cos=cos, sin=cos, positions=pos, axes=binding.axis_sections((32, 32)))
    cache.rope_axes(**args)
    assert len(cache.native.calls) == 1
    args.update({"tables": dict(sin=cos[:3]), "table type": dict(cos=cos.double()), "positions type": dict(positions=pos.long()),
                 "positions shape": dict(positions=pos[:, :1]), "axes": dict(axes=[0] * 63), "q": dict(q=q.float()),
                 "out": dict(out=(q.transpose(1, 2), k, v)), "v alone": dict(out=(q, k, None)), "last dimension": dict(k=k.transpose(2, 3).contiguous().transpose(2, 3))}[bad])
    with pytest.raises(ValueError):
        cache.rope_axes(**args)
    assert len(cache.native.calls) == 1
