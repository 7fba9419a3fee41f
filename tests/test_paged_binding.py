"""The paged cache's and the partial rotation's calls without a GPU: what the binding refuses, what it passes on, null handles, sizes, structures."""
import contextlib
import ctypes as C
import os
import subprocess

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
def native(monkeypatch):
    n = Recorder()
    n.calls = []
    monkeypatch.setattr(binding, "_native", n)
    monkeypatch.setattr(binding, "_stream", lambda: 0)
    monkeypatch.setattr(binding, "_device_of", lambda dev: contextlib.nullcontext())
    return n


@pytest.fixture
def cache(native):
    c = object.__new__(binding.PagedCache)
    c.handle = C.c_void_p(None)
    c.cfg = binding.make_paged_config(1, HQ, HKV, 4, page_tokens=16)
    c.mem = torch.empty(1, dtype=torch.uint8)
    c.native = native
    return c


def tensors(n=N):
    return dict(zip("kvq", (torch.zeros((B, h, n, 128), dtype=torch.bfloat16) for h in (HKV, HKV, HQ))))


def where():
    return dict(pages=torch.zeros((B, 3), dtype=torch.int32), lens=torch.zeros(B, dtype=torch.int32))


def test_arguments_are_passed_on(cache):
    t, w = tensors(), where()
    cos = torch.zeros((7, 32))
    wide = torch.zeros((B, 9), dtype=torch.int32)
    assert cache.append(0, t["k"], t["v"], **w) is None
    q = cache.append(0, **t, pages=wide[:, 2:6], lens=w["lens"], counts=w["lens"], cos=cos, sin=cos, interleaved=True)
    assert q.shape == t["q"].shape and not q.any()
    out = cache.attention(0, t["q"], **w, scale=0.1, dtype=torch.bfloat16)
    assert out.dtype == torch.bfloat16
    cache.step(0, **t, **w, scale=0.1)
    k, v = cache.read(0, **w, n_tokens=3)
    assert k.shape == v.shape == (B, HKV, 3, 128)
    (n0, a0), (n1, a1), (n2, a2), (n3, a3), (n4, a4) = cache.native.calls
    assert (n0, n1, n2, n3, n4) == ("paged_append", "paged_append", "paged_attention", "paged_step", "paged_read")
    assert a0[2:4] == (B, N) and a0[5:7] == (3, 3) and a0[8] is None and a0[11] is None and a0[13:19] == (None,) * 6
    assert a1[5:7] == (4, 9) and a1[8] == w["lens"].data_ptr() and a1[15] == 7 and a1[16] is None and a1[17:19] == (64, 1)
    assert a2[11] == 1 and a2[14] == cache.workspace_bytes(B, N, 3) and len(a3) == 26 and len(a1) == 21 and a4[3] == 3


@pytest.mark.parametrize("bad", ["dtype", "batch", "heads", "tokens", "last dimension", "flat", "pages type", "pages rows", "pages strided", "lens", "lens type", "counts",
                                 "cos alone", "positions alone", "tables", "table type", "positions", "q_out", "q_out strided"])
def test_append_refusals(cache, bad):
    t, cos = tensors(), torch.zeros((7, 32))
    pos = torch.zeros((B, N), dtype=torch.int32)
    args = dict(layer=0, **t, **where(), cos=cos, sin=cos, positions=pos)
    args.update({"dtype": dict(k=t["k"].float()), "batch": dict(v=t["v"][:1]), "heads": dict(k=t["q"]), "tokens": dict(q=t["q"][:, :, :4]),
                 "last dimension": dict(k=t["k"].transpose(2, 3).contiguous().transpose(2, 3)), "flat": dict(k=t["k"][0]), "pages type": dict(pages=torch.zeros((B, 3))),
                 "pages rows": dict(pages=torch.zeros((3, 3), dtype=torch.int32)), "pages strided": dict(pages=torch.zeros((3, B), dtype=torch.int32).T),
                 "lens": dict(lens=torch.zeros(3, dtype=torch.int32)), "lens type": dict(lens=torch.zeros(B, dtype=torch.int64)),
                 "counts": dict(counts=torch.zeros((B, 1), dtype=torch.int32)), "cos alone": dict(sin=None), "positions alone": dict(cos=None, sin=None),
                 "tables": dict(sin=cos[:3]), "table type": dict(cos=cos.double()), "positions": dict(positions=pos[:, :2]),
                 "q_out": dict(q_out=t["k"]), "q_out strided": dict(q_out=torch.zeros((B, N, HQ, 128), dtype=torch.bfloat16).transpose(1, 2))}[bad])
    with pytest.raises(ValueError):
        cache.append(**args)
    with pytest.raises(ValueError):
        cache.step(**args, scale=1.0)
    assert not cache.native.calls


def test_append_and_step_without_queries(cache):
    t = tensors()
    with pytest.raises(ValueError):
        cache.append(0, t["k"], t["v"], **where(), q_out=t["q"])
    with pytest.raises(ValueError):
        cache.step(0, t["k"], t["v"], None, **where(), scale=1.0)
    assert not cache.native.calls


@pytest.mark.parametrize("bad", ["dtype", "heads", "strided", "out shape", "out dtype", "out type", "workspace", "pages", "counts"])
def test_attention_refusals(cache, bad):
    q = tensors()["q"]
    args = dict(layer=0, q=q, **where(), scale=1.0)
    args.update({"dtype": dict(q=q.float()), "heads": dict(q=q[:, :2]), "strided": dict(q=torch.zeros((B, N, HQ, 128), dtype=torch.bfloat16).transpose(1, 2)),
                 "out shape": dict(out=q[:, :1].contiguous()), "out dtype": dict(out=q.half()), "out type": dict(dtype=torch.float16), "workspace": dict(workspace=torch.zeros(1 << 20)),
                 "pages": dict(pages=torch.zeros(3, dtype=torch.int32)), "counts": dict(counts=torch.zeros(B))}[bad])
    with pytest.raises(ValueError):
        cache.attention(**args)
    with pytest.raises(ValueError):
        cache.read(0, **where(), n_tokens=2, out=(q, q))
    assert not cache.native.calls


def test_native_calls_check_their_arguments():
    n = binding._calls()
    seqs = [1, 1, None, 1, 1, None, None]
    rest = {"rope_partial": [None, None, None, None, [0] * 9, 1, None, None, 0, None, 0, 0, None, None, None, 0],
            "paged_append": [None, 0, *seqs, None, None, None, [0] * 9, None, None, 0, None, 0, 0, None, 0], "paged_read": [None, 0, *seqs, None, None, 0],
            "paged_attention": [None, 0, *seqs, None, None, 0, 1.0, None, 0, 0],
            "paged_step": [None, 0, *seqs, None, None, None, [0] * 9, None, None, 0, None, 0, 0, None, None, 0, 1.0, None, 0, 0]}
    for name, args in rest.items():
        call = getattr(n, name)
        assert call(*args) == -1
        with pytest.raises(TypeError):
            call(*args[:-1])
        for i, a in enumerate(args):
            if isinstance(a, list):
                for bad in ([0] * 8, None, [1 << 80] * 9):
                    with pytest.raises((ValueError, TypeError, OverflowError)):
                        call(*args[:i], bad, *args[i + 1:])


def test_null_handles_sizes_and_configurations():
    lib = binding.lib()
    assert lib.mixkvq_paged_append(None, 0, None, None, None, None, None, None, None, None) == -1
    assert lib.mixkvq_paged_read(None, 0, None, None, None, None) == -1
    assert lib.mixkvq_paged_attention(None, 0, None, None, None, 0, 1.0, None, 0, None) == -1
    assert lib.mixkvq_paged_step(None, 0, None, None, None, None, None, None, None, None, 0, 1.0, None, 0, None) == -1
    assert lib.mixkvq_rope_partial(None, None, None, None, None, 1, None, None, None, None, None) == -1
    assert lib.mixkvq_rope_tables(None, 0, 1, None, None, None) == -1
    assert lib.mixkvq_paged_query_status(None, None, None) == -1 and lib.mixkvq_paged_clear_status(None, None) == -1
    assert lib.mixkvq_paged_launch_count(None) == 0 and lib.mixkvq_paged_init(None, None, 0, None, None) == -1
    assert lib.mixkvq_paged_workspace_bytes(None, 1, 1, 1) == 0
    n = C.c_size_t()
    for G, tile in ((32, 2560), (64, 2304), (128, 2176)):
        cfg = binding.make_paged_config(3, 8, 2, 10, page_tokens=64, group_size=G)
        assert lib.mixkvq_paged_bytes(C.byref(cfg), C.byref(n)) == 0 and n.value == 256 + 3 * 10 * 2 * 4 * tile
        assert lib.mixkvq_paged_workspace_bytes(C.byref(cfg), 0, 1, 1) == lib.mixkvq_paged_workspace_bytes(C.byref(cfg), 1, -1, 1) == 0
        assert lib.mixkvq_paged_workspace_bytes(C.byref(cfg), 1, 1, 0) == lib.mixkvq_paged_workspace_bytes(C.byref(cfg), 1, 1, 1 << 30) == 0
        sizes = [lib.mixkvq_paged_workspace_bytes(C.byref(cfg), b, t, p) for b, t, p in ((1, 1, 1), (8, 1, 600), (8, 8, 1), (64, 100, 500), (4096, 2, 9), (1, 5000, 16384), (1, 5000, 1 << 20))]
        assert all(0 < s < 6 << 27 and s % 16 == 0 for s in sizes)
    for field, bad, code in (("n_layers", 0, -1), ("n_q_heads", 7, -1), ("n_q_heads", 32, -2), ("n_kv_heads", 0, -1), ("head_dim", 64, -2), ("n_pages", 0, -1), ("page_tokens", 8, -2),
                             ("page_tokens", 48, -2), ("page_tokens", 512, -2), ("group_size", 16, -2), ("reserved", 1, -1)):
        cfg = binding.make_paged_config(1, 8, 2, 4)
        setattr(cfg, field, bad)
        assert lib.mixkvq_paged_bytes(C.byref(cfg), None) == code, field


def test_structures_match_the_header(tmp_path):
    inc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    names = ["mixkvq_rotation", "mixkvq_rope_scaling", "mixkvq_paged_config", "mixkvq_paged_sequences"]
    src = tmp_path / "t.c"
    src.write_text('#include "mixkvq.h"\n#include <stdio.h>\nint main(void) { printf("' + "%zu " * 4 + '\\n", ' + ", ".join(f"sizeof({n})" for n in names) + "); return 0; }\n")
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-pedantic", "-I", inc, str(src), "-o", str(tmp_path / "t")], check=True)
    sizes = subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout.split()
    assert [int(s) for s in sizes] == [C.sizeof(x) for x in (binding.Rotation, binding.RopeScaling, binding.PagedConfig, binding.Sequences)]


def test_tables_refusals():
    for bad in (dict(scaling="other"), dict(n_positions=0), dict(attention_factor=0.0), dict(out=(torch.zeros((9, 64)), torch.zeros((9, 64))))):
        with pytest.raises(ValueError):
            binding.rope_tables(**{"n_positions": 9, "device": "cpu", **bad})
