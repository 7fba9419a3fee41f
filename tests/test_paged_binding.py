"""The paged cache's and the partial rotation's calls without a GPU: what the binding refuses, what it passes on, null handles, sizes, structures."""
import contextlib
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2512_19206_b200 import binding

B, HQ, HKV, N = 2, 8, 2, 5


@pytest.fixture(scope="module", autouse=True)
def built():
    from paper_2512_19206_b200 import build
    build.build()


@pytest.fixture
def cache(monkeypatch):
    """A cache without a handle, its memory on the CPU: the calls check their arguments and the library refuses the handle (-1)."""
    monkeypatch.setattr(binding, "_device_of", lambda dev: contextlib.nullcontext())
    c = object.__new__(binding.PagedCache)
    c.handle = C.c_void_p(None)
    c.cfg = binding.make_paged_config(1, HQ, HKV, 4, page_tokens=16)
    c.mem = torch.empty(1, dtype=torch.uint8)
    c._sizes = {}
    return c


def passes(call):
    with pytest.raises(binding.MixKVQError) as e:
        call()
    assert e.value.code == -1


def tensors(n=N):
    return dict(zip("kvq", (torch.zeros((B, h, n, 128), dtype=torch.bfloat16) for h in (HKV, HKV, HQ))))


def where():
    return dict(pages=torch.zeros((B, 3), dtype=torch.int32), lens=torch.zeros(B, dtype=torch.int32))


def test_arguments_that_are_in_order(cache):
    t, w = tensors(), where()
    cos = torch.zeros((7, 32))
    wide = torch.zeros((B, 9), dtype=torch.int32)
    x = torch.zeros((B, N, HQ + 2 * HKV, 128), dtype=torch.bfloat16)
    views = dict(zip("qkv", (y.transpose(1, 2) for y in x.split((HQ, HKV, HKV), 2))))
    passes(lambda: cache.append(0, t["k"], t["v"], **w))
    passes(lambda: cache.append(0, **views, pages=wide[:, 2:6], lens=w["lens"], counts=w["lens"], cos=cos, sin=cos, interleaved=True))
    passes(lambda: cache.append(0, **t, **w, cos=cos, sin=cos, positions=torch.zeros((B, N), dtype=torch.int32), q_out=t["q"]))
    passes(lambda: cache.attention(0, t["q"], **w, scale=0.1, dtype=torch.bfloat16))
    passes(lambda: cache.step(0, **views, **w, scale=1))
    passes(lambda: cache.read(0, **w, n_tokens=3))
    one = torch.zeros((1, 1), dtype=torch.int32)
    passes(lambda: cache.read(0, one.expand(1, 1), torch.zeros(1, dtype=torch.int32), 1))


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


def test_append_and_step_without_queries(cache):
    t = tensors()
    with pytest.raises(ValueError):
        cache.append(0, t["k"], t["v"], **where(), q_out=t["q"])
    with pytest.raises(ValueError):
        cache.step(0, t["k"], t["v"], None, **where(), scale=1.0)


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


@pytest.mark.parametrize("bad", ["dtype", "heads", "tokens", "tables", "no tables", "positions", "no positions", "out", "out alone", "last dimension"])
def test_rotation_refusals(monkeypatch, bad):
    monkeypatch.setattr(binding, "_device_of", lambda dev: contextlib.nullcontext())
    c = object.__new__(binding.Cache)
    c.handle, c.cfg, c.mem = C.c_void_p(None), binding.make_config(1, B, HQ, HKV, 16), torch.empty(1, dtype=torch.uint8)
    t, cos, pos = tensors(), torch.zeros((7, 32)), torch.zeros((B, N), dtype=torch.int32)
    args = dict(**t, cos=cos, sin=cos, positions=pos)
    passes(lambda: c.rope_partial(**args))
    passes(lambda: c.rope_partial(**{**args, "v": None}, out=(t["q"], t["k"], None)))
    args.update({"dtype": dict(q=t["q"].float()), "heads": dict(k=t["q"]), "tokens": dict(v=t["v"][:, :, :4]), "tables": dict(sin=cos[:3]), "no tables": dict(cos=None, sin=None),
                 "positions": dict(positions=pos.long()), "no positions": dict(positions=None), "out": dict(out=(t["q"].transpose(1, 2), t["k"], t["v"])),
                 "out alone": dict(out=(t["q"], t["k"], None)), "last dimension": dict(k=t["k"].transpose(2, 3).contiguous().transpose(2, 3))}[bad])
    with pytest.raises(ValueError if bad != "no tables" else (ValueError, binding.MixKVQError)):
        c.rope_partial(**args)


def test_native_calls_check_their_arguments():
    n = binding._calls()
    who = (None, 1, 0, HQ, HKV)
    t, w = tensors(), where()
    seqs, turn, ws = (w["pages"], w["lens"], None), (None, None, None, False), torch.zeros(16, dtype=torch.uint8)
    calls = {"rope_partial": [who, B, t["q"], t["k"], None, torch.zeros((7, 32)), torch.zeros((7, 32)), torch.zeros((B, N), dtype=torch.int32), 0, t["q"], t["k"], None],
             "paged_append": [who, 0, t["k"], t["v"], None, *seqs, *turn, None], "paged_read": [who, 0, w["pages"], w["lens"], N, None, t["k"], t["v"]],
             "paged_attention": [who, 0, t["q"], w["pages"], w["lens"], 1.0, None, t["q"], ws],
             "paged_step": [who, 0, t["k"], t["v"], t["q"], *seqs, *turn, t["q"].clone(), 1.0, t["q"].clone(), ws]}
    for name, args in calls.items():
        call = getattr(n, name)
        assert call(*args) == -1
        with pytest.raises(TypeError):
            call(*args[:-1])
        with pytest.raises(TypeError):
            call(who[:4], *args[1:])
        for i, a in enumerate(args):
            if isinstance(a, torch.Tensor):
                for bad in (3, "x", a.double(), a[None]):
                    with pytest.raises(ValueError):
                        call(*args[:i], bad, *args[i + 1:])
        with pytest.raises(ValueError):                       # another device than the tensors'
            call((None, 2, 0, HQ, HKV), *args[1:])
    x = torch.zeros((9, 64))
    assert n.rope_tables(9, 128, 0, 1e4, 1.0, 0.0, 1.0, 4.0, 0.0, 0, x, x.clone(), 1, 0) in (0, -1, -6)
    for i, bad, error in ((10, x[:3], ValueError), (3, "a", TypeError), (9, 1 << 80, OverflowError), (10, 5, ValueError)):
        args = [9, 128, 0, 1e4, 1.0, 0.0, 1.0, 4.0, 0.0, 0, x, x.clone(), 1, 0]
        args[i] = bad
        with pytest.raises(error):
            n.rope_tables(*args)


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


def test_sizes_beyond_64_bits_are_refused():
    most, n = (1 << 31) - 1, C.c_size_t()
    for shape, code in (((most, 8, 8, 4), 0), ((most, 8, 8, most), -2), ((1, most, most, most), -2), ((1, 8, 8, most), 0)):
        cfg = binding.make_paged_config(*shape)
        assert binding.lib().mixkvq_paged_bytes(C.byref(cfg), C.byref(n)) == code
        if code == 0:
            assert n.value == 256 + shape[0] * shape[2] * shape[3] * (cfg.page_tokens // 16) * (2048 + 32 * 512 // cfg.group_size)
