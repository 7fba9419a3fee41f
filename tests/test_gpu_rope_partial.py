"""GPU tests of the rotation of part of the head (the bits of the defined arithmetic in both pairings and every layout) and of the tables with scaled frequencies."""
import math

import numpy as np
import pytest
import torch

import paged_util as P

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19206_b200 import build
    build.build()
    from paper_2512_19206_b200 import binding as b
    b.lib()
    return b


def tables(n_pos, rotary):
    ang = np.arange(n_pos, dtype=np.float64)[:, None] * 1e4 ** (-np.arange(rotary // 2, dtype=np.float64) * 2 / rotary)[None]
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


@pytest.mark.parametrize("rotary", [16, 32, 48, 64, 96, 112, 128])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("B,Hq,Hkv,n", [(1, 1, 1, 1), (3, 28, 4, 1), (2, 8, 2, 17), (1, 40, 8, 200)])
@pytest.mark.parametrize("layout", ["projection", "heads", "gaps"])
def test_bits_of_the_rotation(binding, rotary, interleaved, B, Hq, Hkv, n, layout):
    cos, sin = tables(300, rotary)
    q, k, v = P.draw(B, Hq, Hkv, n, rotary + n)
    pos = torch.randint(0, 300, (B, n), dtype=torch.int32, generator=torch.Generator().manual_seed(n))
    if layout == "projection":
        x = torch.cat([t.transpose(1, 2) for t in (q, k, v)], 2).contiguous().cuda()
        ins = [t.transpose(1, 2) for t in x.split((Hq, Hkv, Hkv), 2)]
    elif layout == "heads":
        ins = [t.cuda() for t in (q, k, v)]
    else:
        ins = []
        for t in (q, k, v):
            room = torch.zeros((B, t.shape[1], n + 2, 144), dtype=torch.bfloat16, device="cuda")
            room[:, :, :n, :128] = t.cuda()
            ins.append(room[:, :, :n, :128])
    cache = binding.Cache(binding.make_config(1, B, Hq, Hkv, 1))
    turn = (torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), pos.cuda(), interleaved)
    out = cache.rope_partial(*ins, *turn)
    assert cache.status() == 0
    for got, want in zip(out, (P.rotate(q, cos, sin, pos.numpy(), interleaved), P.rotate(k, cos, sin, pos.numpy(), interleaved), v)):
        assert torch.equal(got.cpu(), want)
    if layout == "heads":                                    # in place, and without the values
        again = cache.rope_partial(ins[0], ins[1], None, *turn, out=(ins[0], ins[1], None))
        assert again[2] is None and torch.equal(ins[0], out[0]) and torch.equal(ins[1], out[1])


def test_whole_head_in_halves_is_the_rotation_with_one_axis(binding):
    cos, sin = (torch.from_numpy(t).cuda() for t in tables(64, 128))
    q, k, v = (t.cuda() for t in P.draw(2, 8, 2, 30, 1))
    pos = torch.randint(0, 64, (2, 30), dtype=torch.int32, device="cuda")
    cache = binding.Cache(binding.make_config(1, 2, 8, 2, 1))
    a = cache.rope_axes(q, k, v, cos, sin, pos[None].contiguous(), [0] * 64)
    b = cache.rope_partial(q, k, v, cos, sin, pos)
    assert all(torch.equal(x, y) for x, y in zip(a, b))


def test_padding_and_bad_positions(binding):
    cos, sin = tables(20, 32)
    q, k, v = P.draw(2, 4, 2, 40, 2)
    pos = torch.randint(0, 20, (2, 40), dtype=torch.int32, generator=torch.Generator().manual_seed(1))
    pos[1, 25:], pos[0, 7] = -1, 20
    cache = binding.Cache(binding.make_config(1, 2, 4, 2, 1))
    out = tuple(torch.full(t.shape, 3.0, dtype=torch.bfloat16, device="cuda") for t in (q, k, v))
    cache.rope_partial(q.cuda(), k.cuda(), v.cuda(), torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda(), pos.cuda(), True, out=out)
    assert cache.status() == binding.DEV_BAD_POSITION
    good = ((pos >= 0) & (pos < 20))[:, None, :, None]
    for got, src, turned in zip(out, (q, k, v), (True, True, False)):
        ref = P.rotate(src, cos, sin, pos.clamp(0, 19).numpy(), True) if turned else src
        assert torch.equal(got.cpu(), torch.where(good, ref, torch.full_like(ref, 3.0)))


def frequencies(d, base, scaling, factor=1.0, original=0, low=1.0, high=4.0, fast=32.0, slow=1.0):
    """In Python's floats, pair by pair, and the factor of the entries."""
    out, m = [], 1.0
    for i in range(d // 2):
        f = base ** (-2.0 * i / d)
        if scaling == "linear":
            f /= factor
        elif scaling == "ntk":
            f = (base * factor ** (d / (d - 2.0))) ** (-2.0 * i / d)
        elif scaling == "bands":
            turns = original * f / (2 * math.pi)
            t = min(max((turns - low) / (high - low), 0.0), 1.0)
            f = t * f + (1 - t) * f / factor
        elif scaling == "yarn":
            lo, hi = (d * math.log(original / (2 * math.pi * x)) / (2 * math.log(base)) for x in (fast, slow))
            lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), d - 1)
            t = min(max((i - lo) / max(hi - lo, 1e-3), 0.0), 1.0)
            f = (1 - t) * f + t * f / factor
            m = 0.1 * math.log(factor) + 1
        out.append(f)
    return np.asarray(out), m


@pytest.mark.parametrize("d,base,how", [(128, 1e4, dict(scaling="none")), (64, 1e6, dict(scaling="linear", factor=4.0)), (96, 5e5, dict(scaling="ntk", factor=8.0)),
                                        (128, 5e5, dict(scaling="bands", factor=8.0, original=8192, low=1.0, high=4.0)), (16, 1e4, dict(scaling="yarn", factor=16.0, original=4096)),
                                        (128, 1e6, dict(scaling="yarn", factor=4.0, original=32768, fast=32.0, slow=1.0))])
@pytest.mark.parametrize("n,start", [(1, 0), (7, 100003), (1000, 0), (5001, 1 << 20), (70000, 12345)])
def test_tables(binding, d, base, how, n, start):
    """Entries are rounded to float once: off by at most half a step of an entry (2^-24 of m), and by the angle's own 64-bit rounding."""
    cos, sin = binding.rope_tables(n, d, base, start=start, **how)
    assert cos.shape == sin.shape == (n, d // 2)
    f, m = frequencies(d, base, **how)
    a = np.arange(start, start + n, dtype=np.float64)[:, None] * f[None]
    slack = m * (2.0 ** -24 + 2.0 ** -50 * (start + n) + 2.0 ** -46)      # the angle's rounding and that of pi and of a run's products
    for got, want in ((cos, np.cos(a) * m), (sin, np.sin(a) * m)):
        assert np.abs(got.cpu().numpy().astype(np.float64) - want).max() <= slack


def test_tables_continue_one_another(binding):
    whole = binding.rope_tables(3000, 128, 1e6, "yarn", factor=4.0, original=1024)
    part = binding.rope_tables(1000, 128, 1e6, "yarn", factor=4.0, original=1024, start=2000)
    assert all((a[2000:] - b).abs().max() <= 2.0 ** -23 for a, b in zip(whole, part))
    other = binding.rope_tables(8, 128, attention_factor=0.5)
    plain = binding.rope_tables(8, 128)
    assert all(torch.equal(a, 0.5 * b) for a, b in zip(other, plain))


def test_refusals(binding):
    cache = binding.Cache(binding.make_config(1, 2, 4, 2, 1))
    q, k, v = (torch.zeros((2, h, 5, 128), dtype=torch.bfloat16, device="cuda") for h in (4, 2, 2))
    cos, sin = (torch.zeros((9, 32), device="cuda") for _ in range(2))
    pos = torch.zeros((2, 5), dtype=torch.int32, device="cuda")
    before = cache.launch_count()
    for bad in (dict(cos=cos.double()), dict(sin=sin[:4]), dict(positions=pos.long()), dict(positions=pos[:, :4]), dict(q=q.float()), dict(q=k), dict(k=k.cpu()),
                dict(v=v.transpose(2, 3)), dict(out=(q, k, None)), dict(positions=pos.cpu())):
        with pytest.raises(ValueError):
            cache.rope_partial(**{**dict(q=q, k=k, v=v, cos=cos, sin=sin, positions=pos), **bad})
    odd = torch.zeros((9, 12), device="cuda")
    wide = torch.zeros((2, 4, 5, 132), dtype=torch.bfloat16, device="cuda")
    for bad, code in ((dict(cos=odd, sin=odd), -2), (dict(q=wide[..., :128]), -3), (dict(out=(q, k, k)), -1), (dict(out=(k.new_empty(q.shape), k, k)), -1)):
        with pytest.raises(binding.MixKVQError) as e:
            cache.rope_partial(**{**dict(q=q, k=k, v=v, cos=cos, sin=sin, positions=pos), **bad})
        assert e.value.code == code
    assert cache.launch_count() == before and cache.status() == 0
    for bad in (dict(scaling="other"), dict(attention_factor=-1.0), dict(n_positions=0), dict(out=(cos, sin)), dict(out=(cos.cpu(), sin.cpu()))):
        with pytest.raises(ValueError):
            binding.rope_tables(**{**dict(n_positions=9, rotary_dim=128), **bad})
    for bad, code in ((dict(rotary_dim=24), -2), (dict(base=1.0), -1), (dict(factor=0.0), -1), (dict(scaling="yarn"), -1), (dict(scaling="bands", original=10, low=4.0, high=4.0), -1),
                      (dict(start=-1), -1), (dict(out=(cos, cos), rotary_dim=64), -1)):
        with pytest.raises(binding.MixKVQError) as e:
            binding.rope_tables(**{**dict(n_positions=9, rotary_dim=128), **bad})
        assert e.value.code == code
