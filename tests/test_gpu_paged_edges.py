"""GPU tests of the paged 4-bit cache at the edges of its inputs: zeros, magnitudes, infinities beside large values, NaNs that are appended, rows that a call leaves out."""
import numpy as np
import pytest
import torch

import paged_util as P

pytestmark = pytest.mark.gpu
SCALE = 128 ** -0.5
UNPACKED = 4


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19206_b200 import build
    build.build()
    from paper_2512_19206_b200 import binding as b
    b.lib()
    return b


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def wide(table, page, room):
    more = max(0, room // page - table.shape[1])
    return torch.cat([table, torch.full((table.shape[0], more), -1, dtype=torch.int32)], 1) if more else table


def held(binding, Hq, Hkv, k, v, lens, page=32, G=32):
    """A cache that holds lens[b] tokens of k, v (CPU), and its page table (CPU)."""
    table, n_pages = P.pages_for(lens, page, 3)
    cache = binding.PagedCache(binding.make_paged_config(1, Hq, Hkv, n_pages, page_tokens=page, group_size=G))
    cache.mem[256:] = 0xFF
    cache.append(0, k.cuda(), v.cuda(), table.cuda(), ints([0] * len(lens)), counts=ints(lens))
    return cache, table


@pytest.mark.parametrize("n", [1, 5, 90])
@pytest.mark.parametrize("room", [0, 1 << 16])
@pytest.mark.parametrize("what", ["queries", "keys", "both", "queries, small keys", "keys, small queries", "one tile's keys"])
def test_zeros(binding, n, room, what):
    """Equal logits: the mean of the values seen, whatever factor of the logits a row and a tile of zeros come to."""
    lens, counts = [300, 131], [n, n]
    q, k, v = P.draw(2, 8, 2, 300, 17)
    q = q[:, :, :n].contiguous()
    if what in ("queries", "both", "queries, small keys"):
        q.zero_()
    if what in ("keys", "both", "keys, small queries"):
        k.zero_()
    if what == "one tile's keys":
        k[:, :, 128:] = 0
    if "small" in what:
        q, k = ((x.float() * 2.0 ** -9).to(torch.bfloat16) for x in (q, k))
    cache, table = held(binding, 8, 2, k, v, lens)
    out = cache.attention(0, q.cuda(), wide(table, 32, room).cuda(), ints(lens), SCALE)
    assert cache.status() == 0 and (cache.last_attention() == UNPACKED) == (room > 0 and n == 90)
    P.check(out, q, k, v, 32, SCALE, lens, counts, cache.last_attention() == UNPACKED)


@pytest.mark.parametrize("size", [1e34, 1e35, 1e36])
@pytest.mark.parametrize("n", [1, 4, 40])
@pytest.mark.parametrize("which", ["all", "one"])
def test_queries_near_the_end_of_the_range(binding, size, n, which):
    """Queries as large as bf16 allows before a key: logits that are ordinary, as the keys are as small; or one such row beside ordinary ones."""
    lens = [90, 400]
    q, k, v = P.draw(2, 7, 1, max(lens), 6)
    k = (k.float() / size).to(torch.bfloat16)
    big = (q[:, :, :n].float() * size).to(torch.bfloat16)
    q = big if which == "all" else torch.cat([q[:, :3, :n], big[:, 3:4], q[:, 4:, :n]], 1)
    cache, table = held(binding, 7, 1, k, v, lens)
    for room in (0, 1 << 16):
        out = cache.attention(0, q.contiguous().cuda(), wide(table, 32, room).cuda(), ints(lens), SCALE)
        rounded = cache.last_attention() == UNPACKED
        assert rounded == (room > 0 and n == 40)
        P.check(out, q, k, v, 32, SCALE, lens, [n, n], rounded)


@pytest.mark.parametrize("Hq", [2, 8])
@pytest.mark.parametrize("room", [0, 1 << 10])
@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("bad", ["inf", "-inf", "nan"])
def test_an_infinity_beside_a_large_value(binding, Hq, room, G, bad):
    """The newest value is not finite; the rows that do not see it keep their results, though the same lane of the kernel has a value far larger than the others'."""
    lens, n = [9, 41], 2
    q, k, v = P.draw(2, Hq, 1, 41, 23)
    q = q[:, :, :n].contiguous()
    group = slice(40 // G * G, 40 // G * G + G)
    for b, t in enumerate(lens):
        v[b, :, t - 9] = (v[b, :, t - 9].float() * 2.0 ** 14).to(torch.bfloat16)
        v[b, :, t - 1, group if bad == "nan" else 40] = float(bad)
    cache, table = held(binding, Hq, 1, k, v, lens, G=G)
    out = cache.attention(0, q.cuda(), wide(table, 32, room).cuda(), ints(lens), SCALE).cpu()
    assert cache.status() == 0 and torch.isfinite(out[:, :, 0]).all()
    assert not torch.isfinite(out[:, :, 1, group]).any()
    # (the reference's quantizer has no groups of NaNs: the newest value as zeros, compared in the other channels and rows)
    clean = v.clone()
    for b, t in enumerate(lens):
        clean[b, :, t - 1, group] = 0.0
    rest = [c for c in range(128) if not group.start <= c < group.stop]
    for b, t in enumerate(lens):
        ref, tol = P.reference(q[b], k[b, 0, :t], clean[b, 0, :t], G, SCALE, [t - 1, t])
        err = (out[b].double() - ref).abs() / (tol + 2.0 ** -24 * ref.abs() + 1e-37)
        assert err[:, 0].max() <= 1.0 and (not rest or err[:, 1, rest].max() <= 1.0)


def test_nans_that_are_appended(binding):
    """A NaN is held as the least value of its group, whose other channels are as without it; a group of NaNs alone is NaN, one with an infinity finite nowhere."""
    G = 32
    _, k, v = P.draw(1, 2, 2, 20, 29)
    bad = {}
    for name, x in (("k", k), ("v", v)):
        y = x.clone()
        y[0, 0, 3, 5] = y[0, 1, 19, 64] = y[0, 1, 19, 95] = float("nan")
        y[0, 0, 7, 96:] = float("nan")
        y[0, 1, 8, 33], y[0, 1, 9, 34] = float("inf"), float("-inf")
        y[0, 0, 11, :32] = 2.5
        y[0, 0, 11, 9] = float("nan")
        bad[name] = y
    cache, table = held(binding, 2, 2, bad["k"], bad["v"], [20])
    got = cache.read(0, table.cuda(), ints([0]), 20)
    assert cache.status() == 0
    for y, out in zip(bad.values(), got):
        rows = P.f32(y).reshape(1, 2, 20, 4, G)
        least = np.nanmin(np.where(np.isnan(rows).all(-1, keepdims=True), 0.0, rows), -1, keepdims=True)
        filled = torch.from_numpy(np.where(np.isnan(rows), least, rows).reshape(1, 2, 20, 128)).to(torch.bfloat16)
        finite = torch.isfinite(filled).view(1, 2, 20, 4, G).all(-1, keepdim=True).expand(1, 2, 20, 4, G).reshape(1, 2, 20, 128).clone()
        finite[0, 0, 7, 96:] = False
        calm = torch.where(finite, filled, torch.zeros_like(filled))
        ref = torch.from_numpy(P.values(*P.quantized(calm, G)).astype(np.float32)).to(torch.bfloat16)
        out = out.cpu()
        assert torch.equal(torch.isfinite(out), finite)
        assert torch.equal(out[finite], ref[finite])


def test_keys_alone_and_positions_of_their_own(binding):
    """An append without queries stores what one with them does; a token with a negative position leaves its slot as it was."""
    Hkv, n, page = 2, 8, 32
    _, k, v = P.draw(2, 4, Hkv, n, 5)
    ang = np.arange(50, dtype=np.float64)[:, None] * 1e4 ** (-np.arange(32, dtype=np.float64) / 32)[None]
    cos, sin = np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)
    table, n_pages = P.pages_for([20, 20], page, 1)
    cache = binding.PagedCache(binding.make_paged_config(1, 4, Hkv, n_pages, page_tokens=page))
    cache.mem[256:] = 0x5A
    pos = torch.randint(0, 50, (2, n), dtype=torch.int32, generator=torch.Generator().manual_seed(0))
    pos[0, 3], pos[1, 5] = -1, 49
    want = cache.mem.cpu().numpy().copy()
    lens = [4, 9]
    assert cache.append(0, k.cuda(), v.cuda(), table.cuda(), ints(lens), cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda(), positions=pos.cuda()) is None
    assert cache.status() == 0
    kr = P.rotate(k, cos, sin, pos.clamp(min=0).numpy())
    for b in range(2):
        for i in range(n):
            if pos[b, i] < 0:
                continue
            t = lens[b] + i
            for h in range(Hkv):
                kb, km = P.token_bytes(kr[b, h, i], 32, False, t % 16)
                vb, vm = P.token_bytes(v[b, h, i], 32, True, t % 16)
                for at, data in zip(P.place(cache.cfg, 0, int(table[b, t // page]), h, t % page), (kb, vb, km, vm)):
                    want[at:at + len(data)] = np.frombuffer(data, np.uint8)
    assert np.array_equal(cache.mem.cpu().numpy()[256:], want[256:])


@pytest.mark.parametrize("why", ["tables", "page", "length"])
def test_rows_that_are_left_out_are_zeros(binding, why):
    """Outputs that a call allocates hold zeros where it writes nothing: tokens beyond the tables, on pages that are none, behind the page table."""
    Hq, Hkv, n, page = 4, 2, 6, 16
    q, k, v = (x.cuda() for x in P.draw(2, Hq, Hkv, n, 37))
    table, n_pages = P.pages_for([32, 32], page, 2)
    cache = binding.PagedCache(binding.make_paged_config(1, Hq, Hkv, n_pages, page_tokens=page))
    cache.mem[256:] = 0
    cos, sin = (x[:20 if why == "tables" else 40].contiguous() for x in binding.rope_tables(40))
    pages, lens = table.cuda(), ints([12, 18 if why != "length" else 30])
    if why == "page":
        pages[1, 1] = -3
    left = {"tables": [2, 3, 4, 5], "page": list(range(6)), "length": [2, 3, 4, 5]}[why]       # of sequence 1
    stale = [torch.full((2, h, n, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]
    del stale                                                                    # what the next allocations of these sizes find
    turned = cache.append(0, k, v, pages, lens, q=q, cos=cos, sin=sin)
    assert (turned[1, :, left] == 0).all() and torch.isfinite(turned).all() and (turned[0] != 0).any()
    stale = [torch.full((2, h, n, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]
    del stale
    for out in cache.read(0, pages, lens, n):
        assert (out[1, :, left] == 0).all() and torch.isfinite(out).all() and (out[0] != 0).any()
    stale = [torch.full((2, h, n, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv)]
    del stale
    assert torch.isfinite(cache.step(0, k, v, q, pages, lens, SCALE, cos=cos, sin=sin)).all()
    assert cache.status() != 0


@pytest.mark.parametrize("Hq,Hkv,n,lens,polls", [(7, 1, 60, [700, 300], 100), (28, 4, 300, [5000, 900, 301], 300), (8, 1, 1000, [40000], 1000)])
def test_time_outs_of_many_rows(binding, Hq, Hkv, n, lens, polls):
    """Copies that never arrive in every thread block of the kernel for many rows: the call ends, the status says so, and the next call is as usual."""
    q, k, v = P.draw(len(lens), Hq, Hkv, max(lens), 83)
    q = q[:, :, :n].contiguous().cuda()
    cache, table = held(binding, Hq, Hkv, k, v, lens, page=64)
    pages = wide(table, 64, 1 << 16).cuda()
    want = cache.attention(0, q, pages, ints(lens), SCALE)
    assert cache.last_attention() == UNPACKED
    for _ in range(3):
        cache.test_arm_copy_timeout(16, polls)
        cache.attention(0, q, pages, ints(lens), SCALE)
        assert cache.status() == binding.DEV_COPY_TIMEOUT
        cache.test_arm_copy_timeout(0, 0)
        cache.clear_status()
        assert torch.equal(cache.attention(0, q, pages, ints(lens), SCALE), want) and cache.status() == 0


@pytest.mark.parametrize("n,lens,room,dtype", [(1, [400, 300], 0, torch.float32), (1, [700, 300], 1 << 12, torch.bfloat16), (3, [700, 300], 1 << 12, torch.float32),
                                               (60, [700, 300], 1 << 16, torch.float32), (300, [5000, 900], 1 << 16, torch.bfloat16)])
def test_calls_whose_copies_never_arrive_are_zeros(binding, n, lens, room, dtype):
    """Where no warp contributed the output is 0: nothing of the workspace's former contents, nothing left unwritten."""
    q, k, v = P.draw(2, 28, 4, max(lens), 85)
    q = q[:, :, :n].contiguous().cuda()
    cache, table = held(binding, 28, 4, k, v, lens, page=64)
    pages = wide(table, 64, room).cuda()
    space = torch.full((cache.workspace_bytes(2, n, pages.shape[1]),), 0xFF, dtype=torch.uint8, device="cuda")
    out = torch.full(q.shape, 7.0, dtype=dtype, device="cuda")
    cache.test_arm_copy_timeout(16, 200)
    cache.attention(0, q, pages, ints(lens), SCALE, out=out, workspace=space)
    assert cache.status() == binding.DEV_COPY_TIMEOUT and (cache.last_attention() == UNPACKED) == (n >= 60)
    assert (out == 0).all()
    cache.test_arm_copy_timeout(0, 0)
    cache.clear_status()
    cache.attention(0, q, pages, ints(lens), SCALE, out=out, workspace=space)
    assert cache.status() == 0 and (out.flatten(0, 2).float().abs().amax(1) > 0).all()


def test_one_workspace_for_all_smaller_calls(binding):
    """A workspace of the widest table and the most tokens serves every narrower and shorter call, whatever pass such a call makes."""
    Hq, Hkv, page, lens = 64, 8, 256, [400, 90]
    q, k, v = P.draw(2, Hq, Hkv, 400, 87)
    cache, table = held(binding, Hq, Hkv, k, v, lens, page=page)
    widths = [2, 64, 511, 512, 513, 1025, 2048, 4097]
    space = torch.empty(cache.workspace_bytes(2, 90, widths[-1]), dtype=torch.uint8, device="cuda")
    for n in (1, 30, 90):
        x = q[:, :, :n].contiguous().cuda()
        for width in widths:
            pages = wide(table, 1, width).cuda()
            assert torch.equal(cache.attention(0, x, pages, ints(lens), SCALE, workspace=space), cache.attention(0, x, pages, ints(lens), SCALE))
    assert cache.last_attention() != UNPACKED and cache.status() == 0        # (the widest table holds more than is unpacked)
    cache.attention(0, x, wide(table, 1, 513).cuda(), ints(lens), SCALE, workspace=space)
    assert cache.last_attention() == UNPACKED


@pytest.mark.parametrize("n", [1, 4, 40])
@pytest.mark.parametrize("room", [0, 1 << 16])
@pytest.mark.parametrize("power", [8, 12])
def test_large_values_of_no_weight(binding, n, room, power):
    """The first tokens' values are 2^power times the others' and have next to no weight.  What a token adds is held to 2^-28 of the largest weight times the largest value
    at worst, which for T tokens is T 2^-28 max |v| of the output, beside what the roundings of the others allow."""
    T, heavy = 300, 128
    q, k, v = P.draw(1, 7, 1, T, 91)
    q = q[:, :, :n].contiguous()
    q[..., 0], k[..., 0] = 8.0, 0.0
    k[:, :, :heavy, 0] = -100.0                                       # logits 70 below the others'
    v[:, :, :heavy] = (v[:, :, :heavy].float() * 2.0 ** power).to(torch.bfloat16)
    cache, table = held(binding, 7, 1, k, v, [T])
    out = cache.attention(0, q.cuda(), wide(table, 32, room).cuda(), ints([T]), SCALE)
    rounded = cache.last_attention() == UNPACKED
    assert cache.status() == 0 and rounded == (room > 0 and n == 40)
    ref, _ = P.reference(q[0], k[0, 0], v[0, 0], 32, SCALE, [T - n + i + 1 for i in range(n)], rounded)
    _, tol = P.reference(q[0], k[0, 0, heavy:], v[0, 0, heavy:], 32, SCALE, [T - heavy - n + i + 1 for i in range(n)], rounded)
    most = float(v.double().abs().max())
    assert ((out[0].double().cpu() - ref).abs() <= tol + T * 2.0 ** -28 * most + 2.0 ** -24 * ref.abs()).all()
    assert (out[0].abs().amax(-1) > 0.01).all()
