"""GPU tests of the paged 4-bit cache: the bytes of an append, the values read back, attention against 64 bits, masks, padding, bad pages and lengths, graphs and streams."""
import numpy as np
import pytest
import torch

import paged_util as P
from oracle import mixkvq_oracle as O

pytestmark = pytest.mark.gpu
SCALE = 128 ** -0.5


@pytest.fixture(scope="module")
def binding():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    from paper_2512_19206_b200 import build
    build.build()
    from paper_2512_19206_b200 import binding as b
    b.lib()
    return b


def tables(n_pos, rotary):
    ang = np.arange(n_pos, dtype=np.float64)[:, None] * 1e6 ** (-np.arange(rotary // 2, dtype=np.float64) * 2 / rotary)[None]
    return np.cos(ang).astype(np.float32), np.sin(ang).astype(np.float32)


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def wide(table, page, room):
    """The table with columns (none of them looked at) up to `room` tokens: what a call could have to read chooses its kernel."""
    more = max(0, room // page - table.shape[1])
    return torch.cat([table, torch.full((table.shape[0], more), -1, dtype=torch.int32)], 1) if more else table


def attend(cache, q, table, lens, **kw):
    """attention, and whether it went to the kernel that rounds keys and values."""
    out = cache.attention(0, q.cuda(), table.cuda(), ints(lens), SCALE, **kw)
    return out, cache.last_attention() == 4


def filled(binding, Hq, Hkv, lens, page, G, seed, layers=1, layer=0, extra=0, poison=True):
    """A cache whose sequences hold lens[b] tokens of k, v (CPU), its page table and the rows.  poison: the rest of the pool holds NaNs and infinities."""
    T = max(max(lens), 1)
    table, n_pages = P.pages_for(lens, page, seed, extra=extra)
    q, k, v = P.draw(len(lens), Hq, Hkv, T, seed)
    cache = binding.PagedCache(binding.make_paged_config(layers, Hq, Hkv, n_pages, page_tokens=page, group_size=G))
    if poison:
        cache.mem[256:] = 0xFF
    if max(lens):
        cache.append(layer, k.cuda(), v.cuda(), table.cuda(), ints([0] * len(lens)), counts=ints(lens))
    return cache, table, k, v


@pytest.mark.parametrize("page,G", [(16, 32), (32, 64), (64, 128), (128, 32), (256, 64)])
@pytest.mark.parametrize("pairs", ["none", "halves", "interleaved"])
def test_bytes_of_an_append(binding, page, G, pairs):
    Hq, Hkv, lens, counts, n, rotary = 6, 2, [0, 37, 100, 5], [21, 0, 30, 9], 30, {"none": 0, "halves": 96, "interleaved": 32}[pairs]
    table, n_pages = P.pages_for([t + m for t, m in zip(lens, counts)], page, 7, extra=1)
    q, k, v = P.draw(4, Hq, Hkv, n, 3)
    cos, sin = tables(200, rotary or 16)
    cache = binding.PagedCache(binding.make_paged_config(3, Hq, Hkv, n_pages, page_tokens=page, group_size=G))
    cache.mem[256:] = 0x5A
    before = cache.mem.cpu().numpy().copy()
    x = torch.cat([t.transpose(1, 2) for t in (q, k, v)], 2).contiguous().cuda()                  # the fused projection's output
    qd, kd, vd = (t.transpose(1, 2) for t in x.split((Hq, Hkv, Hkv), 2))
    turn = {} if pairs == "none" else dict(cos=torch.from_numpy(cos).cuda(), sin=torch.from_numpy(sin).cuda(), interleaved=pairs == "interleaved")
    q_out = torch.full((4, Hq, n, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    cache.append(1, kd, vd, table.cuda(), ints(lens), counts=ints(counts), q=qd, q_out=q_out, **turn)
    assert cache.status() == 0
    pos = np.asarray(lens)[:, None] + np.arange(n)[None]
    qr, kr = (q, k) if pairs == "none" else (P.rotate(t, cos, sin, pos, pairs == "interleaved") for t in (q, k))
    want = before
    for b in range(4):
        assert torch.equal(q_out[b, :, :counts[b]].cpu(), qr[b, :, :counts[b]]) and (q_out[b, :, counts[b]:] == 3.0).all()
        for i in range(counts[b]):
            t = lens[b] + i
            for h in range(Hkv):
                at = P.place(cache.cfg, 1, int(table[b, t // page]), h, t % page)
                kb, km = P.token_bytes(kr[b, h, i], G, False, t % 16)
                vb, vm = P.token_bytes(v[b, h, i], G, True, t % 16)
                for o, data in zip(at, (kb, vb, km, vm)):
                    want[o:o + len(data)] = np.frombuffer(data, np.uint8)
    assert np.array_equal(cache.mem.cpu().numpy()[256:], want[256:])                                # and nothing else was written
    ko, vo = (torch.full((4, Hkv, n, 128), 2.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.read(1, table.cuda(), ints(lens), n, counts=ints(counts), out=(ko, vo))
    for b in range(4):
        for got, src in ((ko, kr), (vo, v)):
            ref = torch.from_numpy(P.values(*P.quantized(src[b, :, :counts[b]], G)).astype(np.float32)).to(torch.bfloat16)
            assert torch.equal(got[b, :, :counts[b]].cpu(), ref) and (got[b, :, counts[b]:] == 2.0).all()


def test_append_layouts_and_positions(binding):
    """Head-major tensors, queries turned in place, positions of their own (one is no token, one is beyond the tables), keys alone."""
    Hq, Hkv, n, page = 4, 2, 8, 32
    q, k, v = P.draw(2, Hq, Hkv, n, 5)
    cos, sin = tables(50, 64)
    cd, sd = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    table, n_pages = P.pages_for([20, 20], page, 1)
    cache = binding.PagedCache(binding.make_paged_config(1, Hq, Hkv, n_pages, page_tokens=page))
    pos = torch.randint(0, 50, (2, n), dtype=torch.int32, generator=torch.Generator().manual_seed(0))
    pos[0, 3], pos[1, 5] = -1, 50
    cache.mem[256:] = 0
    qd = q.cuda()
    assert cache.append(0, k.cuda(), v.cuda(), table.cuda(), ints([4, 9]), q=qd, cos=cd, sin=sd, positions=pos.cuda(), q_out=qd) is qd
    assert cache.status() == binding.DEV_BAD_POSITION
    cache.clear_status()
    ko, vo = cache.read(0, table.cuda(), ints([4, 9]), n)
    good = (pos >= 0) & (pos < 50)
    qr, kr = (P.rotate(t, cos, sin, pos.clamp(0, 49).numpy()) for t in (q, k))
    for b in range(2):
        for i in range(n):
            assert torch.equal(qd[b, :, i].cpu(), (qr if good[b, i] else q)[b, :, i])
            for got, src in ((ko, kr), (vo, v)):
                ref = torch.from_numpy(P.values(*P.quantized(src[b, :, i], 32)).astype(np.float32)).to(torch.bfloat16) if good[b, i] else torch.zeros(Hkv, 128)
                assert torch.equal(got[b, :, i].float().cpu(), ref.float())
    first = cache.mem.clone()
    assert cache.append(0, k.cuda(), v.cuda(), table.cuda(), ints([4, 9]), cos=cd, sin=sd, positions=pos.clamp(max=49).cuda()) is None
    ok = torch.ones(2, n, dtype=torch.bool)
    ok[1, 5] = False
    again = cache.read(0, table.cuda(), ints([4, 9]), n)
    assert all(torch.equal(x.transpose(1, 2)[ok.cuda()], y.transpose(1, 2)[ok.cuda()]) for x, y in zip(again, (ko, vo))) and first.shape == cache.mem.shape


CASES = [
    # Hq, Hkv, lens, counts, page, G
    (1, 1, [1], [1], 16, 32), (1, 1, [31], [1], 16, 128), (7, 1, [33, 1, 16], [1, 1, 1], 16, 64), (28, 4, [300, 17, 512], [1, 1, 1], 64, 32),
    (32, 8, [1000], [1], 128, 64), (8, 8, [65, 64, 63], [1, 1, 1], 32, 128), (40, 8, [257, 700], [1, 0], 256, 128), (8, 1, [5000], [1], 64, 32),
    (28, 4, [40, 3, 700], [5, 3, 2], 64, 32), (5, 1, [200, 9], [8, 9], 16, 64), (32, 8, [333], [33], 128, 128), (16, 2, [130, 500], [130, 77], 32, 32),
    (6, 2, [600, 129], [300, 129], 64, 64), (28, 4, [1000, 40, 0, 257], [200, 40, 0, 256], 128, 32), (1, 1, [700], [129], 16, 128), (8, 1, [2100, 5], [700, 1], 256, 64),
    (7, 7, [300, 1500], [150, 300], 32, 32),
]


@pytest.mark.parametrize("Hq,Hkv,lens,counts,page,G", CASES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("room", [0, 1 << 16])
def test_attention(binding, Hq, Hkv, lens, counts, page, G, dtype, room):
    cache, table, k, v = filled(binding, Hq, Hkv, lens, page, G, sum(lens), layers=2, layer=1)
    table = wide(table, page, room)
    q, _, _ = P.draw(len(lens), Hq, Hkv, max(counts), 91)
    out = torch.full(q.shape, 7.0, dtype=dtype, device="cuda")
    cache.attention(1, q.cuda(), table.cuda(), ints(lens), SCALE, counts=ints(counts), out=out)
    assert cache.status() == 0
    rows, form = Hq // Hkv * max(counts), cache.last_attention()
    if rows <= 72:
        assert form == (binding.PAGED_PIECES if table.shape[1] * page > 512 else binding.PAGED_DIRECT)
    elif room and rows > 148:
        assert form == binding.PAGED_UNPACKED
    P.check(out, q, k, v, G, SCALE, lens, counts, form == binding.PAGED_UNPACKED)
    for b, m in enumerate(counts):
        assert (out[b, :, m:] == 7.0).all()
    if min(counts) == max(counts):
        assert torch.equal(cache.attention(1, q.cuda(), table.cuda(), ints(lens), SCALE, dtype=dtype), out)


@pytest.mark.parametrize("n", [5, 70])
def test_rows_that_see_nothing(binding, n):
    """A sequence without tokens, and query rows in front of a sequence's first token, are zeros."""
    cache, table, k, v = filled(binding, 4, 2, [0, 3, 70], 16, 32, 2)
    q, _, _ = P.draw(3, 4, 2, n, 8)
    for room in (0, 1 << 16):
        out, rounded = attend(cache, q, wide(table, 16, room), [0, 3, 70])
        assert cache.status() == 0 and rounded == (room > 0 and n == 70)
        assert (out[0] == 0).all() and (out[1, :, :n - 3] == 0).all()
        P.check(out, q, k, v, 32, SCALE, [0, 3, 70], [0, n, n], rounded)


@pytest.mark.parametrize("size", [1e-30, 1e-6, 1e3, 1e20, 1e36])
@pytest.mark.parametrize("n", [1, 4, 40])
def test_magnitudes(binding, size, n):
    """Values and keys of any magnitude: the softmax's input stays ordinary (queries shrink as keys grow), the output grows with the values."""
    lens = [90, 400]
    table, n_pages = P.pages_for(lens, 32, 4)
    q, k, v = P.draw(2, 7, 1, max(lens), 6)
    k, v, q = (k.float() * size).to(torch.bfloat16), (v.float() * size).to(torch.bfloat16), (q[:, :, :n].float() / size).to(torch.bfloat16)
    v[1, :, 200:] = (v[1, :, 200:].float() * 64).to(torch.bfloat16)                  # values that grow on the way
    cache = binding.PagedCache(binding.make_paged_config(1, 7, 1, n_pages, page_tokens=32))
    cache.append(0, k.cuda(), v.cuda(), table.cuda(), ints([0, 0]), counts=ints(lens))
    for room in (0, 1 << 16):
        out, rounded = attend(cache, q, wide(table, 32, room), lens)
        assert rounded == (room > 0 and n == 40)
        P.check(out, q, k, v, 32, SCALE, lens, [n, n], rounded)


@pytest.mark.parametrize("n", [1, 3, 90])
def test_peaked_and_flat_softmax(binding, n):
    """One key that takes all, logits that rise along the sequence, and equal logits."""
    lens = [500, 500, 500]
    table, n_pages = P.pages_for(lens, 64, 9)
    q, k, v = P.draw(3, 4, 1, 500, 12, outliers=False)
    q = q[:, :, :n].contiguous()
    k[0, 0, 123] = (q[0, 0, 0].float() * 30).to(torch.bfloat16)
    k[1] = (q[1, :1, :1].float() * torch.linspace(-2, 6, 500)[None, :, None]).to(torch.bfloat16)
    k[2] = k[2, :, :1]
    cache = binding.PagedCache(binding.make_paged_config(1, 4, 1, n_pages))
    cache.append(0, k.cuda(), v.cuda(), table.cuda(), ints([0] * 3), counts=ints(lens))
    for room in (0, 1 << 16):
        out, rounded = attend(cache, q, wide(table, 64, room), lens)
        assert rounded == (room > 0 and n == 90)
        P.check(out, q, k, v, 32, SCALE, lens, [n] * 3, rounded)


@pytest.mark.parametrize("n", [2, 50])
@pytest.mark.parametrize("room", [0, 1 << 16])
def test_nan_and_infinity_stay_where_they_are(binding, n, room):
    """A NaN among the queries reaches its own row, an infinite value its group's channels of the rows that see it, an infinite key the rows that see it."""
    lens = [200, 60]
    cache, table, k, v = filled(binding, 8, 2, lens, 32, 32, 21)
    where = wide(table, 32, room)
    q, _, _ = P.draw(2, 8, 2, n, 22)
    ref, rounded = attend(cache, q, where, lens)
    assert rounded == (room > 0 and n == 50)
    bad = q.clone()
    bad[0, 3, 0, 5] = float("nan")
    out, _ = attend(cache, bad, where, lens)
    assert torch.isnan(out[0, 3, 0]).all()
    out[0, 3, 0] = ref[0, 3, 0]
    assert torch.equal(out, ref)
    vi, ki = v.clone(), k.clone()
    vi[1, 1, 59, 40] = float("inf")                                        # the newest token of sequence 1: its last row sees it
    cache.append(0, k.cuda(), vi.cuda(), table.cuda(), ints([0, 0]), counts=ints(lens))
    out, _ = attend(cache, q, where, lens)
    assert not torch.isfinite(out[1, 4:, n - 1, 32:64]).any()
    out[1, 4:, n - 1, 32:64] = ref[1, 4:, n - 1, 32:64]
    assert torch.isfinite(out).all()
    P.check(out, q, k, v, 32, SCALE, lens, [n, n], rounded)
    ki[1, 0, 58, 7] = float("inf")                                         # a key: the last two rows of its heads
    cache.append(0, ki.cuda(), v.cuda(), table.cuda(), ints([0, 0]), counts=ints(lens))
    out, _ = attend(cache, q, where, lens)
    assert not torch.isfinite(out[1, :4, n - 2:]).any()
    out[1, :4, n - 2:] = ref[1, :4, n - 2:]
    assert torch.isfinite(out).all()
    P.check(out, q, k, v, 32, SCALE, lens, [n, n], rounded)


@pytest.mark.parametrize("room", [0, 1 << 16])
def test_bad_pages_of_many_rows(binding, room):
    """Tokens of pages that are none are left out, for many query rows too."""
    cache, table, k, v = filled(binding, 8, 1, [400, 300], 16, 32, 33)
    q, _, _ = P.draw(2, 8, 1, 30, 34)
    table = wide(table, 16, room)
    table[0, 3], table[0, 9], table[1, 18] = -1, cache.cfg.n_pages, -7
    out, rounded = attend(cache, q, table, [400, 300])
    assert rounded == (room > 0) and cache.status() == binding.DEV_BAD_PAGE and torch.isfinite(out).all()
    keep = [t for t in range(400) if t // 16 not in (3, 9)]
    P.check(out[:1], q[:1], k[:1, :, keep], v[:1, :, keep], 32, SCALE, [len(keep)], [30], rounded)
    # sequence 1: page 18 is its last (tokens 288 .. 299); the 30 rows are tokens 270 .. 299
    sees = [min(271 + i, 288) for i in range(30)]
    ref, tol = P.reference(q[1], k[1, 0, :288], v[1, 0, :288], 32, SCALE, sees, rounded)
    assert ((out[1].double().cpu() - ref).abs() <= tol + 2.0 ** -24 * ref.abs()).all()


def test_bad_pages_and_lengths(binding):
    Hq, Hkv, page = 4, 1, 16
    cache, table, k, v = filled(binding, Hq, Hkv, [64, 40], page, 32, 31)
    q, kn, vn = P.draw(2, Hq, Hkv, 1, 32)
    pages, lens = table.cuda(), ints([64, 40])
    ref = cache.attention(0, q.cuda(), pages, lens, SCALE)
    wrong = pages.clone()
    wrong[0, 2] = cache.cfg.n_pages                                        # tokens 32 .. 47 of sequence 0 are left out
    out = cache.attention(0, q.cuda(), wrong, lens, SCALE)
    assert cache.status() == binding.DEV_BAD_PAGE
    cache.clear_status()
    keep = torch.cat([torch.arange(32), torch.arange(48, 64)])
    P.check(out[:1], q[:1], k[:1, :, keep], v[:1, :, keep], 32, SCALE, [48], [1])
    assert torch.equal(out[1], ref[1])
    before = cache.mem.clone()
    wrong[0, 2] = -5
    cache.append(0, kn.cuda(), vn.cuda(), wrong, ints([33, 64]))           # a page that is none, a place behind the table
    assert cache.status() == binding.DEV_BAD_PAGE | binding.DEV_BAD_LENGTH
    cache.clear_status()
    assert torch.equal(cache.mem[256:], before[256:])
    ko, vo = (torch.full((2, Hkv, 1, 128), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.read(0, wrong, ints([33, -1]), 1, out=(ko, vo))
    assert (ko == 5.0).all() and (vo == 5.0).all()
    cache.clear_status()
    out = cache.attention(0, q.cuda(), pages, ints([65, -7]), SCALE, counts=ints([1, 9]))
    assert cache.status() == binding.DEV_BAD_LENGTH                        # 64 tokens and none, one query each
    assert torch.equal(out[0], ref[0]) and (out[1] == 0).all()


def test_pages_in_another_order_and_shared(binding):
    """The result does not depend on where the pages lie; two sequences may share the pages of a common beginning."""
    Hq, Hkv, page, lens = 8, 2, 32, [150, 150]
    outs = []
    q, k, v = P.draw(1, Hq, Hkv, 150, 41)
    for seed in (1, 2):
        table, n_pages = P.pages_for([150], page, seed, spare=20)
        cache = binding.PagedCache(binding.make_paged_config(1, Hq, Hkv, n_pages, page_tokens=page))
        cache.append(0, k.cuda(), v.cuda(), table.cuda(), ints([0]))
        outs.append(cache.attention(0, q[:, :, :1].cuda().contiguous(), table.cuda(), ints([150]), SCALE))
    assert torch.equal(*outs)
    both = table.expand(2, -1).contiguous().cuda()
    qq = q[:, :, :2].transpose(0, 2).transpose(1, 2).contiguous().reshape(2, 1, Hq, 128).transpose(1, 2).contiguous()
    out = cache.attention(0, qq.cuda(), both, ints(lens), SCALE)
    P.check(out, qq, k.expand(2, -1, -1, -1), v.expand(2, -1, -1, -1), 32, SCALE, lens, [1, 1])


def test_steps_are_append_then_attention(binding):
    """Decode steps and drafts through `step`, the lengths on the device, in one captured graph that is replayed as the sequences grow."""
    Hq, Hkv, page, T = 28, 4, 16, 70
    q, k, v = P.draw(2, Hq, Hkv, T, 51)
    cos, sin = tables(T, 128)
    cd, sd = torch.from_numpy(cos).cuda(), torch.from_numpy(sin).cuda()
    table, n_pages = P.pages_for([T, T], page, 3)
    caches = [binding.PagedCache(binding.make_paged_config(1, Hq, Hkv, n_pages, page_tokens=page)) for _ in range(2)]
    pages = table.cuda()
    pos = np.arange(T)[None].repeat(2, 0)
    qr, kr = (P.rotate(t, cos, sin, pos) for t in (q, k))
    start = [31, 12]
    for c in caches:
        c.mem[256:] = 0xFF
        c.append(0, k.cuda(), v.cuda(), pages, ints([0, 0]), counts=ints(start), cos=cd, sin=sd)
    lens, xq, xk, xv = ints(start), *(torch.empty((2, h, 1, 128), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    q_out, out = torch.empty_like(xq), torch.empty(xq.shape, device="cuda")
    ws = torch.empty(caches[0].workspace_bytes(2, 1, pages.shape[1]), dtype=torch.uint8, device="cuda")

    def one():
        caches[0].step(0, xk, xv, xq, pages, lens, SCALE, cos=cd, sin=sd, q_out=q_out, out=out, workspace=ws)
        lens.add_(1)
    graph = torch.cuda.CUDAGraph()
    for i in range(20):
        at = [s + i for s in start]
        for x, src in ((xq, q), (xk, k), (xv, v)):
            x.copy_(torch.stack([src[b, :, at[b]:at[b] + 1] for b in range(2)]))
        if i == 1:
            torch.cuda.synchronize()
            with torch.cuda.graph(graph):
                one()
        one() if i == 0 else graph.replay()
        b = caches[1]
        b.append(0, xk, xv, pages, ints(at), cos=cd, sin=sd)
        qrot = torch.stack([qr[s, :, at[s]:at[s] + 1] for s in range(2)])
        assert torch.equal(q_out.cpu(), qrot)
        want = b.attention(0, q_out, pages, ints([t + 1 for t in at]), SCALE)
        assert torch.equal(out, want) and torch.equal(caches[0].mem, b.mem)
        if i % 9 == 0:
            P.check(out, qrot, kr, v, 32, SCALE, [t + 1 for t in at], [1, 1])
    assert lens.tolist() == [51, 32] and caches[0].status() == 0


@pytest.mark.parametrize("counts_max,room", [(1, 1 << 10), (3, 1 << 10), (40, 1 << 15), (1, 0)])
def test_many_sequences(binding, counts_max, room):
    """More sequences than a warp has lanes, of very different length, some without tokens or queries."""
    B, Hq, Hkv, page, G = 70, 8, 2, 16, 64
    gen = torch.Generator().manual_seed(7)
    lens = torch.randint(0, 130, (B,), generator=gen).tolist()
    lens[3], lens[40], lens[69] = 400, 0, 390
    counts = [min(t, c) for t, c in zip(lens, torch.randint(0, counts_max + 1, (B,), generator=gen).tolist())]
    counts[3] = counts_max
    cache, table, k, v = filled(binding, Hq, Hkv, lens, page, G, 71)
    q, _, _ = P.draw(B, Hq, Hkv, counts_max, 72)
    out, rounded = attend(cache, q, wide(table, page, room), lens, counts=ints(counts))
    assert cache.status() == 0 and rounded == (counts_max == 40)
    assert cache.last_attention() == (binding.PAGED_UNPACKED if rounded else binding.PAGED_PIECES if room else binding.PAGED_DIRECT)
    P.check(out, q, k, v, G, SCALE, lens, counts, rounded)
    for b, m in enumerate(counts):
        assert (out[b, :, m:] == 0).all()


def test_page_table_that_is_a_view_and_a_pool_beyond_four_gigabytes(binding):
    """Pages at the end of a pool of 5 GB, in the second layer; the table's rows lie apart."""
    Hq, Hkv, page, lens = 8, 8, 64, [150, 130]
    n_pages = 31000
    cache = binding.PagedCache(binding.make_paged_config(2, Hq, Hkv, n_pages, page_tokens=page))
    assert cache.mem.numel() > 5e9
    table = torch.tensor([[n_pages - 1, n_pages - 4, n_pages - 2], [n_pages - 3, n_pages - 7, n_pages - 5]], dtype=torch.int32)
    room = torch.full((2, 40), -9, dtype=torch.int32, device="cuda")
    pages = room[:, 5:8]
    pages.copy_(table)
    q, k, v = P.draw(2, Hq, Hkv, 150, 77)
    cache.append(1, k.cuda(), v.cuda(), pages, ints([0, 0]), counts=ints(lens))
    for n, columns in ((1, 3), (3, 20), (140, 3)):
        x = q[:, :, :n].contiguous()
        out = cache.attention(1, x.cuda(), room[:, 5:5 + columns], ints(lens), SCALE, counts=ints([n, min(n, 130)]))
        P.check(out, x, k, v, 32, SCALE, lens, [n, min(n, 130)], cache.last_attention() == binding.PAGED_UNPACKED)
    ko, vo = cache.read(1, pages, ints([149, 129]), 1)
    for got, src in ((ko, k), (vo, v)):
        for b, t in enumerate((149, 129)):
            ref = torch.from_numpy(P.values(*P.quantized(src[b, :, t], 32)).astype(np.float32)).to(torch.bfloat16)
            assert torch.equal(got[b, :, 0].cpu(), ref)
    assert cache.status() == 0


@pytest.mark.parametrize("n,room", [(1, 0), (1, 1 << 12), (3, 1 << 12), (60, 1 << 16)])
def test_waits_that_run_out(binding, n, room):
    """A staged copy that never completes: the call returns, the status says so, and the next call is as usual."""
    lens = [700, 300] if room else [400, 300]
    cache, table, k, v = filled(binding, 7, 1, lens, 64, 32, 81)
    where = wide(table, 64, room)
    q, _, _ = P.draw(2, 7, 1, n, 82)
    want, _ = attend(cache, q, where, lens)
    cache.test_arm_copy_timeout(16, 200)
    attend(cache, q, where, lens)
    assert cache.status() == binding.DEV_COPY_TIMEOUT
    cache.test_arm_copy_timeout(0, 0)
    cache.clear_status()
    again, _ = attend(cache, q, where, lens)
    assert torch.equal(again, want) and cache.status() == 0


def test_long_segments_are_summed_in_parts(binding):
    """More key tiles than are summed up in tensor memory at a time, in one thread block's range: one KV head, 600 tiles, many query rows."""
    T, n = 76900, 256
    table, n_pages = P.pages_for([T], 256, 5)
    gen = torch.Generator(device="cuda").manual_seed(3)
    k, v = (torch.empty((1, 1, T, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=gen) for _ in range(2))
    q = torch.empty((1, 8, 20000, 128), dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    cache = binding.PagedCache(binding.make_paged_config(1, 8, 1, n_pages, page_tokens=256))
    cache.append(0, k, v, table.cuda(), ints([0]))
    out = cache.attention(0, q, table.cuda(), ints([T]), SCALE)
    assert cache.last_attention() == binding.PAGED_UNPACKED and cache.status() == 0
    rows = [0, 1, 4097, 9999, 19998, 19999]
    sees = [T - 20000 + i + 1 for i in rows]
    ref, tol = P.reference(q[0][:, rows].cpu(), k[0, 0].cpu(), v[0, 0].cpu(), 32, SCALE, sees, True)
    assert ((out[0][:, rows].double().cpu() - ref).abs() <= tol + 2.0 ** -24 * ref.abs()).all()


def test_streams_and_two_calls_at_once(binding):
    """Calls on streams of their own with workspaces of their own do not disturb one another."""
    lens = [900, 1500]
    cache, table, k, v = filled(binding, 16, 2, lens, 64, 32, 61)
    qs = [P.draw(2, 16, 2, 1, 70 + i)[0].cuda() for i in range(4)]
    pages, ld = table.cuda(), ints(lens)
    want = [cache.attention(0, x, pages, ld, SCALE) for x in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    outs = [torch.empty_like(w) for w in want]
    spaces = [torch.empty(cache.workspace_bytes(2, 1, pages.shape[1]), dtype=torch.uint8, device="cuda") for _ in qs]
    for _ in range(10):
        for s, x, o, w in zip(streams, qs, outs, spaces):
            with torch.cuda.stream(s):
                cache.attention(0, x, pages, ld, SCALE, out=o, workspace=w)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs, want))


@pytest.mark.parametrize("room", [0, 1 << 17])
def test_prompt_in_chunks_then_steps(binding, room):
    """As a server runs it: tables, a prompt in two chunks from the projection's output, then decode steps, with a part of the head turned."""
    Hq, Hkv, B, T, n = 8, 2, 2, 130, 64
    q, k, v = P.draw(B, Hq, Hkv, T, 81)
    cd, sd = binding.rope_tables(T, 64, 1e4, "linear", factor=2.0)
    cos, sin = cd.cpu().numpy(), sd.cpu().numpy()
    table, n_pages = P.pages_for([T, T], 32, 5)
    cache = binding.PagedCache(binding.make_paged_config(1, Hq, Hkv, n_pages, page_tokens=32, group_size=64))
    cache.mem[256:] = 0xFF
    pages, lens = wide(table, 32, room).cuda(), ints([0, 0])
    qr, kr = (P.rotate(t, cos, sin, np.arange(T)[None].repeat(B, 0), True) for t in (q, k))
    at = 0
    while at < T:
        m = min(n, T - at) if at < 128 else 1
        x = torch.cat([t[:, :, at:at + m].transpose(1, 2) for t in (q, k, v)], 2).contiguous().cuda()
        xq, xk, xv = (t.transpose(1, 2) for t in x.split((Hq, Hkv, Hkv), 2))
        out = cache.step(0, xk, xv, xq, pages, lens, SCALE, cos=cd, sin=sd, interleaved=True, dtype=torch.bfloat16)
        lens.add_(m)
        at += m
        rounded = cache.last_attention() == binding.PAGED_UNPACKED
        assert rounded == (room > 0 and m == n)
        P.check(out, qr[:, :, at - m:at].contiguous(), kr, v, 64, SCALE, [at, at], [m, m], rounded)
    assert cache.status() == 0


def test_refusals(binding):
    Hq, Hkv, n = 4, 2, 3
    cache = binding.PagedCache(binding.make_paged_config(1, Hq, Hkv, 4, page_tokens=16))
    pages, lens = ints([[0, 1], [2, 3]]), ints([0, 0])
    q, k, v = (torch.zeros((2, h, n, 128), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv))
    before = cache.launch_count()
    wide = torch.zeros((2, Hkv, n, 132), dtype=torch.bfloat16, device="cuda")
    pool = cache.mem[256:256 + q.numel() * 2].view(torch.bfloat16).view(q.shape)
    ws = torch.empty(cache.workspace_bytes(2, n, 2), dtype=torch.uint8, device="cuda")
    for call, code in ((lambda: cache.append(1, k, v, pages, lens), -1), (lambda: cache.append(0, wide[..., :128], v, pages, lens), -3),
                       (lambda: cache.append(0, k, v, pages, lens, q=q, q_out=pool), -1),
                       (lambda: cache.append(0, pool[:, :2], v, pages, lens), -1),
                       (lambda: cache.attention(0, q, pages, lens, 0.0), -1), (lambda: cache.attention(0, q, pages, lens, float("nan")), -1),
                       (lambda: cache.attention(0, q, pages, lens, 1.0, out=q), -1), (lambda: cache.attention(0, q, pages, lens, 1.0, workspace=ws[:-16]), -4 if ws.numel() > 16 else -1),
                       (lambda: cache.read(0, pages, lens, n, out=(k, k)), -1), (lambda: cache.read(-1, pages, lens, n), -1), (lambda: cache.read(0, pages, lens, 0), -1),
                       (lambda: cache.step(0, k, v, q, pages, lens, 1.0, q_out=q.clone(), out=torch.zeros(q.shape, device="cuda"), workspace=ws[:-16]), -4)):
        with pytest.raises(binding.MixKVQError) as e:
            call()
        assert e.value.code == code
    assert cache.launch_count() == before and cache.status() == 0


def test_a_step_writes_over_none_of_its_inputs(binding):
    Hq, Hkv, n = 4, 2, 3
    cache = binding.PagedCache(binding.make_paged_config(1, Hq, Hkv, 4, page_tokens=16))
    pages, lens = ints([[0, 1], [2, 3]]), ints([0, 0])
    q, k, v, out = (torch.zeros((2, h, n, 128), dtype=torch.bfloat16, device="cuda") for h in (Hq, Hkv, Hkv, Hq))
    cos = torch.ones((9, 64), device="cuda")
    before = cache.launch_count()
    for over in (dict(k=out[:, :Hkv]), dict(v=out[:, Hkv:]), dict(q=out, q_out=q), dict(q=out, q_out=out), dict(cos=out.view(-1).view(torch.float32)[:9 * 64].view(9, 64))):
        with pytest.raises(binding.MixKVQError) as e:
            cache.step(0, **{**dict(k=k, v=v, q=q, cos=cos, sin=cos), **over}, pages=pages, lens=lens, scale=1.0, out=out)
        assert e.value.code == -1
    assert cache.launch_count() == before and cache.status() == 0


@pytest.mark.parametrize("n,room", [(1, 1 << 10), (4, 1 << 10), (30, 1 << 12), (1, 0)])
def test_as_many_sequences_as_there_may_be(binding, n, room):
    """4096 sequences: every kernel's table of positions at its largest.  A sample of them against 64 bits."""
    B, Hq, Hkv, page, G = 4096, 8, 1, 16, 128
    lens = torch.randint(n, 60, (B,), generator=torch.Generator().manual_seed(8)).tolist()
    lens[17], lens[B - 1] = 130, 120
    cache, table, k, v = filled(binding, Hq, Hkv, lens, page, G, 81)
    q, _, _ = P.draw(B, Hq, Hkv, n, 82)
    table = wide(table, page, room)
    out, rounded = attend(cache, q, table, lens)
    assert cache.status() == 0 and rounded == (n == 30)
    some = [0, 17, 31, 32, 2047, 4000, B - 1]
    P.check(out[some], q[some], k[some], v[some], G, SCALE, [lens[b] for b in some], [n] * len(some), rounded)
    with pytest.raises(binding.MixKVQError):
        cache.attention(0, torch.cat([q, q[:1]]).cuda(), torch.cat([table, table[:1]]).cuda(), ints(lens + lens[:1]), SCALE)
