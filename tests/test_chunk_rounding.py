"""The check that the chunk attention's GPU tests use, on the CPU: it takes the kernel's arithmetic and refuses outputs that are wrong by one key, by one
mask column or by two parts in a thousand."""
import pytest
import torch

import chunk_rounding as CR
import chunk_util as CU
from paper_2512_19206_b200 import workloads as W

SCALE = W.softmax_scale()


def case(name, g, tokens, n, flat, seed, **kw):
    w = W.small(W.CONFIGS[name], n_layers=1, batch=1, n_kv_heads=1, n_q_heads=g, tokens=max(tokens, 1), **kw)
    k, v, q = W.tokens(w, 0, 0, max(tokens, 1))
    st = CU.streams(w, [tokens], k, v, q)[(0, 0)]
    gen = torch.Generator().manual_seed(seed)
    kn, vn = (torch.randn((n, 128), generator=gen).to(torch.bfloat16) for _ in range(2))
    qn = (torch.randn((g, n, 128), generator=gen) * W.layer_gains(w, 0)[2][:g, None]).to(torch.bfloat16)
    if flat:
        qn.zero_()
    K, V, qq = CR.operands(st, kn, vn, qn)
    return K, V, qq, K.shape[0] - n, n


CASES = [("tiny", 1, 513, 129, dict(residual_len=32, **W.P24)), ("qwen7b", 7, 300, 37, W.P24), ("qwen7b", 7, 700, 9, W.P27),
         ("qwen7b", 4, 700, 9, W.P4BASE), ("tiny", 1, 129, 1, dict(residual_len=32, **W.P24)), ("qwen7b", 2, 0, 200, W.P24), ("qwen7b", 3, 2500, 5, W.P24)]


@pytest.mark.parametrize("flat", [False, True])
@pytest.mark.parametrize("name,g,tokens,n,kw", CASES)
def test_the_kernels_arithmetic_is_taken(name, g, tokens, n, kw, flat):
    K, V, q, held, n = case(name, g, tokens, n, flat, tokens + n, **kw)
    rows = slice(max(0, n - 20), n)
    sees = CR.visible(held, n)[rows]
    p, ref, s = CR.attend(K, V, q[:, rows], SCALE, sees)
    got = CR.simulated(K, V, q[:, rows], SCALE, sees)
    assert CR.worst(got, ref, CR.allowed(p, s, K, V, q[:, rows], SCALE)) <= 1.0


MUTATIONS = ["first key dropped", "last held key dropped", "own key dropped", "next key seen", "a tile's first key dropped", "a key twice", "times 1.002"]


@pytest.mark.parametrize("mutation", MUTATIONS)
@pytest.mark.parametrize("name,g,tokens,n,kw", CASES)
def test_wrong_outputs_are_refused(name, g, tokens, n, kw, mutation):
    """With queries of zero every key weighs the same, so that no key's absence can hide behind its weight; a factor shows with any queries."""
    for flat in (True, False):
        K, V, q, held, n = case(name, g, tokens, n, flat, tokens + n, **kw)
        if mutation != "times 1.002" and not flat:
            continue
        if (held == 0 and mutation == "last held key dropped") or (held + n <= 128 and "tile" in mutation) or (n == 1 and mutation == "next key seen"):
            continue
        sees = CR.visible(held, n)
        p, ref, s = CR.attend(K, V, q, SCALE, sees)
        tol = CR.allowed(p, s, K, V, q, SCALE)
        wrong, j = sees.clone(), torch.arange(n)
        factor = 1.0
        if mutation == "first key dropped":
            wrong[:, 0] = False
        elif mutation == "last held key dropped":
            wrong[:, held - 1] = False
        elif mutation == "own key dropped":
            wrong[j, held + j] = False
        elif mutation == "next key seen":
            wrong[j[:-1], held + j[:-1] + 1] = True
        elif mutation == "a tile's first key dropped":
            wrong[:, 128] = False
        elif mutation == "times 1.002":
            factor = 1.002
        if mutation == "a key twice":
            K2, V2, sees2 = torch.cat([K, K[:1]]), torch.cat([V, V[:1]]), torch.cat([sees, sees[:, :1]], 1)
            got = CR.attend(K2, V2, q, SCALE, sees2)[1]
        else:
            got = CR.attend(K, V, q, SCALE, wrong)[1]
        got = torch.where(torch.isnan(got), ref + 1, got) * factor          # (a row without any key)
        changed = (got - ref).abs().amax((0, 2)) > 0                        # rows that the mistake reaches
        share = ((got - ref).abs() / tol).amax(-1)[:, changed]
        share = share.max() if factor != 1.0 else share.min()               # the check refuses it by any row; a key by every row that it is wrong for
        assert changed.any() and float(share) > 1.0, (mutation, flat, float(share))


@pytest.mark.parametrize("preset", ["P24", "P27", "P4BASE"])
def test_wrong_codes_are_refused(preset):
    """A key channel with its neighbour's values, a scale one step off, a key unit in the wrong place: with queries as the model has them."""
    K, V, q, held, n = case("qwen7b", 7, 700, 9, False, 3, **getattr(W, preset))
    sees = CR.visible(held, n)
    p, ref, s = CR.attend(K, V, q, SCALE, sees)
    tol = CR.allowed(p, s, K, V, q, SCALE)
    swapped, scaled, moved = K.clone(), K.clone(), K.clone()
    swapped[:held, [20, 21]] = K[:held, [21, 20]]
    scaled[32:64, 50] *= 1 + 2.0 ** -5
    moved[32:64], moved[64:96] = K[64:96], K[32:64]
    for wrong in (swapped, scaled, moved):
        assert CR.worst(CR.attend(wrong, V, q, SCALE, sees)[1], ref, tol) > 1.5
    values = V.clone()
    values[40, 32:64] = V[41, 32:64]
    assert CR.worst(CR.attend(K, values, q, SCALE, sees)[1], ref, tol) > 1.0


@pytest.mark.parametrize("n4", [64, 37])
def test_keys_rounded_twice_are_refused(n4):
    """(c_lo s + z) rounded, then 4 c_hi s added and rounded again."""
    st, kn, vn, qn = CR.offset_keys(n4)
    K, V, q = CR.operands(st, kn, vn, qn)
    held, n = K.shape[0] - kn.shape[0], kn.shape[0]
    sees = CR.visible(held, n)
    p, ref, s = CR.attend(K, V, q, SCALE, sees)
    tol = CR.allowed(p, s, K, V, q, SCALE)
    assert CR.worst(CR.simulated(K, V, q, SCALE, sees), ref, tol) <= 1.0
    twice, t = K.clone(), 0
    for b in st.blocks:
        scale, zero = (torch.from_numpy(x.astype("float64")).repeat_interleave(st.G, 0) for x in (b.ks, b.kz))
        codes = torch.from_numpy(b.kcodes.reshape(st.R, 128).astype("float64"))
        once = CR.fp16((codes % 4 * scale + zero).numpy())
        again = CR.fp16((once + torch.floor(codes / 4) * 4 * scale).numpy())
        twice[t:t + st.R] = torch.where(torch.from_numpy(b.tiers == 1), again, twice[t:t + st.R])
        t += st.R
    assert CR.worst(CR.attend(twice, V, q, SCALE, sees)[1], ref, tol) > 1.5
