"""GPU tests of the operators for sequences of different lengths where they are read most strictly: orders of NaN, bits that
must not depend on other tokens, values that are not finite under vanishing weights, offsets that fall or lie outside, workspaces
and captured calls."""
import math

import pytest
import torch

import paper_2401_06104_b200 as tova
from test_gpu_serve import (DEV, TD, TT, attention_tolerance, gen, make_table, offsets_of, packed_reference, paged_reference,
                            randn, run_logprobs, within)

pytestmark = pytest.mark.gpu


# ------------------------------------------------------------------------------------------- log probabilities

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T, V, top", [(1, 5, 5), (2, 2000, 20), (200, 2000, 20), (160, 64000, 5), (160, 32000, 20), (2, 128256, 20), (2, 400000, 32)])
def test_logprobs_rows_of_many_nan_are_ordered_by_their_tokens(dtype, T, V, top):
    """NaN come first, equal ones in the order of their tokens: rows of nothing else, of NaN in half or most of the places, of
    both signs; in rows of a block and of a cluster, with more and with fewer of them than are collected at a time."""
    g, n = gen(V + T), torch.arange(V, device=DEV)
    nan = torch.tensor([math.nan, -math.nan], device=DEV)
    one = randn(g, V)
    rows = [torch.full((V,), math.nan, device=DEV), torch.where(n % 2 == 0, nan[0], one), torch.where(n % 3 > 0, nan[1], one),
            torch.where(n >= V // 2, nan[n % 2], torch.full_like(one, math.inf))]
    x = torch.stack([rows[i % len(rows)] for i in range(max(T, len(rows)))]).to(TT[dtype])
    tok = torch.zeros(x.shape[0], dtype=torch.int32, device=DEV)
    lp, ent, ids, tlp = run_logprobs(x, tok, top, dtype)
    assert bool(lp.isnan().all()) and bool(ent.isnan().all()) and bool(tlp.isnan().all())
    key = torch.where(x.isnan(), torch.full((), math.inf, device=DEV, dtype=torch.float64), x.double().clamp(max=1e300))
    assert torch.equal(ids.long(), torch.sort(key, dim=-1, descending=True, stable=True)[1][:, :top])


# -------------------------------------------------------------------------------------------- packed prompts

@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H, Hkv", [(16, 4), (9, 9)])
@pytest.mark.parametrize("far", [30.0, math.nan])
def test_packed_tokens_keep_their_bits_whatever_others_hold(dtype, D, H, Hkv, far):
    """Logits of some size; then other sequences, the later tokens of a sequence from the middle of a warp's rows on (in the first
    tile and in the second), and the rows behind the last sequence get queries and keys far larger, or NaN.  What no token sees
    changes none of its bits."""
    S, L = 50, 200
    g, t, N = gen(D + H), TT[dtype], 50 * 200
    q, k = (randn(g, N + 70, H, D) * 5).to(t), randn(g, N + 70, Hkv, D).to(t)
    v = randn(g, N + 70, Hkv, D).to(t)
    off = offsets_of([L] * S)
    cfg = tova.tova_packed_config(S, H, Hkv, D, TD[dtype], 0.0)
    ws = torch.empty(max(16, tova.tova_packed_workspace_bytes(cfg, N + 70)), dtype=torch.uint8, device=DEV)

    def go(q, k):
        out = torch.full((N + 70, H, D), 77.0, dtype=t, device=DEV)
        tova.tova_packed_attention(cfg, q, k, v, N + 70, off, out, ws)
        return out[:N].view(S, L, H, D)
    clean = go(q, k)
    place = torch.arange(N + 70, device=DEV)
    for first in (48, 150):                        # the first token of each sequence that changes; all of every other sequence
        change = ((place // L) % 2 == 1) | (place % L >= first) | (place >= N)
        q2, k2 = (torch.where(change[:, None, None], x * far, x) for x in (q, k))
        out = go(q2, k2)
        assert torch.equal(out[::2, :first], clean[::2, :first])
    change = ((place // L) % 2 == 1) | (place >= N)
    q2, k2 = (torch.where(change[:, None, None], x * far, x) for x in (q, k))
    assert torch.equal(go(q2, k2)[::2], clean[::2])

# --------------------------------------------------------------------------------------------- a state in pages

WAYS = {"one block": (2, 8, 2, 50), "cluster": (2, 8, 2, 1000), "shares": (1, 8, 2, 40000), "many parts": (1, 32, 1, 70000), "many": (400, 8, 2, 200)}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("logits", ["far below", "minus infinity"])
def test_paged_values_that_are_not_finite_reach_the_result_under_any_weight(dtype, way, logits):
    """All rows but the first 16 have a logit so far below the largest that their weights are 0, or minus infinity; an infinity or
    a NaN in one of them still makes its component, and no other, not finite, wherever the row lies."""
    B, H, Hkv, L = WAYS[way]
    D, rows, t = 64, 16, TT[dtype]
    g = gen(L)
    table, pages = make_table([L] * B, rows, 3)
    K, V = randn(g, pages, Hkv, rows, D).to(t), randn(g, pages, Hkv, rows, D).to(t)
    b, tb = B - 1, table.to(DEV)
    rest = table[b, 1:(L + rows - 1) // rows].long().to(DEV)
    K[rest] = -40.0 if logits == "far below" else -math.inf
    q = (randn(g, B, H, D).abs() + 0.5).to(t)      # logits of the rest: below -8 sqrt(64) * 40 / 16 ln 2 ... far below -2^7 in powers of two
    cfg = tova.tova_paged_config(B, H, Hkv, D, pages, rows, table.shape[1], TD[dtype], 0.0)
    ws = torch.empty(max(16, tova.tova_paged_workspace_bytes(cfg, L)), dtype=torch.uint8, device=DEV)
    lens = torch.full((B,), L, dtype=torch.int32, device=DEV)

    def go():
        out = torch.full((B, H, D), 77.0, dtype=t, device=DEV)
        tova.tova_paged_attention(cfg, K, V, tb, lens, L, q, out, ws)
        return out
    clean = go()
    assert bool(clean.isfinite().all())
    G = H // Hkv
    hk = Hkv - 1
    for j in (16, 33, L // 2, L - 1):
        for bad in (math.inf, -math.inf, math.nan):
            at = (int(table[b, j // rows]), hk, j % rows, 5)
            keep = V[at].clone()
            V[at] = bad
            out = go()
            V[at] = keep
            mine = out[b, hk * G:(hk + 1) * G, 5]
            assert not bool(mine.isfinite().any()), (j, bad, mine)
            mine.copy_(clean[b, hk * G:(hk + 1) * G, 5])
            assert torch.equal(out, clean), (j, bad)


def token_places(off, N):
    """The (sequence, row) pairs that each packed token belongs to: sequence b has the tokens from offsets[b], held to 0..N, to
    the one before offsets[b + 1], held the same way."""
    places = [[] for _ in range(N)]
    for b in range(len(off) - 1):
        a = min(max(off[b], 0), N)
        for i in range(a, min(max(off[b + 1], a), N)):
            places[i].append((b, i - a))
    return places


OFFSETS = {
    "outside": [-4, 100, 200, 2 ** 31 - 1], "far outside": [-2 ** 31, 7, 7, 2 ** 31 - 1], "behind the tokens": [0, 10, 5000, 6000], "below 0": [-9, -3, 60, 250],
    "all the same": [9, 9, 9, 9], "begin late, end early": [7, 20, 20, 240], "one ends before it starts": [-4, 100, 90, 150, 2 ** 31 - 1],
    "many outside": [3 * i - 300 for i in range(230)], "falls back": [0, 200, 90, 120], "falls below 0": [50, -3, 60, 260],
    "many, falling": [0] + [(37 * i) % 257 for i in range(200)] + [230],
}


@pytest.mark.parametrize("case", OFFSETS)
def test_paged_write_reads_offsets_as_packed_attention_does(case):
    """Every token goes to the row that packed attention has it at: values outside 0..N are the nearest of them, a sequence that
    would end before it starts is empty.  Where offsets fall, a token that several sequences hold goes to one of its places, some
    go to none, and nothing else is written."""
    off, N, Hkv, D, rows = OFFSETS[case], 250, 2, 64, 4
    S = len(off) - 1
    g = gen(S)
    first = [(3 * b) % 5 for b in range(S)]
    most = 65                                      # pages a sequence: up to N + 4 rows
    pages = S * most
    table = torch.randperm(pages, generator=torch.Generator().manual_seed(S)).to(torch.int32).view(S, most)
    k, v = randn(g, N, Hkv, D) + 10, randn(g, N, Hkv, D) + 10
    K = torch.zeros(pages, Hkv, rows, D, device=DEV)
    V = torch.zeros_like(K)
    cfg = tova.tova_paged_config(S, Hkv, Hkv, D, pages, rows, most, TD["fp32"], 0.0)
    tova.tova_paged_write(cfg, k, v, N, table.to(DEV), K, V, first_rows=torch.tensor(first, dtype=torch.int32, device=DEV),
                          offsets=torch.tensor(off, dtype=torch.int32, device=DEV))
    for i, places in enumerate(token_places(off, N)):
        found = 0
        for b, r in places:
            j = first[b] + r
            at = (int(table[b, j // rows]), slice(None), j % rows)
            if torch.equal(K[at], k[i]) and torch.equal(V[at], v[i]):
                found += 1
                K[at] = 0.0
                V[at] = 0.0
        assert found == (1 if places else 0) or (found == 0 and "fall" in case), (i, places, found)
    assert not bool(K.any()) and not bool(V.any())
