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


def far_logits(g, N, H, Hkv, D, size, kind, t):
    """Queries and keys along one component, so that logits are whole multiples of 2^size in every arithmetic (-7 .. 7, -7 .. -1, or
    falling and rising with the token): all weight lies on the rows of the largest multiple."""
    c = {"any": lambda: torch.randint(-7, 8, (N, Hkv), generator=g, device=DEV), "negative": lambda: torch.randint(-7, 0, (N, Hkv), generator=g, device=DEV),
         "rising": lambda: (torch.arange(N, device=DEV) // 9)[:, None].expand(N, Hkv), "falling": lambda: -(torch.arange(N, device=DEV) // 9)[:, None].expand(N, Hkv)}[kind]()
    q, k = torch.zeros(N, H, D, device=DEV), torch.zeros(N, Hkv, D, device=DEV)
    q[..., 3], k[..., 3] = 2.0 ** (size - size // 2 + 3), c * 2.0 ** (size // 2)
    return q.to(t), k.to(t), c.double()


FAR = [(size, kind) for size in (7, 19, 27, 31, 40, 100) for kind in ("any", "negative", "rising", "falling")]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("size, kind", FAR)
def test_attention_with_finite_logits_of_any_size(dtype, size, kind):
    """Soft-max of logits that lie 2^7 and more apart is the mean over the rows of the largest, at any size below fp32's range: in
    packed prompts and over pages.  Weights are 1 or 0 (2^-128 and less), so only sums of n values and the result round."""
    t, H, Hkv, D, lens, rows = TT[dtype], 6, 3, 64, [300, 1, 77, 40], 16
    g, N = gen(size), sum(lens)
    q, k, c = far_logits(g, N, H, Hkv, D, size, kind, t)
    v = randn(g, N, Hkv, D).to(t)
    cfg = tova.tova_packed_config(len(lens), H, Hkv, D, TD[dtype], 1.0 / 8)
    ws = torch.empty(max(16, tova.tova_packed_workspace_bytes(cfg, N)), dtype=torch.uint8, device=DEV)
    out = torch.full((N, H, D), 77.0, dtype=t, device=DEV)
    off = offsets_of(lens)
    tova.tova_packed_attention(cfg, q, k, v, N, off, out, ws)
    want, size_v = torch.empty(N, H, D, dtype=torch.float64, device=DEV), torch.empty(N, H, D, dtype=torch.float64, device=DEV)
    a = 0
    for n in lens:
        see = torch.ones(n, n, dtype=torch.bool, device=DEV).tril()
        for h in range(H):
            x = c[a:a + n, h // (H // Hkv)].expand(n, n).masked_fill(~see, -math.inf)
            w = (x == x.amax(-1, keepdim=True)).double()
            w /= w.sum(-1, keepdim=True)
            want[a:a + n, h], size_v[a:a + n, h] = w @ v[a:a + n, h // (H // Hkv)].double(), w @ v[a:a + n, h // (H // Hkv)].double().abs()
        a += n
    half = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -24
    tol = half * want.abs() + (2 * max(lens) + 16) * 2.0 ** -24 * size_v + 1e-30
    within(out, want, tol)
    table, pages = make_table(lens, rows, 1)
    K, V = torch.zeros(pages, Hkv, rows, D, dtype=t, device=DEV), torch.zeros(pages, Hkv, rows, D, dtype=t, device=DEV)
    pc = tova.tova_paged_config(len(lens), H, Hkv, D, pages, rows, table.shape[1], TD[dtype], 1.0 / 8)
    tova.tova_paged_write(pc, k, v, N, table.to(DEV), K, V, offsets=off)
    pw = torch.empty(max(16, tova.tova_paged_workspace_bytes(pc, max(lens))), dtype=torch.uint8, device=DEV)
    last = (off[1:] - 1).long()
    po = torch.full((len(lens), H, D), 77.0, dtype=t, device=DEV)
    tova.tova_paged_attention(pc, K, V, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), max(lens), q[last].contiguous(), po, pw)
    within(po, want[last], tol[last])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_packed_attention_with_a_list_in_captured_graphs_at_once(dtype):
    """Calls that make a list of their tiles first (more sequences, or more work, than blocks find by themselves), captured, and
    replayed over other offsets on two streams at the same time, each with a workspace of its own."""
    t = TT[dtype]
    runs = []
    for seed, (S, H, Hkv, D, N) in enumerate([(300, 8, 2, 64, 3000), (4, 32, 8, 128, 2500)]):
        g = gen(seed)
        cfg = tova.tova_packed_config(S, H, Hkv, D, TD[dtype], 0.0)
        need = tova.tova_packed_workspace_bytes(cfg, N)
        assert need > 0
        s = dict(q=randn(g, N, H, D).to(t), k=randn(g, N, Hkv, D).to(t), v=randn(g, N, Hkv, D).to(t), off=offsets_of([N // S] * S),
                 out=torch.full((N, H, D), 77.0, dtype=t, device=DEV), ws=torch.empty(need, dtype=torch.uint8, device=DEV))

        def go(cfg=cfg, s=s, N=N):
            tova.tova_packed_attention(cfg, s["q"], s["k"], s["v"], N, s["off"], s["out"], s["ws"])
        go()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for _ in range(3):                     # one behind the other in the same workspace
                go()
        lens = [(i * 7) % 19 for i in range(S)] if S > 4 else [0, 1700, 3, 600]
        s["off"].copy_(offsets_of(lens))
        s["out"].fill_(77.0)
        runs.append((s, graph, lens, D))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(4):
        for (s, graph, _, _), st in zip(runs, streams):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for s, _, lens, D in runs:
        n = sum(lens)
        assert n < s["q"].shape[0]
        want, wv, reach = packed_reference(s["q"][:n], s["k"][:n], s["v"][:n], lens)
        within(s["out"][:n], want, attention_tolerance(dtype, D, max(lens), want, wv, reach, True))
        assert bool((s["out"][n:] == 77.0).all())


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
    q = (randn(g, B, H, D).abs() + 0.5).to(t)      # logits of the rest: below -40 * 64 * 0.5 / 8 = -160, weights below 2^-149
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


@pytest.mark.parametrize("dtype, B, H, Hkv, L", [("bf16", 3, 8, 2, 5000), ("fp32", 1, 4, 4, 9000), ("bf16", 60, 32, 8, 2000)])
def test_paged_calls_fit_the_workspace_of_a_longer_bound(dtype, B, H, Hkv, L):
    """A workspace of the size reported for n_live = L serves every call below it, in clusters and in shares, and no byte behind
    it is written."""
    D, rows, t = 128, 16, TT[dtype]
    g = gen(L)
    most = (L + rows - 1) // rows
    K, V = randn(g, 400, Hkv, rows, D).to(t), randn(g, 400, Hkv, rows, D).to(t)
    table = torch.randint(0, 400, (B, most), generator=torch.Generator().manual_seed(B), dtype=torch.int32)
    cfg = tova.tova_paged_config(B, H, Hkv, D, 400, rows, most, TD[dtype], 0.0)
    need = tova.tova_paged_workspace_bytes(cfg, L)
    ws = torch.empty(need + 256, dtype=torch.uint8, device=DEV)
    q = randn(g, B, H, D).to(t)
    for n in (0, 1, 63, 256, 257, 700, 1500, 2000, L // 2, L):
        if n > L:
            continue
        lens = [max(0, n - 13 * b) for b in range(B)]
        ws.fill_(0xff)
        out = torch.full((B, H, D), 77.0, dtype=t, device=DEV)
        tova.tova_paged_attention(cfg, K, V, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), n, q, out, ws[:need])
        want, wv, reach = paged_reference(q, K, V, table, lens, rows)
        within(out, want, attention_tolerance(dtype, D, max(1, n), want, wv, reach, False))
        assert bool((ws[need:] == 0xff).all()), n


def test_paged_bounds_and_their_workspaces_up_to_the_largest():
    """Sizes rise with the bound up to 2^30 rows; above, the size and the call are refused."""
    cfg = tova.tova_paged_config(1, 8, 2, 64, 1, 1 << 15, 1 << 16, TD["bf16"], 0.0)
    need = [tova.tova_paged_workspace_bytes(cfg, n) for n in (1, 1000, 10 ** 6, 2 ** 29, 2 ** 30)]
    assert need == sorted(need)
    K, q = torch.zeros(1, 2, 1 << 15, 64, dtype=torch.bfloat16, device=DEV), torch.zeros(1, 8, 64, dtype=torch.bfloat16, device=DEV)
    table, lens = torch.zeros(1, 1 << 16, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    ws, out = torch.empty(need[-1], dtype=torch.uint8, device=DEV), torch.ones_like(q)
    for n in (2 ** 30 + 1, 2 ** 31 - 1):
        for call in (lambda: tova.tova_paged_workspace_bytes(cfg, n), lambda: tova.tova_paged_attention(cfg, K, K, table, lens, n, q, out, ws)):
            with pytest.raises(tova.TovaError) as e:
                call()
            assert e.value.code == -2
    assert bool((out == 1).all())


# ------------------------------------------------------------------------------------------------ all together

def test_serving_loop_against_the_definition():
    """Three prompts of different lengths and what follows them, token by token: both attentions' outputs against the 64-bit
    definition, element by element, at a bound that notices a single row left out; and the probabilities from the pages against
    those from the whole texts.

    A logit x = sum_d o_d w_d is off by sum_d |w_d| (bound of o_d) and its own rounding 2^-8 |x| (sums in fp32: 2^-10 of the
    terms' sizes is far more than H D 2^-24), and log p = x_t - log sum exp x by twice the largest of these."""
    H, Hkv, D, V, rows, dt = 8, 2, 64, 500, 16, torch.bfloat16
    lens, new = [37, 1, 80], 20
    S, width = len(lens), (H + 2 * Hkv) * D
    g = gen(12)
    embed, wqkv, wout = randn(g, V, 96).to(dt), (randn(g, 96, width) / 10).to(dt), (randn(g, H * D, V) / 20).to(dt)
    qw, kw = (1 + 0.1 * randn(g, D)).to(dt), (1 + 0.1 * randn(g, D)).to(dt)
    whole_lens = [n + new for n in lens]
    starts = [sum(whole_lens[:b]) for b in range(S)]
    N = sum(whole_lens)
    ids = torch.randint(0, V, (N,), generator=g, device=DEV)
    pos = torch.cat([torch.arange(n, device=DEV) for n in whole_lens]).to(torch.int32)
    x = embed[ids] @ wqkv                          # projected once: the same rows go through both ways
    rope = tova.TovaRope(1, H, Hkv, D)

    def project(at):
        n, y = at.shape[0], x[at]
        q, k = y[:, None, :H * D].unflatten(-1, (H, D)), y[:, None, H * D:(H + Hkv) * D].unflatten(-1, (Hkv, D))
        qo, ko = torch.empty(n, 1, H, D, dtype=dt, device=DEV), torch.empty(n, 1, Hkv, D, dtype=dt, device=DEV)
        rope.tova_norm_rope_apply(q, k, n, qo, ko, q_weight=qw, k_weight=kw, positions=pos[at].contiguous())
        return qo[:, 0], ko[:, 0], y[:, (H + Hkv) * D:].unflatten(-1, (Hkv, D))

    def packed(at, lens):
        q, k, v = project(at)
        cfg = tova.tova_packed_config(S, H, Hkv, D, TD["bf16"], 0.0)
        ws = torch.empty(max(16, tova.tova_packed_workspace_bytes(cfg, at.shape[0])), dtype=torch.uint8, device=DEV)
        out = torch.empty(at.shape[0], H, D, dtype=dt, device=DEV)
        tova.tova_packed_attention(cfg, q, k, v, at.shape[0], offsets_of(lens), out, ws)
        return out, q, k, v

    def logprobs(out, tok):
        logits = (out.flatten(1) @ wout).contiguous()
        lp = torch.empty(out.shape[0], device=DEV)
        tova.tova_token_logprobs(tova.tova_logprobs_config(V, TD["bf16"], 0, 0), logits, out.shape[0], tok.to(torch.int32).contiguous(), lp)
        return lp.double(), logits
    whole, q, k, v = packed(torch.arange(N, device=DEV), whole_lens)
    want, wv, reach = packed_reference(q, k, v, whole_lens)
    tol_packed = attention_tolerance("bf16", D, max(whole_lens), want, wv, reach, True)
    tol_paged = attention_tolerance("bf16", D, max(whole_lens), want, wv, reach, False)
    within(whole, want, tol_packed)
    # (the bound notices any row of the longest sequence that its last token would miss)
    b = 2
    last = starts[b] + whole_lens[b] - 1
    kk, vv = k[starts[b]:last + 1, 0].double(), v[starts[b]:last + 1, 0].double()
    s = kk @ q[last, 0].double() * D ** -0.5
    for j in range(whole_lens[b]):
        keep = torch.arange(whole_lens[b], device=DEV) != j
        without = torch.softmax(s[keep], 0) @ vv[keep]
        assert bool(((without - want[last, 0]).abs() > tol_paged[last, 0]).any()), j
    table, pages = make_table(whole_lens, rows, 5)
    table = table.to(DEV)
    K, V_ = (torch.full((pages, Hkv, rows, D), math.nan, dtype=dt, device=DEV) for _ in range(2))
    pcfg = tova.tova_paged_config(S, H, Hkv, D, pages, rows, table.shape[1], TD["bf16"], 0.0)
    at = torch.cat([torch.arange(a, a + n, device=DEV) for a, n in zip(starts, lens)])
    out, _, pk, pv = packed(at, lens)
    assert torch.equal(out, whole[at])             # a token's bits depend on nothing behind it
    tova.tova_paged_write(pcfg, pk, pv, at.shape[0], table, K, V_, offsets=offsets_of(lens))
    held = torch.tensor(lens, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(16, tova.tova_paged_workspace_bytes(pcfg, max(whole_lens))), dtype=torch.uint8, device=DEV)
    for i in range(new - 1):
        at = torch.tensor([a + n + i for a, n in zip(starts, lens)], device=DEV)
        q1, k1, v1 = project(at)
        tova.tova_paged_write(pcfg, k1, v1, S, table, K, V_, first_rows=held)
        held += 1
        o = torch.empty(S, H, D, dtype=dt, device=DEV)
        tova.tova_paged_attention(pcfg, K, V_, table, held, max(whole_lens), q1, o, ws)
        within(o, want[at], tol_paged[at])
        got, logits = logprobs(o, ids[at + 1])
        other, logits2 = logprobs(whole[at], ids[at + 1])
        size = want[at].abs().flatten(1) @ wout.double().abs()
        off = (tol_paged[at] + tol_packed[at]).flatten(1) @ wout.double().abs() + 2.0 ** -8 * (logits.double().abs() + logits2.double().abs()) + 2.0 ** -10 * size
        assert bool(((got - other).abs() <= 2 * off.amax(-1) + 1e-4).all())
        assert bool((got - torch.log_softmax(logits.double(), -1).gather(1, ids[at + 1][:, None])[:, 0]).abs().max() <= 1e-4)
