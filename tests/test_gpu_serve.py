"""GPU tests of the operators for sequences of different lengths, against their definitions in 64 bits.

Tolerances.  A rounding to type t is off by at most half a step, eps(t)/2 relative (bf16 2^-8, fp32 2^-24).  Sums of n
fp32 products are off by at most about n 2^-24 of the sum of the products' sizes, twice that on the tensor cores, whose
adders may truncate."""
import math

import pytest
import torch

import paper_2401_06104_b200 as tova

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TT = {"bf16": torch.bfloat16, "fp32": torch.float32}
TD = {"bf16": tova.TOVA_DTYPE_BF16, "fp32": tova.TOVA_DTYPE_FP32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
U = 2.0 ** -24


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


def within(got, want, tol):
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), float(err.max()), (~(err <= tol)).nonzero()[:3].tolist())


# ------------------------------------------------------------------------------------- norms with the rotation

def turn(x, pos, base, rot, layout, sign):
    """x [T,B,heads,D] turned by sign times the positions' angles, in 64 bits; and the sizes |a| + |b| that roundings scale
    with."""
    w = torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device=DEV)
    z = torch.polar(torch.ones(1, dtype=torch.float64, device=DEV), sign * pos.double()[..., None, None] * w)
    h = rot // 2
    a, b = (slice(0, h), slice(h, rot)) if layout == tova.TOVA_ROPE_HALF else (slice(0, rot, 2), slice(1, rot, 2))
    y, size = x.clone(), x.abs()
    t = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * z
    y[..., a], y[..., b] = t.real, t.imag
    both = x[..., a].abs() + x[..., b].abs()
    size[..., a], size[..., b] = both, both
    return y, size


def norm_forward(x, w, eps, pos, base, rot, layout):
    x, w = x.double(), w.double()
    r = (x.square().mean(-1, keepdim=True) + eps) ** -0.5
    return turn(x * r * w, pos, base, rot, layout, 1.0)


def norm_backward(x, w, eps, pos, base, rot, layout, dy):
    """dx, dw and the sizes that their roundings scale with."""
    x, w = x.double(), w.double()
    r = (x.square().mean(-1, keepdim=True) + eps) ** -0.5
    xh = x * r
    g, gs = turn(dy.double(), pos, base, rot, layout, -1.0)
    dx = r * (g * w - xh * (g * w * xh).mean(-1, keepdim=True))
    size = r * (gs * w.abs() + xh.abs() * (gs * (w * xh).abs()).mean(-1, keepdim=True))
    return dx, size, (g * xh).sum((0, 1, 2)), (gs * xh.abs()).sum((0, 1, 2))


NORM = [(128, 128, "half"), (128, 96, "half"), (128, 20, "half"), (128, 2, "half"), (64, 64, "half"), (64, 62, "half"), (128, 128, "inter"),
        (128, 36, "inter"), (64, 64, "inter")]


def norm_inputs(dtype, D, T, B, H, Hkv, seed, far=200000):
    g, t = gen(seed), TT[dtype]
    s = dict(q=(randn(g, T, B, H, D) * 1.7).to(t), k=(randn(g, T, B, Hkv, D) * 0.3).to(t), qw=(1 + 0.3 * randn(g, D)).to(t),
             kw=randn(g, D).to(t), dq=randn(g, T, B, H, D).to(t), dk=randn(g, T, B, Hkv, D).to(t))
    s["pos"] = torch.randint(-5, far, (T, B), generator=g, device=DEV, dtype=torch.int32)
    return s


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D, rot, layout", NORM)
def test_norm_rope_and_its_gradient(dtype, D, rot, layout):
    """The sum of squares: about D / lanes + log2(lanes) additions, rsqrt 2 steps: r within 16 * 2^-24; three products and the
    turn's (8, as in the rotation's own test) make 28.  The gradient: g 8, r 16, mean of products D/lanes + log2 + 2, again
    r: 64 in all.  dw: a lane's chain of rows (at most 30 here) and the joins' 16 + 8 terms, 8 + 16 for g and xh: 100."""
    lay = tova.TOVA_ROPE_HALF if layout == "half" else tova.TOVA_ROPE_INTERLEAVED
    T, B, H, Hkv, base, eps = 37, 3, 6, 2, 10000.0, 1e-5
    s = norm_inputs(dtype, D, T, B, H, Hkv, rot + D)
    s["q"][3, 1, 2] = 0.0                         # a row of zeros: r = eps^(-1/2)
    r = tova.TovaRope(B, H, Hkv, D, dtype=TD[dtype], rotary_dim=rot, layout=lay)
    qo, ko = torch.full_like(s["q"], 7.0), torch.full_like(s["k"], 7.0)
    r.tova_norm_rope_apply(s["q"], s["k"], T, qo, ko, q_weight=s["qw"], k_weight=s["kw"], eps=eps, positions=s["pos"])
    need = r.tova_norm_rope_workspace_bytes(T)
    ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device=DEV)
    dq, dk = torch.full_like(s["q"], 7.0), torch.full_like(s["k"], 7.0)
    dqw, dkw = torch.full((D,), 7.0, device=DEV), torch.full((D,), 7.0, device=DEV)
    args = (s["q"], s["k"], s["dq"], s["dk"], T, dq, dk, ws[:need])
    kw = dict(q_weight=s["qw"], k_weight=s["kw"], dq_weight=dqw, dk_weight=dkw, eps=eps, positions=s["pos"])
    r.tova_norm_rope_backward(*args, **kw)
    for x, w, y, dy, dx, dw in ((s["q"], s["qw"], qo, s["dq"], dq, dqw), (s["k"], s["kw"], ko, s["dk"], dk, dkw)):
        want, size = norm_forward(x, w, eps, s["pos"], base, rot, lay)
        within(y, want, HALF[dtype] * want.abs() + 28 * U * size + 1e-38)
        want, size, ww, wsize = norm_backward(x, w, eps, s["pos"], base, rot, lay, dy)
        within(dx, want, HALF[dtype] * want.abs() + 64 * U * size + 1e-38)
        within(dw, ww, 100 * U * wsize)
    assert bool((ws[need:] == 0xff).all())
    first = [x.clone() for x in (dq, dk, dqw, dkw)]
    r.tova_norm_rope_backward(*args, **kw)
    assert all(torch.equal(a, b) for a, b in zip(first, (dq, dk, dqw, dkw)))       # the same bits every time


@pytest.mark.parametrize("T, B", [(1, 1), (1, 64), (2500, 2), (5001, 1)])
def test_norm_rope_sizes(T, B):
    """Tokens per block from one to four, ragged ends; without listed positions; the weights' sums over many rows: a lane's
    chain is at most 4 * 4 tokens of a block's walk here, times H + Hkv rows over 16 groups."""
    H, Hkv, D, base, eps = 8, 2, 128, 500000.0, 1e-6
    s = norm_inputs("bf16", D, T, B, H, Hkv, T)
    r = tova.TovaRope(B, H, Hkv, D, base=base)
    qo, ko, dq, dk = (torch.full_like(s[x], 7.0) for x in ("q", "k", "q", "k"))
    dqw, dkw = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
    r.tova_norm_rope_apply(s["q"], s["k"], T, qo, ko, q_weight=s["qw"], k_weight=s["kw"], eps=eps, first_pos=77)
    ws = torch.empty(r.tova_norm_rope_workspace_bytes(T), dtype=torch.uint8, device=DEV)
    r.tova_norm_rope_backward(s["q"], s["k"], s["dq"], s["dk"], T, dq, dk, ws, q_weight=s["qw"], k_weight=s["kw"], dq_weight=dqw,
                              dk_weight=dkw, eps=eps, first_pos=77)
    pos = 77 + torch.arange(T, device=DEV)[:, None].expand(T, B)
    for x, w, y, dy, dx, dw in ((s["q"], s["qw"], qo, s["dq"], dq, dqw), (s["k"], s["kw"], ko, s["dk"], dk, dkw)):
        want, size = norm_forward(x, w, eps, pos, base, D, 0)
        within(y, want, 2.0 ** -8 * want.abs() + 28 * U * size + 1e-38)
        want, size, ww, wsize = norm_backward(x, w, eps, pos, base, D, 0, dy)
        within(dx, want, 2.0 ** -8 * want.abs() + 64 * U * size + 1e-38)
        within(dw, ww, 100 * U * wsize)


def test_norm_rope_strides_aliases_no_keys_no_weights():
    T, B, H, Hkv, D = 9, 2, 8, 2, 64
    g = gen(3)
    qkv = randn(g, T, B, (H + 2 * Hkv) * D).to(torch.bfloat16)
    keep = qkv.clone()
    q, k = qkv[..., :H * D].unflatten(-1, (H, D)), qkv[..., H * D:(H + Hkv) * D].unflatten(-1, (Hkv, D))
    one = torch.ones(D, dtype=torch.bfloat16, device=DEV)
    r = tova.TovaRope(B, H, Hkv, D)
    pos = 11 + torch.arange(T, device=DEV)[:, None].expand(T, B)
    want = [norm_forward(x.clone(), one, 1e-6, pos, 10000.0, D, 0) for x in (q, k)]
    only = torch.empty(T, B, H, D, dtype=torch.bfloat16, device=DEV)
    r.tova_norm_rope_apply(q, None, T, only, None, first_pos=11)
    tol = [2.0 ** -8 * w.abs() + 28 * U * s + 1e-38 for w, s in want]
    within(only, want[0][0], tol[0])
    dy = randn(g, T, B, H, D).to(torch.bfloat16)
    dqw, dkw = torch.full((D,), 7.0, device=DEV), torch.full((D,), 7.0, device=DEV)
    ws = torch.empty(r.tova_norm_rope_workspace_bytes(T), dtype=torch.uint8, device=DEV)
    dx, size, ww, wsize = norm_backward(q.clone(), one, 1e-6, pos, 10000.0, D, 0, dy)
    r.tova_norm_rope_backward(q, None, dy, None, T, dy, None, ws, dq_weight=dqw, dk_weight=dkw, first_pos=11)     # dq over dq_out
    within(dy, dx, 2.0 ** -8 * dx.abs() + 64 * U * size + 1e-38)
    within(dqw, ww, 100 * U * wsize)
    assert bool((dkw == 0).all())                 # no keys
    gq, gk = randn(g, T, B, H, D).to(torch.bfloat16), randn(g, T, B, Hkv, D).to(torch.bfloat16)
    dk, dks, _, _ = norm_backward(k.clone(), one, 1e-6, pos, 10000.0, D, 0, gk)
    r.tova_norm_rope_backward(q, k, gq, gk, T, gq, gk, ws, first_pos=11)       # over both, no weights' gradients asked for
    within(gk, dk, 2.0 ** -8 * dk.abs() + 64 * U * dks + 1e-38)
    assert torch.equal(qkv, keep)
    r.tova_norm_rope_apply(q, k, T, q, k, first_pos=11)         # in place, as slices of the projection
    within(q, want[0][0], tol[0])
    within(k, want[1][0], tol[1])
    assert torch.equal(qkv[..., (H + Hkv) * D:], keep[..., (H + Hkv) * D:])
    dqw.fill_(7.0)
    r.tova_norm_rope_backward(q, None, dy, None, 0, dy, None, ws, dq_weight=dqw)      # no tokens: sums of nothing
    assert bool((dqw == 0).all())
    with pytest.raises(tova.TovaError) as e:
        r.tova_norm_rope_backward(q, None, dy, None, T, dy, None, ws[:64])
    assert e.value.code == -5


def test_norm_rope_gradient_by_differences():
    """loss = <c, y(q, k; weights)> in fp32: the slope along a random direction by central differences at steps h and 2h.  The
    results' roundings (28 2^-24 of their sizes, against c) divided by h are the noise; the steps' disagreement is three
    times the smaller one's own error from the curve's third derivative."""
    T, B, H, Hkv, D = 3, 2, 4, 2, 64
    s = norm_inputs("fp32", D, T, B, H, Hkv, 1, far=500)
    g = gen(9)
    r = tova.TovaRope(B, H, Hkv, D, dtype=TD["fp32"])
    names = ("q", "k", "qw", "kw")
    step = {n: randn(g, *s[n].shape) for n in names}
    noise = [0.0]

    def loss(h):
        x = {n: s[n] + h * step[n] for n in names}
        qo, ko = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        r.tova_norm_rope_apply(x["q"], x["k"], T, qo, ko, q_weight=x["qw"], k_weight=x["kw"], positions=s["pos"])
        noise[0] = max(noise[0], 30 * U * float(sum((norm_forward(x[n], x[n + "w"], 1e-6, s["pos"], 10000.0, D, 0)[1] * s["d" + n].double().abs()).sum()
                                                    for n in "qk")))
        return float((qo.double() * s["dq"]).sum() + (ko.double() * s["dk"]).sum())
    h = 2.0 ** -9
    slope = [(loss(x) - loss(-x)) / (2 * x) for x in (h, 2 * h)]
    dq, dk = torch.empty_like(s["q"]), torch.empty_like(s["k"])
    dw = [torch.empty(D, device=DEV) for _ in range(2)]
    ws = torch.empty(r.tova_norm_rope_workspace_bytes(T), dtype=torch.uint8, device=DEV)
    r.tova_norm_rope_backward(s["q"], s["k"], s["dq"], s["dk"], T, dq, dk, ws, q_weight=s["qw"], k_weight=s["kw"], dq_weight=dw[0],
                              dk_weight=dw[1], positions=s["pos"])
    got = sum(float((a.double() * b.double()).sum()) for a, b in zip((dq, dk, *dw), (step[n] for n in names)))
    assert abs(got - slope[0]) <= noise[0] / h + abs(slope[1] - slope[0]), (got, slope, noise[0] / h)


# --------------------------------------------------------------------------------------------- a state in pages

def make_table(held, rows, seed, spare=2, extra=0):
    """A page table whose pages lie in any order; entries that no row needs are garbage outside the pool."""
    need = [(n + rows - 1) // rows for n in held]
    most = max(1, max(need)) + extra
    total = sum(need) + spare
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed)).to(torch.int32)
    table = torch.full((len(held), most), 2 ** 31 - 1, dtype=torch.int32)
    table[:, 1::2] = -2 ** 31
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D, Hkv", [(64, 1), (128, 8), (128, 32)])
@pytest.mark.parametrize("rows, before, lens", [(16, [0], [1]), (16, [5, 0, 31, 16], [40, 0, 1, 17]), (1, [2, 7], [3, 20]), (64, [63, 64, 1], [130, 1, 700]),
                                                (8, [0] * 70, [3] * 69 + [0]), (4096, [4000, 0], [200, 5])])
def test_paged_write(dtype, D, Hkv, rows, before, lens):
    g, t, S, N = gen(rows + D), TT[dtype], len(lens), sum(lens)
    table, pages = make_table([a + n for a, n in zip(before, lens)], rows, rows)
    pad = 5                                       # tokens that belong to no sequence
    k, v = randn(g, N + pad, Hkv, D).to(t), randn(g, N + pad, 3 * Hkv * D).to(t)[:, Hkv * D:2 * Hkv * D].unflatten(-1, (Hkv, D))
    K, V = randn(g, pages, Hkv, rows, D).to(t), randn(g, pages, Hkv, rows, D).to(t)
    wantK, wantV = K.clone(), V.clone()
    off = [0]
    for n in lens:
        off.append(off[-1] + n)
    for b in range(S):
        for i in range(lens[b]):
            j = before[b] + i
            wantK[table[b, j // rows], :, j % rows] = k[off[b] + i]
            wantV[table[b, j // rows], :, j % rows] = v[off[b] + i]
    cfg = tova.tova_paged_config(S, Hkv, Hkv, D, pages, rows, table.shape[1], TD[dtype], 0.0)
    tova.tova_paged_write(cfg, k, v, N + pad, table.to(DEV), K, V, first_rows=torch.tensor(before, dtype=torch.int32, device=DEV),
                          offsets=torch.tensor(off, dtype=torch.int32, device=DEV))
    assert torch.equal(K, wantK) and torch.equal(V, wantV)


def test_paged_write_one_token_each_and_rows_without_a_place():
    """No offsets: one token a sequence.  Rows behind the table, before row 0, or in pages outside the pool are dropped."""
    S, Hkv, D, rows, pages = 7, 2, 64, 4, 5
    g = gen(1)
    k, v = randn(g, S, Hkv, D), randn(g, S, Hkv, D)
    K = torch.zeros(pages, Hkv, rows, D, device=DEV)
    V = torch.zeros_like(K)
    table = torch.tensor([[0, 9], [1, -1], [5, 2], [-7, 3], [4, 4], [4, 2 ** 31 - 1], [3, 0]], dtype=torch.int32)
    first = [0, 7, 4, 3, 8, -1, 2 ** 31 - 1]       # kept; page -1; kept in page 2; page -7; behind the table; before row 0; far behind
    cfg = tova.tova_paged_config(S, Hkv, Hkv, D, pages, rows, 2, TD["fp32"], 0.0)
    tova.tova_paged_write(cfg, k, v, S, table.to(DEV), K, V, first_rows=torch.tensor(first, dtype=torch.int32, device=DEV))
    want = torch.zeros_like(K)
    want[0, :, 0], want[2, :, 0] = k[0], k[2]
    assert torch.equal(K, want)
    K.zero_()
    tova.tova_paged_write(cfg, k, v, 1, table.to(DEV), K, V)             # fewer tokens than sequences, rows from 0 on
    want.zero_()
    want[0, :, 0] = k[0]
    assert torch.equal(K, want)


def paged_reference(q, K, V, table, lens, rows, scale=None):
    """64-bit attention; the result, sum p |v|, and the largest sum of |q_d k_d| scale."""
    B, H, D = q.shape
    Hkv = K.shape[1]
    scale = scale or D ** -0.5
    out = torch.zeros(B, H, D, dtype=torch.float64, device=DEV)
    wv, reach = torch.zeros_like(out), torch.zeros(B, H, 1, dtype=torch.float64, device=DEV)
    for b, n in enumerate(lens):
        if n == 0:
            continue
        at = [int(table[b, j]) for j in range((n + rows - 1) // rows)]
        keep = torch.tensor([0 <= p < K.shape[0] for p in at for _ in range(rows)][:n], device=DEV)
        pg = torch.tensor([p if 0 <= p < K.shape[0] else 0 for p in at], device=DEV)
        kk = K[pg].transpose(0, 1).reshape(Hkv, -1, D)[:, :n][:, keep].double()
        vv = V[pg].transpose(0, 1).reshape(Hkv, -1, D)[:, :n][:, keep].double()
        if kk.shape[1] == 0:
            continue
        qq = q[b].double().view(Hkv, H // Hkv, D)
        w = torch.softmax(torch.einsum("hgd,hnd->hgn", qq, kk) * scale, -1)
        out[b] = torch.einsum("hgn,hnd->hgd", w, vv).reshape(H, D)
        wv[b] = torch.einsum("hgn,hnd->hgd", w, vv.abs()).reshape(H, D)
        reach[b] = (torch.einsum("hgd,hnd->hgn", qq.abs(), kk.abs()) * scale).amax(-1).reshape(H, 1)
    return out, wv, reach


def attention_tolerance(dtype, D, cols, want, wv, reach, weights_rounded):
    """A logit is off by delta <= 2 (D + 4) 2^-24 reach (products and sums in fp32, truncating adders), a weight by
    e^delta - 1 relative, in numerator and denominator; fp32 sums over the columns add 2 cols 2^-24 at the very most of
    sum p|v|; exp2's own error is 2^-22.  Weights as two bf16 terms are off by 2^-16.  As one they are p (1 + d), |d| <= 2^-8,
    and summed as they are: sum p (1 + d) v / sum p (1 + d) is off from o = sum p v by sum p d (v - o) / sum p (1 + d), that
    is by 2^-8 (sum p|v| + |o|) / (1 - 2^-8).  Then the result's rounding."""
    delta = 2 * (D + 4) * U * reach
    rel = 2 * torch.expm1(delta) + (2 * cols + 16) * U
    if dtype == "bf16":
        rel = rel + (2.0 ** -8 if weights_rounded else 2.0 ** -16)
    sum_rounded = 2.0 ** -8 * want.abs() if dtype == "bf16" and weights_rounded else 0.0
    return (rel * wv + sum_rounded) * 1.01 + HALF[dtype] * want.abs() + 1e-30


def run_paged(dtype, B, H, Hkv, D, lens, rows, seed=0, n_live=None, gain=1.3, sm_scale=0.0, extra=0, bad=()):
    g, t = gen(seed + D + rows), TT[dtype]
    table, pages = make_table(lens, rows, seed, extra=extra)
    K, V = randn(g, pages, Hkv, rows, D).to(t), randn(g, pages, Hkv, rows, D).to(t)
    for b, n in enumerate(lens):                  # rows behind a sequence's last may hold anything, and pages of nobody's
        if n % rows:
            K[table[b, n // rows], :, n % rows:] = math.nan
            V[table[b, n // rows], :, n % rows:] = math.inf
    used = {int(p) for b, n in enumerate(lens) for p in table[b, :(n + rows - 1) // rows]}
    for p in range(pages):
        if p not in used:
            K[p] = V[p] = math.nan
    for b, j, to in bad:
        table[b, j] = to
    q = (randn(g, B, 2 * H * D) * gain).to(t)[:, :H * D].unflatten(-1, (H, D))
    n_live = max(lens) if n_live is None else n_live
    cfg = tova.tova_paged_config(B, H, Hkv, D, pages, rows, table.shape[1], TD[dtype], sm_scale)
    need = tova.tova_paged_workspace_bytes(cfg, n_live)
    ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full((B, H, D), 77.0, dtype=t, device=DEV)
    args = (cfg, K, V, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), n_live, q, out, ws[:need])
    tova.tova_paged_attention(*args)
    want, wv, reach = paged_reference(q, K, V, table, lens, rows, sm_scale or None)
    within(out, want, attention_tolerance(dtype, D, max(lens), want, wv, reach, False))
    assert bool((ws[need:] == 0xff).all())
    first = out.clone()
    tova.tova_paged_attention(*args)
    assert torch.equal(first, out)
    return out


PAGED = [
    # B, H, Hkv, lens, rows
    (1, 4, 4, [0], 16), (1, 1, 1, [1], 16), (2, 32, 8, [1000, 3], 16), (3, 8, 1, [64, 63, 65], 16), (4, 32, 32, [0, 127, 129, 16], 32),
    (2, 12, 4, [515, 33], 64), (3, 16, 1, [100, 257, 0], 128), (2, 24, 1, [300, 17], 16), (1, 40, 2, [70], 1), (2, 6, 3, [50, 9], 2),
    (3, 8, 2, [77, 200, 1], 8), (1, 32, 4, [20011], 16), (5, 8, 8, [9000, 1, 4000, 0, 6500], 256), (70, 8, 2, [(37 * i) % 701 for i in range(70)], 16),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", PAGED, ids=lambda s: f"B{s[0]}H{s[1]}x{s[2]}L{max(s[3])}r{s[4]}")
def test_paged_attention(dtype, D, shape):
    B, H, Hkv, lens, rows = shape
    run_paged(dtype, B, H, Hkv, D, lens, rows)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B, H, Hkv, L", [(1, 32, 32, 30000), (300, 32, 8, 300), (1, 4, 2, 100003), (2000, 2, 1, 40)])
def test_paged_attention_every_way_to_deal_out(dtype, B, H, Hkv, L):
    run_paged(dtype, B, H, Hkv, 128, [max(0, L - 131 * b % L) for b in range(B)], 16, seed=B)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("B, Hkv, long", [(20, 8, 3000), (70, 8, 1500), (9, 2, 20000)])
def test_paged_attention_one_sequence_far_longer_than_the_others(dtype, B, Hkv, long):
    run_paged(dtype, B, 4 * Hkv, Hkv, 128, [long if b == B // 2 else (5 * b) % 40 for b in range(B)], 16, seed=B)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_paged_sequences_share_pages(dtype):
    """The pages of a common beginning are in several sequences' tables, and one sequence is in the batch twice."""
    H, Hkv, D, rows, t = 8, 2, 64, 16, TT[dtype]
    g = gen(3)
    K, V = randn(g, 9, Hkv, rows, D).to(t), randn(g, 9, Hkv, rows, D).to(t)
    table = torch.tensor([[4, 1, 7, 0], [4, 1, 2, 3], [4, 1, 7, 0], [4, 6, 4, 4]], dtype=torch.int32)
    lens = [60, 33, 60, 64]
    q = randn(g, 4, H, D).to(t)
    q[2] = q[0]
    cfg = tova.tova_paged_config(4, H, Hkv, D, 9, rows, 4, TD[dtype], 0.0)
    ws = torch.empty(max(16, tova.tova_paged_workspace_bytes(cfg, 64)), dtype=torch.uint8, device=DEV)
    out = torch.empty(4, H, D, dtype=t, device=DEV)
    tova.tova_paged_attention(cfg, K, V, table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV), 64, q, out, ws)
    want, wv, reach = paged_reference(q, K, V, table, lens, rows)
    within(out, want, attention_tolerance(dtype, D, 64, want, wv, reach, False))
    assert torch.equal(out[0], out[2])


def test_paged_attention_bounds_scale_and_table():
    run_paged("bf16", 2, 8, 2, 128, [300, 20], 16, n_live=320, sm_scale=0.3, extra=3)
    run_paged("fp32", 2, 8, 2, 64, [300, 20], 16, n_live=304, extra=1)
    # pages outside the pool hold no rows: in the middle, all of a sequence's, the first
    for dtype in ("bf16", "fp32"):
        for rows in (16, 4):
            run_paged(dtype, 3, 8, 2, 128, [300, 4, 100], rows, bad=[(0, 3, -1), (0, 4, 2 ** 31 - 1), (1, 0, -5), (2, 0, 10 ** 6)])


def test_paged_attention_lengths_outside_the_bound_are_clamped():
    B, H, Hkv, D, rows, n_live = 4, 8, 2, 64, 16, 40
    g = gen(2)
    K, V = randn(g, 12, Hkv, rows, D), randn(g, 12, Hkv, rows, D)
    table = torch.arange(12, dtype=torch.int32).view(4, 3)
    q = randn(g, B, H, D)
    cfg = tova.tova_paged_config(B, H, Hkv, D, 12, rows, 3, TD["fp32"], 0.0)
    ws = torch.empty(max(16, tova.tova_paged_workspace_bytes(cfg, n_live)), dtype=torch.uint8, device=DEV)
    out = torch.empty(B, H, D, device=DEV)
    tova.tova_paged_attention(cfg, K, V, table.to(DEV), torch.tensor([41, -3, 2 ** 31 - 1, -2 ** 31], dtype=torch.int32, device=DEV), n_live, q, out, ws)
    want, wv, reach = paged_reference(q, K, V, table, [40, 0, 40, 0], rows)
    within(out, want, attention_tolerance("fp32", D, 40, want, wv, reach, False))


WAYS = {"one block": (2, 8, 2, 50), "cluster": (2, 8, 2, 1000), "shares": (1, 8, 2, 40000), "many": (400, 8, 2, 200)}


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("way", WAYS)
def test_paged_values_that_are_not_numbers(dtype, way):
    """NaN in a query, in a visible key, logits that are all minus infinity: NaN rows, and no others."""
    B, H, Hkv, L = WAYS[way]
    D, rows, t = 64, 16, TT[dtype]
    g = gen(5)
    lens = [L] * B
    table, pages = make_table(lens, rows, 3)
    K, V = randn(g, pages, Hkv, rows, D).to(t), randn(g, pages, Hkv, rows, D).to(t)
    q = randn(g, B, H, D).to(t)
    cfg = tova.tova_paged_config(B, H, Hkv, D, pages, rows, table.shape[1], TD[dtype], 0.0)
    ws = torch.empty(max(16, tova.tova_paged_workspace_bytes(cfg, L)), dtype=torch.uint8, device=DEV)
    lt, tb = torch.tensor(lens, dtype=torch.int32, device=DEV), table.to(DEV)

    def go():
        out = torch.full((B, H, D), 77.0, dtype=t, device=DEV)
        tova.tova_paged_attention(cfg, K, V, tb, lt, L, q, out, ws)
        return out
    clean = go()
    b = B - 1
    keep = q[b, 5].clone()
    q[b, 5, 3] = math.nan
    out = go()
    assert bool(out[b, 5].isnan().all())
    out[b, 5] = clean[b, 5]
    assert torch.equal(out, clean)
    q[b, 5] = keep
    j = L - 7
    at = (int(table[b, j // rows]), 0, j % rows)
    row = K[at].clone()
    K[at] = math.nan
    out = go()
    assert bool(out[b, :H // Hkv].isnan().all())
    out[b, :H // Hkv] = clean[b, :H // Hkv]
    assert torch.equal(out, clean)
    K[at] = row
    # minus infinity: components of 1 and minus infinity
    q[b, 5] = 0.0
    q[b, 5, 0] = 1.0
    pg = table[b, :(L + rows - 1) // rows].long().to(DEV)
    old = K[pg, 1, :, 0].clone()
    K[pg, 1, :, 0] = -math.inf
    out = go()
    assert bool(out[b, 5].isnan().all())
    K[pg, 1, :, 0] = old
    K[pg[:1], 1, :, 0] = -math.inf                 # the first tile alone: the rows have no weight
    got = go()[b, 5]
    n = min(L, rows)
    v = V[pg, 1].reshape(-1, D)[n:L].double()
    s = K[pg, 1].reshape(-1, D)[n:L].double() @ q[b, 5].double() * D ** -0.5
    want = torch.softmax(s, 0) @ v
    within(got, want, HALF[dtype] * want.abs() + 2.0 ** -12 * (torch.softmax(s, 0) @ v.abs()))


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_paged_logits_that_grow_along_the_state(dtype):
    """Every tile holds a logit far beyond the ones before: the reference moves each time; and logits of any size."""
    B, H, Hkv, D, L, rows, t = 1, 8, 2, 64, 700, 16, TT[dtype]
    g = gen(8)
    K, V = randn(g, 44, Hkv, rows, D).to(t), randn(g, 44, Hkv, rows, D).to(t)
    q = randn(g, B, H, D).to(t)
    table = torch.arange(44, dtype=torch.int32)[None]
    for gain in (0.02, 1.0, 40.0):
        Kg = (K.float() * (1 + gain * torch.arange(44, device=DEV))[:, None, None, None]).to(t)
        cfg = tova.tova_paged_config(B, H, Hkv, D, 44, rows, 44, TD[dtype], 0.0)
        ws = torch.empty(max(16, tova.tova_paged_workspace_bytes(cfg, L)), dtype=torch.uint8, device=DEV)
        out = torch.empty(B, H, D, dtype=t, device=DEV)
        tova.tova_paged_attention(cfg, Kg, V, table.to(DEV), torch.tensor([L], dtype=torch.int32, device=DEV), L, q, out, ws)
        want, wv, reach = paged_reference(q, Kg, V, table, [L], rows)
        within(out, want, attention_tolerance(dtype, D, L, want, wv, reach, False))


def test_paged_offsets_beyond_32_bits():
    """A pool of more than 2^31 elements; the sequence's rows lie at its end."""
    B, H, Hkv, D, rows, pages = 1, 8, 4, 128, 16, 280000
    g = gen(4)
    K = torch.zeros(pages, Hkv, rows, D, dtype=torch.bfloat16, device=DEV)
    V = torch.zeros_like(K)
    L = 100
    table = torch.arange(pages - 1, pages - 8, -1, dtype=torch.int32)[None].contiguous()
    k, v, q = (randn(g, n, h, D).to(torch.bfloat16) for n, h in ((L, Hkv), (L, Hkv), (B, H)))
    cfg = tova.tova_paged_config(B, H, Hkv, D, pages, rows, 7, TD["bf16"], 0.0)
    tova.tova_paged_write(cfg, k, v, L, table.to(DEV), K, V, offsets=torch.tensor([0, L], dtype=torch.int32, device=DEV))
    assert torch.equal(K[pages - 1, :, 3], k[3]) and torch.equal(V[pages - 7, 3, 3], v[99, 3])
    ws = torch.empty(max(16, tova.tova_paged_workspace_bytes(cfg, L)), dtype=torch.uint8, device=DEV)
    out = torch.empty(B, H, D, dtype=torch.bfloat16, device=DEV)
    tova.tova_paged_attention(cfg, K, V, table.to(DEV), torch.tensor([L], dtype=torch.int32, device=DEV), L, q, out, ws)
    want, wv, reach = paged_reference(q, K, V, table, [L], rows)
    within(out, want, attention_tolerance("bf16", D, L, want, wv, reach, False))


@pytest.mark.parametrize("dtype, B, H, Hkv, L", [("bf16", 3, 8, 2, 30000), ("fp32", 1, 4, 4, 9000), ("bf16", 200, 32, 8, 2000)])
def test_paged_workspace_does_for_every_length_up_to_the_bound(dtype, B, H, Hkv, L):
    cfg = tova.tova_paged_config(B, H, Hkv, 128, 10, 16, (L + 15) // 16, TD[dtype], 0.0)
    need = [tova.tova_paged_workspace_bytes(cfg, n) for n in sorted({0, 1, 64, 100, 1000, L // 2, L})]
    assert need == sorted(need)


def test_paged_workspace_is_checked():
    B, H, Hkv, D, L = 8, 8, 8, 64, 20000
    cfg = tova.tova_paged_config(B, H, Hkv, D, 4, 16, 1250, TD["bf16"], 0.0)
    need = tova.tova_paged_workspace_bytes(cfg, L)
    assert need > 0
    K = torch.zeros(4, Hkv, 16, D, dtype=torch.bfloat16, device=DEV)
    table = torch.zeros(B, 1250, dtype=torch.int32, device=DEV)
    lens = torch.zeros(B, dtype=torch.int32, device=DEV)
    q = torch.zeros(B, H, D, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    for w, code in ((ws[:need - 16], -5), (None, -1)):
        with pytest.raises(tova.TovaError) as e:
            tova.tova_paged_attention(cfg, K, K, table, lens, L, q, torch.empty_like(q), w)
        assert e.value.code == code


# -------------------------------------------------------------------------------------------- packed prompts

def packed_reference(q, k, v, lens, scale=None):
    N, H, D = q.shape
    Hkv = k.shape[1]
    G = H // Hkv
    scale = scale or D ** -0.5
    out = torch.zeros(N, H, D, dtype=torch.float64, device=DEV)
    wv, reach = torch.zeros_like(out), torch.zeros(N, H, 1, dtype=torch.float64, device=DEV)
    at = 0
    for n in lens:
        if n == 0:
            continue
        later = torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1)
        for h in range(H):
            qq, kk, vv = q[at:at + n, h].double(), k[at:at + n, h // G].double(), v[at:at + n, h // G].double()
            w = torch.softmax((qq @ kk.t() * scale).masked_fill(later, -math.inf), -1)
            out[at:at + n, h], wv[at:at + n, h] = w @ vv, w @ vv.abs()
            reach[at:at + n, h] = (qq.abs() @ kk.abs().t() * scale).masked_fill(later, 0.0).amax(-1, keepdim=True)
        at += n
    return out, wv, reach


def offsets_of(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=DEV)


def run_packed(dtype, H, Hkv, D, lens, seed=0, sm_scale=0.0, gain=1.3, pad=3, grow=0.0):
    g, t, N = gen(seed + D), TT[dtype], sum(lens)
    q = (randn(g, N + pad, H * D + 64) * gain).to(t)[:, :H * D].unflatten(-1, (H, D))
    k = randn(g, N + pad, Hkv, D)
    if grow:
        k = k * (1 + grow * torch.arange(N + pad, device=DEV)[:, None, None])
    k = k.to(t)
    v = randn(g, N + pad, (H + 2 * Hkv) * D).to(t)[:, (H + Hkv) * D:].unflatten(-1, (Hkv, D))
    if pad:                                        # rows that belong to no sequence may hold anything
        q[N:] = k[N:] = math.nan
        v[N:] = math.inf
    cfg = tova.tova_packed_config(len(lens), H, Hkv, D, TD[dtype], sm_scale)
    need = tova.tova_packed_workspace_bytes(cfg, N + pad)
    ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full((N + pad, H, D), 77.0, dtype=t, device=DEV)
    off = offsets_of(lens)
    tova.tova_packed_attention(cfg, q, k, v, N + pad, off, out, ws[:need])
    want, wv, reach = packed_reference(q[:N], k[:N], v[:N], lens, sm_scale or None)
    within(out[:N], want, attention_tolerance(dtype, D, max(lens), want, wv, reach, True))
    assert bool((out[N:] == 77.0).all()) and bool((ws[need:] == 0xff).all())
    first = out.clone()
    tova.tova_packed_attention(cfg, q, k, v, N + pad, off, out, ws[:need])
    assert torch.equal(first, out)


PACKED = [
    # H, Hkv, lens
    (4, 4, [1]), (8, 2, [1, 1, 1]), (8, 2, [63, 64, 65, 0, 1]), (6, 2, [127, 128, 129]), (32, 8, [200, 7]), (4, 1, [300]), (5, 5, [257, 255, 256]),
    (2, 2, [1000, 333]), (9, 3, [0, 0, 40, 0]), (8, 4, [640, 383, 385]), (3, 1, [5] * 90), (2, 1, [2100]),
]


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", PACKED, ids=lambda s: f"H{s[0]}x{s[1]}S{len(s[2])}L{max(s[2])}")
def test_packed_attention(dtype, D, shape):
    H, Hkv, lens = shape
    run_packed(dtype, H, Hkv, D, lens)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_packed_attention_scale_and_logits_of_any_size(dtype):
    run_packed(dtype, 4, 2, 128, [130, 400], sm_scale=0.5)
    run_packed(dtype, 4, 2, 64, [700, 3], grow=0.05)            # every tile's logits beyond the ones before
    run_packed(dtype, 4, 2, 128, [700, 3], grow=1.0)
    run_packed(dtype, 4, 2, 128, [260], gain=30.0)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H, Hkv, lens", [(32, 32, [1] * 40 + [114, 5]), (32, 32, [3] * 28), (9, 3, [100] * 200), (32, 32, [129, 1, 128, 300, 2] * 9)])
def test_packed_many_items_a_block_some_without_a_second_tile(D, H, Hkv, lens):
    run_packed("bf16", H, Hkv, D, lens)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_packed_attention_many_sequences(dtype):
    run_packed(dtype, 4, 2, 64, [(7 * i) % 40 for i in range(2000)])
    run_packed(dtype, 4, 2, 64, [0] * 3000 + [9, 0, 70] + [0] * 2000, pad=0)      # nearly all of them empty
    run_packed(dtype, 2, 2, 128, [0] * 200 + [130] + [0] * 50)


def test_packed_offsets_that_are_not_rising_or_lie_outside():
    H, Hkv, D, N = 4, 2, 64, 500
    for dtype in ("bf16", "fp32"):
        g, t = gen(2), TT[dtype]
        q, k, v = randn(g, N, H, D).to(t), randn(g, N, Hkv, D).to(t), randn(g, N, Hkv, D).to(t)
        off = torch.tensor([-4, 100, 90, 300, 2 ** 31 - 1], dtype=torch.int32, device=DEV)     # 0..100, none, 90..300, 300..500
        cfg = tova.tova_packed_config(4, H, Hkv, D, TD[dtype], 0.0)
        ws = torch.empty(max(16, tova.tova_packed_workspace_bytes(cfg, N)), dtype=torch.uint8, device=DEV)
        out = torch.full((N, H, D), 77.0, dtype=t, device=DEV)
        tova.tova_packed_attention(cfg, q, k, v, N, off, out, ws)
        for a, b in ((0, 90), (100, 300), (300, 500)):           # (90..99 belong to two sequences: either's)
            s = {0: 0, 100: 90, 300: 300}[a]
            want, wv, reach = packed_reference(q[s:b], k[s:b], v[s:b], [b - s])
            tol = attention_tolerance(dtype, D, b - s, want, wv, reach, True)
            within(out[a:b], want[a - s:], tol[a - s:])


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H, Hkv", [(2, 1), (2, 2), (3, 1)])
@pytest.mark.parametrize("L, at", [(300, 150), (300, 299), (130, 64), (600, 255), (600, 256), (600, 130)])
def test_packed_values_that_are_not_numbers_reach_only_later_tokens(dtype, D, H, Hkv, L, at):
    """A token whose key or value is not finite: earlier tokens, and other sequences, keep their bits; later tokens of its
    sequence get its infinity (value) or NaN (key)."""
    g, t, lens = gen(L + at), TT[dtype], [77, L, 50]
    N = sum(lens)
    q, k, v = randn(g, N, H, D).to(t), randn(g, N, Hkv, D).to(t), randn(g, N, Hkv, D).to(t)
    off, x = offsets_of(lens), 77 + at
    cfg = tova.tova_packed_config(3, H, Hkv, D, TD[dtype], 0.0)
    ws = torch.empty(max(16, tova.tova_packed_workspace_bytes(cfg, N)), dtype=torch.uint8, device=DEV)

    def go():
        out = torch.full((N, H, D), 77.0, dtype=t, device=DEV)
        tova.tova_packed_attention(cfg, q, k, v, N, off, out, ws)
        return out
    clean = go()
    hk, G = Hkv - 1, H // Hkv
    mine = slice(hk * G, H)                        # the query heads that read this KV head
    unseen = torch.ones(N, H, dtype=torch.bool, device=DEV)
    unseen[x:77 + L, mine] = False
    for bad, seen in ((math.inf, lambda o: o == math.inf), (-math.inf, lambda o: o == -math.inf), (math.nan, torch.isnan)):
        keep = v[x, hk, 5].clone()
        v[x, hk, 5] = bad
        out = go()
        v[x, hk, 5] = keep
        assert torch.equal(out[unseen], clean[unseen])
        got = out[x:77 + L, mine]
        assert bool(seen(got[..., 5]).all())
        got[..., 5] = clean[x:77 + L, mine, 5]
        assert torch.equal(got, clean[x:77 + L, mine])           # the other components
    keep = k[x, hk].clone()
    k[x, hk, 3] = math.nan
    out = go()
    assert torch.equal(out[unseen], clean[unseen]) and bool(out[x:77 + L, mine].isnan().all())
    k[x, hk] = keep
    keep = q[x, H - 1].clone()
    q[x, H - 1, 1] = math.nan
    out = go()
    assert bool(out[x, H - 1].isnan().all())
    out[x, H - 1] = clean[x, H - 1]
    assert torch.equal(out, clean)
    # all logits minus infinity: NaN for the rows that see nothing else
    q[x, H - 1] = 0.0
    q[x, H - 1, 1] = 1.0
    k[77:x + 1, hk, 1] = -math.inf
    assert bool(go()[x, H - 1].isnan().all())


def test_packed_offsets_beyond_32_bits():
    """Rows of a projection so wide that the last token's lie more than 2^31 elements in."""
    H, Hkv, D, N, wide = 2, 1, 64, 600, 4 * 1024 * 1024
    g = gen(6)
    x = torch.zeros(N, wide, dtype=torch.bfloat16, device=DEV)
    q, k, v = x[:, :H * D].unflatten(-1, (H, D)), x[:, 128:192].unflatten(-1, (1, D)), x[:, 192:256].unflatten(-1, (1, D))
    for y in (q, k, v):
        y.copy_(randn(g, *y.shape))
    cfg = tova.tova_packed_config(1, H, Hkv, D, TD["bf16"], 0.0)
    ws = torch.empty(max(16, tova.tova_packed_workspace_bytes(cfg, N)), dtype=torch.uint8, device=DEV)
    out = torch.empty(N, H, D, dtype=torch.bfloat16, device=DEV)
    tova.tova_packed_attention(cfg, q, k, v, N, offsets_of([N]), out, ws)
    want, wv, reach = packed_reference(q, k, v, [N])
    within(out, want, attention_tolerance("bf16", D, N, want, wv, reach, True))


def test_packed_workspace_is_checked():
    cfg = tova.tova_packed_config(4, 32, 8, 128, TD["bf16"], 0.0)
    N = 5000
    need = tova.tova_packed_workspace_bytes(cfg, N)
    assert need > 0
    q, k = torch.zeros(N, 32, 128, dtype=torch.bfloat16, device=DEV), torch.zeros(N, 8, 128, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(need, dtype=torch.uint8, device=DEV)
    for w, code in ((ws[:need - 16], -5), (None, -1)):
        with pytest.raises(tova.TovaError) as e:
            tova.tova_packed_attention(cfg, q, k, k, N, offsets_of([N, 0, 0, 0]), torch.empty_like(q), w)
        assert e.value.code == code


# ------------------------------------------------------------------------------------------- log probabilities

def run_logprobs(x, tok, top, dtype, row_stride=0, with_entropy=True):
    T, V = tok.shape[0], x.shape[1]
    cfg = tova.tova_logprobs_config(V, TD[dtype], top, row_stride)
    flat = x
    if row_stride:
        flat = torch.full((T, row_stride), 1e30, dtype=TT[dtype], device=DEV)      # what lies between rows is not looked at
        flat[:, :V] = x
    lp = torch.full((T,), 7.0, device=DEV)
    ent = torch.full((T,), 7.0, device=DEV) if with_entropy else None
    ids = torch.full((T, top), -7, dtype=torch.int32, device=DEV) if top else None
    tlp = torch.full((T, top), 7.0, device=DEV) if top else None
    tova.tova_token_logprobs(cfg, flat, T, tok, lp, ent, ids, tlp)
    return lp, ent, ids, tlp


def check_logprobs(x, tok, got, top, dtype):
    """d = x - m is rounded once (2^-24 |d|), so is its product with log2 e, exp2 adds 2^-22; terms with d beyond -100 are
    nothing.  A thread's chain has at most V / 512 + 40 terms, the joins 16 + 8 more.  So S is off by (V/512 + 400) 2^-24
    relative (|d| <= 100: 200 for the exponents of what counts at all), E by the same of sum w |d|.  log: 2^-22."""
    lp, ent, ids, tlp = got
    xd = x.double()
    V = x.shape[1]
    y = xd - torch.logsumexp(xd, -1, keepdim=True)
    rel = (V / 512 + 400) * U
    want = y.gather(1, tok.long().clamp(0, V - 1)[:, None])[:, 0]
    ok = (tok >= 0) & (tok < V)
    tol = rel + 4 * U * (want.abs() + xd.abs().amax(-1)) + 2.0 ** -22 * math.log(V + 1)
    fin = ok & torch.isfinite(want)
    within(lp[fin], want[fin], tol[fin])
    assert bool((lp[~fin] == -math.inf).all())
    p = torch.exp(y)
    if ent is not None:
        h = -(p * torch.where(p > 0, y, torch.zeros_like(y))).sum(-1)
        size = (p * torch.where(p > 0, y, torch.zeros_like(y)).abs()).sum(-1)
        within(ent, h, 2 * rel * (1 + size) + 8 * U * xd[xd.isfinite()].abs().max() + 2.0 ** -21 * math.log(V + 1))
    if top:
        order = torch.sort(x.float() + 0.0, dim=-1, descending=True, stable=True)[1][:, :top]
        assert torch.equal(ids.long(), order), (ids.long() != order).nonzero()[:3].tolist()
        wt = y.gather(1, order)
        m = torch.isfinite(wt)
        within(tlp[m], wt[m], (rel + 4 * U * (wt.abs() + xd[xd.isfinite()].abs().max()) + 2.0 ** -22 * math.log(V + 1))[m])
        assert bool((tlp[~m] == -math.inf).all())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("T, V, top", [(1, 1, 1), (3, 2, 2), (5, 31, 31), (2, 100, 32), (7, 1000, 0), (4, 4095, 20), (1, 32000, 20), (9, 4097, 5),
                                       (200, 32001, 5), (75, 5000, 32), (3, 128256, 20), (300, 50257, 1), (1, 1000003, 32)])
def test_logprobs(dtype, T, V, top):
    g = gen(T + V)
    x = (randn(g, T, V) * 2.5).to(TT[dtype])
    tok = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
    tok[-1] = V - 1
    check_logprobs(x, tok, run_logprobs(x, tok, top, dtype), top, dtype)
    if T > 1 and V < 50000:
        check_logprobs(x, tok, run_logprobs(x, tok, top, dtype, row_stride=V + 3, with_entropy=T % 2 == 0), top, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [50, 3001, 40001])
@pytest.mark.parametrize("T", [2, 90])
def test_logprobs_ties_and_orders(dtype, V, T):
    """Rows of equal logits, of few different ones, rising, falling, with the largest in one thread's share, zeros of both
    signs, tokens outside."""
    g, t = gen(V), TT[dtype]
    n = torch.arange(V, device=DEV).float()
    rows = [torch.zeros(V, device=DEV), torch.full((V,), -3.0, device=DEV), torch.randint(0, 3, (V,), generator=g, device=DEV).float(), n / V, -n / V,
            torch.where(n % 4096 < 8, 5.0 + n / V, torch.zeros_like(n)), torch.where(n % 2 == 0, torch.zeros_like(n), -torch.zeros_like(n)),
            torch.where(n == V - 1, torch.full_like(n, 60.0), -n / 100), torch.where(n % 7 == 3, n * 0 + 1, n * 0 - math.inf)]
    x = torch.stack([rows[i % len(rows)] for i in range(max(T, len(rows)))]).to(t)
    tok = torch.tensor([[-1, V, 0, 3 % V, V - 1, 2 ** 31 - 1, -2 ** 31][i % 7] for i in range(x.shape[0])], dtype=torch.int32, device=DEV)
    for top in (1, 7, 32):
        check_logprobs(x, tok, run_logprobs(x, tok, top, dtype), top, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("V", [900, 9000])
def test_logprobs_rows_that_are_not_finite(dtype, V):
    g = gen(V)
    x = (randn(g, 5, V) * 2).to(TT[dtype])
    x[0, 17] = math.nan
    x[1, 5] = math.inf
    x[2] = -math.inf
    x[3, 3::2] = -math.inf
    x[3, 1] = -math.inf
    tok = torch.tensor([3, 5, 2, 7, 1], dtype=torch.int32, device=DEV)
    lp, ent, ids, tlp = run_logprobs(x, tok, 6, dtype)
    for i in range(3):
        assert bool(lp[i].isnan()) and bool(ent[i].isnan())
    assert torch.equal(ids.long(), torch.sort(x.float(), dim=-1, descending=True, stable=True)[1][:, :6])
    check_logprobs(x[3:], tok[3:], tuple(y[3:] for y in (lp, ent, ids, tlp)), 6, dtype)
    assert float(lp[3]) == -math.inf


def test_logprobs_offsets_beyond_32_bits():
    T, V, ld = 3, 1000, 1 << 30
    x = torch.zeros(2 * ld + V, dtype=torch.bfloat16, device=DEV)
    g = gen(1)
    rows = (randn(g, T, V) * 2).to(torch.bfloat16)
    for i in range(T):
        x[i * ld:i * ld + V] = rows[i]
    tok = torch.tensor([1, 999, 5], dtype=torch.int32, device=DEV)
    cfg = tova.tova_logprobs_config(V, TD["bf16"], 3, ld)
    lp, ent, ids, tlp = torch.empty(T, device=DEV), torch.empty(T, device=DEV), torch.empty(T, 3, dtype=torch.int32, device=DEV), torch.empty(T, 3, device=DEV)
    tova.tova_token_logprobs(cfg, x, T, tok, lp, ent, ids, tlp)
    check_logprobs(rows, tok, (lp, ent, ids, tlp), 3, "bf16")


# ------------------------------------------------------------------------------------------------ all together

def test_serving_prompts_and_new_tokens_over_pages():
    """Three prompts of different lengths through one layer and on, token by token: what the pages answer is what the packed
    attention of the whole texts gives, and the probabilities of the chosen tokens add up to the texts'."""
    H, Hkv, D, V, rows, dt = 8, 2, 64, 500, 16, torch.bfloat16
    lens, new = [37, 1, 80], 20
    S, width = len(lens), (H + 2 * Hkv) * D
    g = gen(12)
    embed, wqkv, wout = randn(g, V, 96).to(dt), (randn(g, 96, width) / 10).to(dt), (randn(g, H * D, V) / 20).to(dt)
    qw, kw = (1 + 0.1 * randn(g, D)).to(dt), (1 + 0.1 * randn(g, D)).to(dt)
    texts = [torch.randint(0, V, (n + new,), generator=g, device=DEV) for n in lens]
    table, pages = make_table([n + new for n in lens], rows, 5)
    table = table.to(DEV)
    K, V_ = torch.full((pages, Hkv, rows, D), math.nan, dtype=dt, device=DEV), torch.full((pages, Hkv, rows, D), math.nan, dtype=dt, device=DEV)

    def project(ids, pos):                         # packed tokens -> normed, rotated q and k, and v as it lies
        n = ids.shape[0]
        x = embed[ids] @ wqkv
        q, k = x[:, None, :H * D].unflatten(-1, (H, D)), x[:, None, H * D:(H + Hkv) * D].unflatten(-1, (Hkv, D))
        rope = tova.TovaRope(1, H, Hkv, D)
        qo, ko = torch.empty(n, 1, H, D, dtype=dt, device=DEV), torch.empty(n, 1, Hkv, D, dtype=dt, device=DEV)
        rope.tova_norm_rope_apply(q, k, n, qo, ko, q_weight=qw, k_weight=kw, positions=pos.to(torch.int32))
        return qo[:, 0], ko[:, 0], x[:, (H + Hkv) * D:].unflatten(-1, (Hkv, D))

    def packed(ids):
        off = offsets_of([t.shape[0] for t in ids])
        n = int(off[-1])
        q, k, v = project(torch.cat(ids), torch.cat([torch.arange(t.shape[0], device=DEV) for t in ids]))
        cfg = tova.tova_packed_config(S, H, Hkv, D, TD["bf16"], 0.0)
        ws = torch.empty(max(16, tova.tova_packed_workspace_bytes(cfg, n)), dtype=torch.uint8, device=DEV)
        out = torch.empty(n, H, D, dtype=dt, device=DEV)
        tova.tova_packed_attention(cfg, q, k, v, n, off, out, ws)
        return out, k, v, off

    def logprobs(out, tok):
        n = out.shape[0]
        cfg = tova.tova_logprobs_config(V, TD["bf16"], 0, 0)
        lp = torch.empty(n, device=DEV)
        tova.tova_token_logprobs(cfg, (out.flatten(1) @ wout).contiguous(), n, tok.to(torch.int32), lp)
        return lp
    whole, _, _, _ = packed(texts)
    pcfg = tova.tova_paged_config(S, H, Hkv, D, pages, rows, table.shape[1], TD["bf16"], 0.0)
    out, k, v, off = packed([t[:n] for t, n in zip(texts, lens)])
    tova.tova_paged_write(pcfg, k, v, k.shape[0], table, K, V_, offsets=off)
    held = torch.tensor(lens, dtype=torch.int32, device=DEV)
    most = max(lens) + new
    ws = torch.empty(max(16, tova.tova_paged_workspace_bytes(pcfg, most)), dtype=torch.uint8, device=DEV)
    starts = [0]
    for t in texts:
        starts.append(starts[-1] + t.shape[0])
    total = 0.0
    want_total = 0.0
    for i in range(new - 1):
        ids = torch.stack([t[n + i] for t, n in zip(texts, lens)])
        q, k, v = project(ids, held)
        tova.tova_paged_write(pcfg, k, v, S, table, K, V_, first_rows=held)
        held += 1
        o = torch.empty(S, H, D, dtype=dt, device=DEV)
        tova.tova_paged_attention(pcfg, K, V_, table, held, most, q, o, ws)
        rows_ = torch.tensor([starts[b] + lens[b] + i for b in range(S)], device=DEV)
        same = whole[rows_]
        # two roundings to bf16 of the same sums, and the packed kernel's weights (2^-8 of sum p|v|, here at most max |v|)
        tol = 2 * 2.0 ** -8 * same.double().abs() + 2.0 ** -8 * v.float().abs().max().double() * 4
        assert bool(((o.double() - same.double()).abs() <= tol).all())
        nxt = torch.stack([t[n + i + 1] for t, n in zip(texts, lens)])
        total += float(logprobs(o, nxt).sum())
        want_total += float(torch.log_softmax((o.flatten(1) @ wout).double(), -1).gather(1, nxt[:, None]).sum())
    assert abs(total - want_total) <= 1e-4 * (new - 1) * S


def serve_state(seed, dtype="bf16"):
    B, H, Hkv, D, rows, V = 3, 8, 2, 64, 16, 5000
    g, t = gen(seed), TT[dtype]
    lens = [700, 5, 3000]
    table, pages = make_table([n + 1 for n in lens], rows, seed)
    s = dict(q=randn(g, B, 1, H, D).to(t), k=randn(g, B, 1, Hkv, D).to(t), v=randn(g, B, Hkv, D).to(t), K=randn(g, pages, Hkv, rows, D).to(t),
             V=randn(g, pages, Hkv, rows, D).to(t), table=table.to(DEV), held=torch.tensor(lens, dtype=torch.int32, device=DEV),
             x=(randn(g, B, V) * 2).to(t), tok=torch.randint(0, V, (B,), generator=g, device=DEV, dtype=torch.int32),
             pq=randn(g, 400, H, D).to(t), pk=randn(g, 400, Hkv, D).to(t), off=offsets_of([150, 0, 249]), gy=randn(g, B, 1, H, D).to(t))
    s["lens"] = s["held"] + 1
    cfg = tova.tova_paged_config(B, H, Hkv, D, pages, rows, table.shape[1], TD[dtype], 0.0)
    pc, lc = tova.tova_packed_config(3, H, Hkv, D, TD[dtype], 0.0), tova.tova_logprobs_config(V, TD[dtype], 4, 0)
    rope = tova.TovaRope(1, H, Hkv, D, dtype=TD[dtype])
    s.update(qo=torch.zeros_like(s["q"]), ko=torch.zeros_like(s["k"]), out=torch.zeros(B, H, D, dtype=t, device=DEV),
             pout=torch.zeros(400, H, D, dtype=t, device=DEV), lp=torch.zeros(B, device=DEV), ent=torch.zeros(B, device=DEV),
             ids=torch.zeros(B, 4, dtype=torch.int32, device=DEV), tlp=torch.zeros(B, 4, device=DEV), dq=torch.zeros_like(s["q"]),
             dqw=torch.zeros(D, device=DEV))
    s["ws"] = [torch.empty(max(16, n), dtype=torch.uint8, device=DEV) for n in
               (tova.tova_paged_workspace_bytes(cfg, 3001), tova.tova_packed_workspace_bytes(pc, 400), rope.tova_norm_rope_workspace_bytes(B))]

    def go(stream=None):
        rope.tova_norm_rope_apply(s["q"], s["k"], B, s["qo"], s["ko"], first_pos=9, stream=stream)
        tova.tova_paged_write(cfg, s["ko"][:, 0], s["v"], B, s["table"], s["K"], s["V"], first_rows=s["held"], stream=stream)
        tova.tova_paged_attention(cfg, s["K"], s["V"], s["table"], s["lens"], 3001, s["qo"][:, 0], s["out"], s["ws"][0], stream=stream)
        tova.tova_packed_attention(pc, s["pq"], s["pk"], s["pk"], 400, s["off"], s["pout"], s["ws"][1], stream=stream)
        tova.tova_token_logprobs(lc, s["x"], B, s["tok"], s["lp"], s["ent"], s["ids"], s["tlp"], stream=stream)
        rope.tova_norm_rope_backward(s["q"], None, s["gy"], None, B, s["dq"], None, s["ws"][2], dq_weight=s["dqw"], first_pos=9, stream=stream)
    return s, go, ("qo", "ko", "K", "V", "out", "pout", "lp", "ent", "ids", "tlp", "dq", "dqw")


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_serving_operators_in_captured_graphs_and_on_other_streams(dtype):
    """Captured once and replayed on new inputs, lengths and offsets; two graphs with workspaces of their own at once on two
    streams; the same bits as calls on a stream given explicitly."""
    runs = [serve_state(seed, dtype) for seed in (1, 2)]
    graphs = []
    for s, go, names in runs:
        go()                                       # (first calls set kernels' attributes)
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            go()
        graphs.append(gr)
    for s, _, _ in runs:                           # other inputs than at capture
        s["q"].mul_(0.5)
        s["pk"].mul_(1.5)
        s["held"].sub_(3)
        s["lens"].sub_(3)
        s["off"].copy_(offsets_of([3, 390, 2]))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    got = [{x: s[x].clone() for x in names} for s, _, names in runs]
    for (s, go, names), seen, st in zip(runs, got, streams):
        for x in names:
            if x not in ("K", "V"):
                s[x].zero_()
        st.wait_stream(torch.cuda.current_stream())
        go(st)
        st.synchronize()
        assert all(torch.equal(s[x], seen[x]) for x in names if x != "pout")
        assert torch.equal(s["pout"][:395], seen["pout"][:395])
