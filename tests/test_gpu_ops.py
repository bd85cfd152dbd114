"""GPU tests of the operators around the decode step, against their definitions in 64 bits.

Tolerances.  A rounding to type t is off by at most half a step, eps(t)/2 relative (bf16 2^-8, fp32 2^-24).  Sums of n
fp32 products are off by at most about n 2^-24 of the sum of the products' sizes, twice that on the tensor cores, whose
adders may truncate."""
import ctypes
import math

import pytest
import torch

import paper_2401_06104_b200 as tova
from paper_2401_06104_b200 import workloads as W

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TT = {"bf16": torch.bfloat16, "fp32": torch.float32}
TD = {"bf16": tova.TOVA_DTYPE_BF16, "fp32": tova.TOVA_DTYPE_FP32}
HALF = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
FMT = {"plain": tova.TOVA_FORMAT_PLAIN, "int8": tova.TOVA_FORMAT_INT8, "e4m3": tova.TOVA_FORMAT_E4M3}


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV)


# ------------------------------------------------------------------------------------------------ rotary positions

def frequencies(rot, base, scaling, factor, orig):
    i = torch.arange(rot // 2, dtype=torch.float64)
    if scaling == tova.TOVA_ROPE_NTK:
        base = base * factor ** (rot / (rot - 2))
    w = base ** (-2.0 * i / rot)
    m = 1.0
    if scaling == tova.TOVA_ROPE_LINEAR:
        w = w / factor
    elif scaling == tova.TOVA_ROPE_YARN:
        lo = max(math.floor(rot * math.log(orig / (32 * 2 * math.pi)) / (2 * math.log(base))), 0)
        hi = min(math.ceil(rot * math.log(orig / (1 * 2 * math.pi)) / (2 * math.log(base))), rot - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        w = w / factor * ramp + w * (1 - ramp)
        m = 0.1 * math.log(factor) + 1
    elif scaling == tova.TOVA_ROPE_BANDS:
        s = ((orig * w / (2 * math.pi) - 1) / 3).clamp(0, 1)
        w = (1 - s) * w / factor + s * w
    return w.to(DEV), m


def rope_reference(x, pos, w, m, rot, layout, inverse=False):
    """x [T,B,heads,D] in double, pos [T,B]: pairs as complex numbers.  Also the size that roundings scale with."""
    x = x.double()
    ang = pos.double()[..., None] * w * (-1.0 if inverse else 1.0)
    z = torch.polar(torch.full_like(ang, m), ang)[:, :, None]
    y, size = x.clone(), x.abs()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == tova.TOVA_ROPE_HALF else (slice(0, rot, 2), slice(1, rot, 2))
    t = torch.complex(x[..., a].contiguous(), x[..., b].contiguous()) * z
    y[..., a], y[..., b] = t.real, t.imag
    both = m * (x[..., a].abs() + x[..., b].abs())
    size[..., a], size[..., b] = both, both
    return y, size


def check_rope(got, want, size, dtype):
    # angle: a turn rounded to fp32 (2^-25 of a half turn, times pi) and sincospi's own 2^-23 or so; two products and a
    # sum; the result's rounding
    tol = HALF[dtype] * want.abs() + 8 * 2.0 ** -24 * size + 1e-38
    assert bool(((got.double() - want).abs() <= tol).all()), float(((got.double() - want).abs() - tol).max())


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("layout", [tova.TOVA_ROPE_HALF, tova.TOVA_ROPE_INTERLEAVED])
@pytest.mark.parametrize("D, rot", [(128, 128), (128, 96), (128, 2), (128, 20), (64, 64), (64, 32), (64, 62)])
def test_rope_layouts_and_parts(dtype, layout, D, rot):
    g = gen(rot + D)
    T, B, H, Hkv = 5, 3, 8, 2
    q, k = randn(g, T, B, H, D).to(TT[dtype]), randn(g, T, B, Hkv, D).to(TT[dtype])
    pos = torch.randint(0, 2 ** 31 - 1, (T, B), generator=g, device=DEV, dtype=torch.int32)
    pos[0, 0], pos[1, 1], pos[2, 2] = 0, 2 ** 31 - 1, -5
    r = tova.TovaRope(B, H, Hkv, D, dtype=TD[dtype], rotary_dim=rot, layout=layout)
    w, m = frequencies(rot, 10000.0, 0, 1.0, 0)
    for inverse in (False, True):
        qo, ko = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
        r.tova_rope_apply(q, k, T, qo, ko, positions=pos, inverse=inverse)
        for x, y in ((q, qo), (k, ko)):
            check_rope(y, *rope_reference(x, pos, w, m, rot, layout, inverse), dtype)


@pytest.mark.parametrize("scaling", [tova.TOVA_ROPE_LINEAR, tova.TOVA_ROPE_NTK, tova.TOVA_ROPE_YARN, tova.TOVA_ROPE_BANDS])
def test_rope_scalings(scaling):
    g = gen(scaling)
    T, B, H, Hkv, D = 700, 2, 4, 4, 128
    q, k = randn(g, T, B, H, D), randn(g, T, B, Hkv, D)
    r = tova.TovaRope(B, H, Hkv, D, dtype=tova.TOVA_DTYPE_FP32, base=500000.0, scaling=scaling, factor=8.0, original_context=4096)
    w, m = frequencies(D, 500000.0, scaling, 8.0, 4096)
    first = 31000
    pos = first + torch.arange(T, device=DEV)[:, None].expand(T, B)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    r.tova_rope_apply(q, k, T, qo, ko, first_pos=first)
    check_rope(qo, *rope_reference(q, pos, w, m, D, 0), "fp32")
    check_rope(ko, *rope_reference(k, pos, w, m, D, 0), "fp32")


def test_rope_amplitude_strides_in_place_and_no_keys():
    g = gen(3)
    T, B, H, Hkv, D = 9, 2, 8, 2, 64
    qkv = randn(g, T, B, (H + 2 * Hkv) * D).to(torch.bfloat16)
    keep = qkv.clone()
    q, k = qkv[..., :H * D].unflatten(-1, (H, D)), qkv[..., H * D:(H + Hkv) * D].unflatten(-1, (Hkv, D))
    r = tova.TovaRope(B, H, Hkv, D, amplitude=0.5)
    w, _ = frequencies(D, 10000.0, 0, 1.0, 0)
    pos = 11 + torch.arange(T, device=DEV)[:, None].expand(T, B)
    want = [rope_reference(x.clone(), pos, w, 0.5, D, 0) for x in (q, k)]
    only = torch.empty(T, B, H, D, dtype=torch.bfloat16, device=DEV)
    r.tova_rope_apply(q, None, T, only, None, first_pos=11)
    check_rope(only, *want[0], "bf16")
    assert torch.equal(qkv, keep)
    r.tova_rope_apply(q, k, T, q, k, first_pos=11)         # in place, as slices of the projection
    check_rope(q, *want[0], "bf16")
    check_rope(k, *want[1], "bf16")
    assert torch.equal(qkv[..., (H + Hkv) * D:], keep[..., (H + Hkv) * D:])       # the values between stay as they were
    r.tova_rope_apply(q, k, 0, q, k)                       # no tokens: nothing happens
    check_rope(q, *want[0], "bf16")


def test_rope_inverse_is_the_gradient():
    """loss = <w, rope(x)>: the gradient is the inverse applied to w, by the formula and by differences (the map is
    linear, so a difference of any size is exact up to rounding)."""
    g = gen(4)
    T, B, H, D = 3, 2, 2, 64
    x, w = randn(g, T, B, H, D), randn(g, T, B, H, D)
    r = tova.TovaRope(B, H, H, D, dtype=tova.TOVA_DTYPE_FP32, rotary_dim=32, layout=tova.TOVA_ROPE_INTERLEAVED,
                      scaling=tova.TOVA_ROPE_YARN, factor=4.0, original_context=100)
    grad, y0, y1 = torch.empty_like(x), torch.empty_like(x), torch.empty_like(x)
    r.tova_rope_apply(w, None, T, grad, None, first_pos=77, inverse=True)
    r.tova_rope_apply(x, None, T, y0, None, first_pos=77)
    for at in ((0, 0, 0, 0), (1, 1, 1, 31), (2, 0, 1, 32), (2, 1, 0, 63), (0, 1, 0, 17)):
        x1 = x.clone()
        x1[at] += 1.0
        r.tova_rope_apply(x1, None, T, y1, None, first_pos=77)
        diff = float(((y1.double() - y0.double()) * w.double()).sum())
        # two outputs of size <= 2 m max|x| change; each is off by 8 2^-24 of its size in both evaluations
        tol = 2 * 2 * 8 * 2.0 ** -24 * 2 * 1.2 * float(x1.abs().max()) * float(w.abs().max()) + 8 * 2.0 ** -24 * 2.5 * float(w.abs().max())
        assert abs(diff - float(grad[at])) <= tol, (at, diff, float(grad[at]), tol)


# ------------------------------------------------------------------------------------------------ the 8-bit state

def quantise(x, fmt):
    """Codes as floats and scales, from the definition: the fp32 roundings through 64 bits."""
    qmax = 127.0 if fmt == "int8" else 448.0
    x = x.double()
    a = x.abs().amax(-1)
    good = torch.isfinite(a) & (a >= 2.0 ** -100)
    top = torch.full_like(a, qmax)
    one = torch.ones_like(a)
    scale = torch.where(good, (torch.where(good, a, one) / top).float(), torch.zeros_like(a, dtype=torch.float32))
    scale = torch.where(torch.isfinite(a), scale, torch.full_like(scale, math.nan))
    r = torch.where(good, (top / torch.where(good, a, one)).float(), torch.zeros_like(scale))
    y = torch.where(good[..., None], (x * r.double()[..., None]).float(), torch.zeros_like(x, dtype=torch.float32))
    code = torch.round(y) if fmt == "int8" else y.clamp(-448, 448).to(torch.float8_e4m3fn).float()
    return code, scale


def codes_as_floats(c, fmt):
    return c.float() if fmt == "int8" else c.view(torch.float8_e4m3fn).float()


def new_state(B, Hkv, cap, D, fmt):
    codes = [torch.full((B, Hkv, cap, D), 3, dtype=torch.int8, device=DEV) for _ in range(2)]
    scales = [torch.full((B, Hkv, cap), 0.25, device=DEV) for _ in range(2)]
    return codes, scales


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("T, B, Hkv, cap, listed", [(1, 1, 1, 1, False), (1, 5, 4, 37, True), (77, 3, 2, 101, True), (300, 1, 8, 300, False)])
def test_quant_write_and_read(fmt, dtype, D, T, B, Hkv, cap, listed):
    g = gen(T + D)
    k, v = (randn(g, T, B, Hkv, D).to(TT[dtype]) for _ in range(2))
    codes, scales = new_state(B, Hkv, cap, D, fmt)
    first = cap - T
    slots = torch.argsort(torch.rand(B, cap, generator=g, device=DEV), 1)[:, :T].t().to(torch.int32).contiguous() if listed else None
    cfg = tova.tova_quant_config(B, Hkv, D, cap, TD[dtype], FMT[fmt])
    tova.tova_quant_write(cfg, k, v, T, codes[0], scales[0], codes[1], scales[1], slots=slots, first_slot=0 if listed else first)
    at = slots.long() if listed else (first + torch.arange(T, device=DEV))[:, None].expand(T, B)
    b = torch.arange(B, device=DEV)[None].expand(T, B)
    back = [torch.empty(T, B, Hkv, D, dtype=TT[dtype], device=DEV) for _ in range(2)]
    tova.tova_quant_read(cfg, codes[0], scales[0], codes[1], scales[1], T, back[0], back[1], slots=slots, first_slot=0 if listed else first)
    for x, c, s, y in zip((k, v), codes, scales, back):
        code, scale = quantise(x, fmt)
        assert torch.equal(codes_as_floats(c, fmt)[b, :, at], code)
        assert torch.equal(s[b, :, at], scale)
        assert torch.equal(y, (code * scale[..., None]).to(TT[dtype]))
        hit = torch.zeros(B, cap, dtype=torch.bool, device=DEV)
        hit[b, at] = True
        assert bool((c.permute(0, 2, 1, 3)[~hit] == 3).all()) and bool((s.permute(0, 2, 1)[~hit] == 0.25).all())


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_quant_rows_at_the_edges(fmt):
    """Zeros, the smallest and largest values, ties, infinities and NaN."""
    D, B, Hkv = 64, 1, 1
    rows = torch.zeros(12, D)
    rows[1, 3] = 2.0 ** -149                                   # the smallest number: stored as zero
    rows[2] = 2.0 ** -101
    rows[3] = 2.0 ** -100
    rows[4] = torch.linspace(-1, 1, D) * 3e38
    rows[5, 7] = math.inf
    rows[6, 8] = -math.inf
    rows[7, 9] = math.nan
    rows[8] = (torch.arange(D) - 31.5) * 2 + 0.0               # with 127 on top: scale 1, every value a tie
    rows[8, 0] = 127.0
    rows[9] = torch.where(torch.arange(D) % 2 == 0, 448.0, 17.0)   # e4m3: 17 lies between 16 and 18
    rows[10] = -rows[8]
    rows[11] = 1.0
    x = rows[:, None, None, :].to(DEV)
    T = rows.shape[0]
    codes, scales = new_state(B, Hkv, T, D, fmt)
    cfg = tova.tova_quant_config(B, Hkv, D, T, tova.TOVA_DTYPE_FP32, FMT[fmt])
    tova.tova_quant_write(cfg, x, x, T, codes[0], scales[0], codes[1], scales[1])
    code, scale = quantise(x, fmt)
    got = codes_as_floats(codes[0], fmt)[0, 0]
    assert torch.equal(got, code[:, 0, 0])
    assert torch.equal(scales[0][0, 0].isnan().cpu(), torch.tensor([t in (5, 6, 7) for t in range(T)]))
    assert torch.equal(torch.nan_to_num(scales[0][0, 0]), torch.nan_to_num(scale[:, 0, 0]))
    y = torch.empty_like(x)
    tova.tova_quant_read(cfg, codes[0], scales[0], None, None, T, y, None)
    assert bool(y[5:8].isnan().all()) and bool(y[8:].isfinite().all()) and bool((y[:3] == 0).all())
    assert torch.equal(codes[0], codes[1])


def test_quant_slots_named_twice_and_slots_outside():
    """The later token's row stands (near and far apart in the call), rows without a slot are skipped, and reading a
    slot outside the state gives zeros."""
    g = gen(8)
    T, B, Hkv, D, cap = 700, 3, 2, 128, 50
    k = randn(g, T, B, Hkv, D).to(torch.bfloat16)
    v = randn(g, T, B, Hkv, D).to(torch.bfloat16)
    slots = torch.randint(-3, cap + 3, (T, B), generator=g, device=DEV, dtype=torch.int32)
    slots[100:160, 1] = 7
    slots[:, 2] = torch.where(slots[:, 2] == 11, 12, slots[:, 2])
    slots[0, 2], slots[1, 2] = 11, 2 ** 31 - 1
    codes, scales = new_state(B, Hkv, cap, D, "int8")
    cfg = tova.tova_quant_config(B, Hkv, D, cap, tova.TOVA_DTYPE_BF16, tova.TOVA_FORMAT_INT8)
    for _ in range(3):                                       # the same bits every time
        tova.tova_quant_write(cfg, k, v, T, codes[0], scales[0], codes[1], scales[1], slots=slots)
        for x, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
            code, scale = quantise(x, "int8")
            want_c, want_s = torch.full_like(c, 3), torch.full_like(s, 0.25)
            for b in range(B):
                for t, slot in enumerate(slots[:, b].tolist()):
                    if 0 <= slot < cap:
                        want_c[b, :, slot], want_s[b, :, slot] = code[t, b].to(torch.int8), scale[t, b]
            assert torch.equal(c, want_c) and torch.equal(s, want_s)
    y = torch.full((T, B, Hkv, D), 9.0, dtype=torch.bfloat16, device=DEV)
    tova.tova_quant_read(cfg, codes[0], scales[0], codes[1], scales[1], T, None, y, slots=slots)
    out = (slots < 0) | (slots >= cap)
    assert bool((y[out] == 0).all()) and bool((y[~out].float().abs().amax((-1, -2)) > 0).all())


def test_quant_write_takes_slices_of_a_projection():
    g = gen(9)
    T, B, H, Hkv, D = 6, 2, 4, 2, 64
    qkv = randn(g, T, B, (H + 2 * Hkv) * D)
    k, v = qkv[..., H * D:(H + Hkv) * D].unflatten(-1, (Hkv, D)), qkv[..., (H + Hkv) * D:].unflatten(-1, (Hkv, D))
    codes, scales = new_state(B, Hkv, 8, D, "e4m3")
    cfg = tova.tova_quant_config(B, Hkv, D, 8, tova.TOVA_DTYPE_FP32, tova.TOVA_FORMAT_E4M3)
    tova.tova_quant_write(cfg, k, v, T, codes[0], scales[0], codes[1], scales[1], first_slot=2)
    for x, c, s in ((k, codes[0], scales[0]), (v, codes[1], scales[1])):
        code, scale = quantise(x, "e4m3")
        assert torch.equal(codes_as_floats(c, "e4m3")[:, :, 2:], code.permute(1, 2, 0, 3))
        assert torch.equal(s[:, :, 2:], scale.permute(1, 2, 0))


# ------------------------------------------------------------------------------- attention of drafted tokens

def ancestors(par):
    """[N][..] lists of visible nodes per node for one sequence's parents (empty: padding)."""
    out = []
    for i in range(len(par)):
        j, chain = i, []
        while j >= 0:
            chain.append(j)
            if not -1 <= par[j] < j:
                chain = []
                break
            j = par[j]
        out.append(chain)
    return out


def tree_reference(q, k, v, K, V, lens, parents, scale=None):
    """64-bit attention; K, V [B,Hkv,cap,D] in double.  Returns the result and, per output row, sum p|v| per component
    and the largest sum of |q_d k_d| scale among visible columns (what roundings scale with)."""
    N, B, H, D = q.shape
    Hkv = k.shape[2]
    G = H // Hkv
    scale = scale or D ** -0.5
    out = torch.zeros(N, B, H, D, dtype=torch.float64, device=DEV)
    wv, reach, vmax = torch.zeros_like(out), torch.zeros(N, B, H, 1, dtype=torch.float64, device=DEV), torch.zeros(N, B, H, 1, dtype=torch.float64, device=DEV)
    for b in range(B):
        par = [i - 1 for i in range(N)] if parents is None else parents[:, b].tolist()
        for i, chain in enumerate(ancestors(par)):
            if not chain:
                continue
            n = lens[b]
            kk = torch.cat([K[b, :, :n], k[chain, b].double().transpose(0, 1)], 1)        # [Hkv,n+c,D]
            vv = torch.cat([V[b, :, :n], v[chain, b].double().transpose(0, 1)], 1)
            qq = q[i, b].double().view(Hkv, G, D)
            x = torch.einsum("hgd,hld->hgl", qq, kk) * scale
            w = torch.softmax(x, -1)
            out[i, b] = torch.einsum("hgl,hld->hgd", w, vv).reshape(H, D)
            wv[i, b] = torch.einsum("hgl,hld->hgd", w, vv.abs()).reshape(H, D)
            reach[i, b] = (torch.einsum("hgd,hld->hgl", qq.abs(), kk.abs()) * scale).amax(-1).reshape(H, 1)
            vmax[i, b] = vv.abs().amax((1, 2))[:, None].expand(Hkv, G).reshape(H, 1)
    return out, wv, reach, vmax


def tree_tolerance(dtype, D, cols, want, wv, reach):
    """A logit is off by delta <= 2 (D + 4) 2^-24 reach (products and sums in fp32, truncating adders), a weight by
    e^delta - 1 relative, in numerator and denominator; fp32 sums over the columns add 2 cols 2^-24 at the very most of
    sum p|v| (pairwise in tiles: far less); bf16 rounds weights and result by 2^-8 each.  exp2's own error is 2^-22."""
    delta = 2 * (D + 4) * 2.0 ** -24 * reach
    rel = 2 * torch.expm1(delta) + (2 * cols + 16) * 2.0 ** -24
    if dtype == "bf16":
        rel = rel + 2.0 ** -8
    return rel * wv * 1.01 + HALF[dtype] * want.abs() + 1e-30


def random_parents(N, B, seed, padding=True):
    g = torch.Generator().manual_seed(seed)
    par = torch.empty(N, B, dtype=torch.int32)
    for b in range(B):
        for i in range(N):
            par[i, b] = int(torch.randint(max(-1, i - 5), i, (1,), generator=g)) if i else -1
        if padding and N > 3 and b % 2 == 1:
            par[N - 1, b] = -2
            par[N // 2, b] = N // 2            # its own parent: padding, and so are the nodes below it
    return par.to(DEV)


def run_tree(dtype, fmt, N, B, H, Hkv, D, lens, cap, parents, seed=0, sm_scale=0.0, gain=1.0, n_live=None, poison=True):
    g = gen(seed)
    t = TT[dtype]
    q, k, v = (randn(g, N, B, H, D) * gain).to(t), randn(g, N, B, Hkv, D).to(t), randn(g, N, B, Hkv, D).to(t)
    Kf, Vf = randn(g, B, Hkv, cap, D), randn(g, B, Hkv, cap, D)
    ks = vs = None
    if fmt == "plain":
        K, V = Kf.to(t), Vf.to(t)
        Kd, Vd = K.double(), V.double()
    else:
        cfg = tova.tova_quant_config(B, Hkv, D, cap, tova.TOVA_DTYPE_FP32, FMT[fmt])
        (K, V), (ks, vs) = new_state(B, Hkv, cap, D, fmt)
        tova.tova_quant_write(cfg, Kf.permute(2, 0, 1, 3).contiguous(), Vf.permute(2, 0, 1, 3).contiguous(), cap, K, ks, V, vs)
        Kd, Vd = codes_as_floats(K, fmt).double() * ks.double()[..., None], codes_as_floats(V, fmt).double() * vs.double()[..., None]
    if poison:                                  # rows behind a sequence's last may hold anything
        for b in range(B):
            for X, s in ((K, ks), (V, vs)):
                if lens[b] < cap:
                    if fmt == "plain":
                        X[b, :, lens[b]:] = math.nan
                        X[b, :, lens[b]::2] = math.inf
                    else:
                        X[b, :, lens[b]:] = 127
                        s[b, :, lens[b]:] = math.nan
    cfg = tova.tova_tree_config(B, H, Hkv, D, cap, TD[dtype], FMT[fmt], sm_scale)
    n_live = max(lens) if n_live is None else n_live
    need = tova.tova_tree_workspace_bytes(cfg, n_live, N)
    ws = torch.full((need + 64,), 0xff, dtype=torch.uint8, device=DEV)
    out = torch.full((N, B, H, D), 77.0, dtype=t, device=DEV)
    lt = None if all(x == n_live for x in lens) else torch.tensor(lens, dtype=torch.int32, device=DEV)
    args = (cfg, K, V, n_live, q, k, v, N, out, ws[:need])
    tova.tova_tree_attention(*args, parents=parents, lens=lt, k_scale=ks, v_scale=vs)
    want, wv, reach, _ = tree_reference(q, k, v, Kd, Vd, lens, None if parents is None else parents.cpu(), sm_scale or None)
    tol = tree_tolerance(dtype, D, max(lens) + N, want, wv, reach)
    err = (out.double() - want).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), float(err.max()), (err > tol).nonzero()[:3].tolist())
    assert bool((ws[need:] == 0xff).all())
    first = out.clone()
    tova.tova_tree_attention(*args, parents=parents, lens=lt, k_scale=ks, v_scale=vs)
    assert torch.equal(first, out)              # the same bits every time
    return out, want


TREE_SHAPES = [
    # N, B, H, Hkv, lens, cap
    (1, 1, 4, 4, [0], 1),                         # an empty state: only itself
    (1, 1, 1, 1, [1], 1),
    (1, 2, 32, 8, [1000, 3], 1003),               # a plain step
    (1, 3, 8, 1, [64, 63, 65], 65),               # tile edges
    (3, 2, 8, 8, [127, 0], 129),
    (5, 1, 32, 8, [2500], 2500),
    (16, 2, 4, 4, [200, 31], 200),
    (17, 3, 8, 2, [33, 128, 1], 130),
    (31, 1, 32, 4, [700], 711),
    (64, 2, 16, 4, [90, 257], 300),
    (65, 1, 4, 2, [1], 5),
    (130, 2, 4, 1, [40, 513], 520),
    (256, 1, 2, 1, [300], 300),
]


@pytest.mark.parametrize("fmt", ["plain", "int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("shape", TREE_SHAPES, ids=lambda s: f"N{s[0]}B{s[1]}H{s[2]}x{s[3]}L{max(s[4])}")
def test_tree_attention(dtype, fmt, D, shape):
    N, B, H, Hkv, lens, cap = shape
    run_tree(dtype, fmt, N, B, H, Hkv, D, lens, cap, random_parents(N, B, N), seed=N)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("N, lens", [(1, [5000]), (8, [4097]), (40, [20001])])
def test_tree_chain_over_a_long_state(dtype, N, lens):
    run_tree(dtype, "plain", N, 1, 8, 2, 128, lens, lens[0], None, seed=N, gain=2.0)


@pytest.mark.parametrize("fmt", ["plain", "int8", "e4m3"])
@pytest.mark.parametrize("D, N, H, Hkv", [(128, 20, 8, 2), (64, 20, 8, 2), (128, 40, 8, 2), (64, 150, 4, 2), (128, 25, 6, 2), (64, 30, 12, 4)])
def test_tree_many_short_sequences(fmt, D, N, H, Hkv):
    """More than 64 rows of the product over many sequences of a tile or two: a block walks through many jobs, most of
    them ending inside a tile, some empty, some cut by the end of its run; query groups that do not divide 128 too."""
    B = 41
    g = torch.Generator().manual_seed(N)
    lens = [int(x) for x in torch.randint(0, 300, (B,), generator=g)]
    lens[3], lens[4], lens[5], lens[6] = 0, 128, 256, 1
    run_tree("bf16", fmt, N, B, H, Hkv, D, lens, 301, random_parents(N, B, N), seed=N)


@pytest.mark.parametrize("fmt", ["plain", "int8"])
@pytest.mark.parametrize("N, H", [(3, 4096), (16, 4096), (2, 1000)])
def test_tree_more_rows_than_the_gpu_has_blocks_for(fmt, N, H):
    """One KV head under thousands of query heads: more row blocks than SMs, groups larger than a row tile."""
    run_tree("bf16", fmt, N, 1, H, 1, 64, [70], 80, random_parents(N, 1, N), seed=N)


@pytest.mark.parametrize("dtype, fmt, N", [("bf16", "plain", 4), ("bf16", "plain", 24), ("bf16", "plain", 50), ("bf16", "int8", 50), ("fp32", "plain", 5)])
def test_tree_logits_that_grow_along_the_state(dtype, fmt, N):
    """Later columns outweigh earlier ones by far more than any slack in the running reference: keys grow along the state."""
    g = gen(N)
    B, H, Hkv, D, L = 1, 8, 2, 128, 1500
    t = TT[dtype]
    q, k, v = (randn(g, N, B, n, D).to(t) for n in (H, Hkv, Hkv))
    grow = torch.linspace(0.01, 60.0, L, device=DEV)[None, None, :, None]
    Kf, Vf = randn(g, B, Hkv, L, D) * grow, randn(g, B, Hkv, L, D)
    ks = vs = None
    if fmt == "plain":
        K, V = Kf.to(t), Vf.to(t)
        Kd, Vd = K.double(), V.double()
    else:
        (K, V), (ks, vs) = new_state(B, Hkv, L, D, fmt)
        tova.tova_quant_write(tova.tova_quant_config(B, Hkv, D, L, tova.TOVA_DTYPE_FP32, FMT[fmt]), Kf.permute(2, 0, 1, 3).contiguous(),
                              Vf.permute(2, 0, 1, 3).contiguous(), L, K, ks, V, vs)
        Kd, Vd = codes_as_floats(K, fmt).double() * ks.double()[..., None], codes_as_floats(V, fmt).double() * vs.double()[..., None]
    cfg = tova.tova_tree_config(B, H, Hkv, D, L, TD[dtype], FMT[fmt], 0.0)
    ws = torch.empty(max(16, tova.tova_tree_workspace_bytes(cfg, L, N)), dtype=torch.uint8, device=DEV)
    out = torch.empty(N, B, H, D, dtype=t, device=DEV)
    tova.tova_tree_attention(cfg, K, V, L, q, k, v, N, out, ws, k_scale=ks, v_scale=vs)
    want, wv, reach, _ = tree_reference(q, k, v, Kd, Vd, [L], None)
    assert bool(((out.double() - want).abs() <= tree_tolerance(dtype, D, L + N, want, wv, reach)).all())


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype, N", [("bf16", 3), ("bf16", 12), ("bf16", 50), ("fp32", 3), ("fp32", 12)])
def test_tree_value_scales_of_any_size(dtype, fmt, N):
    """Value scales from zero and below the normal numbers up to 2^60, each row's its own, under codes that are not zero."""
    g = gen(N)
    B, H, Hkv, D, L = 2, 8, 2, 128, 330
    t = TT[dtype]
    q, k, v = (randn(g, N, B, n, D).to(t) for n in (H, Hkv, Hkv))
    (K, V), (ks, vs) = new_state(B, Hkv, L, D, fmt)
    Kf, Vf = randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D)
    tova.tova_quant_write(tova.tova_quant_config(B, Hkv, D, L, tova.TOVA_DTYPE_FP32, FMT[fmt]), Kf, Vf, L, K, ks, V, vs)
    sizes = torch.tensor([0.0, 2.0 ** -140, 2.0 ** -126, 2.0 ** -101, 2.0 ** -90, 2.0 ** -20, 2.0 ** -6, -2.0 ** -7], device=DEV)
    vs.copy_(sizes[torch.arange(L, device=DEV) % 8].expand(B, Hkv, L))
    vs[1, :, 77] = 2.0 ** 60
    Kd, Vd = codes_as_floats(K, fmt).double() * ks.double()[..., None], codes_as_floats(V, fmt).double() * vs.double()[..., None]
    cfg = tova.tova_tree_config(B, H, Hkv, D, L, TD[dtype], FMT[fmt], 0.0)
    ws = torch.empty(max(16, tova.tova_tree_workspace_bytes(cfg, L, N)), dtype=torch.uint8, device=DEV)
    out = torch.empty(N, B, H, D, dtype=t, device=DEV)
    par = random_parents(N, B, N)
    tova.tova_tree_attention(cfg, K, V, L, q, k, v, N, out, ws, parents=par, k_scale=ks, v_scale=vs)
    want, wv, reach, _ = tree_reference(q, k, v, Kd, Vd, [L] * B, par.cpu())
    assert bool(((out.double() - want).abs() <= tree_tolerance(dtype, D, L + N, want, wv, reach)).all())


def test_tree_scale_and_live_bound():
    """A scale of the caller's; n_live above every length (the launch is cut for it, the lengths decide)."""
    run_tree("bf16", "plain", 7, 2, 8, 2, 64, [40, 0], 3000, random_parents(7, 2, 1), sm_scale=0.31, n_live=3000)
    run_tree("fp32", "int8", 7, 2, 8, 2, 128, [400, 9], 3000, random_parents(7, 2, 1), sm_scale=0.02, n_live=2999)
    run_tree("bf16", "e4m3", 30, 2, 8, 2, 128, [40, 0], 3000, random_parents(30, 2, 1), n_live=3000)


def test_tree_lengths_outside_the_bound_are_clamped():
    g = gen(5)
    B, H, Hkv, D, cap = 3, 4, 2, 64, 20
    q, k, v = (randn(g, 2, B, n, D) for n in (H, Hkv, Hkv))
    K, V = randn(g, B, Hkv, cap, D), randn(g, B, Hkv, cap, D)
    cfg = tova.tova_tree_config(B, H, Hkv, D, cap, tova.TOVA_DTYPE_FP32, tova.TOVA_FORMAT_PLAIN, 0.0)
    out, same = torch.empty(2, B, H, D, device=DEV), torch.empty(2, B, H, D, device=DEV)
    tova.tova_tree_attention(cfg, K, V, 10, q, k, v, 2, out, None, lens=torch.tensor([2 ** 30, -4, 10], dtype=torch.int32, device=DEV))
    tova.tova_tree_attention(cfg, K, V, 10, q, k, v, 2, same, None, lens=torch.tensor([10, 0, 10], dtype=torch.int32, device=DEV))
    assert torch.equal(out, same)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("H, Hkv, N", [(4, 4, 6), (8, 2, 40)])
def test_tree_values_of_unseen_drafts_do_not_leak(dtype, H, Hkv, N):
    """Infinities and NaN in drafts reach the nodes that see them and no others."""
    g = gen(6)
    B, D, L = 2, 128, 70
    t = TT[dtype]
    q, k, v = (randn(g, N, B, n, D).to(t) for n in (H, Hkv, Hkv))
    K, V = randn(g, B, Hkv, L, D).to(t), randn(g, B, Hkv, L, D).to(t)
    par = random_parents(N, B, 3, padding=False)
    cfg = tova.tova_tree_config(B, H, Hkv, D, L, TD[dtype], tova.TOVA_FORMAT_PLAIN, 0.0)
    ws = torch.empty(max(16, tova.tova_tree_workspace_bytes(cfg, L, N)), dtype=torch.uint8, device=DEV)
    clean, out = torch.empty(N, B, H, D, dtype=t, device=DEV), torch.empty(N, B, H, D, dtype=t, device=DEV)
    tova.tova_tree_attention(cfg, K, V, L, q, k, v, N, clean, ws, parents=par)
    bad = 2
    k2, v2 = k.clone(), v.clone()
    k2[bad, 0] = math.nan
    v2[bad, 1, :, 5], v2[bad, 1, :, 6] = math.inf, math.nan
    tova.tova_tree_attention(cfg, K, V, L, q, k2, v2, N, out, ws, parents=par)
    for b in range(B):
        sees = torch.tensor([bad in c for c in ancestors(par[:, b].tolist())], device=DEV)
        assert torch.equal(out[:, b][~sees], clean[:, b][~sees])
        if b == 0:
            assert bool(out[:, b][sees].isnan().all())
        else:
            assert bool(out[:, b][sees][..., 5].isinf().all()) and bool(out[:, b][sees][..., 6].isnan().all())
            keep = [d for d in range(D) if d not in (5, 6)]
            assert torch.equal(out[:, b][sees][..., keep], clean[:, b][sees][..., keep])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype, H, Hkv, N", [("bf16", 4, 4, 6), ("bf16", 8, 2, 40), ("fp32", 8, 2, 40)])
def test_tree_values_of_unseen_drafts_do_not_leak_over_an_8_bit_state(dtype, fmt, H, Hkv, N):
    """The same over codes: a NaN key and infinite values of one draft reach the nodes that see it and no others."""
    g = gen(16)
    B, D, L = 2, 128, 270
    t = TT[dtype]
    q, k, v = (randn(g, N, B, n, D).to(t) for n in (H, Hkv, Hkv))
    (K, V), (ks, vs) = new_state(B, Hkv, L, D, fmt)
    tova.tova_quant_write(tova.tova_quant_config(B, Hkv, D, L, tova.TOVA_DTYPE_FP32, FMT[fmt]), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D),
                          L, K, ks, V, vs)
    par = random_parents(N, B, 3, padding=False)
    cfg = tova.tova_tree_config(B, H, Hkv, D, L, TD[dtype], FMT[fmt], 0.0)
    ws = torch.empty(max(16, tova.tova_tree_workspace_bytes(cfg, L, N)), dtype=torch.uint8, device=DEV)
    clean, out = torch.empty(N, B, H, D, dtype=t, device=DEV), torch.empty(N, B, H, D, dtype=t, device=DEV)
    tova.tova_tree_attention(cfg, K, V, L, q, k, v, N, clean, ws, parents=par, k_scale=ks, v_scale=vs)
    bad = 2
    k2, v2 = k.clone(), v.clone()
    k2[bad, 0] = math.nan
    v2[bad, 1, :, 5] = -math.inf
    tova.tova_tree_attention(cfg, K, V, L, q, k2, v2, N, out, ws, parents=par, k_scale=ks, v_scale=vs)
    for b in range(B):
        sees = torch.tensor([bad in c for c in ancestors(par[:, b].tolist())], device=DEV)
        assert torch.equal(out[:, b][~sees], clean[:, b][~sees])
        if b == 0:
            assert bool(out[:, b][sees].isnan().all())
        else:
            assert bool((out[:, b][sees][..., 5] == -math.inf).all())
            keep = [d for d in range(D) if d != 5]
            assert torch.equal(out[:, b][sees][..., keep], clean[:, b][sees][..., keep])


def test_tree_offsets_beyond_32_bits():
    """A state of more than 2^31 elements: the last sequence's rows lie behind that."""
    B, H, Hkv, D, cap, L = 2, 4, 2, 128, 4300000, 300
    g = gen(7)
    K = torch.zeros(B, Hkv, cap, D, dtype=torch.int8, device=DEV)
    V = torch.zeros_like(K)
    ks, vs = torch.zeros(B, Hkv, cap, device=DEV), torch.zeros(B, Hkv, cap, device=DEV)
    rows = randn(g, L, B, Hkv, D).to(torch.bfloat16)
    qc = tova.tova_quant_config(B, Hkv, D, cap, tova.TOVA_DTYPE_BF16, tova.TOVA_FORMAT_INT8)
    tova.tova_quant_write(qc, rows, rows, L, K, ks, V, vs)
    back = torch.empty_like(rows)
    tova.tova_quant_read(qc, K, ks, V, vs, L, back, None)
    code, scale = quantise(rows, "int8")
    assert torch.equal(back, (code * scale[..., None]).to(torch.bfloat16))
    far = torch.full((1, B), cap - 1, dtype=torch.int32, device=DEV)
    tova.tova_quant_write(qc, rows[:1], rows[:1], 1, K, ks, V, vs, slots=far)
    assert torch.equal(K[1, 1, cap - 1].float(), code[0, 1, 1])
    q, k, v = (randn(g, 3, B, n, D).to(torch.bfloat16) for n in (H, Hkv, Hkv))
    cfg = tova.tova_tree_config(B, H, Hkv, D, cap, tova.TOVA_DTYPE_BF16, tova.TOVA_FORMAT_INT8, 0.0)
    ws = torch.empty(max(16, tova.tova_tree_workspace_bytes(cfg, L, 3)), dtype=torch.uint8, device=DEV)
    out = torch.empty(3, B, H, D, dtype=torch.bfloat16, device=DEV)
    tova.tova_tree_attention(cfg, K, V, L, q, k, v, 3, out, ws, k_scale=ks, v_scale=vs)
    vals = code.double() * scale.double()[..., None]
    want, wv, reach, _ = tree_reference(q, k, v, vals.permute(1, 2, 0, 3), vals.permute(1, 2, 0, 3), [L] * B, None)
    assert bool(((out.double() - want).abs() <= tree_tolerance("bf16", D, L + 3, want, wv, reach)).all())


@pytest.mark.parametrize("policy", [tova.TOVA_POLICY_TOVA, tova.TOVA_POLICY_TOVA_HEAD])
@pytest.mark.parametrize("deferred", [False, True])
def test_tree_attention_over_a_cache(policy, deferred):
    """The handle's form sees the state as the last step left it, evictions included (deferred ones too), leaves it as it
    is, and agrees with the tensors' form on the state read out."""
    w = W.WORKLOADS["mistral_7b_gqa"].scaled(batch=2, n_q_heads=8, n_kv_heads=2, capacity=70)
    N, T = 9, 100
    q, k, v = (tova.to_device(a, w.dtype) for a in W.tokens(w, 0, T + N))
    c = tova.TovaCache(w.batch, w.n_q_heads, w.n_kv_heads, w.head_dim, w.capacity, dtype=w.dtype)
    c.tova_cache_set_policy(policy, 0)
    c.tova_cache_set_deferred_eviction(deferred)
    ws = torch.empty(max(16, c.tova_cache_tree_workspace_bytes(N)), dtype=torch.uint8, device=DEV)
    out = torch.empty(N, w.batch, w.n_q_heads, w.head_dim, dtype=torch.bfloat16, device=DEV)
    step = torch.empty(w.batch, w.n_q_heads, w.head_dim, device=DEV)
    par = random_parents(N, w.batch, 5, padding=False)
    lens = []
    for t in range(T):
        c.tova_decode_step(q[t], k[t], v[t], t, step)
        if t in (0, 40, 69, 99):
            c.tova_cache_tree_attention(q[T:], k[T:], v[T:], N, out, ws, parents=par)
            state = c.tova_cache_read(want_kv=True)
            n = int(state["len"][0])
            lens.append(n)
            want, wv, reach, _ = tree_reference(q[T:], k[T:], v[T:], state["K"].double().to(DEV), state["V"].double().to(DEV),
                                                [n] * w.batch, par.cpu())
            assert bool(((out.double() - want).abs() <= tree_tolerance("bf16", w.head_dim, n + N, want, wv, reach)).all())
            again = c.tova_cache_read(want_kv=True)
            assert all(torch.equal(state[x], again[x]) for x in ("len", "positions", "K", "V"))
    assert lens == [1, 41, 70, 70]
    c.tova_cache_join()


def test_tree_attention_refuses_position_compression():
    c = tova.TovaCache(1, 4, 4, 64, 32, dtype=tova.TOVA_DTYPE_FP32)
    c.tova_cache_set_position_compression()
    x = torch.zeros(1, 1, 4, 64, device=DEV)
    with pytest.raises(tova.TovaError) as e:
        c.tova_cache_tree_attention(x, x, x, 1, torch.empty_like(x))
    assert e.value.code == -3


def test_tree_workspace_is_checked():
    cfg = tova.tova_tree_config(1, 4, 4, 128, 9000, tova.TOVA_DTYPE_BF16, tova.TOVA_FORMAT_PLAIN, 0.0)
    need = tova.tova_tree_workspace_bytes(cfg, 9000, 2)
    assert need > 0
    K = torch.zeros(1, 4, 9000, 128, dtype=torch.bfloat16, device=DEV)
    x = torch.zeros(2, 1, 4, 128, dtype=torch.bfloat16, device=DEV)
    for ws, code in ((None, -1), (torch.empty(need - 1, dtype=torch.uint8, device=DEV), -5)):
        with pytest.raises(tova.TovaError) as e:
            tova.tova_tree_attention(cfg, K, K, 9000, x, x, x, 2, torch.empty_like(x), ws)
        assert e.value.code == code


@pytest.mark.parametrize("dtype, B, H, N, D", [("bf16", 1, 4, 2, 128), ("bf16", 2, 3, 5, 64), ("bf16", 1, 1, 40, 64), ("bf16", 7, 4, 2, 64), ("bf16", 50, 4, 1, 64),
                                                ("bf16", 1, 2, 70, 64), ("fp32", 1, 2, 3, 64), ("fp32", 3, 4, 20, 64), ("fp32", 80, 4, 1, 64)])
def test_tree_workspace_does_for_every_length_up_to_the_bound(dtype, B, H, N, D):
    """A state that grows: one workspace, sized for the most rows it will hold."""
    t = TT[dtype]
    top = 24000 // B
    cfg = tova.tova_tree_config(B, H, H, D, top, TD[dtype], tova.TOVA_FORMAT_PLAIN, 0.0)
    K = torch.zeros(B, H, top, D, dtype=t, device=DEV)
    x = torch.zeros(N, B, H, D, dtype=t, device=DEV)
    out = torch.empty_like(x)
    for most in (top, top // 2 + 1, top // 3):
        ws = torch.empty(tova.tova_tree_workspace_bytes(cfg, most, N), dtype=torch.uint8, device=DEV)
        for n in list(range(most, 0, -max(1, most // 150))) + [1, 0]:
            tova.tova_tree_attention(cfg, K, K, n, x, x, x, N, out, ws)
    torch.cuda.synchronize()


# -------------------------------------------------------------------------------------------- verification

def verify_reference(p, q, tokens, parents, u, us):
    """One sequence, from the definition, with exact sums: p, q [N+1][V] lists of floats (q may be None)."""
    N, V = len(tokens), len(p[0])
    node, path, out = -1, [], []
    while True:
        r, Z, S = list(p[node + 1]), 1.0, 0.0
        r = [x if x > 0 else 0.0 for x in r]
        got = -1
        for c in range(N):
            if parents[c] != node or not -1 <= parents[c] < c:
                continue
            x = tokens[c]
            qx = 1.0 if q is None or not 0 <= x < V else q[node + 1][x]
            if 0 <= x < V and u[c] * qx * Z < r[x]:
                got = c
                break
            if q is None:
                if 0 <= x < V:
                    Z -= r[x]
                    r[x] = 0.0
            else:
                S += Z
                r = [max(0.0, a - S * b) for a, b in zip(p[node + 1], q[node + 1])]
                Z = math.fsum(r)
        if got < 0:
            break
        path.append(got)
        out.append(tokens[got])
        node = got
    if not math.fsum(r) > 0:
        r = [x if x > 0 else 0.0 for x in p[node + 1]]
    whole, run, last = math.fsum(r), 0.0, -1
    goal = us * whole
    if whole > 0:
        part = []
        for x in range(V):
            if r[x] > 0:
                last = x
                part.append(r[x])
                run += r[x]
                if run > goal:
                    break
    return len(path), path + [-1] * (N - len(path)), out + [last] + [-1] * (N - len(path))


def run_verify(p, q, tok, par, u, us, dtype, row_stride=0):
    R, B, V = p.shape
    N = tok.shape[0]
    cfg = tova.tova_verify_config(B, N, V, TD[dtype], row_stride)
    n = torch.full((B,), 99, dtype=torch.int32, device=DEV)
    path = torch.full((N, B), 99, dtype=torch.int32, device=DEV)
    out = torch.full((N + 1, B), 99, dtype=torch.int32, device=DEV)
    if row_stride:
        def padded(x):
            y = torch.full((x.shape[0] * B * row_stride,), math.nan, dtype=x.dtype, device=DEV).view(x.shape[0], B, row_stride)
            y[..., :V] = x
            return y
        p, q = padded(p), None if q is None else padded(q)
    tova.tova_verify_draft(cfg, p, q, tok, u, us, n, path, out, parents=par)
    return n, path, out


def verify_inputs(N, B, V, dtype, seed, chain, draft, sharp=2.0):
    g = gen(seed)
    logits = randn(g, N + 1, B, V) * sharp
    p = torch.softmax(logits, -1).to(TT[dtype])
    q = torch.softmax(logits + randn(g, N + 1, B, V), -1).to(TT[dtype])
    par = None if chain else random_parents(N, B, seed)
    pc = torch.arange(-1, N - 1)[:, None].expand(N, B) if chain else par.cpu()
    tok = torch.zeros(N, B, dtype=torch.int32, device=DEV)
    for i in range(N):
        for b in range(B):
            row = min(max(int(pc[i, b]), -1), N - 1) + 1
            tok[i, b] = torch.multinomial(q[row, b].float(), 1, generator=g)[0].int()
    u, us = torch.rand(N, B, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
    return p, (q if draft else None), tok, par, pc, u, us


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("N, B, V, chain", [(0, 3, 17, True), (1, 1, 1, True), (1, 4, 2, False), (5, 3, 1000, True), (12, 4, 7, False),
                                            (33, 3, 4099, False), (40, 2, 50, False), (7, 2, 32000, False), (90, 2, 33, True)])
def test_verify_against_the_definition(dtype, draft, N, B, V, chain):
    p, q, tok, par, pc, u, us = verify_inputs(N, B, V, dtype, N + V, chain, draft)
    for stride in (0, (V + 15) // 8 * 8):
        n, path, out = run_verify(p, q, tok, par, u, us, dtype, row_stride=stride)
        for b in range(B):
            want = verify_reference(p[:, b].double().tolist(), None if q is None else q[:, b].double().tolist(), tok[:, b].tolist(),
                                    pc[:, b].tolist(), u[:, b].double().tolist(), float(us[b].double()))
            assert (int(n[b]), path[:, b].tolist(), out[:, b].tolist()) == want, b


def test_verify_edges():
    V, N, B = 300, 3, 8
    g = gen(1)
    p = torch.softmax(randn(g, N + 1, B, V), -1)
    q = torch.softmax(randn(g, N + 1, B, V), -1)
    tok = torch.randint(0, V, (N, B), generator=g, device=DEV, dtype=torch.int32)
    u, us = torch.rand(N, B, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
    u[:, 0] = 0.0                                  # u = 0 accepts whatever has probability
    p[:, 1], q[:, 1] = 0.0, 0.0
    p[:, 1, 7] = 1.0                               # a certain target: only token 7 passes
    tok[:, 1] = torch.tensor([7, 7, 8], device=DEV)
    q[:, 1, 7], q[:, 1, 8] = 0.5, 0.5
    p[0, 2] = 0.0                                  # nothing to draw from
    u[0, 2] = 0.999
    p[0, 3] = q[0, 3]                              # the residual is zero: the last token comes from p
    tok[0, 3] = V + 5                              # a token outside the vocabulary is not accepted
    p[0, 4, :200] = math.nan                       # NaN counts as nothing
    tok[0, 4] = 3
    us[5] = 0.0
    us[6] = 1.0 - 2.0 ** -24
    tok[:, 7] = -1
    par = torch.tensor([[-1, 0, 1]], device=DEV, dtype=torch.int32).t().expand(N, B).contiguous()
    n, path, out = run_verify(p, q, tok, par, u, us, "fp32")
    again = run_verify(p, q, tok, None, u, us, "fp32")          # the same chain without parents
    assert all(torch.equal(x, y) for x, y in zip((n, path, out), again))
    assert int(n[0]) == 3 and path[:, 0].tolist() == [0, 1, 2]
    assert int(n[1]) == 2 and out[:, 1].tolist() == [7, 7, 7, -1]
    assert int(n[2]) == 0 and out[:, 2].tolist() == [-1, -1, -1, -1]
    assert int(n[3]) == 0 and 0 <= int(out[0, 3]) < V
    assert int(n[4]) == 0 and 200 <= int(out[0, 4]) < V
    assert int(n[7]) == 0 and 0 <= int(out[0, 7]) < V
    for b in (0, 1, 3, 5, 6, 7):
        want = verify_reference(p[:, b].double().tolist(), q[:, b].double().tolist(), tok[:, b].tolist(), [-1, 0, 1],
                                u[:, b].double().tolist(), float(us[b].double()))
        assert (int(n[b]), path[:, b].tolist(), out[:, b].tolist()) == want, b


@pytest.mark.parametrize("draft", [True, False])
def test_verify_keeps_the_target_distribution(draft):
    """The first token of many sequences with one target is distributed as the target says, whatever the drafts: two
    children of the root, drawn independently from q (or, without q, always the two likeliest tokens of another
    distribution).  Five standard deviations of a binomial count, for each of 6 tokens: a chance below 1e-5."""
    B, V, N = 60000, 6, 2
    g = gen(11)
    p1 = torch.tensor([0.05, 0.3, 0.1, 0.25, 0.05, 0.25], device=DEV)
    q1 = torch.tensor([0.4, 0.1, 0.2, 0.1, 0.15, 0.05], device=DEV)
    p, q = p1.expand(N + 1, B, V).contiguous(), q1.expand(N + 1, B, V).contiguous()
    tok = torch.multinomial(q1, N * B, replacement=True, generator=g).view(N, B).to(torch.int32)
    if not draft:
        tok[0], tok[1] = 0, 2
    par = torch.full((N, B), -1, dtype=torch.int32, device=DEV)
    u, us = torch.rand(N, B, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
    _, _, out = run_verify(p, q if draft else None, tok, par, u, us, "fp32")
    counts = torch.bincount(out[0].long(), minlength=V).double()
    want = B * p1.double()
    assert bool(((counts - want).abs() <= 5 * torch.sqrt(want * (1 - p1.double()))).all()), (counts.tolist(), want.tolist())


# ------------------------------------------------------------------------------------------------- together

def test_speculative_decoding_over_a_state():
    """Rotary positions, attention of the drafts over the cache and over its 8-bit copy, verification, and the accepted
    path through the ordinary prompt route: the cache ends up as if the accepted tokens had been fed one by one, and
    while the state has free rows the drafts' outputs are those of ordinary steps."""
    B, H, Hkv, D, cap, V, N = 1, 8, 2, 128, 96, 64, 10
    g = gen(21)
    rope = tova.TovaRope(B, H, Hkv, D)
    cache = tova.TovaCache(B, H, Hkv, D, cap)
    plain = tova.TovaCache(B, H, Hkv, D, cap)
    qcfg = tova.tova_quant_config(B, Hkv, D, cap, tova.TOVA_DTYPE_BF16, tova.TOVA_FORMAT_INT8)
    (K8, V8), (ks, vs) = new_state(B, Hkv, cap, D, "int8")
    tcfg = tova.tova_tree_config(B, H, Hkv, D, cap, tova.TOVA_DTYPE_BF16, tova.TOVA_FORMAT_INT8, 0.0)
    vcfg = tova.tova_verify_config(B, N, V, tova.TOVA_DTYPE_FP32, 0)
    ws = torch.empty(max(16, cache.tova_cache_tree_workspace_bytes(N), tova.tova_tree_workspace_bytes(tcfg, cap, N)),
                     dtype=torch.uint8, device=DEV)
    settled, steps, taken = 0, 0, 0
    while settled < 60:
        qkv = randn(g, N, B, (H + 2 * Hkv) * D).to(torch.bfloat16)
        par = random_parents(N, B, steps, padding=False)
        depth = [len(c) for c in ancestors(par[:, 0].tolist())]
        pos = (settled + torch.tensor(depth, device=DEV, dtype=torch.int32) - 1)[:, None].contiguous()
        q, k = torch.empty(N, B, H, D, dtype=torch.bfloat16, device=DEV), torch.empty(N, B, Hkv, D, dtype=torch.bfloat16, device=DEV)
        v = qkv[..., (H + Hkv) * D:].unflatten(-1, (Hkv, D)).contiguous()
        rope.tova_rope_apply(qkv[..., :H * D].unflatten(-1, (H, D)), qkv[..., H * D:(H + Hkv) * D].unflatten(-1, (Hkv, D)), N, q, k,
                             positions=pos)
        out, out8 = torch.empty_like(q), torch.empty_like(q)
        cache.tova_cache_tree_attention(q, k, v, N, out, ws, parents=par)
        tova.tova_tree_attention(tcfg, K8, V8, settled, q, k, v, N, out8, ws, parents=par, k_scale=ks, v_scale=vs)
        # int8 rounds keys and values by at most half a step of their row's scale, 1/254 of its largest entry
        assert float((out8.float() - out.float()).norm() / out.float().norm()) < 0.02
        p = torch.softmax(randn(g, N + 1, B, V), -1)
        dq = torch.softmax(torch.log(p) + 0.2 * randn(g, N + 1, B, V), -1)
        tok = torch.stack([torch.multinomial(dq[int(par[i, 0]) + 1], 1, generator=g)[:, 0] for i in range(N)]).to(torch.int32)
        u, us = torch.rand(N, B, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
        n, path, toks = (torch.empty(s, dtype=torch.int32, device=DEV) for s in ((B,), (N, B), (N + 1, B)))
        tova.tova_verify_draft(vcfg, p, dq, tok, u, us, n, path, toks, parents=par)
        got = int(n[0])
        if got:
            way = path[:got, 0].long()
            ko, vo = k[way], v[way]
            ev = torch.empty(got, B, dtype=torch.int32, device=DEV)
            cache.tova_prefill(q[way], ko, vo, got, settled, None, ev)
            tova.tova_quant_write(qcfg, ko, vo, got, K8, ks, V8, vs, first_slot=settled)
            step = torch.empty(B, H, D, device=DEV)
            for i in range(got):
                plain.tova_decode_step(q[way[i]], ko[i], vo[i], settled + i, step)
                # both are within the bf16 tolerance of the same 64-bit value; the step's own is 2e-3
                o = out[way[i]].float()
                assert float((o - step).abs().max()) <= 2e-3 + 2.0 ** -7 * float(step.abs().max()) + 2.0 ** -8 * 3.0
            settled += got
            taken += got
        steps += 1
        assert steps < 200
    a, b = cache.tova_cache_read(want_kv=True), plain.tova_cache_read(want_kv=True)
    assert all(torch.equal(a[x], b[x]) for x in ("len", "positions", "K", "V")) and a["status"] == b["status"] == 0
    assert taken > steps                                      # drafts were accepted


def test_operators_in_a_captured_graph_and_on_another_stream():
    """Captured once and replayed on new inputs; two graphs with workspaces of their own replayed on two streams at once."""
    B, H, Hkv, D, L, N, V = 2, 8, 2, 128, 3000, 12, 500
    runs = []
    for seed in (1, 2):
        g = gen(seed)
        s = dict(q=randn(g, N, B, H, D).to(torch.bfloat16), k=randn(g, N, B, Hkv, D).to(torch.bfloat16), v=randn(g, N, B, Hkv, D).to(torch.bfloat16))
        s["K"], s["V"] = randn(g, B, Hkv, L, D).to(torch.bfloat16), randn(g, B, Hkv, L, D).to(torch.bfloat16)
        s["par"] = random_parents(N, B, seed, padding=False)
        s["p"], s["dq"] = torch.softmax(randn(g, N + 1, B, V), -1), torch.softmax(randn(g, N + 1, B, V), -1)
        s["tok"] = torch.randint(0, V, (N, B), generator=g, device=DEV, dtype=torch.int32)
        s["u"], s["us"] = torch.rand(N, B, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
        cfg = tova.tova_tree_config(B, H, Hkv, D, L, tova.TOVA_DTYPE_BF16, tova.TOVA_FORMAT_PLAIN, 0.0)
        s["ws"] = torch.empty(max(16, tova.tova_tree_workspace_bytes(cfg, L, N)), dtype=torch.uint8, device=DEV)
        s["rq"], s["rk"], s["out"] = torch.empty_like(s["q"]), torch.empty_like(s["k"]), torch.empty_like(s["q"])
        s["n"], s["path"], s["toks"] = (torch.empty(x, dtype=torch.int32, device=DEV) for x in ((B,), (N, B), (N + 1, B)))
        (s["K8"], s["V8"]), (s["ks"], s["vs"]) = new_state(B, Hkv, N, D, "e4m3")
        rope, qc = tova.TovaRope(B, H, Hkv, D), tova.tova_quant_config(B, Hkv, D, N, tova.TOVA_DTYPE_BF16, tova.TOVA_FORMAT_E4M3)
        vc = tova.tova_verify_config(B, N, V, tova.TOVA_DTYPE_FP32, 0)

        def go(s=s, rope=rope, cfg=cfg, qc=qc, vc=vc):
            rope.tova_rope_apply(s["q"], s["k"], N, s["rq"], s["rk"], first_pos=9)
            tova.tova_quant_write(qc, s["rk"], s["v"], N, s["K8"], s["ks"], s["V8"], s["vs"])
            tova.tova_tree_attention(cfg, s["K"], s["V"], L, s["rq"], s["rk"], s["v"], N, s["out"], s["ws"], parents=s["par"])
            tova.tova_verify_draft(vc, s["p"], s["dq"], s["tok"], s["u"], s["us"], s["n"], s["path"], s["toks"], parents=s["par"])
        runs.append((s, go))
    names = ("rq", "rk", "K8", "ks", "out", "n", "path", "toks")
    graphs = []
    for s, go in runs:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            go()
        graphs.append(gr)
    for s, _ in runs:                              # other inputs than at capture
        s["q"].mul_(0.5)
        s["u"].mul_(0.7)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    for _ in range(5):
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
    torch.cuda.synchronize()
    got = [{x: s[x].clone() for x in names} for s, _ in runs]
    for (s, go), seen, st in zip(runs, got, streams):
        for x in names:
            s[x].zero_()
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            go()
        st.synchronize()
        assert all(torch.equal(s[x], seen[x]) for x in names)


def test_operators_take_an_explicit_stream():
    B, H, D, T = 2, 4, 64, 50
    x = randn(gen(1), T, B, H, D)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    r = tova.TovaRope(B, H, H, D, dtype=tova.TOVA_DTYPE_FP32)
    a, b = torch.empty_like(x), torch.empty_like(x)
    r.tova_rope_apply(x, None, T, a, None, stream=st)
    st.synchronize()
    r.tova_rope_apply(x, None, T, b, None)
    torch.cuda.synchronize()
    assert torch.equal(a, b)


# ------------------------------------------------------------------- drafted tokens: values that are not finite

# One shape for each way that a call is cut: one run of columns; runs joined in a cluster, few rows and many; runs joined by
# the second kernel; the tcgen05 kernel, with whole jobs and with cut ones.  N, B, H, Hkv, L.
CUTS = {"one run": (3, 2, 8, 2, 50), "cluster": (3, 2, 8, 2, 1000), "cluster, one token": (1, 1, 32, 8, 1000),
        "cluster, 48 rows": (12, 2, 8, 2, 500), "second kernel": (5, 1, 8, 2, 9000), "tcgen05": (40, 2, 8, 2, 300),
        "tcgen05, cut jobs": (40, 1, 8, 2, 9000)}


def cut_inputs(cut, dtype, fmt, seed):
    """Inputs of a call cut that way, the function that makes the call on given q, k, v and state, and its tree's parents
    (a padding node in every other sequence, where there are more than three nodes)."""
    N, B, H, Hkv, L = CUTS[cut]
    D, g, t = 128, gen(seed), TT[dtype]
    q, k, v = (randn(g, N, B, n, D).to(t) for n in (H, Hkv, Hkv))
    ks = vs = None
    if fmt == "plain":
        K, V = randn(g, B, Hkv, L, D).to(t), randn(g, B, Hkv, L, D).to(t)
    else:
        (K, V), (ks, vs) = new_state(B, Hkv, L, D, fmt)
        tova.tova_quant_write(tova.tova_quant_config(B, Hkv, D, L, tova.TOVA_DTYPE_FP32, FMT[fmt]), randn(g, L, B, Hkv, D), randn(g, L, B, Hkv, D),
                              L, K, ks, V, vs)
    par = random_parents(N, B, seed)
    cfg = tova.tova_tree_config(B, H, Hkv, D, L, TD[dtype], FMT[fmt], 0.0)
    ws = torch.empty(max(16, tova.tova_tree_workspace_bytes(cfg, L, N)), dtype=torch.uint8, device=DEV)

    def call(q, k, v, K, V, ks, vs):
        out = torch.full((N, B, H, D), 7.0, dtype=t, device=DEV)
        tova.tova_tree_attention(cfg, K, V, L, q, k, v, N, out, ws, parents=par, k_scale=ks, v_scale=vs)
        return out
    real = torch.tensor([[bool(ancestors(par[:, b].tolist())[i]) for b in range(B)] for i in range(N)], device=DEV)
    return (q, k, v, K, V, ks, vs), call, real


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("dtype, fmt", [("bf16", "plain"), ("bf16", "int8"), ("bf16", "e4m3"), ("fp32", "plain"), ("fp32", "e4m3")])
def test_tree_queries_that_are_not_numbers(dtype, fmt, cut):
    """A NaN in a query makes that row NaN, whichever way the call is cut; every other row keeps its bits, padding its zeros."""
    (q, k, v, *state), call, real = cut_inputs(cut, dtype, fmt, 31)
    N, B, H, D = q.shape
    clean = call(q, k, v, *state)
    assert bool(clean.isfinite().all())
    bad = torch.zeros(N, B, H, dtype=torch.bool, device=DEV)
    bad.view(-1)[::5] = True
    q2 = q.clone()
    q2[..., 77] = torch.where(bad, torch.full_like(q[..., 77], math.nan), q[..., 77])
    out = call(q2, k, v, *state)
    nan = bad & real[..., None]
    assert bool(out[nan].isnan().all())
    assert torch.equal(out[~nan], clean[~nan])
    assert bool((out[~real] == 0).all())


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("dtype, fmt", [("bf16", "plain"), ("bf16", "int8"), ("fp32", "plain"), ("fp32", "int8")])
def test_tree_keys_of_the_state_that_are_not_numbers(dtype, fmt, cut):
    """Every key of a stretch of the state is NaN: all that see it come back NaN.  The whole state of a KV head, so that only the
    drafts have finite logits; a stretch that is all that one run of columns has; one that begins and ends within runs."""
    (q, k, v, K, V, ks, vs), call, real = cut_inputs(cut, dtype, fmt, 32)
    L, G = K.shape[2], q.shape[2] // K.shape[1]
    clean = call(q, k, v, K, V, ks, vs)
    for a, b in ((0, L), (min(128, L // 2), min(256, L)), (L // 8, L // 2), (L - 1, L)):
        K2, ks2 = K.clone(), None if ks is None else ks.clone()
        if ks is None:
            K2[0, 0, a:b] = math.nan
        else:
            ks2[0, 0, a:b] = math.nan
        out = call(q, k, v, K2, V, ks2, vs)
        hit = real[..., None].expand(out.shape[:3]).clone()
        hit[:, 1:], hit[:, :, G:] = False, False
        assert bool(out[hit].isnan().all()), (a, b)
        assert torch.equal(out[~hit], clean[~hit])


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("dtype, fmt", [("bf16", "plain"), ("bf16", "int8"), ("fp32", "plain"), ("fp32", "e4m3")])
def test_tree_logits_that_are_all_minus_infinity(dtype, fmt, cut):
    """A row that sees columns, all of them with the logit minus infinity, has no soft-max: NaN by the formula, not the zeros
    of a row that sees nothing."""
    (q, k, v, K, V, ks, vs), call, real = cut_inputs(cut, dtype, fmt, 33)
    N, B, H, D = q.shape
    # component 5 of every key is negative, and an infinite query there makes every logit of its row minus infinity
    k[..., 5] = -1.0
    K[..., 5] = -1
    if fmt == "e4m3":
        K[..., 5] = -72                               # 0xb8: -1
    clean = call(q, k, v, K, V, ks, vs)
    bad = torch.zeros(N, B, H, dtype=torch.bool, device=DEV)
    bad.view(-1)[::3] = True
    q2 = q.clone()
    q2[..., 5] = torch.where(bad, torch.full_like(q[..., 5], math.inf), q[..., 5])
    out = call(q2, k, v, K, V, ks, vs)
    nan = bad & real[..., None]
    assert bool(out[nan].isnan().all())
    assert torch.equal(out[~nan], clean[~nan])
    assert bool((out[~real] == 0).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("V", [300, 40000])
def test_verify_probabilities_that_are_not_finite(dtype, draft, V):
    """An entry that is an infinity or NaN counts as nothing, for its own token and in every sum: the results are those of
    the same rows with zeros there, and every output is written."""
    B, N = 6, 4
    g = gen(41)
    p = (torch.softmax(randn(g, N + 1, B, V), -1)).to(TT[dtype])
    q = (torch.softmax(randn(g, N + 1, B, V), -1)).to(TT[dtype])
    tok = torch.randint(0, V, (N, B), generator=g, device=DEV, dtype=torch.int32)
    tok[1, 4] = tok[0, 4]
    par = torch.tensor([-1, -1, 0, -1], device=DEV, dtype=torch.int32)[:, None].expand(N, B).contiguous()
    u, us = torch.rand(N, B, generator=g, device=DEV), torch.rand(B, generator=g, device=DEV)
    us[0], us[1] = 0.0, 1.0 - 2.0 ** -24
    u[:, 5] = 0.0
    bad_p, bad_q = p.clone(), q.clone()
    bad_p[:, :, 17], bad_p[:, 1, 3], bad_p[:, 2, V - 1], bad_p[:, 3, ::7] = math.inf, -math.inf, math.nan, math.inf
    for i in range(N):                               # tokens of the drafts among them
        bad_p[0, 4, tok[i, 4].long()] = math.inf
        bad_p[:, 5, tok[i, 5].long()] = math.inf
    p = torch.where(bad_p.isfinite(), bad_p, torch.zeros_like(p))
    got, want = run_verify(bad_p, q if draft else None, tok, par, u, us, dtype), run_verify(p, q if draft else None, tok, par, u, us, dtype)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    n, path, out = got
    assert int(n[5]) == 0 and bool((out != 99).all()) and bool((path != 99).all())
    pc, b = [-1, -1, 0, -1], 4
    assert (int(n[b]), path[:, b].tolist(), out[:, b].tolist()) == verify_reference(
        p[:, b].double().tolist(), q[:, b].double().tolist() if draft else None, tok[:, b].tolist(), pc, u[:, b].double().tolist(), float(us[b].double()))
    all_bad = torch.full_like(p, math.inf)           # nothing to draw from
    n, path, out = run_verify(all_bad, q if draft else None, tok, par, u, us, dtype)
    assert bool((n == 0).all()) and bool((out == -1).all()) and bool((path == -1).all())
    if draft:                                        # a draft's entries: the token is not accepted, the rest is the target's
        bad_q[0, :, 17], bad_q[0, :, 20], bad_q[0, :, 23] = math.inf, -math.inf, math.nan
        tok[0], tok[1], tok[3] = 17, 20, 23
        n, path, out = run_verify(p, bad_q, tok, par, u, us, dtype)
        assert bool((n == 0).all()) and bool(((out[0] >= 0) & (out[0] < V)).all()) and bool((out[1:] == -1).all())


@pytest.mark.parametrize("base, rot, orig", [(10000.0, 128, 1), (10000.0, 128, 4), (10000.0, 64, 4), (1.5, 64, 2 ** 31 - 1), (1.01, 128, 100000)])
def test_rope_yarn_where_all_pairs_turn_less_or_more_than_the_blend(base, rot, orig):
    """Contexts so short that even the first pair turns less than once are divided by the factor throughout; with
    frequencies so close together that the last pair still turns more than 32 times nothing is."""
    g = gen(51)
    T, B, H, D, factor = 40, 2, 2, 128, 4.0
    x = randn(g, T, B, H, D)
    r = tova.TovaRope(B, H, H, D, dtype=tova.TOVA_DTYPE_FP32, rotary_dim=rot, base=base, scaling=tova.TOVA_ROPE_YARN, factor=factor, original_context=orig)
    w = base ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64) / rot)
    turns = orig * w / (2 * math.pi)
    assert bool((turns < 1).all()) or bool((turns > 32).all())
    if bool((turns < 1).all()):
        w = w / factor
    y = torch.empty_like(x)
    r.tova_rope_apply(x, None, T, y, None, first_pos=1000)
    pos = 1000 + torch.arange(T, device=DEV)[:, None].expand(T, B)
    check_rope(y, *rope_reference(x, pos, w.to(DEV), 0.1 * math.log(factor) + 1, rot, 0), "fp32")


@pytest.mark.parametrize("cut", CUTS)
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_tree_e4m3_codes_that_are_not_numbers(dtype, cut):
    """0x7f and 0xff are NaN wherever codes are read: a key that holds one makes every row that sees it NaN, a value the one
    component.  (The library's own writer stores neither; codes converted elsewhere may hold them.)"""
    (q, k, v, K, V, ks, vs), call, real = cut_inputs(cut, dtype, "e4m3", 34)
    B, Hkv, L, D = K.shape
    G = q.shape[2] // Hkv
    K[K.view(torch.uint8) % 128 == 127] = 0
    K[0, 0, L // 2], V[0, 0, L // 2] = 126, -2                 # the largest numbers, 0x7e and 0xfe, are none
    clean = call(q, k, v, K, V, ks, vs)
    assert bool(clean.isfinite().all())
    for row, d, code in ((0, 0, 127), (L - 1, 127, -1), (L // 2, 63, 127), (L // 3, 70, -1)):
        K2, V2 = K.clone(), V.clone()
        K2[0, Hkv - 1, row, d] = code
        V2[0, 0, row, d] = code
        V2[B - 1, Hkv - 1, row, (d + 9) % D] = code
        out = call(q, k, v, K2, V, ks, vs)
        hit = real[..., None].expand(out.shape[:3]).clone()
        hit[:, 1:], hit[:, :, :(Hkv - 1) * G] = False, False
        assert bool(out[hit].isnan().all())
        assert torch.equal(out[~hit], clean[~hit])
        out = call(q, k, v, K, V2, ks, vs)
        want = clean.clone()
        want[:, 0, :G, d] = torch.where(real[:, 0, None], torch.full_like(want[:, 0, :G, d], math.nan), want[:, 0, :G, d])
        x = want[:, B - 1, (Hkv - 1) * G:]
        x[..., (d + 9) % D] = torch.where(real[:, B - 1, None], torch.full_like(x[..., 0], math.nan), x[..., (d + 9) % D])
        assert torch.equal(out.isnan(), want.isnan())
        assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))
    back = torch.empty(L, B, Hkv, D, device=DEV)
    cfg = tova.tova_quant_config(B, Hkv, D, L, tova.TOVA_DTYPE_FP32, tova.TOVA_FORMAT_E4M3)
    tova.tova_quant_read(cfg, K2, ks, V2, vs, L, back, None)
    assert int(back.isnan().sum()) == 1 and bool(back[row, 0, Hkv - 1, d].isnan())


@pytest.mark.parametrize("fmt", ["plain", "int8"])
@pytest.mark.parametrize("N", [1, 6, 14, 30])
def test_tree_results_under_other_cuts(fmt, N):
    """The same sequence under other bounds on the length, and beside other sequences: the columns are cut differently, so
    fp32 sums come in another order and a weight may be rounded to bf16 against another reference, and that is all."""
    H, Hkv, D, L, cap = 8, 2, 128, 777, 20000
    g = gen(61)
    one = [randn(g, N, 1, n, D).bfloat16() for n in (H, Hkv, Hkv)]
    Kf, Vf = randn(g, L, 1, Hkv, D).bfloat16(), randn(g, L, 1, Hkv, D).bfloat16()
    got, ref = [], None
    for B, n_live in ((1, L), (1, 3000), (1, cap), (2, cap), (9, 5000), (150, 1000)):
        c = min(cap, n_live)
        q, k, v = (torch.cat([x, randn(g, N, B - 1, x.shape[2], D).bfloat16()], 1).contiguous() for x in one)
        Kb, Vb = (torch.cat([x, randn(g, L, B - 1, Hkv, D).bfloat16()], 1) for x in (Kf, Vf))
        ks = vs = None
        if fmt == "plain":
            K, V = (torch.zeros(B, Hkv, c, D, dtype=torch.bfloat16, device=DEV) for _ in range(2))
            K[:, :, :L], V[:, :, :L] = Kb.permute(1, 2, 0, 3), Vb.permute(1, 2, 0, 3)
            Kd, Vd = K[:1, :, :L].double(), V[:1, :, :L].double()
        else:
            (K, V), (ks, vs) = new_state(B, Hkv, c, D, fmt)
            tova.tova_quant_write(tova.tova_quant_config(B, Hkv, D, c, tova.TOVA_DTYPE_BF16, FMT[fmt]), Kb.contiguous(), Vb.contiguous(), L, K, ks, V, vs)
            Kd, Vd = K[:1, :, :L].double() * ks[:1, :, :L, None].double(), V[:1, :, :L].double() * vs[:1, :, :L, None].double()
        lens = torch.tensor([L] + [max(1, (L * b) // B) for b in range(1, B)], dtype=torch.int32, device=DEV)
        cfg = tova.tova_tree_config(B, H, Hkv, D, c, tova.TOVA_DTYPE_BF16, FMT[fmt], 0.0)
        ws = torch.empty(max(16, tova.tova_tree_workspace_bytes(cfg, c, N)), dtype=torch.uint8, device=DEV)
        out = torch.empty_like(q)
        tova.tova_tree_attention(cfg, K, V, c, q, k, v, N, out, ws, lens=lens, k_scale=ks, v_scale=vs)
        got.append(out[:, :1].double())
        ref = ref or tree_reference(*one, Kd, Vd, [L], None)
    want, wv, reach, _ = ref
    # Either result is off the exact one by the tolerance, and by what the rounded weights' sum adds: with weights w (1 + d),
    # |d| <= 2^-8, the result moves by sum w d (v - out) / (1 + sum w d), at most 2^-8 (sum w |v| + |out|) / (1 - 2^-8), of which
    # tree_tolerance counts the first term.
    tol = tree_tolerance("bf16", D, L + N, want, wv, reach) + 2.0 ** -8 * 1.01 * want.abs()
    for x in got:
        assert bool(((x - want).abs() <= tol).all())
        assert bool(((x - got[0]).abs() <= 2 * tol).all())


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("N, B, V, chain", [(6, 2, 32769, False), (9, 2, 50001, False), (3, 1, 128256, True), (20, 2, 131072, False)])
def test_verify_large_vocabularies(dtype, draft, N, B, V, chain):
    """Rows longer than the registers of a cluster hold are read again for every sum."""
    p, q, tok, par, pc, u, us = verify_inputs(N, B, V, dtype, N + V, chain, draft)
    n, path, out = run_verify(p, q, tok, par, u, us, dtype)
    for b in range(B):
        want = verify_reference(p[:, b].double().tolist(), None if q is None else q[:, b].double().tolist(), tok[:, b].tolist(),
                                pc[:, b].tolist(), u[:, b].double().tolist(), float(us[b].double()))
        assert (int(n[b]), path[:, b].tolist(), out[:, b].tolist()) == want, b
