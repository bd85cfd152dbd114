"""Work of the operators around the decode step: rotary positions, the 8-bit state, attention of drafted tokens over a
state, verification of drafted tokens.

`run` computes a case either in plain torch operations (own = False) or through the library's entry points (own = True)
on the same inputs; `exact` gives the same outputs from the definitions in 64 bits.  Layer shapes are those of the
package's workloads (LLaMA-2-7B, Mistral-7B, Yi-6B layers) and small generic ones.  Token-major layouts throughout:
[T,B,...] for prompt tokens, [N,B,...] for the N drafted tokens of every sequence.
"""
import math

import torch

own = False

DEV = "cuda:0"
QMAX = {"int8": 127.0, "e4m3": 448.0}


# ----------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one decode step's new token of 64 sequences, LLaMA-2-7B heads: the smallest call, once per layer and step
        dict(name="rope_step", op="rope", T=1, B=64, H=32, Hkv=32, D=128, rot=128, dtype="bf16", layout="half",
             scaling="none", base=10000.0, factor=1.0, far=4096, listed_positions=False, fused=True, inverse=False),
        # a long prompt of four sequences, GQA heads cut out of one fused projection, context stretched 8 times
        dict(name="rope_prompt", op="rope", T=4096, B=4, H=32, Hkv=8, D=128, rot=128, dtype="bf16", layout="half",
             scaling="bands", base=10000.0, factor=8.0, far=32768, listed_positions=False, fused=True, inverse=False),
        # the gradient's way back of a partly rotated head in adjacent pairs, odd length, fp32
        dict(name="rope_back_fp32", op="rope", T=517, B=3, H=32, Hkv=4, D=128, rot=64, dtype="fp32",
             layout="interleaved", scaling="yarn", base=10000.0, factor=4.0, far=900000, listed_positions=True,
             fused=False, inverse=True),
        # the rows of one decode step go into 32 sequences' states, each into the slot that its eviction freed
        dict(name="quant_write_step", op="qwrite", T=1, B=32, Hkv=8, D=128, cap=1024, dtype="bf16", format="e4m3",
             slots=True),
        # a whole prompt goes into the state
        dict(name="quant_write_prompt", op="qwrite", T=4096, B=8, Hkv=8, D=128, cap=4096, dtype="bf16", format="int8",
             slots=False),
        # a state is read back in the model's type
        dict(name="quant_read_state", op="qread", T=4001, B=4, Hkv=32, D=128, cap=4096, dtype="bf16", format="e4m3",
             slots=False),
        # one plain step (a tree of one node) of one sequence over an 8-bit state: latency
        dict(name="tree_single_int8", op="tree", B=1, H=32, Hkv=8, D=128, L=1000, cap=1024, N=1, dtype="bf16",
             format="int8", tree="chain", ragged=False),
        # 8 chained drafts of 64 sequences, MHA
        dict(name="tree_chain_mha", op="tree", B=64, H=32, Hkv=32, D=128, L=1024, cap=1024, N=8, dtype="bf16",
             format="plain", tree="chain", ragged=True),
        # a tree of 63 drafts of 32 sequences, GQA
        dict(name="tree_63_gqa", op="tree", B=32, H=32, Hkv=8, D=128, L=4000, cap=4096, N=63, dtype="bf16",
             format="plain", tree="random", ragged=True),
        # the same kind over an 8-bit state, long, few sequences, wide query groups
        dict(name="tree_25_long_e4m3", op="tree", B=4, H=32, Hkv=4, D=128, L=16001, cap=16384, N=25, dtype="bf16",
             format="e4m3", tree="random", ragged=False),
        # a chain of five drafts of one sequence
        dict(name="verify_chain", op="verify", B=1, N=5, V=32000, dtype="fp32", tree="chain", draft=True),
        # trees of 63 drafts of 32 sequences
        dict(name="verify_tree", op="verify", B=32, N=63, V=32000, dtype="fp32", tree="random", draft=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges; its long axis is halved while it would be more work than the largest listed cases."""
    top = [max(work(c)[k] for c in listed()) for k in ("bytes", "flops")]
    case = _draw(rng)
    axis = {"tree": "L", "verify": "B"}.get(case["op"], "T")
    while case[axis] > 1 and any(work(case)[k] > t for k, t in zip(("bytes", "flops"), top)):
        case[axis] = (case[axis] + 1) // 2
        if axis == "L":
            case["cap"] = case["L"] + 5
    return case


def _draw(rng):
    op = rng.choice(["rope", "qwrite", "qread", "tree", "tree", "tree", "verify", "verify"])
    if op == "rope":
        H, Hkv = rng.choice([(32, 32), (32, 8), (32, 4), (8, 2), (4, 4)])
        D = rng.choice([64, 128, 128])
        B = _log(rng, 1, 64)
        T = _log(rng, 1, max(1, 16384 * 40 // (B * (H + Hkv))))
        dtype = rng.choice(["bf16", "bf16", "fp32"])
        return dict(op="rope", T=T, B=B, H=H, Hkv=Hkv, D=D, rot=rng.choice([D, D, D // 2, D // 4 * 3]), dtype=dtype,
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "ntk", "yarn", "bands"]),
                    base=rng.choice([10000.0, 500000.0]), factor=rng.choice([2.0, 4.0, 8.0]), far=_log(rng, 4096, 1000000),
                    listed_positions=rng.random() < 0.5, fused=rng.random() < 0.5, inverse=rng.random() < 0.3)
    if op in ("qwrite", "qread"):
        Hkv, D = rng.choice([32, 8, 4]), rng.choice([64, 128])
        B = _log(rng, 1, 32)
        cap = _log(rng, 33, max(40, 262144 // (B * Hkv)))
        return dict(op=op, T=min(cap, _log(rng, 1, cap)), B=B, Hkv=Hkv, D=D, cap=cap,
                    dtype=rng.choice(["bf16", "bf16", "fp32"]), format=rng.choice(["int8", "e4m3"]),
                    slots=rng.random() < 0.5)
    if op == "tree":
        H, Hkv = rng.choice([(32, 32), (32, 8), (32, 4), (8, 2), (4, 4)])
        D = rng.choice([64, 128, 128])
        dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
        B = _log(rng, 1, 64)
        N = _log(rng, 1, 200)
        L = _log(rng, 1, 32768 if dtype == "bf16" else 4096)
        return dict(op="tree", B=B, H=H, Hkv=Hkv, D=D, L=L, cap=L + rng.choice([0, 1, 7, 64]), N=N, dtype=dtype,
                    format=rng.choice(["plain", "plain", "int8", "e4m3"]), tree=rng.choice(["chain", "random", "random"]),
                    ragged=rng.random() < 0.6)
    V = _log(rng, 1000, 64000)
    N = _log(rng, 1, 64)
    B = min(_log(rng, 1, 64), max(1, 64 * 32 * 32000 // ((N + 1) * V)))
    return dict(op="verify", B=B, N=N, V=V, dtype=rng.choice(["fp32", "fp32", "bf16"]),
                tree=rng.choice(["chain", "random"]), draft=rng.random() < 0.75)


# ---------------------------------------------------------------------------------------------------- inputs

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _lens(case):
    """Rows each sequence holds: all alike, or spread between a third of L and L."""
    B, L = case["B"], case["L"]
    if not case["ragged"]:
        return [L] * B
    return [L - (2 * L * b) // (3 * B) for b in range(B)]


def _parents(case, seed):
    """[N,B] on the CPU: chains, or random trees (a few recent nodes may be the parent) whose last nodes are padding in
    some sequences (-2)."""
    N, B = case["N"], case["B"]
    if case["tree"] == "chain":
        return torch.arange(-1, N - 1, dtype=torch.int32)[:, None].repeat(1, B).contiguous()
    g = torch.Generator().manual_seed(seed * 7 + 3)
    i = torch.arange(N)[:, None]
    back = 1 + (torch.rand(N, B, generator=g) * torch.clamp(i + 1, max=6)).floor().long()
    par = torch.clamp(i - back, min=-1)
    pad = (torch.rand(B, generator=g) < 0.25).long() * (N // 8)
    par = torch.where(i >= N - pad[None, :], torch.full_like(par, -2), par)
    return par.to(torch.int32).contiguous()


def _depths(par):
    """Depth of every node (1 for children of the root, 0 for padding), as lists [N][B]."""
    N, B = par.shape
    p, d = par.tolist(), []
    for i in range(N):
        d.append([0 if p[i][b] < -1 else 1 if p[i][b] == -1 else (d[p[i][b]][b] + 1 if d[p[i][b]][b] else 0)
                  for b in range(B)])
    return d


def _rope_frequencies(case):
    """Inverse frequencies in double and the factor on cosine and sine.  Definitions: base^(-2i/rot); "linear": all
    divided by the factor; "ntk": base times factor^(rot/(rot-2)); "yarn" (arXiv 2309.00071): between the pairs that
    turn beta_fast = 32 and beta_slow = 1 times over the original context, from plain to divided, cosine and sine times
    0.1 ln(factor) + 1; "bands": by wavelength, plain below original/4, divided above original, blended between."""
    rot, base, f, kind = case["rot"], case["base"], case["factor"], case["scaling"]
    orig = max(1, int(case["far"] / f))
    if kind == "ntk":
        base = base * f ** (rot / (rot - 2))
    inv = [base ** (-2.0 * i / rot) for i in range(rot // 2)]
    att = 1.0
    if kind == "linear":
        inv = [w / f for w in inv]
    elif kind == "yarn":
        at = lambda turns: rot * math.log(orig / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rot - 1)
        if hi == lo:
            hi = lo + 0.001
        ramp = [min(1.0, max(0.0, (i - lo) / (hi - lo))) for i in range(rot // 2)]
        inv = [w / f * r + w * (1 - r) for w, r in zip(inv, ramp)]
        att = 0.1 * math.log(f) + 1.0 if f > 1 else 1.0
    elif kind == "bands":
        out = []
        for w in inv:
            wave = 2 * math.pi / w
            if wave < orig / 4.0:
                out.append(w)
            elif wave > orig:
                out.append(w / f)
            else:
                s = (orig / wave - 1.0) / (4.0 - 1.0)
                out.append((1 - s) * w / f + s * w)
        inv = out
    return inv, att, orig


def _quantise(x, fmt):
    """Codes and scales of rows x[..., D]: scale = fp32(amax / qmax), code = round(fp32(x * fp32(qmax / amax)))."""
    x = x.float()
    qmax = QMAX[fmt]
    amax = x.abs().amax(-1, keepdim=True)
    top = torch.full_like(amax, qmax)           # (a tensor: a quotient with a plain number is formed by its reciprocal)
    scale = amax / top
    r = torch.where(amax > 0, top / amax, torch.zeros_like(amax))
    y = x * r
    if fmt == "int8":
        return torch.round(y).clamp(-127, 127).to(torch.int8), scale.squeeze(-1)
    return y.clamp(-448, 448).to(torch.float8_e4m3fn), scale.squeeze(-1)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    op, B = case["op"], case["B"]
    s = {"case": case, "op": op}
    if own:
        import paper_2401_06104_b200 as tova
        s["tova"] = tova
    t = _type(case["dtype"])
    if op == "rope":
        T, H, Hkv, D = case["T"], case["H"], case["Hkv"], case["D"]
        if case["fused"]:       # q and k are slices of one projection's output
            qkv = (rnd(T, B, (H + 2 * Hkv) * D) * math.sqrt(2.0)).to(t)
            q = qkv[..., :H * D].unflatten(-1, (H, D))
            k = qkv[..., H * D:(H + Hkv) * D].unflatten(-1, (Hkv, D))
        else:
            q, k = rnd(T, B, H, D).to(t), rnd(T, B, Hkv, D).to(t)
        first = int(torch.randint(0, max(1, case["far"] - T), (1,), generator=torch.Generator().manual_seed(seed)))
        s.update(q=q, k=k, first=first, pos=None)
        if case["listed_positions"]:
            s["pos"] = torch.randint(0, case["far"], (T, B), generator=g, device=DEV, dtype=torch.int32)
        inv, att, orig = _rope_frequencies(case)
        s.update(inv=torch.tensor(inv, dtype=torch.float64, device=DEV), att=att)
        if own:
            kinds = dict(none=tova.TOVA_ROPE_PLAIN, linear=tova.TOVA_ROPE_LINEAR, ntk=tova.TOVA_ROPE_NTK,
                         yarn=tova.TOVA_ROPE_YARN, bands=tova.TOVA_ROPE_BANDS)
            s["rope"] = tova.TovaRope(B, H, Hkv, D, dtype=tova.TOVA_DTYPE_BF16 if t == torch.bfloat16 else tova.TOVA_DTYPE_FP32,
                                      rotary_dim=case["rot"], layout=tova.TOVA_ROPE_HALF if case["layout"] == "half" else tova.TOVA_ROPE_INTERLEAVED,
                                      base=case["base"], scaling=kinds[case["scaling"]], factor=case["factor"], original_context=orig)
            s["qo"] = torch.empty(T, B, H, D, dtype=t, device=DEV)
            s["ko"] = torch.empty(T, B, Hkv, D, dtype=t, device=DEV)
    elif op in ("qwrite", "qread"):
        T, Hkv, D, cap, fmt = case["T"], case["Hkv"], case["D"], case["cap"], case["format"]
        ct = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
        if op == "qread":
            s["kq"], s["ks"] = _quantise(rnd(B, Hkv, cap, D), fmt)
            s["vq"], s["vs"] = _quantise(rnd(B, Hkv, cap, D), fmt)
            s["k"] = torch.empty(T, B, Hkv, D, dtype=t, device=DEV)
            s["v"] = torch.empty_like(s["k"])
        else:
            for n in ("kq", "vq"):
                s[n] = torch.zeros(B, Hkv, cap, D, dtype=torch.int8, device=DEV).view(ct)
                s[n[0] + "s"] = torch.zeros(B, Hkv, cap, device=DEV)
            s["k"], s["v"] = (rnd(T, B, Hkv, D) * math.sqrt(2.0)).to(t), rnd(T, B, Hkv, D).to(t)
        if case["slots"]:       # every sequence has an order of its own
            s["slots"] = torch.argsort(torch.rand(B, cap, generator=g, device=DEV), dim=1)[:, :T].t().to(torch.int32).contiguous()
        else:
            s["slots"] = None
        if own:
            s["cfg"] = tova.tova_quant_config(B, Hkv, D, cap, tova.TOVA_DTYPE_BF16 if t == torch.bfloat16 else tova.TOVA_DTYPE_FP32,
                                              tova.TOVA_FORMAT_INT8 if fmt == "int8" else tova.TOVA_FORMAT_E4M3)
    elif op == "tree":
        H, Hkv, D, cap, N, fmt = case["H"], case["Hkv"], case["D"], case["cap"], case["N"], case["format"]
        s["q"], s["k"], s["v"] = (rnd(N, B, H, D) * 1.3).to(t), rnd(N, B, Hkv, D).to(t), rnd(N, B, Hkv, D).to(t)
        K, V = rnd(B, Hkv, cap, D), rnd(B, Hkv, cap, D)
        K[:, :, 0] *= 3.0       # the first token stays attended
        s["ks"] = s["vs"] = None
        if fmt == "plain":
            s["K"], s["V"] = K.to(t), V.to(t)
        else:
            (s["K"], s["ks"]), (s["V"], s["vs"]) = _quantise(K, fmt), _quantise(V, fmt)
        lens = _lens(case)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV) if case["ragged"] else None
        s["par"] = None if case["tree"] == "chain" else _parents(case, seed).to(DEV)
        if own:
            f = dict(plain=tova.TOVA_FORMAT_PLAIN, int8=tova.TOVA_FORMAT_INT8, e4m3=tova.TOVA_FORMAT_E4M3)[fmt]
            s["cfg"] = tova.tova_tree_config(B, H, Hkv, D, cap, tova.TOVA_DTYPE_BF16 if t == torch.bfloat16 else tova.TOVA_DTYPE_FP32, f, 0.0)
            s["ws"] = torch.empty(max(16, tova.tova_tree_workspace_bytes(s["cfg"], case["L"], N)), dtype=torch.uint8, device=DEV)
            s["out"] = torch.empty(N, B, H, D, dtype=t, device=DEV)
    else:
        N, V = case["N"], case["V"]
        par = _parents(case, seed)
        s["par"] = None if case["tree"] == "chain" else par.to(DEV)
        dep = _depths(par)
        s["depth"] = max(max(r) for r in dep)
        s["wide"] = 6 if case["tree"] != "chain" else 1            # children of a node at most
        logits = rnd(N + 1, B, V) * 2.5
        s["p"] = torch.softmax(logits, -1).to(t)
        q = torch.softmax(logits + 0.8 * rnd(N + 1, B, V), -1).to(t)
        del logits
        # every node's token is drawn from its parent's draft distribution (the largest q / exponential)
        row = torch.clamp(par.to(DEV).long() + 1, min=0)
        toks = [torch.argmax(q[row[i], torch.arange(B, device=DEV)].float() /
                             torch.empty(B, V, device=DEV).exponential_(generator=g), -1) for i in range(N)]
        s["tok"] = torch.stack(toks).to(torch.int32)
        s["q"] = q if case["draft"] else None
        s["u"] = torch.rand(N, B, generator=g, device=DEV)
        s["us"] = torch.rand(B, generator=g, device=DEV)
        if own:
            s["cfg"] = tova.tova_verify_config(B, N, V, tova.TOVA_DTYPE_BF16 if t == torch.bfloat16 else tova.TOVA_DTYPE_FP32, 0)
            s["n"] = torch.empty(B, dtype=torch.int32, device=DEV)
            s["path"] = torch.empty(N, B, dtype=torch.int32, device=DEV)
            s["toks"] = torch.empty(N + 1, B, dtype=torch.int32, device=DEV)
    return s


# --------------------------------------------------------------------------------------------- the operators

def run(s):
    if s["op"] == "rope":
        return _run_rope(s)
    if s["op"] == "qwrite":
        return _run_write(s)
    if s["op"] == "qread":
        return _run_read(s)
    if s["op"] == "tree":
        return _run_tree(s)
    return _run_verify(s)


def _turn(x, c, si, rot, layout):
    """x [T,B,heads,D] turned by the angles whose cosines and sines are c, si [T,B|1,1,rot/2]."""
    x = x.float()
    r, rest = x[..., :rot], x[..., rot:]
    if layout == "half":
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat([a * c - b * si, b * c + a * si], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * c - b * si, b * c + a * si], -1).flatten(-2)
    return torch.cat([r, rest], -1)


def _run_rope(s):
    c = s["case"]
    if own:
        s["rope"].tova_rope_apply(s["q"], s["k"], c["T"], s["qo"], s["ko"], positions=s["pos"], first_pos=s["first"],
                                  inverse=c["inverse"])
        return s["qo"], s["ko"]
    pos = s["pos"] if s["pos"] is not None else s["first"] + torch.arange(c["T"], device=DEV)[:, None]
    ang = pos.double()[..., None] * s["inv"]                       # far positions: the angle in 64 bits
    if c["inverse"]:
        ang = -ang
    co, si = (torch.cos(ang) * s["att"]).float()[:, :, None], (torch.sin(ang) * s["att"]).float()[:, :, None]
    return tuple(_turn(x, co, si, c["rot"], c["layout"]).to(x.dtype) for x in (s["q"], s["k"]))


def _run_write(s):
    c = s["case"]
    if own:
        s["tova"].tova_quant_write(s["cfg"], s["k"], s["v"], c["T"], s["kq"], s["ks"], s["vq"], s["vs"], slots=s["slots"])
        return s["kq"], s["ks"], s["vq"], s["vs"]
    T, B = c["T"], c["B"]
    slots = s["slots"].long() if s["slots"] is not None else torch.arange(T, device=DEV)[:, None].expand(T, B)
    b = torch.arange(B, device=DEV)[None].expand(T, B)
    kc, ksc = _quantise(s["k"], c["format"])
    vc, vsc = _quantise(s["v"], c["format"])
    s["kq"].view(torch.int8)[b, :, slots] = kc.view(torch.int8)
    s["vq"].view(torch.int8)[b, :, slots] = vc.view(torch.int8)
    s["ks"][b, :, slots] = ksc
    s["vs"][b, :, slots] = vsc
    return s["kq"], s["ks"], s["vq"], s["vs"]


def _run_read(s):
    c = s["case"]
    if own:
        s["tova"].tova_quant_read(s["cfg"], s["kq"], s["ks"], s["vq"], s["vs"], c["T"], s["k"], s["v"], slots=s["slots"])
        return s["k"], s["v"]
    T, B = c["T"], c["B"]
    slots = s["slots"].long() if s["slots"] is not None else torch.arange(T, device=DEV)[:, None].expand(T, B)
    b = torch.arange(B, device=DEV)[None].expand(T, B)
    got = []
    got.append((s["kq"].view(torch.int8)[b, :, slots].view(s["kq"].dtype).float() * s["ks"][b, :, slots][..., None]).to(s["k"].dtype))
    got.append((s["vq"].view(torch.int8)[b, :, slots].view(s["vq"].dtype).float() * s["vs"][b, :, slots][..., None]).to(s["v"].dtype))
    return tuple(got)


def _ancestors(par, N, B):
    """[B,N,N] bool: node j is node i itself or above it; rows of padding nodes are empty."""
    if par is None:
        return torch.ones(N, N, dtype=torch.bool, device=DEV).tril().expand(B, N, N)
    p = par.t().long()                                             # [B,N]
    i = torch.arange(N, device=DEV)
    up = (p[:, :, None] == i) & (p >= 0)[:, :, None]               # direct parent
    m = (up | torch.eye(N, dtype=torch.bool, device=DEV)).float()
    for _ in range(max(1, (N - 1).bit_length())):                  # every pass doubles the reach
        m = (torch.matmul(m, m) > 0).float()
    bad = ((p < -1) | (p >= i)).float()[:, :, None]
    return (m > 0) & (torch.matmul(m, bad) == 0)


def _run_tree(s):
    c = s["case"]
    N, B, H, Hkv, D, L = c["N"], c["B"], c["H"], c["Hkv"], c["D"], c["L"]
    if own:
        s["tova"].tova_tree_attention(s["cfg"], s["K"], s["V"], L, s["q"], s["k"], s["v"], N, s["out"], s["ws"],
                                      parents=s["par"], lens=s["lens"], k_scale=s["ks"], v_scale=s["vs"])
        return s["out"]
    K, V = s["K"][:, :, :L].float(), s["V"][:, :, :L].float()
    if s["ks"] is not None:
        K, V = K * s["ks"][:, :, :L, None], V * s["vs"][:, :, :L, None]
    K = torch.cat([K, s["k"].float().permute(1, 2, 0, 3)], 2)      # [B,Hkv,L+N,D]
    V = torch.cat([V, s["v"].float().permute(1, 2, 0, 3)], 2)
    q = s["q"].float().permute(1, 2, 0, 3).reshape(B, Hkv, (H // Hkv) * N, D)
    x = torch.matmul(q, K.transpose(2, 3)) * (1.0 / math.sqrt(D))
    x = x.view(B, Hkv, H // Hkv, N, L + N)
    tree = _ancestors(s["par"], N, B)
    live = tree.any(-1)                                            # padding nodes attend to nothing
    rows = torch.arange(L, device=DEV)
    held = (rows < s["lens"][:, None]) if s["lens"] is not None else torch.ones(B, L, dtype=torch.bool, device=DEV)
    see = torch.cat([held[:, None, :] & live[:, :, None], tree], 2)[:, None, None]
    x = x.masked_fill(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    o = torch.matmul(e.view(B, Hkv, -1, L + N), V).view(B, H, N, D)
    o = o / e.sum(-1).view(B, H, N, 1).clamp_min(1e-30)
    return o.permute(2, 0, 1, 3).to(s["q"].dtype).contiguous()


def _run_verify(s):
    c = s["case"]
    N, B = c["N"], c["B"]
    if own:
        s["tova"].tova_verify_draft(s["cfg"], s["p"], s["q"], s["tok"], s["u"], s["us"], s["n"], s["path"], s["toks"],
                                    parents=s["par"])
        return s["n"], s["path"], s["toks"]
    # which child every row of the tree would take, from scalars: row r stands for the root (0) or node r - 1
    bi = torch.arange(B, device=DEV)
    node = torch.arange(N, device=DEV)[:, None].expand(N, B)
    par = s["par"].long() if s["par"] is not None else node - 1
    real = (par >= -1) & (par < node)
    row = torch.where(real, par + 1, torch.zeros_like(par))
    tok = s["tok"].long()
    P, Q = s["p"], s["q"]
    px = P[row, bi, tok].double()
    qx = Q[row, bi, tok].double() if Q is not None else torch.ones_like(px)
    older = real[:, None] & real[None] & (par[:, None] == par[None]) & (node[:, None] > node[None])   # [n,m]: m before n
    rank = older.sum(1)
    S = torch.zeros(N + 1, B, dtype=torch.float64, device=DEV)
    Z = torch.ones_like(S)
    take = torch.full((N + 1, B), -1, dtype=torch.long, device=DEV)
    kids = torch.zeros(N + 2, B, dtype=torch.long, device=DEV).scatter_add_(0, torch.where(real, par + 1, torch.full_like(par, N + 1)), real.long())[:N + 1]
    if Q is None:
        again = (older & (tok[:, None] == tok[None])).any(1)
        px = torch.where(again, torch.zeros_like(px), px)
        before = 1.0 - (older * px[None]).sum(1)
    for j in range(s["wide"]):
        if j and Q is not None:
            S = torch.where(kids >= j, S + Z, S)
            Z = torch.clamp(P.double() - S[..., None] * Q, min=0).sum(-1)
        if Q is not None:
            Sx, Zx = S[row, bi], Z[row, bi]
            yes = s["u"].double() * qx * Zx < torch.clamp(px - Sx * qx, min=0)
        else:
            yes = s["u"].double() * before < px
        yes = yes & real & (rank == j)
        slot = torch.where(yes, row, torch.full_like(row, N + 1))
        got = torch.full((N + 2, B), -1, dtype=torch.long, device=DEV).scatter_(0, slot, node)[:N + 1]
        take = torch.where(take < 0, got, take)
    if Q is not None:
        S = torch.where(kids >= s["wide"], S + Z, S)
    # the walk
    cur = torch.zeros(B, dtype=torch.long, device=DEV)
    path = []
    for _ in range(s["depth"]):
        nxt = torch.where(cur >= 0, take[cur.clamp_min(0), bi], cur)
        path.append(nxt)
        cur = torch.where(nxt >= 0, nxt + 1, torch.minimum(cur, -1 - cur))     # a stopped walk keeps its row as -1 - row
    at = torch.where(cur >= 0, cur, -1 - cur)
    path = torch.stack([torch.where(p >= 0, p, torch.full_like(p, -1)) for p in path])
    count = (path >= 0).sum(0)
    # the last token
    last = P[at, bi].double()
    if Q is not None:
        rest = torch.clamp(last - S[at, bi][:, None] * Q[at, bi], min=0)
    else:
        tried = real & (row == at)
        hide = torch.zeros(B, last.shape[-1], device=DEV).scatter_add_(1, torch.where(tried, tok, torch.zeros_like(tok)).t(), tried.t().float())
        rest = torch.where(hide > 0, torch.zeros_like(last), last)
    last = torch.where((rest.sum(-1) > 0)[:, None], rest, last)
    cum = torch.cumsum(last, -1)
    hit = cum > (s["us"].double() * cum[:, -1])[:, None]
    some = last > 0
    V = last.shape[-1]
    final = torch.where(hit.any(-1), hit.long().argmax(-1), V - 1 - some.flip(-1).long().argmax(-1))
    final = torch.where(some.any(-1), final, torch.full_like(final, -1))
    nodes = torch.full((N + 1, B), -1, dtype=torch.long, device=DEV)
    nodes[:path.shape[0]] = path
    toks = torch.where(nodes >= 0, torch.cat([tok, tok[:1]])[nodes.clamp_min(0), bi], nodes)
    toks[count, bi] = final
    return count.to(torch.int32), nodes[:N].to(torch.int32).contiguous(), toks.to(torch.int32)


def work(case):
    op, B = case["op"], case["B"]
    E = 2 if case["dtype"] == "bf16" else 4
    if op == "rope":
        n = case["T"] * B * (case["H"] + case["Hkv"])
        return {"bytes": 2.0 * n * case["D"] * E + (4.0 * case["T"] * B if case["listed_positions"] else 0), "flops": 3.0 * n * case["rot"]}
    if op in ("qwrite", "qread"):
        rows = 2.0 * case["T"] * B * case["Hkv"]
        return {"bytes": rows * (case["D"] * (E + 1) + 4) + (4.0 * case["T"] * B if case["slots"] else 0), "flops": 3.0 * rows * case["D"]}
    if op == "tree":
        H, Hkv, D, N = case["H"], case["Hkv"], case["D"], case["N"]
        held = float(sum(_lens(case)))
        row = D * E if case["format"] == "plain" else D + 4
        return {"bytes": 2 * held * Hkv * row + B * N * D * E * (2.0 * H + 2.0 * Hkv), "flops": 4.0 * held * N * H * D}
    # what the walk cannot do without: the row that the last token is drawn from, of one or both distributions
    return {"bytes": float(B) * case["V"] * E * (2 if case["draft"] else 1) + 20.0 * B * case["N"], "flops": 4.0 * B * case["V"]}


# --------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    op, B = case["op"], case["B"]
    if op == "rope":
        # a pair is a complex number, the rotation a product with att * exp(i * angle)
        pos = s["pos"].double() if s["pos"] is not None else (s["first"] + torch.arange(case["T"], device=DEV).double())[:, None].expand(-1, B)
        ang = torch.einsum("tb,i->tbi", pos, s["inv"]) * (-1.0 if case["inverse"] else 1.0)
        w = torch.polar(torch.full_like(ang, s["att"]), ang)[:, :, None]
        got = []
        for x in (s["q"], s["k"]):
            y = x.double().clone()
            h = case["rot"] // 2
            lo, hi = (slice(0, h), slice(h, 2 * h)) if case["layout"] == "half" else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))
            z = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * w
            y[..., lo], y[..., hi] = z.real, z.imag
            got.append(y)
            del z
        return tuple(got)
    if op == "qwrite":
        # scale = fp32(amax / qmax) and code = nearest(fp32(x * fp32(qmax / amax))): the two roundings to fp32 belong
        # to the definition (a quotient or a product of two fp32 values, formed in 64 bits and rounded once more, is
        # the correctly rounded fp32 one)
        qmax = QMAX[case["format"]]
        for n in "kv":
            x = s[n].double()
            amax = x.abs().amax(-1)
            top = torch.full_like(amax, qmax)
            sc = (amax / top).float()
            r = torch.where(amax > 0, top / amax, torch.zeros_like(amax)).float().double()
            y = (x * r[..., None]).float().double()
            code = torch.round(y) if case["format"] == "int8" else _nearest_e4m3(y)
            full = torch.zeros(*s[n + "q"].shape, dtype=torch.float64, device=DEV)
            fs = s[n + "s"].double()
            if s["slots"] is None:
                full[:, :, :case["T"]] = code.permute(1, 2, 0, 3)
                fs[:, :, :case["T"]] = sc.double().permute(1, 2, 0)
            else:
                at = s["slots"].t().long()[:, None].expand(-1, case["Hkv"], -1)
                full.scatter_(2, at[..., None].expand(-1, -1, -1, case["D"]), code.permute(1, 2, 0, 3))
                fs.scatter_(2, at, sc.double().permute(1, 2, 0))
            s[n + "q64"], s[n + "s64"] = full, fs
        whole = case["format"] == "int8"
        return (None if whole else s["kq64"]), s["ks64"], (None if whole else s["vq64"]), s["vs64"]
    if op == "qread":
        got = []
        for n in "kv":
            x = s[n + "q"].to(torch.float32).double() * s[n + "s"].double()[..., None]
            if s["slots"] is None:
                x = x[:, :, :case["T"]].permute(2, 0, 1, 3)
            else:
                x = torch.stack([x[b].index_select(1, s["slots"][:, b].long()) for b in range(B)]).permute(2, 0, 1, 3)
            got.append(x)
        return tuple(got)
    if op == "tree":
        N, H, Hkv, D = case["N"], case["H"], case["Hkv"], case["D"]
        par = _parents(case, seed).tolist()
        lens = _lens(case)
        out = torch.zeros(N, B, H, D, dtype=torch.float64, device=DEV)
        group = max(1, int(2e8) // max(1, N * (H // Hkv) * (case["L"] + N)))
        for b in range(B):
            # the ancestors of every node by walking up
            see = torch.zeros(N, N, dtype=torch.bool)
            for i in range(N):
                j, ok = i, True
                chain = []
                while j >= 0 and ok:
                    chain.append(j)
                    ok = -1 <= par[j][b] < j
                    j = par[j][b]
                if ok:
                    see[i, chain] = True
            see = see.to(DEV)
            n = lens[b]
            for h0 in range(0, Hkv, group):
                h1 = min(Hkv, h0 + group)
                K, V = s["K"][b, h0:h1, :n].to(torch.float32).double(), s["V"][b, h0:h1, :n].to(torch.float32).double()
                if s["ks"] is not None:
                    K, V = K * s["ks"][b, h0:h1, :n, None].double(), V * s["vs"][b, h0:h1, :n, None].double()
                K = torch.cat([K, s["k"][:, b, h0:h1].double().transpose(0, 1)], 1)
                V = torch.cat([V, s["v"][:, b, h0:h1].double().transpose(0, 1)], 1)
                q = s["q"][:, b].double().view(N, Hkv, H // Hkv, D)[:, h0:h1]
                x = torch.einsum("nhgd,hld->hgnl", q, K) * D ** -0.5
                ok = torch.cat([torch.ones(N, n, dtype=torch.bool, device=DEV), see], 1)
                w = torch.exp(x - torch.logsumexp(x.masked_fill(~ok, -math.inf), -1, keepdim=True)) * ok
                o = torch.einsum("hgnl,hld->nhgd", w, V) * see.any(-1)[:, None, None, None]
                out[:, b].view(N, Hkv, H // Hkv, D)[:, h0:h1] = o
        return out
    return None     # whole numbers


def _nearest_e4m3(y):
    """The nearest e4m3 value (3 bits after the point, smallest normal 2^-6, largest 448), ties to even."""
    step = torch.exp2(torch.clamp(torch.floor(torch.log2(y.abs().clamp_min(1e-300))), min=-6.0) - 3.0)
    return (torch.round(y / step) * step).clamp(-448.0, 448.0)
