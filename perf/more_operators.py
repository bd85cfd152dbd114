"""Work of the operators that serve sequences of different lengths over an unbounded state: norms of queries and keys with
the rotation in the same pass (and the gradient), rows written to a state kept in pages, attention of one new token over the
pages, causal attention of packed prompts, log probabilities of given tokens.

`run` computes a case either in plain torch operations (own = False) or through the library's entry points (own = True)
on the same inputs; `exact` gives the same outputs from the definitions in 64 bits.  Layer shapes are those of the
package's workloads (LLaMA-2-7B, Mistral-7B, Yi-6B layers) and small generic ones.  Token-major layouts: [T,B,...] for
tokens of sequences in lock step, [N,...] for packed tokens of sequences of different lengths, one sequence behind the
other; pages [pages,Hkv,rows,D].
"""
import math
import random

import torch

own = False

DEV = "cuda:0"
EPS = 1e-6


# ----------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one decode step's new tokens of 64 sequences, each at a position of its own: once per layer and step
        dict(name="norm_rope_step", op="norm", T=1, B=64, H=32, Hkv=8, D=128, rot=128, dtype="bf16", layout="half",
             base=500000.0, far=8192, listed_positions=True, fused=True, back=False),
        # a long prompt of four sequences; q and k are cut out of one fused projection
        dict(name="norm_rope_prompt", op="norm", T=4096, B=4, H=32, Hkv=8, D=128, rot=128, dtype="bf16", layout="half",
             base=10000.0, far=32768, listed_positions=False, fused=True, back=False),
        # the gradient's way back through the same, odd length
        dict(name="norm_rope_back", op="norm", T=2047, B=4, H=32, Hkv=8, D=128, rot=128, dtype="bf16", layout="half",
             base=10000.0, far=32768, listed_positions=False, fused=False, back=True),
        # the rows of one decode step go behind 64 sequences' last ones
        dict(name="paged_write_step", op="write", S=64, L=1, held=5000, Hkv=8, D=128, rows=16, dtype="bf16", spread="even"),
        # the rows of seven packed prompts go into their pages
        dict(name="paged_write_prompts", op="write", S=7, L=8191, held=0, Hkv=8, D=128, rows=16, dtype="bf16",
             spread="steep"),
        # one new token of one sequence: latency
        dict(name="paged_single", op="paged", B=1, H=32, Hkv=8, D=128, L=1000, rows=16, dtype="bf16", ragged=False),
        # a serving batch, Mistral-7B heads, lengths from a third of the longest; one place of the batch is idle
        dict(name="paged_batch_gqa", op="paged", B=64, H=32, Hkv=8, D=128, L=8192, rows=16, dtype="bf16", ragged=True),
        # LLaMA-2-7B heads in fp32, wide pages
        dict(name="paged_mha_fp32", op="paged", B=8, H=32, Hkv=32, D=128, L=2001, rows=64, dtype="fp32", ragged=True),
        # nine short prompts: latency
        dict(name="packed_short", op="packed", S=9, L=200, H=8, Hkv=2, D=64, dtype="bf16", spread="linear", fused=True),
        # seven prompts from 8191 tokens down, Mistral-7B heads
        dict(name="packed_prompts", op="packed", S=7, L=8191, H=32, Hkv=8, D=128, dtype="bf16", spread="steep", fused=True),
        # one step's logits of one sequence, with the alternatives that an API reports
        dict(name="logprobs_step", op="logprobs", T=1, V=32000, top=20, dtype="fp32"),
        # a text's tokens, for its perplexity, with the five best alternatives
        dict(name="logprobs_text", op="logprobs", T=4095, V=64000, top=5, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """A case of the same ranges; its long axis is halved while it would be more work than the largest listed cases."""
    top = [max(work(c)[k] for c in listed()) for k in ("bytes", "flops")]
    case = _draw(rng)
    axis = {"norm": "T", "logprobs": "T"}.get(case["op"], "L")
    while case[axis] > 1 and any(work(case)[k] > t for k, t in zip(("bytes", "flops"), top)):
        case[axis] = (case[axis] + 1) // 2
    return case


def _draw(rng):
    op = rng.choice(["norm", "norm", "write", "paged", "paged", "packed", "packed", "logprobs"])
    H, Hkv = rng.choice([(32, 32), (32, 8), (32, 4), (8, 2), (4, 4)])
    D = rng.choice([64, 128, 128])
    dtype = rng.choice(["bf16", "bf16", "bf16", "fp32"])
    if op == "norm":
        B = _log(rng, 1, 64)
        T = _log(rng, 1, max(1, 16384 * 40 // (B * (H + Hkv))))
        return dict(op="norm", T=T, B=B, H=H, Hkv=Hkv, D=D, rot=rng.choice([D, D, D // 2, D // 4 * 3]), dtype=dtype,
                    layout=rng.choice(["half", "half", "interleaved"]), base=rng.choice([10000.0, 500000.0]),
                    far=_log(rng, 4096, 1000000), listed_positions=rng.random() < 0.5, fused=rng.random() < 0.5,
                    back=rng.random() < 0.4)
    if op == "write":
        S = _log(rng, 1, 64)
        return dict(op="write", S=S, L=_log(rng, 1, max(2, 8192 // S)), held=_log(rng, 1, 2000) - 1, Hkv=Hkv, D=D,
                    rows=rng.choice([1, 8, 16, 32, 64, 256]), dtype=dtype, spread=rng.choice(["even", "linear", "steep"]))
    if op == "paged":
        return dict(op="paged", B=_log(rng, 1, 128), H=H, Hkv=Hkv, D=D, L=_log(rng, 1, 32768 if dtype == "bf16" else 8192),
                    rows=rng.choice([1, 8, 16, 16, 32, 64, 256]), dtype=dtype, ragged=rng.random() < 0.6)
    if op == "packed":
        if dtype == "fp32":
            S, L = _log(rng, 1, 16), _log(rng, 1, 1500)
        else:
            S = _log(rng, 1, 64)
            L = _log(rng, 1, 8192)
        return dict(op="packed", S=S, L=L, H=H, Hkv=Hkv, D=D, dtype=dtype, spread=rng.choice(["even", "linear", "steep"]),
                    fused=rng.random() < 0.5)
    V = _log(rng, 1000, 128000)
    return dict(op="logprobs", T=_log(rng, 1, max(1, 4095 * 32000 // V)), V=V, top=rng.choice([0, 1, 5, 20, 32]), dtype=dtype)


# ---------------------------------------------------------------------------------------------------- inputs

def _type(name):
    return torch.bfloat16 if name == "bf16" else torch.float32


def _lens(case):
    """Rows each sequence of a batch holds: all alike, or spread between a third of L and L, the second of four and
    more none (a place of the batch that is idle)."""
    B, L = case["B"], case["L"]
    if not case["ragged"]:
        return [L] * B
    n = [L - (2 * L * b) // (3 * B) for b in range(B)]
    if B >= 4:
        n[1] = 0
    return n


def _prompts(case):
    """Lengths of the packed sequences, the longest L: alike, falling evenly, or each about six tenths of the one before;
    in an order of their own."""
    S, L = case["S"], case["L"]
    if case["spread"] == "even":
        return [L] * S
    n = [max(1, L * (S - i) // S) if case["spread"] == "linear" else max(1, int(L * 0.61 ** i)) for i in range(S)]
    random.Random(S * 1000003 + L).shuffle(n)
    return n


def _offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _table(held, rows, seed):
    """A page table [sequences, most pages] whose pages lie in any order, -1 where a sequence has none; pages in all."""
    need = [(n + rows - 1) // rows for n in held]
    most, total = max(1, max(need)), sum(need) + 3
    order = torch.randperm(total, generator=torch.Generator().manual_seed(seed * 11 + 5)).to(torch.int32)
    table = torch.full((len(held), most), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, total


def _frequencies(case):
    """Inverse frequencies of the pairs in 64 bits."""
    return [case["base"] ** (-2.0 * i / case["rot"]) for i in range(case["rot"] // 2)]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device=DEV)  # noqa: E731
    op, t = case["op"], _type(case["dtype"])
    s = {"case": case, "op": op}
    if own:
        import paper_2401_06104_b200 as tova
        s["tova"] = tova
        dt = tova.TOVA_DTYPE_BF16 if t == torch.bfloat16 else tova.TOVA_DTYPE_FP32
    if op == "norm":
        T, B, H, Hkv, D = case["T"], case["B"], case["H"], case["Hkv"], case["D"]
        if case["fused"]:       # q and k are slices of one projection's output
            qkv = (rnd(T, B, (H + 2 * Hkv) * D) * 1.7).to(t)
            q = qkv[..., :H * D].unflatten(-1, (H, D))
            k = qkv[..., H * D:(H + Hkv) * D].unflatten(-1, (Hkv, D))
        else:
            q, k = (rnd(T, B, H, D) * 1.7).to(t), (rnd(T, B, Hkv, D) * 0.6).to(t)
        first = int(torch.randint(0, max(1, case["far"] - T), (1,), generator=torch.Generator().manual_seed(seed)))
        s.update(q=q, k=k, first=first, pos=None, qw=(1 + 0.2 * rnd(D)).to(t), kw=(1 + 0.2 * rnd(D)).to(t),
                 inv=torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV))
        if case["listed_positions"]:
            s["pos"] = torch.randint(0, case["far"], (T, B), generator=g, device=DEV, dtype=torch.int32)
        if case["back"]:
            s["dqo"], s["dko"] = rnd(T, B, H, D).to(t), rnd(T, B, Hkv, D).to(t)
        if own:
            s["rope"] = tova.TovaRope(B, H, Hkv, D, dtype=dt, rotary_dim=case["rot"], base=case["base"],
                                      layout=tova.TOVA_ROPE_HALF if case["layout"] == "half" else tova.TOVA_ROPE_INTERLEAVED)
            s["qo"] = torch.empty(T, B, H, D, dtype=t, device=DEV)
            s["ko"] = torch.empty(T, B, Hkv, D, dtype=t, device=DEV)
            if case["back"]:
                s["dqw"], s["dkw"] = torch.empty(D, device=DEV), torch.empty(D, device=DEV)
                s["ws"] = torch.empty(s["rope"].tova_norm_rope_workspace_bytes(T), dtype=torch.uint8, device=DEV)
    elif op == "write":
        lens, Hkv, D, rows = _prompts(case), case["Hkv"], case["D"], case["rows"]
        # the sequences hold between none and `held` rows already
        before = [(case["held"] * (i + 1)) // case["S"] for i in range(case["S"])]
        table, pages = _table([a + n for a, n in zip(before, lens)], rows, seed)
        N = sum(lens)
        s["k"] = rnd(N, Hkv, D).to(t)
        s["v"] = (rnd(N, 2 * Hkv * D)).to(t)[:, Hkv * D:].unflatten(-1, (Hkv, D))      # a slice of the projection's output
        s["K"], s["V"] = torch.zeros(pages, Hkv, rows, D, dtype=t, device=DEV), torch.zeros(pages, Hkv, rows, D, dtype=t, device=DEV)
        s["table"] = table.to(DEV)
        s["first"] = torch.tensor(before, dtype=torch.int32, device=DEV)
        s["offsets"] = None if case["spread"] == "even" and case["L"] == 1 else torch.tensor(_offsets(lens), dtype=torch.int32, device=DEV)
        s["N"] = N
        if own:
            s["cfg"] = tova.tova_paged_config(case["S"], Hkv, Hkv, D, pages, rows, table.shape[1], dt, 0.0)
    elif op == "paged":
        B, H, Hkv, D, rows = case["B"], case["H"], case["Hkv"], case["D"], case["rows"]
        lens = _lens(case)
        table, pages = _table(lens, rows, seed)
        s["K"], s["V"] = rnd(pages, Hkv, rows, D).to(t), rnd(pages, Hkv, rows, D).to(t)
        first = table[:, 0].clamp_min(0).long().to(DEV)
        s["K"][first, :, 0] *= 3.0      # the first token stays attended
        s["q"] = (rnd(B, H, D) * 1.3).to(t)
        s["table"], s["lens"] = table.to(DEV), torch.tensor(lens, dtype=torch.int32, device=DEV)
        if own:
            s["cfg"] = tova.tova_paged_config(B, H, Hkv, D, pages, rows, table.shape[1], dt, 0.0)
            s["ws"] = torch.empty(max(16, tova.tova_paged_workspace_bytes(s["cfg"], case["L"])), dtype=torch.uint8, device=DEV)
            s["out"] = torch.empty(B, H, D, dtype=t, device=DEV)
    elif op == "packed":
        H, Hkv, D = case["H"], case["Hkv"], case["D"]
        lens = _prompts(case)
        N = sum(lens)
        if case["fused"]:       # v is a slice of the projection's output, q and k come from the rotation
            v = rnd(N, (H + 2 * Hkv) * D).to(t)[:, (H + Hkv) * D:].unflatten(-1, (Hkv, D))
        else:
            v = rnd(N, Hkv, D).to(t)
        s.update(q=(rnd(N, H, D) * 1.3).to(t), k=rnd(N, Hkv, D).to(t), v=v, N=N,
                 offsets=torch.tensor(_offsets(lens), dtype=torch.int32, device=DEV))
        if own:
            s["cfg"] = tova.tova_packed_config(case["S"], H, Hkv, D, dt, 0.0)
            s["ws"] = torch.empty(max(16, tova.tova_packed_workspace_bytes(s["cfg"], N)), dtype=torch.uint8, device=DEV)
            s["out"] = torch.empty(N, H, D, dtype=t, device=DEV)
    else:
        T, V = case["T"], case["V"]
        s["x"] = (rnd(T, V) * 2.5).to(t)
        s["tok"] = torch.randint(0, V, (T,), generator=g, device=DEV, dtype=torch.int32)
        likely = s["x"][:, :V // 2].argmax(-1).to(torch.int32)       # most tokens of a text are likely ones
        s["tok"] = torch.where(torch.rand(T, generator=g, device=DEV) < 0.7, likely, s["tok"])
        if own:
            s["cfg"] = tova.tova_logprobs_config(V, dt, case["top"], 0)
            s["lp"], s["ent"] = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
            s["ids"] = torch.empty(T, case["top"], dtype=torch.int32, device=DEV) if case["top"] else None
            s["tlp"] = torch.empty(T, case["top"], device=DEV) if case["top"] else None
    return s


# --------------------------------------------------------------------------------------------- the operators

def run(s):
    return dict(norm=_run_norm, write=_run_write, paged=_run_paged, packed=_run_packed, logprobs=_run_logprobs)[s["op"]](s)


def _turn(x, c, si, rot, layout):
    """x [T,B,heads,D] turned by the angles whose cosines and sines are c, si [T,B|1,1,rot/2]."""
    r, rest = x[..., :rot], x[..., rot:]
    if layout == "half":
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        r = torch.cat([a * c - b * si, b * c + a * si], -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack([a * c - b * si, b * c + a * si], -1).flatten(-2)
    return torch.cat([r, rest], -1)


def _run_norm(s):
    c = s["case"]
    if own:
        if c["back"]:
            s["rope"].tova_norm_rope_backward(s["q"], s["k"], s["dqo"], s["dko"], c["T"], s["qo"], s["ko"], s["ws"],
                                              q_weight=s["qw"], k_weight=s["kw"], dq_weight=s["dqw"], dk_weight=s["dkw"],
                                              eps=EPS, positions=s["pos"], first_pos=s["first"])
            return s["qo"], s["ko"], s["dqw"], s["dkw"]
        s["rope"].tova_norm_rope_apply(s["q"], s["k"], c["T"], s["qo"], s["ko"], q_weight=s["qw"], k_weight=s["kw"], eps=EPS,
                                       positions=s["pos"], first_pos=s["first"])
        return s["qo"], s["ko"]
    pos = s["pos"] if s["pos"] is not None else s["first"] + torch.arange(c["T"], device=DEV)[:, None]
    ang = pos.double()[..., None] * s["inv"]                       # far positions: the angle in 64 bits
    co, si = torch.cos(ang).float()[:, :, None], torch.sin(ang).float()[:, :, None]
    got, weights = [], []
    for n in "qk":
        x, w = s[n].float(), s[n + "w"].float()
        r = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
        if not c["back"]:
            got.append(_turn(x * r * w, co, si, c["rot"], c["layout"]).to(s[n].dtype))
            continue
        xh = x * r
        gr = _turn(s["d" + n + "o"].float(), co, -si, c["rot"], c["layout"])
        weights.append((gr * xh).double().sum((0, 1, 2)).float())     # a long sum
        gr = gr * w
        got.append((r * (gr - xh * (gr * xh).mean(-1, keepdim=True))).to(s[n].dtype))
    return tuple(got + weights)


def _run_write(s):
    c = s["case"]
    if own:
        s["tova"].tova_paged_write(s["cfg"], s["k"], s["v"], s["N"], s["table"], s["K"], s["V"], first_rows=s["first"],
                                   offsets=s["offsets"])
        return s["K"], s["V"]
    i = torch.arange(s["N"], device=DEV)
    if s["offsets"] is None:
        b, j = i, s["first"].long()
    else:
        off = s["offsets"].long()
        b = (i[:, None] >= off[None, 1:]).sum(1)
        j = s["first"].long()[b] + i - off[b]
    page = s["table"].long()[b, j // c["rows"]]
    s["K"][page, :, j % c["rows"]] = s["k"]
    s["V"][page, :, j % c["rows"]] = s["v"]
    return s["K"], s["V"]


def _run_paged(s):
    c = s["case"]
    B, H, Hkv, D, L = c["B"], c["H"], c["Hkv"], c["D"], c["L"]
    if own:
        s["tova"].tova_paged_attention(s["cfg"], s["K"], s["V"], s["table"], s["lens"], L, s["q"], s["out"], s["ws"])
        return s["out"]
    at = s["table"].long().clamp_min(0)
    K = s["K"][at].permute(0, 2, 1, 3, 4).flatten(2, 3).float()   # [B,Hkv,rows,D]
    x = torch.matmul(s["q"].float().view(B, Hkv, H // Hkv, D), K.transpose(2, 3)) * (1.0 / math.sqrt(D))
    del K
    see = (torch.arange(x.shape[-1], device=DEV) < s["lens"][:, None])[:, None, None]
    x = x.masked_fill(~see, -math.inf)
    top = x.amax(-1, keepdim=True)
    e = torch.exp(x - torch.where(torch.isfinite(top), top, torch.zeros_like(top)))
    V = s["V"][at].permute(0, 2, 1, 3, 4).flatten(2, 3).float()
    o = torch.matmul(e, V) / e.sum(-1, keepdim=True).clamp_min(1e-30)
    return o.view(B, H, D).to(s["q"].dtype)


def _run_packed(s):
    c = s["case"]
    H, Hkv, D = c["H"], c["Hkv"], c["D"]
    G = H // Hkv
    if own:
        s["tova"].tova_packed_attention(s["cfg"], s["q"], s["k"], s["v"], s["N"], s["offsets"], s["out"], s["ws"])
        return s["out"]
    out = torch.empty(s["N"], H, D, dtype=s["q"].dtype, device=DEV)
    at = 0
    for n in _prompts(c):                                          # (the program has the lengths on the host, too)
        q = s["q"][at:at + n].float().transpose(0, 1).reshape(Hkv, G * n, D)
        k = s["k"][at:at + n].float().permute(1, 2, 0)
        v = s["v"][at:at + n].float().transpose(0, 1)
        later = torch.ones(n, n, dtype=torch.bool, device=DEV).triu(1)
        step = max(1, (1 << 30) // (G * n * n))                    # KV heads at a time
        for h in range(0, Hkv, step):
            x = torch.matmul(q[h:h + step], k[h:h + step]) * (1.0 / math.sqrt(D))
            m = x.shape[0]
            x = x.view(m, G, n, n).masked_fill_(later, -math.inf)
            x = torch.exp(x - x.amax(-1, keepdim=True))
            o = torch.matmul(x.view(m, G * n, n), v[h:h + step]).view(m, G, n, D) / x.sum(-1, keepdim=True)
            out[at:at + n, h * G:(h + m) * G] = o.reshape(m * G, n, D).transpose(0, 1).to(out.dtype)
            del x
        at += n
    return out


def _run_logprobs(s):
    c = s["case"]
    if own:
        s["tova"].tova_token_logprobs(s["cfg"], s["x"], c["T"], s["tok"], s["lp"], s["ent"], s["ids"], s["tlp"])
        return (s["lp"], s["ent"], s["ids"], s["tlp"]) if c["top"] else (s["lp"], s["ent"])
    x = s["x"].float()
    d = x - x.amax(-1, keepdim=True)
    e = torch.exp(d)
    z = e.sum(-1, keepdim=True)
    lz = torch.log(z)
    lp = torch.gather(d, 1, s["tok"].long()[:, None]) - lz
    ent = lz - (e * d).sum(-1, keepdim=True) / z
    if not c["top"]:
        return lp[:, 0], ent[:, 0]
    ids = torch.sort(x, dim=-1, descending=True, stable=True)[1][:, :c["top"]]      # ties: the lowest token first
    return lp[:, 0], ent[:, 0], ids.to(torch.int32), torch.gather(d, 1, ids) - lz


def work(case):
    op = case["op"]
    E = 2 if case["dtype"] == "bf16" else 4
    if op == "norm":
        n = float(case["T"] * case["B"] * (case["H"] + case["Hkv"]))
        D = case["D"]
        b = (3.0 if case["back"] else 2.0) * n * D * E + 2.0 * D * E + (8.0 * D if case["back"] else 0)
        return {"bytes": b + (4.0 * case["T"] * case["B"] if case["listed_positions"] else 0),
                "flops": n * ((11.0 if case["back"] else 4.0) * D + 3.0 * case["rot"])}
    if op == "write":
        lens = _prompts(case)
        return {"bytes": 4.0 * sum(lens) * case["Hkv"] * case["D"] * E + 8.0 * len(lens) + 4.0 * sum(-(-n // case["rows"]) for n in lens),
                "flops": 0.0}
    if op == "paged":
        held, D = float(sum(_lens(case))), case["D"]
        return {"bytes": 2.0 * held * case["Hkv"] * D * E + 2.0 * case["B"] * case["H"] * D * E + 4.0 * (case["B"] + held / case["rows"]),
                "flops": 4.0 * held * case["H"] * D}
    if op == "packed":
        lens, D = _prompts(case), case["D"]
        return {"bytes": sum(lens) * D * E * (2.0 * case["H"] + 2.0 * case["Hkv"]) + 4.0 * (len(lens) + 1),
                "flops": sum(2.0 * n * (n + 1) * case["H"] * D for n in lens)}
    T, V = case["T"], case["V"]
    return {"bytes": float(T) * V * E + T * (12.0 + 8.0 * case["top"]), "flops": 5.0 * T * V}


# --------------------------------------------------------------------------------- the definitions in 64 bits

def exact(case, seed):
    global own
    keep, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = keep
    op = case["op"]
    if op == "norm":
        # a pair is a complex number; the gradient's pair goes through the product with the conjugate
        T, B, D, h = case["T"], case["B"], case["D"], case["rot"] // 2
        pos = s["pos"].double() if s["pos"] is not None else (s["first"] + torch.arange(T, device=DEV).double())[:, None].expand(T, B)
        ang = torch.einsum("tb,i->tbi", pos, s["inv"])
        unit = torch.polar(torch.ones_like(ang), ang)[:, :, None]
        lo, hi = (slice(0, h), slice(h, 2 * h)) if case["layout"] == "half" else (slice(0, 2 * h, 2), slice(1, 2 * h, 2))

        def turned(y, by):
            y = y.clone()
            z = torch.complex(y[..., lo].contiguous(), y[..., hi].contiguous()) * by
            y[..., lo], y[..., hi] = z.real, z.imag
            return y
        got, weights = [], []
        for n in "qk":
            x, w = s[n].double(), s[n + "w"].double()
            size = torch.sqrt(x.square().sum(-1, keepdim=True) / D + EPS)
            if not case["back"]:
                got.append(turned(x / size * w, unit))
                continue
            gr = turned(s["d" + n + "o"].double(), unit.conj())
            weights.append(torch.einsum("tbhd,tbhd->d", gr, x / size))
            a = gr * w
            along = torch.einsum("tbhd,tbhd->tbh", a, x)[..., None]       # d size / d x = x / (D size)
            got.append(a / size - x * along / (D * size ** 3))
        return tuple(got + weights)
    if op == "write":
        K, V = torch.zeros_like(s["K"], dtype=torch.float64), torch.zeros_like(s["V"], dtype=torch.float64)
        table, before, rows = s["table"].tolist(), s["first"].tolist(), case["rows"]
        place = [(table[b][j // rows], j % rows) for b, n in enumerate(_prompts(case)) for j in range(before[b], before[b] + n)]
        page, row = (torch.tensor(x, device=DEV) for x in zip(*place))
        for h in range(case["Hkv"]):
            K[page, h, row] = s["k"][:, h].double()
            V[page, h, row] = s["v"][:, h].double()
        return K, V
    if op == "paged":
        B, H, Hkv, D, rows = case["B"], case["H"], case["Hkv"], case["D"], case["rows"]
        out = torch.zeros(B, H, D, dtype=torch.float64, device=DEV)
        for b, n in enumerate(_lens(case)):
            if n == 0:
                continue
            pages = s["table"][b, :(n + rows - 1) // rows].long()
            step = max(1, (1 << 28) // (n * D))
            for h in range(0, Hkv, step):
                K = s["K"].index_select(0, pages)[:, h:h + step].transpose(0, 1).reshape(-1, len(pages) * rows, D)[:, :n].double()
                V = s["V"].index_select(0, pages)[:, h:h + step].transpose(0, 1).reshape(-1, len(pages) * rows, D)[:, :n].double()
                q = s["q"][b].double().view(Hkv, H // Hkv, D)[h:h + step]
                w = torch.softmax(torch.einsum("hgd,hnd->hgn", q, K) * D ** -0.5, -1)
                out[b].view(Hkv, H // Hkv, D)[h:h + step] = torch.einsum("hgn,hnd->hgd", w, V)
        return out
    if op == "packed":
        H, Hkv, D = case["H"], case["Hkv"], case["D"]
        out = torch.empty(s["N"], H, D, dtype=torch.float64, device=DEV)
        at = 0
        for n in _prompts(case):
            i = torch.arange(n, device=DEV)
            for h in range(H):
                hk = h // (H // Hkv)
                x = (s["q"][at:at + n, h].double() @ s["k"][at:at + n, hk].double().t()) * D ** -0.5
                x = torch.where(i[None] <= i[:, None], x, torch.full_like(x, -math.inf))
                w = torch.exp(x - torch.logsumexp(x, -1, keepdim=True))
                out[at:at + n, h] = w @ s["v"][at:at + n, hk].double()
                del x, w
            at += n
        return out
    # a slice of the rows at a time
    T, V, top = case["T"], case["V"], case["top"]
    lp, ent, tlp = [], [], []
    for a in range(0, T, max(1, (1 << 27) // V)):
        x = s["x"][a:a + max(1, (1 << 27) // V)].double()
        y = x - torch.logsumexp(x, -1, keepdim=True)
        lp.append(y.gather(1, s["tok"][a:a + x.shape[0]].long()[:, None])[:, 0])
        ent.append(-(torch.exp(y) * y).sum(-1))
        if top:
            tlp.append(torch.topk(y, top, -1)[0])
    if not top:
        return torch.cat(lp), torch.cat(ent)
    return torch.cat(lp), torch.cat(ent), None, torch.cat(tlp)
