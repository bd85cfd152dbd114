"""Host-side checks of the operators for sequences of different lengths (norms with the rotation, a state in pages, packed
prompts, log probabilities): every refusal comes before anything is launched, so none of them needs a GPU."""
import ctypes

import pytest
import torch

import paper_2401_06104_b200 as tova

NULL, UNSUPPORTED, SHAPE, ALIGN = -1, -3, -2, -4
A = ctypes.c_void_p(4096)          # never dereferenced: the calls below are refused
ODD = ctypes.c_void_p(4104)
NO_SIZE = ctypes.c_size_t(-1).value


def rope_handle(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=4, head_dim=128, dtype=tova.TOVA_DTYPE_BF16, rotary_dim=0, layout=0, scaling=0,
                base=10000.0, factor=1.0, blend_low=0.0, blend_high=0.0, amplitude=0.0, original_context=0)
    base.update(kw)
    h = ctypes.c_void_p()
    assert tova.lib().tova_rope_init(ctypes.byref(h), ctypes.byref(tova.tova_rope_config(**base))) == 0
    return h


def test_norm_rope_refuses():
    L, h = tova.lib(), rope_handle()

    def go(r=h, q=A, qs=0, k=A, ks=0, qw=A, kw=A, eps=1e-6, T=1, pos=None, first=0, qo=A, qos=0, ko=A, kos=0):
        return L.tova_norm_rope_apply(r, q, qs, k, ks, qw, kw, eps, T, pos, first, qo, qos, ko, kos, None)
    assert go(r=None) == NULL
    assert go(T=0) == 0 and go(T=0, q=None) == 0
    assert go(T=-1) == SHAPE and go(eps=-1e-6) == SHAPE and go(eps=float("nan")) == SHAPE and go(eps=float("inf")) == SHAPE
    assert go(q=None) == NULL and go(qo=None) == NULL and go(k=None) == NULL and go(ko=None) == NULL
    for name in ("q", "k", "qw", "kw", "qo", "ko"):
        assert go(**{name: ODD}) == ALIGN
    assert go(qs=8 * 128 - 8) == ALIGN and go(kos=4 * 128 + 4) == ALIGN and go(ks=-1024) == SHAPE
    assert go(T=2, first=2**31 - 1) == SHAPE

    def back(r=h, q=A, qs=0, k=A, ks=0, qw=A, kw=A, eps=1e-6, T=1, first=0, gq=A, gqs=0, gk=A, gks=0, dq=A, dqs=0, dk=A, dks=0,
             dqw=A, dkw=A, ws=A, n=1 << 40):
        return L.tova_norm_rope_backward(r, q, qs, k, ks, qw, kw, eps, T, None, first, gq, gqs, gk, gks, dq, dqs, dk, dks, dqw, dkw,
                                         ws, n, None)
    assert back(r=None) == NULL
    assert back(T=-1) == SHAPE and back(eps=-1.0) == SHAPE and back(T=2, first=2**31 - 1) == SHAPE
    for name in ("q", "gq", "dq", "k", "gk", "dk"):
        assert back(**{name: None}) == NULL
    for name in ("q", "gq", "dq", "k", "gk", "dk", "qw", "kw", "dqw", "dkw", "ws"):
        assert back(**{name: ODD}) == ALIGN
    assert back(gqs=100) == ALIGN and back(dks=4 * 128 + 4) == ALIGN and back(dqs=-8) == SHAPE
    assert L.tova_norm_rope_workspace_bytes(None, 1) == NO_SIZE and L.tova_norm_rope_workspace_bytes(h, -1) == NO_SIZE
    assert L.tova_rope_destroy(h) == 0


def paged_cfg(**kw):
    base = dict(batch=3, n_q_heads=8, n_kv_heads=4, head_dim=128, n_pages=10, page_rows=16, max_pages=5, dtype=tova.TOVA_DTYPE_BF16,
                sm_scale=0.0)
    base.update(kw)
    return tova.tova_paged_config(**base)


@pytest.mark.parametrize("bad, code", [
    (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(n_q_heads=6), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(n_pages=0), SHAPE),
    (dict(page_rows=0), SHAPE), (dict(page_rows=24), SHAPE), (dict(page_rows=1 << 16), SHAPE), (dict(page_rows=-16), SHAPE),
    (dict(max_pages=0), SHAPE), (dict(sm_scale=-1.0), SHAPE), (dict(sm_scale=float("inf")), SHAPE), (dict(head_dim=96), UNSUPPORTED),
    (dict(dtype=2), UNSUPPORTED)])
def test_paged_refuses_configurations(bad, code):
    L, c = tova.lib(), paged_cfg(**bad)
    r = ctypes.byref(c)
    assert L.tova_paged_write(r, A, 0, A, 0, 1, None, None, A, A, A, None) == code
    assert L.tova_paged_attention(r, A, A, A, A, 1, A, 0, A, A, 1 << 40, None) == code
    assert L.tova_paged_workspace_bytes(r, 1) == NO_SIZE


def test_paged_refuses_arguments():
    L, c = tova.lib(), paged_cfg()
    r = ctypes.byref(c)

    def write(cfg=r, k=A, ks=0, v=A, vs=0, n=3, off=None, first=A, table=A, K=A, V=A):
        return L.tova_paged_write(cfg, k, ks, v, vs, n, off, first, table, K, V, None)
    assert write(cfg=None) == NULL
    assert write(n=0) == 0 and write(n=-1) == SHAPE and write(n=4) == SHAPE      # without offsets: one token a sequence at most
    for name in ("k", "v", "table", "K", "V"):
        assert write(**{name: None}) == NULL
    for name in ("k", "v", "K", "V"):
        assert write(**{name: ODD}) == ALIGN
    assert write(ks=4 * 128 - 8) == ALIGN and write(vs=4 * 128 + 4) == ALIGN and write(ks=-512) == SHAPE

    def read(cfg=r, K=A, V=A, table=A, lens=A, n=80, q=A, qs=0, out=A, ws=A, size=1 << 40):
        return L.tova_paged_attention(cfg, K, V, table, lens, n, q, qs, out, ws, size, None)
    assert read(cfg=None) == NULL
    assert read(n=81) == SHAPE and read(n=-1) == SHAPE
    for name in ("K", "V", "table", "lens", "q", "out"):
        assert read(**{name: None}) == NULL
    for name in ("K", "V", "q", "out", "ws"):
        assert read(**{name: ODD}) == ALIGN
    assert read(qs=1000) == ALIGN and read(qs=8 * 128 + 4) == ALIGN and read(qs=-1024) == SHAPE
    assert L.tova_paged_workspace_bytes(r, 81) == NO_SIZE and L.tova_paged_workspace_bytes(None, 1) == NO_SIZE


def packed_cfg(**kw):
    base = dict(n_seqs=3, n_q_heads=8, n_kv_heads=4, head_dim=128, dtype=tova.TOVA_DTYPE_BF16, sm_scale=0.0)
    base.update(kw)
    return tova.tova_packed_config(**base)


@pytest.mark.parametrize("bad, n, code", [
    (dict(n_seqs=0), 1, SHAPE), (dict(n_seqs=65536), 1, SHAPE), (dict(n_q_heads=6), 1, SHAPE), (dict(n_kv_heads=0), 1, SHAPE),
    (dict(sm_scale=-1.0), 1, SHAPE), (dict(sm_scale=float("nan")), 1, SHAPE), (dict(head_dim=80), 1, UNSUPPORTED),
    (dict(dtype=7), 1, UNSUPPORTED), (dict(), -1, SHAPE), (dict(), (1 << 24) + 1, SHAPE)])
def test_packed_refuses_configurations(bad, n, code):
    L, c = tova.lib(), packed_cfg(**bad)
    assert L.tova_packed_attention(ctypes.byref(c), A, 0, A, 0, A, 0, n, A, A, A, 1 << 40, None) == code
    assert L.tova_packed_workspace_bytes(ctypes.byref(c), n) == NO_SIZE


def test_packed_refuses_arguments():
    L, c = tova.lib(), packed_cfg()

    def go(cfg=ctypes.byref(c), q=A, qs=0, k=A, ks=0, v=A, vs=0, n=5, off=A, out=A, ws=A, size=1 << 40):
        return L.tova_packed_attention(cfg, q, qs, k, ks, v, vs, n, off, out, ws, size, None)
    assert go(cfg=None) == NULL and go(n=0) == 0
    for name in ("q", "k", "v", "off", "out"):
        assert go(**{name: None}) == NULL
    for name in ("q", "k", "v", "out", "ws"):
        assert go(**{name: ODD}) == ALIGN
    assert go(qs=8 * 128 - 8) == ALIGN and go(ks=4 * 128 + 4) == ALIGN and go(vs=-512) == SHAPE


@pytest.mark.parametrize("bad, n, code", [
    (dict(vocab=0), 1, SHAPE), (dict(vocab=(1 << 24) + 1), 1, SHAPE), (dict(n_top=-1), 1, SHAPE), (dict(n_top=33), 1, SHAPE),
    (dict(vocab=4, n_top=5), 1, SHAPE), (dict(row_stride=999), 1, SHAPE), (dict(row_stride=-1), 1, SHAPE), (dict(dtype=3), 1, UNSUPPORTED),
    (dict(), -1, SHAPE), (dict(), (1 << 24) + 1, SHAPE)])
def test_logprobs_refuses_configurations(bad, n, code):
    base = dict(vocab=1000, dtype=tova.TOVA_DTYPE_FP32, n_top=5, row_stride=0)
    base.update(bad)
    c = tova.tova_logprobs_config(**base)
    assert tova.lib().tova_token_logprobs(ctypes.byref(c), A, n, A, A, A, A, A, None) == code


def test_logprobs_refuses_arguments():
    L = tova.lib()
    c = tova.tova_logprobs_config(1000, tova.TOVA_DTYPE_FP32, 5, 0)
    r = ctypes.byref(c)
    assert L.tova_token_logprobs(None, A, 1, A, A, A, A, A, None) == NULL
    assert L.tova_token_logprobs(r, A, 0, A, A, A, A, A, None) == 0
    for i in (0, 1, 2, 4, 5):
        p = [A] * 6
        p[i] = None
        assert L.tova_token_logprobs(r, p[0], 1, p[1], p[2], p[3], p[4], p[5], None) == NULL
    assert L.tova_token_logprobs(r, ODD, 1, A, A, A, A, A, None) == ALIGN


def test_bindings_refuse_tensors_that_do_not_fit():
    """The binding checks types, shapes and devices before an address reaches the library; CPU tensors are on no GPU."""
    x = torch.zeros(4, 2, 64)
    i = torch.zeros(4, dtype=torch.int32)
    r = tova.TovaRope(1, 2, 2, 64, dtype=tova.TOVA_DTYPE_FP32)
    with pytest.raises((TypeError, ValueError)):
        r.tova_norm_rope_apply(x[:, None], None, 4, x[:, None], None)
    with pytest.raises((TypeError, ValueError)):
        tova.tova_paged_write(tova.tova_paged_config(4, 2, 2, 64, 1, 4, 1, tova.TOVA_DTYPE_FP32, 0.0), x, x, 4, i, x, x)
    with pytest.raises((TypeError, ValueError)):
        tova.tova_packed_attention(tova.tova_packed_config(1, 2, 2, 64, tova.TOVA_DTYPE_FP32, 0.0), x, x, x, 4, i, x)
    with pytest.raises((TypeError, ValueError)):
        tova.tova_token_logprobs(tova.tova_logprobs_config(64, tova.TOVA_DTYPE_FP32, 0, 0), x, 4, i, x)
