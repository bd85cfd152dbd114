"""Host-side checks of the operators around the decode step (rotary positions, 8-bit state, drafted tokens): every
refusal comes before anything is launched, so none of them needs a GPU."""
import ctypes
import os
import random
import subprocess

import pytest
import torch

import paper_2401_06104_b200 as tova
from paper_2401_06104_b200 import build as tbuild

NULL, UNSUPPORTED, SHAPE, ALIGN, CUDA = -1, -3, -2, -4, -7
A = ctypes.c_void_p(4096)          # never dereferenced: the calls below are refused
ODD = ctypes.c_void_p(4104)


def rope_cfg(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=4, head_dim=128, dtype=tova.TOVA_DTYPE_BF16, rotary_dim=0, layout=0, scaling=0,
                base=10000.0, factor=2.0, blend_low=0.0, blend_high=0.0, amplitude=0.0, original_context=4096)
    base.update(kw)
    return tova.tova_rope_config(**base)


@pytest.mark.parametrize("bad, code", [
    (dict(head_dim=96), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED), (dict(layout=2), UNSUPPORTED), (dict(scaling=5), UNSUPPORTED),
    (dict(scaling=-1), UNSUPPORTED), (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(n_q_heads=6), SHAPE),
    (dict(n_kv_heads=0), SHAPE), (dict(rotary_dim=3), SHAPE), (dict(rotary_dim=130), SHAPE), (dict(rotary_dim=-2), SHAPE),
    (dict(base=1.0), SHAPE), (dict(base=float("nan")), SHAPE), (dict(scaling=1, factor=0.5), SHAPE), (dict(scaling=1, factor=float("inf")), SHAPE),
    (dict(amplitude=-1.0), SHAPE), (dict(scaling=3, original_context=0), SHAPE), (dict(scaling=4, blend_low=5.0), SHAPE),
    (dict(scaling=2, rotary_dim=2), SHAPE), (dict(blend_low=float("nan")), SHAPE)])
def test_rope_init_refuses(bad, code):
    h = ctypes.c_void_p()
    assert tova.lib().tova_rope_init(ctypes.byref(h), ctypes.byref(rope_cfg(**bad))) == code
    assert not h.value


def test_rope_apply_refuses_before_any_launch():
    L = tova.lib()
    assert L.tova_rope_init(None, ctypes.byref(rope_cfg())) == NULL
    h = ctypes.c_void_p()
    assert L.tova_rope_init(ctypes.byref(h), None) == NULL
    assert L.tova_rope_apply(None, A, 0, A, 0, 1, None, 0, 0, A, 0, A, 0, None) == NULL
    assert L.tova_rope_destroy(None) == NULL
    assert L.tova_rope_init(ctypes.byref(h), ctypes.byref(rope_cfg())) == 0

    def go(q=A, qs=0, k=A, ks=0, T=1, pos=None, first=0, qo=A, qos=0, ko=A, kos=0):
        return L.tova_rope_apply(h, q, qs, k, ks, T, pos, first, 0, qo, qos, ko, kos, None)
    assert go(T=0) == 0                                   # nothing to do
    assert go(T=-1) == SHAPE
    assert go(q=None) == NULL and go(qo=None) == NULL and go(k=None) == NULL and go(ko=None) == NULL
    assert go(q=ODD) == ALIGN and go(ko=ODD) == ALIGN
    assert go(qs=8 * 128 - 8) == ALIGN                    # rows would overlap
    assert go(qs=8 * 128 + 4) == ALIGN                    # rows would leave the 16-byte grid
    assert go(ks=-1024) == SHAPE
    assert go(T=2, first=2**31 - 1) == SHAPE              # the last position leaves int32
    assert L.tova_rope_destroy(h) == 0


def quant_cfg(**kw):
    base = dict(batch=2, n_kv_heads=4, head_dim=128, capacity=100, dtype=tova.TOVA_DTYPE_BF16, format=tova.TOVA_FORMAT_INT8)
    base.update(kw)
    return tova.tova_quant_config(**base)


@pytest.mark.parametrize("bad, code", [
    (dict(batch=0), SHAPE), (dict(batch=65536), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(capacity=0), SHAPE), (dict(capacity=(1 << 24) + 1), SHAPE),
    (dict(head_dim=32), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(format=0), UNSUPPORTED), (dict(format=3), UNSUPPORTED)])
def test_quant_refuses_configurations(bad, code):
    L, c = tova.lib(), quant_cfg(**bad)
    assert L.tova_quant_write(ctypes.byref(c), A, 0, A, 0, 1, None, 0, A, A, A, A, None) == code
    assert L.tova_quant_read(ctypes.byref(c), A, A, A, A, 1, None, 0, A, A, None) == code


def test_quant_refuses_arguments():
    L, c = tova.lib(), quant_cfg()
    r = ctypes.byref(c)
    assert L.tova_quant_write(None, A, 0, A, 0, 1, None, 0, A, A, A, A, None) == NULL
    assert L.tova_quant_write(r, A, 0, A, 0, 0, None, 0, A, A, A, A, None) == 0
    assert L.tova_quant_write(r, A, 0, A, 0, -1, None, 0, A, A, A, A, None) == SHAPE
    for first, T in ((-1, 1), (100, 1), (90, 11), (2**31 - 1, 5)):
        assert L.tova_quant_write(r, A, 0, A, 0, T, None, first, A, A, A, A, None) == SHAPE
        assert L.tova_quant_read(r, A, A, A, A, T, None, first, A, A, None) == SHAPE
    for i in range(6):
        p = [A] * 6
        p[i] = None
        assert L.tova_quant_write(r, p[0], 0, p[1], 0, 1, None, 0, p[2], p[3], p[4], p[5], None) == NULL
        p[i] = ODD
        assert L.tova_quant_write(r, p[0], 0, p[1], 0, 1, None, 0, p[2], p[3], p[4], p[5], None) == ALIGN
    assert L.tova_quant_write(r, A, 4 * 128 - 8, A, 0, 1, None, 0, A, A, A, A, None) == ALIGN
    assert L.tova_quant_write(r, A, 0, A, -512, 1, None, 0, A, A, A, A, None) == SHAPE
    assert L.tova_quant_read(r, None, A, A, A, 1, None, 0, A, A, None) == NULL
    assert L.tova_quant_read(r, A, A, A, None, 1, None, 0, A, A, None) == NULL
    assert L.tova_quant_read(r, None, None, None, None, 1, None, 0, None, None, None) == 0
    assert L.tova_quant_read(r, A, A, A, A, 1, None, 0, ODD, A, None) == ALIGN


def tree_cfg(**kw):
    base = dict(batch=2, n_q_heads=8, n_kv_heads=4, head_dim=128, capacity=100, dtype=tova.TOVA_DTYPE_BF16, format=tova.TOVA_FORMAT_PLAIN,
                sm_scale=0.0)
    base.update(kw)
    return tova.tova_tree_config(**base)


@pytest.mark.parametrize("bad, n_live, nodes, code", [
    (dict(batch=0), 1, 1, SHAPE), (dict(batch=20000), 1, 1, SHAPE), (dict(n_q_heads=6), 1, 1, SHAPE), (dict(capacity=0), 0, 1, SHAPE),
    (dict(sm_scale=-1.0), 1, 1, SHAPE), (dict(sm_scale=float("nan")), 1, 1, SHAPE), (dict(head_dim=80), 1, 1, UNSUPPORTED),
    (dict(dtype=9), 1, 1, UNSUPPORTED), (dict(format=3), 1, 1, UNSUPPORTED), (dict(), 101, 1, SHAPE), (dict(), -1, 1, SHAPE),
    (dict(), 1, 257, SHAPE), (dict(), 1, -1, SHAPE)])
def test_tree_refuses_configurations(bad, n_live, nodes, code):
    L, c = tova.lib(), tree_cfg(**bad)
    assert L.tova_tree_attention(ctypes.byref(c), A, A, A, A, None, n_live, A, A, A, nodes, None, A, A, 1 << 40, None) == code
    assert L.tova_tree_workspace_bytes(ctypes.byref(c), n_live, nodes) == ctypes.c_size_t(-1).value


def test_tree_refuses_arguments():
    L, c = tova.lib(), tree_cfg()
    r = ctypes.byref(c)
    assert L.tova_tree_attention(None, A, A, A, A, None, 1, A, A, A, 1, None, A, A, 1 << 40, None) == NULL
    assert L.tova_tree_attention(r, A, A, None, None, None, 1, A, A, A, 0, None, A, None, 0, None) == 0
    for i in range(6):
        p = [A] * 6
        p[i] = None
        assert L.tova_tree_attention(r, p[0], p[1], None, None, None, 1, p[2], p[3], p[4], 1, None, p[5], A, 1 << 40, None) == NULL
        p[i] = ODD
        assert L.tova_tree_attention(r, p[0], p[1], None, None, None, 1, p[2], p[3], p[4], 1, None, p[5], A, 1 << 40, None) == ALIGN
    q = ctypes.byref(tree_cfg(format=tova.TOVA_FORMAT_E4M3))
    assert L.tova_tree_attention(q, A, A, None, A, None, 1, A, A, A, 1, None, A, A, 1 << 40, None) == NULL
    assert L.tova_tree_attention(q, A, A, A, ODD, None, 1, A, A, A, 1, None, A, A, 1 << 40, None) == ALIGN
    assert L.tova_cache_tree_attention(None, A, A, A, 1, None, A, A, 0, None) == NULL
    assert L.tova_cache_tree_workspace_bytes(None, 1) == ctypes.c_size_t(-1).value


def test_verify_refuses():
    L = tova.lib()

    def go(target=A, draft=A, tokens=A, u=A, us=A, n=A, path=A, out=A, **kw):
        base = dict(batch=2, n_nodes=3, vocab=50, dtype=tova.TOVA_DTYPE_FP32, row_stride=0)
        base.update(kw)
        c = tova.tova_verify_config(**base)
        return L.tova_verify_draft(ctypes.byref(c), target, draft, tokens, None, u, us, n, path, out, None)
    assert L.tova_verify_draft(None, A, A, A, None, A, A, A, A, A, None) == NULL
    assert go(batch=0) == SHAPE and go(batch=65536) == SHAPE and go(n_nodes=-1) == SHAPE and go(n_nodes=1025) == SHAPE
    assert go(vocab=0) == SHAPE and go(vocab=(1 << 24) + 1) == SHAPE and go(row_stride=49) == SHAPE
    assert go(dtype=3) == UNSUPPORTED
    assert go(target=None) == NULL and go(us=None) == NULL and go(n=None) == NULL and go(out=None) == NULL
    assert go(tokens=None) == NULL and go(u=None) == NULL
    assert go(target=ODD) == ALIGN and go(draft=ODD) == ALIGN


def test_binding_refuses_tensors_that_do_not_fit():
    """Types, devices and sizes are checked before an address reaches the library."""
    cfg = quant_cfg()
    k = torch.zeros(1, 2, 4, 128, dtype=torch.bfloat16)
    codes, scale = torch.zeros(2, 4, 100, 128, dtype=torch.int8), torch.zeros(2, 4, 100)
    with pytest.raises(TypeError):
        tova.tova_quant_write(cfg, k.float(), k, 1, codes, scale, codes, scale)
    with pytest.raises(ValueError):                        # not on a GPU
        tova.tova_quant_write(cfg, k, k, 1, codes, scale, codes, scale)
    q = torch.zeros(1, 2, 8, 128, dtype=torch.bfloat16)
    with pytest.raises((TypeError, ValueError)):
        tova.tova_tree_attention(tree_cfg(), k, k, 1, q, k, k, 1, q)
    with pytest.raises(TypeError):
        tova.tova_verify_draft(tova.tova_verify_config(1, 1, 8, tova.TOVA_DTYPE_BF16, 0), torch.zeros(2, 1, 8), None, None, None,
                               None, None, None, None)


@pytest.mark.skipif(torch.cuda.is_available(), reason="only meaningful without a GPU")
def test_valid_calls_fail_loudly_without_a_device():
    L = tova.lib()
    h = ctypes.c_void_p()
    assert L.tova_rope_init(ctypes.byref(h), ctypes.byref(rope_cfg())) == 0
    assert L.tova_rope_apply(h, A, 0, A, 0, 1, None, 0, 0, A, 0, A, 0, None) == CUDA
    L.tova_rope_destroy(h)
    assert L.tova_quant_write(ctypes.byref(quant_cfg()), A, 0, A, 0, 1, None, 0, A, A, A, A, None) == CUDA
    assert L.tova_tree_attention(ctypes.byref(tree_cfg()), A, A, None, None, None, 1, A, A, A, 1, None, A, A, 1 << 40, None) == CUDA
    c = tova.tova_verify_config(1, 1, 8, tova.TOVA_DTYPE_FP32, 0)
    assert L.tova_verify_draft(ctypes.byref(c), A, A, A, None, A, A, A, A, A, None) == CUDA


@pytest.fixture(scope="module")
def tree_runs(tmp_path_factory):
    src = os.path.join(os.path.dirname(os.path.abspath(__file__)), "tree_runs_host.cu")
    so = str(tmp_path_factory.mktemp("tree_runs") / "tree_runs.so")
    flags = [f for f in tbuild.NVCC_FLAGS if f not in ("-O3", "-lineinfo")]
    subprocess.run([tbuild._nvcc(), *flags, "-O1", "-o", so, src], check=True, capture_output=True, text=True)
    f = ctypes.CDLL(so).check_tree_runs
    f.argtypes = [ctypes.c_int] * 5 + [ctypes.c_void_p] + [ctypes.c_int] * 6
    return f


def test_tree_runs_cover_every_job_whatever_wait_runs_out(tree_runs):
    """More than 64 rows of drafts: the tiles of all jobs are dealt out to the blocks exactly once, and the list for the joining
    kernel holds every job that was cut - also where a wait of the block ran out before it came to that job, since the NaN
    that its pieces then hold must reach the result.  (The wait is the host's stand-in: none runs out on a GPU here.)"""
    rng = random.Random(5)
    for case in range(400):
        B, Hkv, G = rng.choice([1, 2, 7, 41]), rng.choice([1, 2, 8]), rng.choice([1, 4, 8, 32])
        N = rng.randint(1, 256)
        cap = rng.choice([1, 130, 700, 5000, 70000])
        n_live = rng.randint(0, cap)
        lens = (ctypes.c_int * B)(*[rng.choice([0, 1, 128, n_live, rng.randint(0, cap)]) for _ in range(B)]) if rng.random() < 0.7 else None
        sm = rng.choice([1, 5, 100, 148])
        row_blocks = -(-N * G // rng.choice([128, 256]))
        rounds = -(-row_blocks // sm)
        group = -(-row_blocks // rounds)
        blocks = sm // group * group
        for fail_at in (-1, 0, 1, 5):
            rc = tree_runs(B, Hkv, G, N, cap, lens, n_live, blocks, group, rounds, rng.choice([1, 4]), fail_at)
            assert rc == 0, (rc, B, Hkv, G, N, cap, lens and list(lens), n_live, blocks, group, rounds, fail_at)
