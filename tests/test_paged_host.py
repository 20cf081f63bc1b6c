"""Argument checks of the operators around paged caches: all of them run on the host, before any CUDA call."""
import ctypes as C
import math

import pytest

from paper_2604_21215_b200 import rt

BUF = (C.c_char * 8192)()
ADDR = (C.addressof(BUF) + 255) & ~255


def cache(**kw):
    c = rt.RtPagedCache(ADDR, ADDR, None, None, ADDR, ADDR, 8, 16, 2, 64, rt.RT_BF16, 3, 4)
    for n, x in kw.items():
        setattr(c, n, x)
    return c


def query(**kw):
    q = rt.RtPagedQuery(ADDR, None, None, ADDR, None, ADDR + 4096, None, 128, 0, 0, 128, rt.RT_BF16, 2, 0.125)
    for n, x in kw.items():
        setattr(q, n, x)
    return q


BAD, UNSUPPORTED = rt.RT_ERR_INVALID_ARG, rt.RT_ERR_UNSUPPORTED
CACHES = [(dict(k=None), BAD), (dict(v=None), BAD), (dict(page_table=None), BAD), (dict(n_pages=0), BAD), (dict(page_size=-16), BAD), (dict(n_kv_heads=0), BAD),
          (dict(n_seqs=0), BAD), (dict(max_pages=0), BAD), (dict(dtype=3), BAD), (dict(dtype=-1), BAD), (dict(k=ADDR + 8), BAD), (dict(v=ADDR + 4), BAD),
          (dict(dtype=rt.RT_E4M3), BAD), (dict(dtype=rt.RT_E4M3, k_exp=ADDR), BAD), (dict(k_exp=ADDR, v_exp=ADDR), BAD), (dict(page_table=ADDR + 2), BAD),
          (dict(status=ADDR + 1), BAD), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=32), UNSUPPORTED), (dict(page_size=8), UNSUPPORTED),
          (dict(page_size=48), UNSUPPORTED), (dict(page_size=512), UNSUPPORTED), (dict(n_kv_heads=1 << 20), UNSUPPORTED)]


@pytest.mark.parametrize("change,want", CACHES)
def test_caches_that_are_refused(change, want):
    c = cache(**change)
    rows = lambda f: f(c, rt.RT_BF16, ADDR, ADDR, 1 << 20, 1 << 20, ADDR, ADDR, 1, None)
    assert rows(rt.rt_cache_write) == want and rows(rt.rt_cache_read) == want
    assert rt.rt_paged_attention(c, query(), ADDR, 1 << 40, None) == want
    assert rt.rt_paged_attention_workspace_bytes(c, 2) == 0


@pytest.mark.parametrize("f", [rt.rt_cache_write, rt.rt_cache_read])
def test_rows_that_are_refused(f):
    call = lambda dtype=rt.RT_BF16, k=ADDR, v=ADDR, ks=128, vs=128, seq=ADDR, pos=ADDR, rows=4: f(cache(), dtype, k, v, ks, vs, seq, pos, rows, None)
    for kw in (dict(dtype=rt.RT_E4M3), dict(dtype=7), dict(k=None), dict(v=None), dict(seq=None), dict(pos=None), dict(rows=-1), dict(ks=127), dict(vs=132),
               dict(ks=64), dict(ks=0), dict(ks=-128), dict(k=ADDR + 8), dict(pos=ADDR + 2), dict(ks=1 << 62)):
        assert call(**kw) == BAD, kw
    assert call(rows=0) == rt.RT_OK and call(rows=0, k=None, v=None, seq=None, pos=None) == rt.RT_OK


def test_queries_that_are_refused():
    call = lambda need=1 << 40, ws=ADDR, **kw: rt.rt_paged_attention(cache(), query(**kw), ws, need, None)
    for kw in (dict(q=None), dict(out=None), dict(lens=None), dict(dtype=rt.RT_E4M3), dict(n_heads=0), dict(n_heads=3), dict(n_heads=-2), dict(k_own=ADDR),
               dict(v_own=ADDR), dict(k_own=ADDR, v_own=ADDR), dict(k_own=ADDR, v_own=ADDR, k_own_stride=128, v_own_stride=64), dict(q_stride=64),
               dict(q_stride=130), dict(out_stride=0), dict(q=ADDR + 2), dict(out=ADDR + 8), dict(lens=ADDR + 1), dict(alibi_slopes=ADDR + 2),
               dict(lse=ADDR + 3), dict(softmax_scale=math.inf), dict(softmax_scale=math.nan), dict(ws=None), dict(ws=ADDR + 8),
               # out on the queries, on their last row, on the own pairs
               dict(out=ADDR), dict(out=ADDR + 512), dict(out=ADDR, out_stride=256),
               dict(k_own=ADDR + 4096, v_own=ADDR, k_own_stride=128, v_own_stride=128)):
        assert call(**kw) == BAD, kw
    assert call(n_heads=2 * 2048, q_stride=2 * 2048 * 64, out_stride=2 * 2048 * 64) == UNSUPPORTED
    need = rt.rt_paged_attention_workspace_bytes(cache(), 2)
    assert need > 0 and call(need=need - 1) == rt.RT_ERR_WORKSPACE
    assert rt.rt_paged_attention_workspace_bytes(cache(), 3) == 0 and rt.rt_paged_attention_workspace_bytes(cache(), 0) == 0


def config(**kw):
    c = rt.RtRotateConfig(rt.RT_BF16, 4, 2, 64, rt.RT_NORM_QK, 1e-6, 64, rt.RT_PAIRS_HALVES, (C.c_double * 64)(*[0.5] * 64))
    for n, x in kw.items():
        setattr(c, n, x)
    return c


@pytest.mark.parametrize("change,want", [
    (dict(dtype=rt.RT_E4M3), BAD), (dict(n_heads=0), BAD), (dict(n_kv_heads=-1), BAD), (dict(norm_flags=rt.RT_NORM_PRE), BAD), (dict(rms_eps=-1.0), BAD),
    (dict(rms_eps=math.nan), BAD), (dict(rot_dim=-16), BAD), (dict(rot_dim=80), BAD), (dict(pairs=2), BAD), (dict(freq=C.POINTER(C.c_double)()), BAD),
    (dict(freq=(C.c_double * 64)(*[math.nan] * 64)), BAD), (dict(head_dim=32, rot_dim=32), UNSUPPORTED), (dict(rot_dim=24), UNSUPPORTED),
    (dict(n_heads=70000), UNSUPPORTED)])
def test_rotations_that_are_refused(change, want):
    c = config(**change)
    assert rt.rt_qk_rotate(c, ADDR, ADDR, 1 << 24, 1 << 24, None, None, ADDR, 1, ADDR, ADDR, 1 << 24, 1 << 24, None) == want
    assert rt.rt_qk_rotate_backward_workspace_bytes(c, 1) == 0
    assert rt.rt_qk_rotate_backward(c, ADDR, ADDR, 1 << 24, 1 << 24, None, None, ADDR, 1, ADDR, ADDR, ADDR, ADDR, None, None, ADDR, 1 << 40, None) == want


def test_rows_to_rotate_that_are_refused():
    base = dict(q=ADDR, k=ADDR + 256, qs=256, ks=128, gq=None, gk=None, pos=ADDR, rows=3, qo=ADDR, ko=ADDR + 256, qos=256, kos=128)
    call = lambda **kw: rt.rt_qk_rotate(config(), *{**base, **kw}.values(), None)
    for kw in (dict(q=None), dict(k=None), dict(pos=None), dict(rows=-1), dict(qo=None), dict(ko=None), dict(qs=128), dict(qs=260), dict(ks=100), dict(qos=0),
               dict(kos=64), dict(gq=ADDR + 2), dict(gk=ADDR + 8), dict(q=ADDR + 8), dict(pos=ADDR + 2), dict(qos=264), dict(kos=136), dict(qo=ADDR + 32), dict(qo=ADDR + 256), dict(ko=ADDR),
               dict(qo=ADDR + 4096, ko=ADDR + 4096)):
        assert call(**kw) == BAD, kw
    assert call(rows=0) == rt.RT_OK
    need = rt.rt_qk_rotate_backward_workspace_bytes(config(), 1000)
    assert need >= rt.rt_qk_rotate_backward_workspace_bytes(config(), 10) >= rt.rt_qk_rotate_backward_workspace_bytes(config(), 0) > 0
    sizes = [rt.rt_qk_rotate_backward_workspace_bytes(config(), r) for r in (0, 1, 16, 17, 1000, 18943, 18944, 18945, 40000, 1 << 30)]
    assert sizes == sorted(sizes)                              # a workspace for many rows serves fewer
    grad = dict(q=ADDR, k=ADDR, qs=256, ks=128, gq=None, gk=None, pos=ADDR, rows=1000, dqo=ADDR, dko=ADDR + (1 << 24), dq=ADDR + (1 << 25), dk=ADDR + (1 << 26), dgq=None, dgk=None, ws=ADDR, n=need)
    call = lambda **kw: rt.rt_qk_rotate_backward(config(), *{**grad, **kw}.values(), None)
    for kw in (dict(q=None), dict(dqo=None), dict(dko=None), dict(dq=None), dict(dk=None), dict(dqo=ADDR + 4), dict(dk=ADDR + 8), dict(dgq=ADDR + 4), dict(ws=None),
               dict(ws=ADDR + 16 + 4), dict(rows=-1), dict(qs=0), dict(dq=ADDR + 16), dict(dk=ADDR), dict(dq=ADDR + (1 << 24)), dict(dk=ADDR + (1 << 25))):
        assert call(**kw) == BAD, kw
    assert call(n=need - 1) == rt.RT_ERR_WORKSPACE


def test_outputs_that_lie_in_the_pools_or_on_inputs_of_the_other_kind():
    big = 1 << 24
    apart = lambda **kw: cache(**{**dict(v=ADDR + big), **kw})                # pools of 32 KB
    write = lambda c, k, v: rt.rt_cache_write(c, rt.RT_BF16, k, v, 128, 128, ADDR, ADDR, 4, None)
    read = lambda c, k, v: rt.rt_cache_read(c, rt.RT_BF16, k, v, 128, 128, ADDR, ADDR, 4, None)
    assert write(cache(), ADDR + 2 * big, ADDR + 3 * big) == BAD             # keys and values in one pool
    for f in (write, read):
        assert f(apart(), ADDR + 16, ADDR + 3 * big) == BAD and f(apart(), ADDR + 3 * big, ADDR + big + 32768 - 16) == BAD
        assert f(apart(), ADDR + big - 512, ADDR + 3 * big) == BAD             # the last row reaches the values' first
    f8 = apart(dtype=rt.RT_E4M3, k_exp=ADDR + 4 * big, v_exp=ADDR + 5 * big)
    assert write(f8, ADDR + 5 * big, ADDR + 3 * big) == BAD and write(apart(dtype=rt.RT_E4M3, k_exp=ADDR + 4 * big, v_exp=ADDR + 4 * big), ADDR + 2 * big, ADDR + 3 * big) == BAD
    attend = lambda **kw: rt.rt_paged_attention(apart(), query(**{**dict(q=ADDR + 2 * big, out=ADDR + 3 * big), **kw}), ADDR, 1 << 40, None)
    assert attend(out=ADDR + 4096) == BAD and attend(out=ADDR + big - 16) == BAD and attend(lse=ADDR + big + 32764) == BAD
    grad = dict(q=ADDR, k=ADDR + big, qs=256, ks=128, gq=None, gk=None, pos=ADDR, rows=100, dqo=ADDR + 2 * big, dko=ADDR + 3 * big, dq=ADDR + 4 * big, dk=ADDR + 5 * big,
                dgq=None, dgk=None, ws=ADDR, n=1 << 40)
    call = lambda **kw: rt.rt_qk_rotate_backward(config(), *{**grad, **kw}.values(), None)
    for kw in (dict(dq=ADDR + big), dict(dk=ADDR), dict(dgq=ADDR + 6 * big, dgk=ADDR + 6 * big), dict(dgq=ADDR + 6 * big, dgk=ADDR + 6 * big + 256)):
        assert call(**kw) == BAD, kw
