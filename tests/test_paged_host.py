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


def places(n):
    """n addresses with 16 MB between them (nothing is read through them)."""
    return [ADDR + (i << 24) for i in range(n)]


def on_the_host(status):
    """What a call with addresses of nothing ends with once its arguments have passed: there is no device here (and with one, no such memory)."""
    import torch
    return status == (BAD if torch.cuda.is_available() else rt.RT_ERR_CUDA)


def test_attention_outputs_on_anything_else():
    k, v, table, status, ke, ve, q, ko, vo, lens, slopes, out, lse, ws, free = places(15)
    names = dict(q=q, k_own=ko, v_own=vo, lens=lens, alibi_slopes=slopes, out=out, lse=lse)
    for f8 in (False, True):
        c = rt.RtPagedCache(k, v, ke if f8 else None, ve if f8 else None, table, status, 8, 16, 2, 64, rt.RT_E4M3 if f8 else rt.RT_BF16, 3, 4)
        need = rt.rt_paged_attention_workspace_bytes(c, 4)
        call = lambda work=ws, **kw: rt.rt_paged_attention(c, rt.RtPagedQuery(*{**names, **kw}.values(), 256, 128, 128, 256, rt.RT_BF16, 4, 0.125), work, need, None)
        assert on_the_host(call()) and on_the_host(call(lse=None, alibi_slopes=None)) and on_the_host(call(out=free)) and on_the_host(call(work=free, lse=ws))
        pool = 8 * 2 * 16 * 64 * (1 if f8 else 2)
        sizes = dict(k=(k, pool), v=(v, pool), table=(table, 48), status=(status, 4), q=(q, 3 * 512), k_own=(ko, 3 * 256), v_own=(vo, 3 * 256), lens=(lens, 12), slopes=(slopes, 16))
        if f8:
            sizes.update(k_exp=(ke, 256), v_exp=(ve, 256))
        for name, (at, n) in sizes.items():
            for there in (at, (at + n - 1) & ~15):                       # its first and its last 16 bytes
                assert call(out=there) == BAD and call(lse=there) == BAD and call(work=there) == BAD, name
            assert call(out=at - 3 * 512 + 16) == BAD and call(lse=at - 44) == BAD and call(work=at - need + 16) == BAD, name      # (its own last 16 bytes, the last number)
            assert on_the_host(call(out=at - 3 * 512)) and on_the_host(call(lse=at - 48)) and on_the_host(call(work=at - need)), name
            assert on_the_host(call(out=at + (n + 15) // 16 * 16)) and on_the_host(call(lse=at + (n + 3) // 4 * 4)), name
        assert call(lse=out + 512) == BAD and call(work=out) == BAD and call(work=lse) == BAD


def test_row_outputs_on_indexes_and_tables():
    k, v, table, status, kr, vr, seq, pos, free = places(9)
    c = rt.RtPagedCache(k, v, None, None, table, status, 8, 16, 2, 64, rt.RT_BF16, 3, 4)
    names = dict(k=kr, v=vr, seq=seq, pos=pos)
    for f in (rt.rt_cache_write, rt.rt_cache_read):
        call = lambda c=c, ks=128, vs=128, **kw: f(c, rt.RT_BF16, *list({**names, **kw}.values())[:2], ks, vs, *list({**names, **kw}.values())[2:], 40, None)
        assert on_the_host(call()) and on_the_host(call(k=kr, v=kr + 256, ks=256, vs=256))
    read = lambda **kw: rt.rt_cache_read(c, rt.RT_BF16, *{**dict(k=kr, v=vr, ks=128, vs=128, seq=seq, pos=pos), **kw}.values(), 40, None)
    for at in (seq, seq + 144, pos, table, table + 32, status):
        assert read(k=at) == BAD and read(v=at) == BAD
    # rows of two strides that lie in one stretch of memory: in the gaps, or on one another far from the beginning
    assert on_the_host(read(k=kr, ks=512, v=kr + 256, vs=1024)) and on_the_host(read(k=kr, ks=1024, v=kr + 256, vs=512))
    assert read(k=kr, ks=512, v=kr + 256, vs=136) == BAD and read(k=kr, ks=136, v=kr + 256, vs=512) == BAD
    # rows of 256 bytes, 1280 and 1296 apart: the second ones begin 256 - 16 i bytes behind the first ones, or 256 + 16 i (and row 49 reaches row 50 of the others: 16 * 49 > 1280 - 512)
    assert read(k=kr, ks=648, v=kr + 256, vs=640) == BAD and on_the_host(read(k=kr, ks=640, v=kr + 256, vs=648))
    assert rt.rt_cache_read(c, rt.RT_BF16, kr, kr + 256, 640, 648, seq, pos, 51, None) == BAD and on_the_host(rt.rt_cache_read(c, rt.RT_BF16, kr, kr + 256, 640, 648, seq, pos, 50, None))
    for kw in (dict(k=seq), dict(v=pos), dict(k=table), dict(v=table - 32752), dict(k=status), dict(k_exp=seq, v_exp=free, dtype=rt.RT_E4M3), dict(k_exp=free, v_exp=pos - 240, dtype=rt.RT_E4M3),
               dict(k_exp=free, v_exp=table, dtype=rt.RT_E4M3)):
        other = rt.RtPagedCache(k, v, None, None, table, status, 8, 16, 2, 64, rt.RT_BF16, 3, 4)
        for n, x in kw.items():
            setattr(other, n, x)
        assert rt.rt_cache_write(other, rt.RT_BF16, kr, vr, 128, 128, seq, pos, 40, None) == BAD, kw


def test_rotation_outputs_on_gains_and_positions():
    q, k, gq, gk, pos, qo, ko, free = places(8)
    base = dict(q=q, k=k, qs=256, ks=128, gq=gq, gk=gk, pos=pos, rows=40, qo=qo, ko=ko, qos=256, kos=128)
    call = lambda cfg={}, **kw: rt.rt_qk_rotate(config(**cfg), *{**base, **kw}.values(), None)
    assert on_the_host(call()) and on_the_host(call(qo=q, ko=k)) and on_the_host(call(qo=gk, ko=gk, cfg=dict(n_kv_heads=0)))
    for at in (gq, gq + 496, gk, gk + 240, pos, pos + 144):
        assert call(qo=at) == BAD and call(ko=at) == BAD
    assert call(qo=q, qs=256, qos=264) == BAD and call(qo=q + 256, qs=264) == BAD and call(ko=k + 128 * 39, ks=136) == BAD
    # rows of 512 bytes, 2048 apart: others in their gaps every 1024 or 4096 bytes, but not every 1536
    assert on_the_host(call(q=q, qs=1024, qo=q + 512, qos=512)) and on_the_host(call(q=q, qs=1024, qo=q + 512, qos=2048)) and call(q=q, qs=1024, qo=q + 512, qos=768) == BAD


def test_gradients_on_anything_else():
    q, k, gq, gk, pos, dqo, dko, dq, dk, dgq, dgk, ws, free = places(13)
    base = dict(q=q, k=k, qs=256, ks=128, gq=gq, gk=gk, pos=pos, rows=40, dqo=dqo, dko=dko, dq=dq, dk=dk, dgq=dgq, dgk=dgk, ws=ws)
    need = rt.rt_qk_rotate_backward_workspace_bytes(config(), 40)
    call = lambda cfg={}, **kw: rt.rt_qk_rotate_backward(config(**cfg), *{**base, **kw}.values(), need, None)
    assert on_the_host(call()) and on_the_host(call(dq=dqo, dk=dko)) and on_the_host(call(dgq=None, dgk=None, ws=q)) and on_the_host(call(dgq=None))
    sizes = dict(q=(q, 40 * 512), k=(k, 40 * 256), gq=(gq, 512), gk=(gk, 256), pos=(pos, 160), dqo=(dqo, 40 * 1024), dko=(dko, 40 * 512), dq=(dq, 40 * 1024), dk=(dk, 40 * 512),
                 dgq=(dgq, 1024), dgk=(dgk, 512))
    outs = dict(dq=40 * 1024, dk=40 * 512, dgq=1024, dgk=512, ws=need)
    for out, n in outs.items():
        for name, (at, size) in sizes.items():
            if name == out:
                continue
            assert call(**{out: at + size - 16}) == BAD and call(**{out: at - n + 16}) == BAD, (out, name)
            assert on_the_host(call(**{out: at + size})) and on_the_host(call(**{out: at - n // 16 * 16})), (out, name)
            if (out, name) not in (("dq", "dqo"), ("dk", "dko")):
                assert call(**{out: at}) == BAD, (out, name)
    # without rows the gains' gradients are written all the same
    assert call(rows=0, dgq=gq) == BAD and call(rows=0, dgq=free, dgk=free + 512) == BAD and on_the_host(call(rows=0, q=None, k=None, dqo=None, dko=None, dq=None, dk=None, pos=None))
