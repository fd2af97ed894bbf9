"""What the calls around a step's attention refuse (stores of projection rows, weights of cached keys, eviction), before anything is
queued: addresses are never dereferenced here."""
import ctypes as C

import numpy as np
import pytest

from paper_2603_16104_amd import binding as hkv

from test_host_library import fake_pool

A = 0x100000


def code(f, *args, **kw):
    with pytest.raises(hkv.HkvError) as e:
        f(*args, **kw)
    return e.value.code


def rows(**kw):
    x = dict(q=A, k=A, v=A, q_out=2 * A, rotary_dim=128, inv_freq=A)
    x.update(kw)
    return hkv.qkv_rows(**x)


@pytest.fixture
def prefill():
    pool = fake_pool()
    plan = hkv.hkv_prefill_plan_create(pool, [0, 5, 9], [[0, 1], [2, 3]], [20, 9], 8, hkv.PLAN_HOST_ONLY)
    yield plan
    hkv.hkv_prefill_plan_destroy(plan)
    hkv.kv_pool_destroy(pool)


def decode_plan(pool, T=1, n_tokens=(32, 20, 7), leaves=(1, 2), pages=(0, 1, 2, 3, 4), reserve=0, **kw):
    nodes, begin = [], 0
    for i, n in enumerate(n_tokens):
        nodes.append((-1 if i == 0 else 0, begin, (n + 15) // 16, n))
        begin += (n + 15) // 16
    return hkv.hkv_decode_plan_create_ex(pool, nodes, list(pages)[:begin], list(leaves), 8, hkv.PLAN_HOST_ONLY, tokens_per_req=T, reserve_tokens=reserve, **kw)


BAD_ROWS = [
    (dict(q=None), hkv.EINVAL), (dict(k=None), hkv.EINVAL), (dict(v=None), hkv.EINVAL), (dict(q_out=None), hkv.EINVAL),
    (dict(q=A + 8), hkv.EINVAL), (dict(k_norm=A + 2), hkv.EINVAL), (dict(q_out=A + 4), hkv.EINVAL),
    (dict(rotary_dim=24), hkv.ESHAPE), (dict(rotary_dim=144), hkv.ESHAPE), (dict(rotary_dim=-16), hkv.ESHAPE),
    (dict(inv_freq=None), hkv.EINVAL), (dict(inv_freq=A + 4), hkv.EINVAL), (dict(positions=A + 1), hkv.EINVAL),
    (dict(q_norm=A, eps=float("nan")), hkv.EINVAL), (dict(k_norm=A, eps=-1.0), hkv.EINVAL), (dict(q_norm=A, eps=float("inf")), hkv.EINVAL),
    (dict(n_axes=5), hkv.EINVAL), (dict(n_axes=-1), hkv.EINVAL), (dict(n_axes=2), hkv.EINVAL), (dict(n_axes=2, positions=A), hkv.EINVAL),
    (dict(n_axes=3, positions=A, axis=[0, 1, 3] + [0] * 61), hkv.EINVAL), (dict(axis=[-1] * 64), hkv.EINVAL), (dict(axis=[1] * 64), hkv.EINVAL),
]


@pytest.mark.parametrize("bad, want", BAD_ROWS)
def test_store_refuses_bad_rows(prefill, bad, want):
    x = rows(**bad)
    assert code(hkv.hkv_prefill_plan_store, prefill, x, 0) == want
    pool = fake_pool()
    plan = decode_plan(pool)
    assert code(hkv.hkv_decode_plan_store, plan, x, 0) == want
    grow = decode_plan(pool, reserve=4)
    assert code(hkv.hkv_decode_plan_append_qkv, grow, None, x, 0) == want
    for p in (plan, grow):
        hkv.hkv_decode_plan_destroy(p)
    hkv.kv_pool_destroy(pool)


@pytest.mark.parametrize("field, value", [("q_stride", 1016), ("q_stride", 1028), ("k_stride", 128), ("v_stride", -256), ("position_stride", -1)])
def test_store_refuses_bad_strides(prefill, field, value):
    x = rows()
    setattr(x, field, value)
    assert code(hkv.hkv_prefill_plan_store, prefill, x, 0) == hkv.EINVAL


def test_store_refuses_queries_in_place_with_gaps(prefill):
    x = rows(q_out=A)
    x.q_stride = 2048
    assert code(hkv.hkv_prefill_plan_store, prefill, x, 0) == hkv.EINVAL


def test_store_refuses_plans_without_a_device_and_null_arguments(prefill):
    assert code(hkv.hkv_prefill_plan_store, prefill, rows(), 0) == hkv.EINVAL and "host-only" in hkv.last_error()
    assert code(hkv.hkv_prefill_plan_store, prefill, None, 0) == hkv.EINVAL
    assert code(hkv.hkv_prefill_plan_store, None, rows(), 0) == hkv.EINVAL
    assert code(hkv.hkv_decode_plan_store, None, rows(), 0) == hkv.EINVAL
    assert code(hkv.hkv_decode_plan_append_qkv, None, None, rows(), 0) == hkv.EINVAL
    pool = fake_pool()
    plan = decode_plan(pool)
    assert code(hkv.hkv_decode_plan_append_qkv, plan, None, rows(), 0) == hkv.EINVAL and "growing" in hkv.last_error()
    hkv.hkv_decode_plan_destroy(plan)
    hkv.kv_pool_destroy(pool)


def test_rows_are_checked_by_shape():
    import torch
    t = torch.zeros(4, 1536, dtype=torch.bfloat16)
    q, k, v = (x.unflatten(1, (-1, 128)) for x in t.split([1024, 256, 256], dim=1))
    x = hkv.qkv_rows(q, k, v, torch.zeros(4, 8, 128, dtype=torch.bfloat16))
    assert (x.q_stride, x.k_stride, x.v_stride, x.n_axes) == (1536, 1536, 1536, 1)
    out = torch.zeros(4, 8, 128, dtype=torch.bfloat16)
    for bad in (dict(q=q.transpose(0, 1)), dict(k=k[:1].expand(4, -1, -1)), dict(q=q[:, ::2]), dict(q=t), dict(q_out=out[:, ::2]), dict(inv_freq=torch.zeros(64)),
                dict(q_out=out.float()), dict(q_out=out[:, :4].contiguous()), dict(q_norm=torch.zeros(128)), dict(k_norm=out[0, 0, :64]), dict(v=v.float()),
                dict(inv_freq=torch.zeros(32, dtype=torch.float64)), dict(positions=torch.zeros(4, dtype=torch.int64)),
                dict(positions=torch.zeros(4)), dict(axis=[0] * 63)):
        with pytest.raises(ValueError):
            hkv.qkv_rows(**{**dict(q=q, k=k, v=v, q_out=out, rotary_dim=128, inv_freq=torch.zeros(64, dtype=torch.float64)), **bad})
    p = torch.zeros(3, 8, dtype=torch.int32)[:, :4]
    x = hkv.qkv_rows(q, k, v, out, positions=p, axis=np.arange(64) % 3, rotary_dim=128, inv_freq=torch.zeros(64, dtype=torch.float64))
    assert x.n_axes == 3 and x.position_stride == 8 and C.cast(x.axis, C.POINTER(C.c_int32))[2] == 2


def test_a_single_row_has_the_plans_heads(prefill):
    import torch
    q, k = torch.zeros(1, 8, 128, dtype=torch.bfloat16), torch.zeros(1, 2, 128, dtype=torch.bfloat16)
    for q_, k_ in ((q[:, :4], k), (q, k[:, :1])):
        assert code(hkv.hkv_prefill_plan_store, prefill, hkv.qkv_rows(q_, k_, k, q_.clone()), 0) == hkv.EINVAL and "stride" in hkv.last_error()


def test_weights_refusals():
    pool = fake_pool()
    plan = decode_plan(pool, T=3)
    run = lambda p=plan, q=A, lse=A, decay=1.0, n_new=0, w=A: hkv.attn_decode_plan_weights(p, q, 0.1, lse, decay, n_new, w, 0)  # noqa: E731
    assert code(run) == hkv.EINVAL and "track_weights" in hkv.last_error()
    hkv.hkv_decode_plan_track_weights(plan)
    hkv.hkv_decode_plan_track_weights(plan)
    for kw in (dict(q=None), dict(lse=None), dict(w=None), dict(q=A + 8), dict(w=A + 4), dict(lse=A + 2), dict(decay=-0.1), dict(decay=1.1), dict(decay=float("nan")),
               dict(n_new=-1), dict(n_new=4), dict(p=None)):
        assert code(run, **kw) == hkv.EINVAL, kw
    assert code(run, n_new=3) == hkv.EINVAL and "host-only" in hkv.last_error()
    assert code(hkv.hkv_decode_plan_track_weights, None) == hkv.EINVAL
    twice = decode_plan(pool, pages=(0, 1, 2, 3, 1))
    assert code(hkv.hkv_decode_plan_track_weights, twice) == hkv.EINVAL and "twice" in hkv.last_error()
    for p in (plan, twice):
        hkv.hkv_decode_plan_destroy(p)
    hkv.kv_pool_destroy(pool)
    pool = fake_pool(dtype=hkv.FP32)
    plan = decode_plan(pool)
    hkv.hkv_decode_plan_track_weights(plan)
    assert code(run, p=plan) == hkv.EINVAL and "host-only" in hkv.last_error()
    twice = decode_plan(pool, pages=(0, 1, 2, 3, 1))
    assert code(hkv.hkv_decode_plan_track_weights, twice) == hkv.EINVAL and "twice" in hkv.last_error()
    for p in (plan, twice):
        hkv.hkv_decode_plan_destroy(p)
    hkv.kv_pool_destroy(pool)


def test_evict_refusals():
    pool = fake_pool()
    evict = lambda src=(0, 1), n=(20,), dst=(2,), m=(10,), first=0, recent=0, w=A, kept=A, p=pool: hkv.kv_pool_evict(p, src, n, dst, m, first, recent, w, kept, 0)  # noqa: E731
    for kw in (dict(n=(-1,)), dict(m=(-1,)), dict(m=(21,), dst=(2, 3)), dict(first=-1), dict(recent=-1), dict(first=6, recent=5), dict(m=(0,), first=1),
               dict(w=None), dict(kept=None), dict(w=A + 8), dict(kept=A + 2), dict(dst=(1,)), dict(n=(20, 20)), dict(src=(0,)), dict(dst=())):
        assert code(evict, **kw) == hkv.EINVAL, kw
    assert code(evict, n=(20, 17), src=(0, 1, 2, 3), dst=(5, 5), m=(3, 3)) == hkv.EINVAL and "twice" in hkv.last_error()
    for kw in (dict(src=(0, 64)), dict(src=(-1, 0)), dict(dst=(64,)), dict(dst=(-1,))):
        assert code(evict, **kw) == hkv.ERANGE, kw
    shared = hkv.kv_pool_alloc(pool, 3)[2:]
    hkv.kv_pool_retain(pool, shared)
    assert code(evict, dst=shared) == hkv.EINVAL and "owners" in hkv.last_error()
    assert code(evict, n=(1 << 20,), src=np.zeros(65536, dtype=np.int32)) == hkv.EINVAL
    evict(n=(), src=(), dst=(), m=())                       # nothing to do
    evict(n=(20,), m=(0,), dst=())
    hkv.kv_pool_destroy(pool)
    assert code(evict, p=None) == hkv.EINVAL
