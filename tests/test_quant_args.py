"""Calls on a cache that is generated into refuse on the host what they do not support, with a text.  Nothing here reaches a GPU: pointers are
made up, every refusal comes before a launch."""
import ctypes as C
import os

import pytest

import paper_2503_23956_amd as A
from paper_2503_23956_amd import binding

P = 4096  # an aligned address that is never read
INVALID, SHAPE, WORKSPACE = binding.AIR_ERR_INVALID_ARG, binding.AIR_ERR_SHAPE, binding.AIR_ERR_WORKSPACE


def _lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2503_23956_amd.build import build

        build(verbose=False)
    return A.load_library()


def _cache(**kw):
    f = dict(batch=2, n_kv_heads=2, capacity=100, head_dim=128, group=32, dtype=A.AIR_BF16, k_codes=P, v_codes=P, k_scales=P, v_scales=P)
    f.update(kw)
    return A.air_quant_cache(**f)


def _rows(**kw):
    f = dict(k=P, v=P, k_b=1280, k_h=128, k_t=256, v_b=1280, v_h=128, v_t=256, n_tokens=5, lens=P, counts=P, positions=0, first_positions=0, weights=0)
    f.update(kw)
    return A.air_quant_rows(**f)


def _query(**kw):
    f = dict(n_q_heads=4, n_tokens=5, causal=1, max_len=0, scale=0.0, q=P, out=P, q_b=2560, q_h=128, q_t=512, out_b=2560, out_h=128, out_t=512,
             lens=P, counts=P, weights=0)
    f.update(kw)
    return A.air_quant_query(**f)


BAD_CACHES = [dict(head_dim=96), dict(group=16), dict(group=128), dict(dtype=2), dict(batch=-1), dict(n_kv_heads=0), dict(batch=300, n_kv_heads=300),
              dict(capacity=0), dict(capacity=(1 << 24) + 1), dict(k_codes=0), dict(v_scales=0), dict(v_codes=P + 8), dict(k_scales=P + 4)]


@pytest.mark.parametrize("bad", BAD_CACHES)
def test_bad_caches(bad):
    lib, c = _lib(), _cache(**bad)
    for name, more in (("air_quant_append", (C.byref(_rows()),)), ("air_quant_read", (C.byref(_rows()),)),
                       ("air_quant_attn", (C.byref(_query()), None, None, 0))):
        assert getattr(lib, name)(None, C.byref(c), *more) == SHAPE
        assert lib.air_last_error(None).startswith(name.encode() + b": ")


@pytest.mark.parametrize("status,bad,names", [
    (SHAPE, dict(n_tokens=-1), "ar"), (SHAPE, dict(n_tokens=1 << 27), "ar"), (INVALID, dict(k=P + 8), "ar"), (INVALID, dict(lens=P + 2), "ar"),
    (INVALID, dict(counts=P + 1), "ar"), (SHAPE, dict(k_t=-256), "ar"), (SHAPE, dict(v_h=132), "ar"),
    (INVALID, dict(k=0), "a"), (INVALID, dict(v=0), "a"), (INVALID, dict(positions=P), "a"), (INVALID, dict(weights=P + 2), "a"),
    (INVALID, dict(positions=P, first_positions=P), "r"), (INVALID, dict(weights=P), "r"), (INVALID, dict(k=0, v=0), "r"),
    (SHAPE, dict(k_t=0), "r"), (SHAPE, dict(v_h=64), "r"), (SHAPE, dict(v_b=0), "r"),
])
def test_bad_rows(status, bad, names):
    lib = _lib()
    for n in names:
        fn = lib.air_quant_append if n == "a" else lib.air_quant_read
        assert fn(None, C.byref(_cache()), C.byref(_rows(**bad))) == status
    assert lib.air_quant_append(None, None, C.byref(_rows())) == INVALID and lib.air_quant_read(None, C.byref(_cache()), None) == INVALID


@pytest.mark.parametrize("status,bad", [
    (SHAPE, dict(n_q_heads=3)), (SHAPE, dict(n_q_heads=0)), (SHAPE, dict(n_q_heads=32768)), (SHAPE, dict(n_tokens=-1)), (SHAPE, dict(n_tokens=1 << 24)),
    (INVALID, dict(causal=2)), (INVALID, dict(max_len=-1)), (INVALID, dict(scale=-1.0)), (INVALID, dict(scale=float("nan"))),
    (INVALID, dict(scale=3e38)), (SHAPE, dict(q_t=-512)), (SHAPE, dict(out_h=4)), (SHAPE, dict(out_t=0)), (SHAPE, dict(out_h=64)),
    (INVALID, dict(q=0)), (INVALID, dict(lens=0)), (INVALID, dict(out=0)), (INVALID, dict(q=P + 8)), (INVALID, dict(weights=P + 2)),
    (INVALID, dict(counts=P + 2)), (WORKSPACE, dict()),
])
def test_bad_queries(status, bad):
    lib = _lib()
    assert lib.air_quant_attn(None, C.byref(_cache(capacity=10000)), C.byref(_query(**bad)), None, None, 0) == status
    assert lib.air_last_error(None).startswith(b"air_quant_attn: ")


def test_bad_appends_of_a_query():
    lib = _lib()
    for bad in (dict(n_tokens=4), dict(lens=2 * P), dict(counts=0), dict(k=0), dict(positions=P), dict(v_t=4)):
        st = lib.air_quant_attn(None, C.byref(_cache()), C.byref(_query()), C.byref(_rows(**bad)), None, 0)
        assert st == (SHAPE if "v_t" in bad else INVALID), bad


def test_workspaces():
    lib = _lib()
    size = lambda q, c: lib.air_quant_workspace_bytes(C.byref(c), C.byref(q))  # noqa: E731
    big = _cache(capacity=10000)
    need = size(_query(), big)
    assert need > 0 and need == size(_query(), _cache(capacity=10000, k_codes=0, v_codes=0, k_scales=0, v_scales=0))
    assert size(_query(max_len=1), big) == 0  # one workgroup a row block
    assert size(_query(max_len=1, weights=P), big) > 0
    assert size(_query(n_q_heads=3), big) == 0 and size(_query(n_tokens=0), big) == 0
    for ws, n in ((None, need), (P + 16, need), (P, need - 1)):
        assert lib.air_quant_attn(None, C.byref(big), C.byref(_query()), None, ws, n) == WORKSPACE


def test_workspaces_of_few_rows_do_not_grow_without_bound():
    lib = _lib()
    size = lambda q, c: lib.air_quant_workspace_bytes(C.byref(c), C.byref(q))  # noqa: E731
    most = 0
    for log2 in range(8, 25):
        for batch in (1, 3, 64):
            most = max(most, size(_query(n_tokens=1, weights=P), _cache(batch=batch, capacity=1 << log2)))
    assert 2 ** 29 < most < 2 ** 30 + 2 ** 24


def test_workspaces_of_many_rows_do_not_follow_the_capacity():
    lib = _lib()
    q = _query(n_tokens=2000, weights=P, max_len=100, q_b=2000 * 512, out_b=2000 * 512)
    assert 0 < lib.air_quant_workspace_bytes(C.byref(_cache(capacity=1 << 24)), C.byref(q)) < 2 ** 29 + 2 ** 26


def _evict(n_planes=1, plane=None, w=P, pos=P, lens=P, out=2 * P, ws=None, nbytes=0, **kw):
    f = dict(batch=2, n_heads=2, capacity=100, keep=40, limit=50, first=2, recent=8)
    f.update(kw)
    p = dict(rows=P, b=100 * 512, h=100 * 256, t=256, row_bytes=256)
    p.update(plane or {})
    cfg = A.air_evict_config(n_planes=n_planes, **f)
    cfg.planes[0] = A.air_evict_plane(**p)
    lib = _lib()
    return lib.air_evict(None, C.byref(cfg), w, pos, lens, out, ws, nbytes), lib.air_evict_workspace_bytes(C.byref(cfg))


@pytest.mark.parametrize("status,kw", [
    (SHAPE, dict(batch=-1)), (SHAPE, dict(n_heads=0)), (SHAPE, dict(batch=300, n_heads=300)), (SHAPE, dict(capacity=0)), (SHAPE, dict(capacity=1 << 25)),
    (INVALID, dict(keep=0, first=0, recent=0)), (INVALID, dict(limit=39)), (INVALID, dict(first=-1)), (INVALID, dict(recent=-1)),
    (INVALID, dict(first=33)), (INVALID, dict(first=2 ** 31 - 1, recent=2 ** 31 - 1)), (INVALID, dict(n_planes=-1)), (INVALID, dict(n_planes=9)),
    (INVALID, dict(plane=dict(rows=P + 2))), (INVALID, dict(plane=dict(rows=0))), (SHAPE, dict(plane=dict(row_bytes=0))),
    (SHAPE, dict(plane=dict(row_bytes=6))), (SHAPE, dict(plane=dict(row_bytes=1028))), (SHAPE, dict(plane=dict(t=-256))), (SHAPE, dict(plane=dict(t=258))),
    (SHAPE, dict(plane=dict(t=252))), (SHAPE, dict(plane=dict(h=0))), (SHAPE, dict(capacity=1 << 24, plane=dict(t=1024, h=1 << 34, b=1 << 35, row_bytes=1024))),
    (INVALID, dict(w=0)), (INVALID, dict(lens=0)), (INVALID, dict(out=0)), (INVALID, dict(out=P)), (INVALID, dict(w=P + 2)), (INVALID, dict(pos=P + 1)),
    (INVALID, dict(pos=0)),
])
def test_bad_evictions(status, kw):
    assert _evict(**kw)[0] == status
    lib = _lib()
    _evict(**kw)
    lib.air_evict(None, None, P, P, P, 2 * P, None, 0)
    assert lib.air_last_error(None).startswith(b"air_evict: ")


def test_an_evictions_lengths_lie_apart():
    assert all(_evict(lens=P, out=P + at)[0] == INVALID for at in (-4, 0, 4))  # two sequences


def test_eviction_workspaces():
    assert _evict(capacity=40, n_planes=0, batch=0)[1] == 0 and _evict(batch=0)[1] == 0
    big = dict(capacity=20000, keep=9000, limit=9000, plane=dict(h=20000 * 256, b=20000 * 512))
    st, need = _evict(**big)
    assert st == WORKSPACE and need >= 2 * 2 * 2 * 9000 * 4
    assert _evict(ws=P + 8, nbytes=need, **big)[0] == WORKSPACE and _evict(ws=P, nbytes=need - 1, **big)[0] == WORKSPACE


def test_nothing_to_do_is_no_error():
    lib = _lib()
    empty = _cache(batch=0, k_codes=0, v_codes=0, k_scales=0, v_scales=0)
    assert lib.air_quant_append(None, C.byref(empty), C.byref(_rows(k=0, v=0))) == 0
    assert lib.air_quant_read(None, C.byref(_cache()), C.byref(_rows(n_tokens=0, k=0, v=0))) == 0
    assert lib.air_quant_attn(None, C.byref(_cache()), C.byref(_query(n_tokens=0, q=0, out=0)), None, None, 0) == 0
    assert lib.air_quant_attn(None, C.byref(empty), C.byref(_query(q=0)), C.byref(_rows(k=0, v=0)), None, 0) == 0
    assert _evict(batch=0, w=0, lens=0, out=0)[0] == 0


def test_the_binding_refuses_what_it_cannot_marshal():
    import torch

    cache = A.QuantCache(2, 2, 20, 64, A.AIR_F32, device="cpu")
    x = torch.zeros((2, 2, 3, 64))
    q = torch.zeros((2, 4, 3, 64))
    lens, w = torch.zeros(2, dtype=torch.int32), torch.zeros((2, 2, 20))
    bad = [
        lambda: A.QuantCache(1, 1, 1, 96, device="cpu"), lambda: A.QuantCache(0, 1, 1, 64, device="cpu"),
        lambda: A.prepare_quant_append(cache, x, None), lambda: A.prepare_quant_append(cache, x.bfloat16(), x.bfloat16()),
        lambda: A.prepare_quant_append(cache, x, x[:, :, :2]), lambda: A.prepare_quant_append(cache, x[:1], x[:1]),
        lambda: A.prepare_quant_append(cache, x, x, lens=lens.long()), lambda: A.prepare_quant_append(cache, x, x, lens=lens[:1]),
        lambda: A.prepare_quant_append(cache, x, x, weights=w[:, :, :19]), lambda: A.prepare_quant_read(cache),
        lambda: A.prepare_quant_attn(cache, q, q[:, :, :2], lens=lens), lambda: A.prepare_quant_attn(cache, q, q, lens=None),
        lambda: A.prepare_quant_attn(cache, q, q, lens=lens, k=x), lambda: A.prepare_quant_attn(cache, q, q, lens=lens, positions=lens),
        lambda: A.prepare_quant_attn(cache, q, q, lens=lens, weights=w.double()),
        lambda: A.prepare_evict([x], w, lens=lens, lens_out=lens.clone(), keep=5), lambda: A.prepare_evict([], w[0], lens=lens, lens_out=lens, keep=5),
        lambda: A.prepare_evict([], w, lens=lens, lens_out=None, keep=5), lambda: A.prepare_evict([w[..., None]] * 9, w, lens=lens, lens_out=lens, keep=5),
        lambda: A.air_quant_append(cache, x, x),  # not on a GPU
        lambda: A.air_evict([], w, lens=lens, lens_out=lens.clone(), keep=5),
        lambda: A.prepare_quant_append(cache, x, x)(0, w),
    ]
    for i, f in enumerate(bad):
        with pytest.raises(A.AirError):
            f()
            pytest.fail(f"case {i} was taken")
