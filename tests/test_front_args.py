"""The calls that need no context refuse on the host what they do not support, with a text, and the frequencies follow their
formulas.  Nothing here reaches a GPU: pointers are made up, every refusal comes before a launch."""
import ctypes as C
import os
import re

import numpy as np
import pytest

import paper_2503_23956_amd as A
from paper_2503_23956_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 4096  # an aligned address that is never read


def _lib():
    if not os.path.exists(binding.LIB_PATH):
        from paper_2503_23956_amd.build import build

        build(verbose=False)
    return A.load_library()


def _rope(null=(), pos=P, freqs=P, tensors=None, **kw):
    f = dict(n_q_heads=4, n_kv_heads=2, head_dim=128, dtype=A.AIR_BF16, batch=2, n_tokens=5, layout=0, n_axes=1,
             axis_pairs=(64, 0, 0), norm_eps=1e-6, scale=1.0)
    f.update(kw)
    f["axis_pairs"] = (C.c_int32 * 3)(*f["axis_pairs"])
    cfg = A.air_rope_config(**f)
    ts = {}
    for name, heads in (("q", 4), ("k", 2), ("v", 2)):
        t = dict(src=P, dst=2 * P, weight=0, src_b=5 * heads * 128, src_h=128, src_t=heads * 128, dst_b=5 * heads * 128, dst_h=5 * 128, dst_t=128)
        t.update((tensors or {}).get(name, {}))
        ts[name] = A.air_rope_tensor(**t)
    return _lib().air_rope(None, C.byref(cfg), *(None if n in null else C.byref(ts[n]) for n in ("q", "k", "v")), pos, freqs)


def _attn(seqs=((0, 0, 0, 0, 3, 3),), n=None, q=P, k=P, v=P, out=P, ws=None, nbytes=0, **kw):
    f = dict(n_q_heads=4, n_kv_heads=2, head_dim=128, dtype=A.AIR_BF16, scale=0.0, q_h=128, q_t=512, k_h=128, k_t=256, v_h=128, v_t=256,
             out_h=128, out_t=512)
    f.update(kw)
    arr = (A.air_prompt_seq * max(1, len(seqs)))(*(A.air_prompt_seq(*s) for s in seqs))
    n = len(seqs) if n is None else n
    cfg = A.air_prompt_config(**f)
    return (_lib().air_prompt_attn(None, C.byref(cfg), arr, n, q, k, v, out, ws, nbytes),
            _lib().air_prompt_workspace_bytes(C.byref(cfg), arr, n))


INVALID, SHAPE, WORKSPACE = binding.AIR_ERR_INVALID_ARG, binding.AIR_ERR_SHAPE, binding.AIR_ERR_WORKSPACE


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(null=("q", "k", "v"))),
    (INVALID, dict(pos=None)), (INVALID, dict(freqs=None)), (INVALID, dict(pos=P + 2)), (INVALID, dict(freqs=P + 4)),
    (SHAPE, dict(dtype=2)), (SHAPE, dict(head_dim=96)), (SHAPE, dict(n_q_heads=5)), (SHAPE, dict(n_kv_heads=0)),
    (SHAPE, dict(n_q_heads=32768, n_kv_heads=32768)),
    (SHAPE, dict(batch=-1)), (SHAPE, dict(n_tokens=-1)), (SHAPE, dict(batch=1 << 16, n_tokens=1 << 16)), (SHAPE, dict(batch=3, n_tokens=1 << 26)),
    (INVALID, dict(layout=2)), (INVALID, dict(n_axes=0)), (INVALID, dict(n_axes=4)),
    (SHAPE, dict(axis_pairs=(60, 0, 0))), (SHAPE, dict(axis_pairs=(72, 0, 0))), (SHAPE, dict(axis_pairs=(-8, 0, 0))),
    (SHAPE, dict(n_axes=3, axis_pairs=(32, 40, -8))),
    (INVALID, dict(norm_eps=-1.0)), (INVALID, dict(norm_eps=float("nan"))), (INVALID, dict(scale=float("inf"))),
    (INVALID, dict(tensors=dict(q=dict(src=0)))), (INVALID, dict(tensors=dict(k=dict(dst=0)))),
    (INVALID, dict(tensors=dict(q=dict(src=P + 8)))), (INVALID, dict(tensors=dict(k=dict(weight=P + 2)))),
    (INVALID, dict(tensors=dict(v=dict(weight=P)))),
    (SHAPE, dict(tensors=dict(q=dict(src_t=-128)))), (SHAPE, dict(tensors=dict(q=dict(src_h=132)))),
    (SHAPE, dict(tensors=dict(q=dict(dst_t=0)))), (SHAPE, dict(tensors=dict(k=dict(dst_h=64)))), (SHAPE, dict(tensors=dict(v=dict(dst_b=0)))),
    (SHAPE, dict(tensors=dict(q=dict(dst=P)))),  # in place with other strides
])
def test_rope_refusals(status, kw):
    assert _rope(**kw) == status
    assert _lib().air_last_error(None).startswith(b"air_rope: ")


def test_nothing_to_do_is_no_error():
    assert _rope(batch=0) == 0 and _rope(n_tokens=0) == 0
    assert _rope(n_tokens=0, pos=None, freqs=None, tensors=dict(q=dict(src=0, dst=0))) == 0
    assert _attn(seqs=()) == (0, 0)
    assert _attn(seqs=((0, 0, 0, 0, 0, 7),), q=None, k=None, v=None, out=None) == (0, 0)


@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(q=None)), (INVALID, dict(k=None)), (INVALID, dict(v=None)), (INVALID, dict(out=None)),
    (INVALID, dict(q=P + 2)), (INVALID, dict(k=P + 4)), (INVALID, dict(v=P + 8)), (INVALID, dict(out=P + 1)),
    (SHAPE, dict(dtype=-1)), (SHAPE, dict(head_dim=80)), (SHAPE, dict(n_q_heads=3)), (SHAPE, dict(n_kv_heads=-2)),
    (SHAPE, dict(n=65)), (SHAPE, dict(n=-1)),
    (INVALID, dict(scale=-0.1)), (INVALID, dict(scale=float("nan"))), (INVALID, dict(scale=float("inf"))),
    (SHAPE, dict(q_t=-512)), (SHAPE, dict(k_h=4)), (SHAPE, dict(out_t=120)), (SHAPE, dict(k_t=1 << 24)), (SHAPE, dict(v_t=1 << 24)), (SHAPE, dict(out_h=0)), (SHAPE, dict(out_t=0)),
    (SHAPE, dict(seqs=((0, 0, 0, 0, -1, 3),))), (SHAPE, dict(seqs=((0, 0, 0, 0, 1, -3),))), (SHAPE, dict(seqs=((0, 0, 0, 0, 1, (1 << 30) + 1),))),
    (SHAPE, dict(seqs=((0, 0, 0, 0, 1 << 24, 1),))),
    (SHAPE, dict(seqs=((-8, 0, 0, 0, 1, 3),))), (SHAPE, dict(seqs=((0, 4, 0, 0, 1, 3),))), (SHAPE, dict(seqs=((0, 0, 0, 0, 1 << 29, 1),))),
    (WORKSPACE, dict(seqs=((0, 0, 0, 0, 1, 5000),))),
    (WORKSPACE, dict(seqs=((0, 0, 0, 0, 1, 5000),), ws=P, nbytes=256)),
    (WORKSPACE, dict(seqs=((0, 0, 0, 0, 1, 5000),), ws=P + 16, nbytes=1 << 30)),
])
def test_prompt_attention_refusals(status, kw):
    got, nbytes = _attn(**kw)
    assert got == status
    if status == WORKSPACE:
        assert nbytes > 0
    text = _lib().air_last_error(None)
    assert text.startswith(b"air_prompt_"), text


def test_null_descriptors():
    lib = _lib()
    assert lib.air_rope(None, None, None, None, None, None, None) == INVALID
    assert lib.air_prompt_attn(None, None, None, 0, None, None, None, None, None, 0) == INVALID
    assert lib.air_prompt_workspace_bytes(None, None, 0) == 0
    assert lib.air_rope_frequencies(4, 1e4, 0, 1.0, 0, 0.0, 0.0, None, None) == INVALID


def test_structs_follow_the_header_field_by_field():
    text = open(os.path.join(ROOT, "include", "aircache.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    ctype = {"int32_t": C.c_int32, "int64_t": C.c_int64, "float": C.c_float, "void": C.c_void_p}
    for name in ("air_rope_config", "air_rope_tensor", "air_prompt_config", "air_prompt_seq"):
        m = re.search(r"typedef struct\s*\{([^}]*)\}\s*" + name + r"\s*;", text)
        fields = []
        for decl in filter(None, (d.strip() for d in m.group(1).split(";"))):
            base, rest = re.match(r"(?:const\s+)?(\w+)\s+(.*)", decl, flags=re.S).groups()
            for var in (x.strip() for x in rest.split(",")):
                n = re.match(r"\**\s*(\w+)(?:\[(\d+)\])?$", var)
                t = C.c_void_p if var.startswith("*") else ctype[base]
                fields.append((n.group(1), t * int(n.group(2)) if n.group(2) else t))
        assert [f[0] for f in getattr(binding, name)._fields_] == [f[0] for f in fields], name
        for (_, got), (_, want) in zip(getattr(binding, name)._fields_, fields):
            assert got is want or (got._type_ is want._type_ and got._length_ == want._length_), name


def test_binding_refuses_what_it_cannot_marshal():
    torch = pytest.importorskip("torch")
    q, k = torch.zeros(1, 4, 3, 64), torch.zeros(1, 2, 3, 64)
    for bad in (lambda: A.prepare_rope(), lambda: A.prepare_rope(q.half()), lambda: A.prepare_rope(q[0]), lambda: A.prepare_rope(q, q_out=k),
                lambda: A.prepare_rope(q, k.bfloat16()), lambda: A.prepare_rope(q, q_weight=torch.zeros(32)), lambda: A.prepare_rope(k_out=k, q=q),
                lambda: A.prepare_rope(q, axis_pairs=(8, 8, 8, 8)), lambda: A.prepare_rope(q, axis_pairs=(32,), positions=torch.zeros(1, 3)),
                lambda: A.prepare_rope(q, axis_pairs=(32,), freqs=torch.zeros(32)), lambda: A.prepare_rope(q, axis_pairs=(32,), freqs=torch.zeros(31).double()),
                lambda: A.prepare_rope(q, k, q[:, :1]),
                lambda: A.prepare_prompt_attn(q, k, k, q.transpose(2, 3)), lambda: A.prepare_prompt_attn(q, k, k[:, :1], q),
                lambda: A.prepare_prompt_attn(q, k, k, q.double()), lambda: A.prepare_prompt_attn(q, k, k, q, spans=[(1, 0, 1, 0, 1)]),
                lambda: A.prepare_prompt_attn(q, k, k, q, spans=[(0, 1, 3, 0, 3)]), lambda: A.prepare_prompt_attn(q, k, k, q, spans=[(0, 0, 1, 0, 4)]),
                lambda: A.air_prompt_attn(q, k, k, q.clone())):  # the last: tensors of the host
        with pytest.raises(A.AirError):
            bad()


def test_frequencies_follow_the_formulas():
    n, theta = 48, 1e6
    plain = theta ** (-np.arange(n) / n)
    f, s = A.air_rope_frequencies(n, theta)
    np.testing.assert_allclose(f, plain, rtol=1e-14)
    assert s == 1.0
    f, s = A.air_rope_frequencies(n, theta, A.AIR_ROPE_LINEAR, 4.0)
    np.testing.assert_allclose(f, plain / 4.0, rtol=1e-14)
    assert s == 1.0
    f, s = A.air_rope_frequencies(n, theta, A.AIR_ROPE_BY_PARTS, 8.0, 32768)
    turns = 32768 * plain / (2 * np.pi)
    keep = np.clip((turns - 1.0) / 31.0, 0.0, 1.0)
    np.testing.assert_allclose(f, plain * keep + plain / 8.0 * (1.0 - keep), rtol=1e-13)
    assert f[0] == plain[0] and abs(f[-1] * 8.0 / plain[-1] - 1.0) < 1e-14
    assert abs(s - (0.1 * np.log(8.0) + 1.0)) < 1e-6
    assert A.air_rope_frequencies(0, theta)[0].size == 0
    for bad in (dict(theta=0.0), dict(theta=float("nan")), dict(scaling=3), dict(scaling=-1), dict(factor=0.5), dict(factor=float("inf")),
                dict(scaling=2, original_len=0), dict(scaling=2, original_len=9, slow_turns=2.0, fast_turns=2.0), dict(n_pairs=-1)):
        with pytest.raises(A.AirError):
            A.air_rope_frequencies(**{**dict(n_pairs=n, theta=theta), **bad})


def test_error_text_belongs_to_the_thread():
    import threading

    assert _rope(head_dim=96) == SHAPE
    seen = []
    t = threading.Thread(target=lambda: seen.append(_lib().air_last_error(None)))
    t.start()
    t.join()
    assert seen == [b"null context"] and b"head_dim" in _lib().air_last_error(None)


def test_workspace_that_is_not_one_piece_of_the_device():
    torch = pytest.importorskip("torch")
    q, k = torch.zeros(1, 4, 1, 64), torch.zeros(1, 2, 9000, 64)
    call = A.prepare_prompt_attn(q, k, k, q.clone())
    assert call.workspace_bytes > 0
    for ws in (torch.empty(2 * call.workspace_bytes, dtype=torch.uint8)[::2], torch.empty(call.workspace_bytes, dtype=torch.uint8, device="meta")):
        with pytest.raises(A.AirError, match="workspace"):
            A.air_prompt_attn(prepared=call, workspace=ws)
