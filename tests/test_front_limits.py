"""What the header of air_rope and air_prompt_attn allows is accepted, and what it does not is refused for the reason that it gives.  Host only:
nothing here reaches a GPU."""
import ctypes as C
import random
import time

import pytest
import torch

import paper_2503_23956_amd as A
from paper_2503_23956_amd import binding
from test_front_args import SHAPE, _attn, _lib


def _config(dtype, d, hq, hkv, **kw):
    """Token-major tensors."""
    return dict(dict(n_q_heads=hq, n_kv_heads=hkv, head_dim=d, dtype=A.AIR_F32 if dtype == "f32" else A.AIR_BF16, scale=0.0,
                     q_h=d, q_t=hq * d, k_h=d, k_t=hkv * d, v_h=d, v_t=hkv * d, out_h=d, out_t=hq * d), **kw)


def _workspace(cfg, seqs):
    """(bytes, text of the refusal or None) of air_prompt_workspace_bytes, which checks what air_prompt_attn checks but the pointers."""
    arr = (A.air_prompt_seq * max(1, len(seqs)))(*(A.air_prompt_seq(*s) for s in seqs))
    lib = _lib()
    assert lib.air_prompt_workspace_bytes(None, None, 0) == 0
    before = lib.air_last_error(None)
    nbytes = lib.air_prompt_workspace_bytes(C.byref(A.air_prompt_config(**cfg)), arr, len(seqs))
    text = lib.air_last_error(None)
    return nbytes, None if text == before else text.decode()


def _prompts(cfg, lens):
    """Sequences one behind the other."""
    out, q0, k0 = [], 0, 0
    for n, m in lens:
        out.append((q0 * cfg["q_t"], k0 * cfg["k_t"], k0 * cfg["v_t"], q0 * cfg["out_t"], n, m))
        q0, k0 = q0 + n, k0 + m
    return out


def _log_int(rng, lo, hi):
    return int(round(2.0 ** rng.uniform(lo, hi)))


@pytest.mark.parametrize("dtype,d,hq,hkv,lens", [
    ("f32", 128, 40, 5, [(463172, 924067)]), ("f32", 64, 16, 2, [(1051463, 1051463)]), ("bf16", 128, 64, 8, [((1 << 20) - 1, 1 << 30)]),
    ("bf16", 64, 1, 1, [((1 << 26) - 1, 1 << 30)]), ("f32", 128, 16384, 16384, [(63, 1 << 20)] * 64), ("bf16", 64, 16384, 1, [(4095, 4095)]),
])
def test_calls_at_the_limits_are_accepted(dtype, d, hq, hkv, lens):
    cfg = _config(dtype, d, hq, hkv)
    assert _workspace(cfg, _prompts(cfg, lens))[1] is None


def test_no_call_inside_the_limits_is_refused():
    rng = random.Random(3)
    for _ in range(3000):
        hkv = rng.choice([1, 2, 4, 5, 8, 16, 128, 16384])
        hq = min(16384 // hkv, rng.choice([1, 2, 5, 7, 8, 16, 64])) * hkv
        most = ((1 << 26) - 1) // hq
        n_seqs = rng.choice([1, 1, 2, 7, 33, 64])
        lens = [(min(_log_int(rng, 0, 26), most // n_seqs), _log_int(rng, 0, 30)) for _ in range(n_seqs)]
        cfg = _config(rng.choice(["bf16", "f32"]), rng.choice([64, 128]), hq, hkv)
        if cfg["k_t"] < 1 << 24:
            assert _workspace(cfg, _prompts(cfg, lens))[1] is None, (cfg, lens)


def test_more_rows_than_a_call_takes():
    for dtype, d, hq, hkv, lens in (("bf16", 64, 2, 1, [((1 << 26) - 1, 100)]), ("bf16", 64, 1, 1, [(1 << 26, 100)]), ("f32", 128, 16384, 1, [(1, 1)] * 64),
                                    ("f32", 128, 28, 4, [(1 << 21, 1 << 21)] * 2), ("bf16", 128, 16384, 16384, [((1 << 31) - 1, 1)] * 64)):
        cfg = _config(dtype, d, hq, hkv)
        rows = sum(n for n, _ in lens) * hq
        _, text = _workspace(cfg, _prompts(cfg, lens))
        assert (text is not None and "too many rows" in text) == (rows >= 1 << 26), (text, rows)
    # with out rows of their own, so that the number of rows is what is refused
    status, _ = _attn(seqs=((0, 0, 0, 0, 1 << 24, 1),))
    assert status == SHAPE and b"too many rows" in _lib().air_last_error(None)


def test_splits_are_worth_their_workspace():
    """Long prompts take none, and no call takes more than 256 MiB; few rows over many keys, which need splits, still have them."""
    for dtype, d, hq, hkv, n, m in (("bf16", 128, 64, 8, 21839, 249226), ("f32", 128, 64, 8, 97499, 258675), ("f32", 128, 28, 4, 131295, 250773)):
        cfg = _config(dtype, d, hq, hkv)
        assert _workspace(cfg, _prompts(cfg, [(n, m)])) == (0, None)
    rng = random.Random(4)
    for _ in range(3000):
        hkv = rng.choice([1, 2, 3, 4, 8])
        cfg = _config(rng.choice(["bf16", "f32"]), rng.choice([64, 128]), hkv * rng.choice([1, 2, 5, 7, 8, 16]), hkv)
        lens = [(_log_int(rng, 0, 18), _log_int(rng, 0, 22)) for _ in range(rng.choice([1, 1, 2, 8, 33]))]
        assert _workspace(cfg, _prompts(cfg, lens))[0] <= 256 << 20, (cfg, lens)
    for dtype, d, hq, hkv, lens in (("bf16", 128, 28, 4, [(1, 7432)]), ("bf16", 64, 14, 2, [(1, 7432), (1, 33), (1, 4000)]), ("f32", 64, 4, 2, [(656, 656)]), ("f32", 64, 14, 2, [(8000, 8000)]),
                                    ("bf16", 128, 64, 8, [(512, 16910)]), ("bf16", 128, 64, 8, [(1, 1 << 20)] * 8)):
        cfg = _config(dtype, d, hq, hkv)
        assert _workspace(cfg, _prompts(cfg, lens))[0] > 0


def _rows_overlap(rows, d):
    rows = sorted(rows)
    return any(b - a < d for a, b in zip(rows, rows[1:]))


def test_output_rows_that_overlap_are_refused():
    cfg = _config("bf16", 128, 4, 2)
    assert "output rows overlap" in _workspace(dict(cfg, out_h=128, out_t=128), [(0, 0, 0, 0, 3, 3)])[1]  # head 1 of a token is head 0 of the next
    same = [(0, 0, 0, 0, 3, 3)] * 2  # an output that is expanded over the batch
    assert "two sequences" in _workspace(cfg, same)[1]
    assert "two sequences" in _workspace(cfg, [(0, 0, 0, 0, 3, 3), (0, 0, 0, 2 * 512, 3, 3)])[1]
    assert _workspace(cfg, [(0, 0, 0, 0, 3, 3), (0, 0, 0, 3 * 512, 3, 3)])[1] is None
    assert _workspace(cfg, [(0, 0, 0, 0, 0, 3), (0, 0, 0, 0, 3, 3)])[1] is None  # no queries, no rows
    assert "output rows overlap" in _workspace(dict(cfg, out_h=2 ** 61, out_t=2 ** 61), [(0, 0, 0, 0, 3, 3)])[1]
    assert _workspace(dict(cfg, out_h=2 ** 62, out_t=2 ** 61), [(2 ** 62, 0, 0, 2 ** 62, 1, 3)])[1] is None


def test_output_rows_of_any_layout():
    """Against the rows themselves: heads inside tokens, tokens inside heads, strides that are no multiples of each other."""
    rng = random.Random(5)
    seen = [0, 0]
    for _ in range(6000):
        d = rng.choice([64, 128])
        heads, n_seqs = rng.choice([1, 2, 3, 5, 8]), rng.choice([1, 1, 2, 3])
        unit = 8 * rng.choice([1, 1, 2, 4, 8])
        out_h, out_t = (rng.choice([unit * rng.randint(1, 900 // unit * 2), d * rng.randint(1, 9)]) for _ in range(2))
        seqs = [(0, 0, 0, unit * rng.randint(0, rng.choice([10, 4000 // unit])), rng.choice([0, 1, 2, 3, 7, 12]), 5) for _ in range(n_seqs)]
        rows = [o + h * out_h + t * out_t for _, _, _, o, n, _ in seqs for h in range(heads) for t in range(n)]
        text = _workspace(_config("bf16", d, heads, 1, out_h=out_h, out_t=out_t), seqs)[1]
        want = _rows_overlap(rows, d)
        assert (text is not None and "overlap" in text) == want, (d, heads, out_h, out_t, seqs, text)
        seen[want] += 1
    assert min(seen) > 1000


@pytest.mark.skipif(torch.cuda.is_available(), reason="made-up pointers: what is accepted would run")
def test_rotated_rows_of_any_layout():
    rng = random.Random(6)
    seen = [0, 0]
    for i in range(4000):
        d = rng.choice([64, 128])
        n = [rng.choice([1, 2, 3, 5, 9]) for _ in range(3)]
        unit = 8 * rng.choice([1, 1, 2, 8])
        s = [rng.choice([unit * rng.randint(1, 2400 // unit), d * rng.randint(1, 30)]) for _ in range(3)]
        if i % 4 == 0:  # nested in some order
            at = d
            for j in rng.sample(range(3), 3):
                s[j] = at + 8 * rng.choice([0, 0, 1, 5])
                at = s[j] * n[j]
        rows = [a * s[0] + b * s[1] + c * s[2] for a in range(n[0]) for b in range(n[1]) for c in range(n[2])]
        cfg = A.air_rope_config(n[1], n[1], d, A.AIR_BF16, n[0], n[2], 0, 1, (C.c_int32 * 3)(0, 0, 0), 1e-6, 1.0)
        t = A.air_rope_tensor(4096, 8192, None, 0, 0, 0, *s)
        status = _lib().air_rope(None, C.byref(cfg), None, C.byref(t), None, None, None)
        want = _rows_overlap(rows, d)
        assert status == (SHAPE if want else binding.AIR_ERR_HIP), (d, n, s, want)  # (no GPU here: what is accepted stops at the launch)
        seen[want] += 1
    assert min(seen) > 800


def test_overlap_in_large_calls_takes_no_time():
    t = A.air_rope_tensor(4096, 8192, None, 0, 0, 0, 11616 * 64 + 8, 11584 * 64, 11600 * 64)
    cfg = A.air_rope_config(11585, 11585, 64, A.AIR_BF16, 11585, 11585, 0, 1, (C.c_int32 * 3)(0, 0, 0), 1e-6, 1.0)
    start = time.perf_counter()
    assert _lib().air_rope(None, C.byref(cfg), None, C.byref(t), None, None, None) == SHAPE
    assert time.perf_counter() - start < 0.5
    cfg = _config("bf16", 128, 28, 4, out_h=128 * 64, out_t=128)  # 64 decoded tokens, head-major
    seqs = [(0, 0, 0, 128 * i, 1, 500) for i in range(64)]
    start = time.perf_counter()
    for _ in range(100):
        assert _workspace(cfg, seqs)[1] is None
    assert time.perf_counter() - start < 0.5


def test_scales_whose_base_2_factor_overflows_are_refused():
    for scale, text in ((2.0 ** 127, None), (2.4e38, "scale must be"), (3.4e38, "scale must be"), (float("inf"), "scale must be"), (1e-45, None)):
        got = _workspace(_config("bf16", 64, 4, 2, scale=scale), [(0, 0, 0, 0, 1, 9)])[1]
        assert got is None if text is None else text in got, (scale, got)


class _OnGpu:
    """What PreparedCall asks of torch, without a GPU."""

    def __init__(self):
        self.made = []

    class cuda:
        current_device = staticmethod(lambda: 0)

    uint8 = torch.uint8

    def empty(self, n, dtype, device):
        self.made.append(torch.empty(n, dtype=dtype))
        return self.made[-1]


def test_a_prepared_attention_may_be_called():
    q, k = torch.zeros(1, 4, 1, 64), torch.zeros(1, 2, 9000, 64)
    lib = _lib()
    for m in (9000, 3):
        call = A.prepare_prompt_attn(q, k, k, q.clone(), spans=[(0, 0, 1, 0, m)])
        seen = []
        call.torch, call.on_gpu, call.raw_stream = _OnGpu(), True, lambda i: 77
        call.fn = C.CFUNCTYPE(C.c_int, *lib.air_prompt_attn.argtypes)(lambda *args: seen.append((args[0], args[8], args[9])) or 0)
        call()
        made = call.torch.made
        assert seen == [(77, made[0].data_ptr(), made[0].numel())] if m == 9000 else seen == [(77, None, 0)] and not made


# calls of several sequences, unequal lengths, more keys than queries and fewer, one without queries: one of every kernel, without splits and with
MIXED = [(dt, d, hq, hkv, [*pairs, (0, 5), (9, 4)], rows, split) for dt, d, hq, hkv, pairs, rows, split in (
    ("bf16", 128, 8, 8, [(40, 41), (77, 77)], 32, False),
    ("bf16", 128, 8, 8, [(40, 540), (77, 1077)], 32, True),
    ("bf16", 128, 16, 1, [(40, 40), (77, 90), (114, 114), (151, 200), (188, 188)], 128, False),
    ("bf16", 128, 8, 8, [(40, 3040), (77, 6077), (114, 3114)], 128, True),
    ("bf16", 128, 64, 8, [(40, 40), (77, 90), (114, 114), (151, 200), (188, 188)], 256, False),
    ("bf16", 128, 28, 4, [(901, 901), (1333, 1400), (612, 1000), (1100, 1107)], 256, False),
    ("bf16", 128, 16, 2, [(200, 3100), (237, 6137), (274, 3174), (311, 6211), (248, 3248)], 256, True),
    ("bf16", 64, 8, 8, [(40, 41), (77, 77)], 32, False),
    ("bf16", 64, 8, 8, [(40, 540), (77, 1077)], 32, True),
    ("bf16", 64, 64, 8, [(100, 110), (137, 137), (174, 200)], 128, False),
    ("bf16", 64, 14, 2, [(300, 3100), (200, 4000)], 128, True),
    ("bf16", 64, 64, 8, [(40, 40), (77, 90), (114, 114), (151, 200), (188, 188)], 256, False),
    ("bf16", 64, 16, 1, [(40, 3040), (77, 6077), (114, 3114), (151, 6151), (188, 3188)], 256, True),
    ("f32", 128, 8, 8, [(40, 40), (77, 77)], 32, False),
    ("f32", 128, 8, 8, [(40, 71), (77, 139)], 32, True),
    ("f32", 128, 64, 8, [(100, 110), (137, 137), (174, 200)], 128, False),
    ("f32", 128, 14, 2, [(40, 540), (77, 1077), (114, 614)], 128, True),
    ("f32", 64, 8, 8, [(40, 41), (77, 77)], 32, False),
    ("f32", 64, 8, 8, [(40, 540), (77, 1077)], 32, True),
    ("f32", 64, 64, 8, [(40, 71), (77, 139), (114, 145), (151, 213), (188, 219)], 128, False),
    ("f32", 64, 8, 8, [(400, 900), (437, 1437), (474, 974)], 128, True),
)]


@pytest.mark.parametrize("dtype,d,hq,hkv,pairs,rows,split", MIXED)
def test_plans_of_mixed_calls(dtype, d, hq, hkv, pairs, rows, split):
    cfg = _config(dtype, d, hq, hkv)
    seqs = _prompts(cfg, pairs)
    arr = (A.air_prompt_seq * len(seqs))(*(A.air_prompt_seq(*s) for s in seqs))
    got, splits = C.c_int32(), C.c_int32()
    assert _lib().air_prompt_plan(C.byref(A.air_prompt_config(**cfg)), arr, len(seqs), C.byref(got), C.byref(splits)) == 0
    assert (got.value, splits.value > 1) == (rows, split), splits.value
    assert (_workspace(cfg, seqs)[0] > 0) == split


def test_plans_are_refused_as_calls_are():
    lib, n = _lib(), C.c_int32()
    cfg = A.air_prompt_config(**_config("bf16", 64, 4, 2))
    arr = (A.air_prompt_seq * 1)(A.air_prompt_seq(0, 0, 0, 0, -1, 3))
    assert lib.air_prompt_plan(C.byref(cfg), arr, 1, C.byref(n), C.byref(n)) == SHAPE and b"length" in lib.air_last_error(None)
    assert lib.air_prompt_plan(C.byref(cfg), arr, 0, None, C.byref(n)) == binding.AIR_ERR_INVALID_ARG
    assert lib.air_prompt_plan(None, arr, 1, C.byref(n), C.byref(n)) == binding.AIR_ERR_INVALID_ARG


@pytest.mark.parametrize("text,kw", [
    ("dtype", dict(dtype=-1)), ("head_dim", dict(head_dim=80)), ("multiple of KV heads", dict(n_q_heads=3)), ("multiple of KV heads", dict(n_kv_heads=-2)),
    ("n_seqs", dict(n=65)), ("n_seqs", dict(n=-1)), ("strides must be", dict(q_t=-512)), ("strides must be", dict(k_h=4)), ("output rows overlap", dict(out_t=120)),
    ("token strides", dict(k_t=1 << 24)), ("token strides", dict(v_t=1 << 24)), ("output rows overlap", dict(out_h=0)),
    ("a length", dict(seqs=((0, 0, 0, 0, -1, 3),))), ("a length", dict(seqs=((0, 0, 0, 0, 1, (1 << 30) + 1),))),
    ("offsets", dict(seqs=((-8, 0, 0, 0, 1, 3),))), ("offsets", dict(seqs=((0, 4, 0, 0, 1, 3),))), ("too many rows", dict(seqs=((0, 0, 0, 0, 1 << 24, 1),))),
])
def test_refusals_name_their_reason(text, kw):
    assert _attn(**kw)[0] == SHAPE
    assert text in _lib().air_last_error(None).decode()
