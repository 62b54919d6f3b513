"""air_prompt_attn against attention in fp64, with bounds derived from the roundings it makes."""
import math

import pytest

pytestmark = pytest.mark.gpu


def _plain(q, k, v, spans, scale=None):
    """[(span, rows in fp64, bound)] of every span: q [B][Hq][T][d] and so on."""
    import torch

    step = 2.0 ** -8 if q.dtype == torch.bfloat16 else 2.0 ** -24
    d, g = q.shape[3], q.shape[1] // k.shape[1]
    scale = scale or d ** -0.5
    out = []
    for b, q0, n, k0, m in spans:
        qs = q[b, :, q0:q0 + n].double()
        ks, vs = (x[b, :, k0:k0 + m].double().repeat_interleave(g, dim=0) for x in (k, v))
        seen = torch.arange(m, device=q.device)[None, :] <= torch.arange(n, device=q.device)[:, None] + (m - n)
        s = (qs @ ks.transpose(1, 2).contiguous() * scale).masked_fill(~seen, -math.inf)
        top = s.amax(-1, keepdim=True) if m else s.new_zeros((*s.shape[:2], 1))
        p = torch.exp(s - torch.where(torch.isinf(top) & (top < 0), 0.0, top))
        l = p.sum(-1, keepdim=True)
        p = torch.where(l > 0, p / l, p)
        o, a = p @ vs, p @ vs.abs()
        # logits: d products and sums of |q||k|, the factor, the reference and the exponent in fp32 (the scaled logit itself rounded once or
        # twice); exp2 to 2^-22; sums of n terms; bf16 rounds the probabilities and the outputs, fp32 the outputs
        dot = (qs.abs() @ ks.abs().transpose(1, 2).contiguous() * scale).masked_fill(~seen, 0.0)
        logit = dot.amax(-1, keepdim=True) * ((d + 4) * 2.0 ** -24) if m else l * 0.0
        size = torch.where(seen, s, torch.zeros_like(s)).abs().amax(-1, keepdim=True) * 2.0 ** -22 if m else l * 0.0
        rel = 2 * (torch.expm1(logit + size) + 2.0 ** -22 + (m + 64) * 2.0 ** -24)
        if q.dtype == torch.bfloat16:
            rel = rel + 2.0 ** -8
        out.append((o, a * rel * 1.01 + (o.abs() + a * rel) * step + 1e-37))
    return out


def _run(A, q, k, v, spans, out=None, **kw):
    import torch

    if out is None:
        out = torch.full((q.shape[0], q.shape[2], q.shape[1], q.shape[3]), 42.0, dtype=q.dtype, device=q.device).transpose(1, 2)
    A.air_prompt_attn(q, k, v, out, spans=spans, **kw)
    torch.cuda.synchronize()
    return out


def _check(q, k, v, spans, out, scale=None):
    import torch

    left = torch.ones(out.shape[:3], dtype=torch.bool, device=out.device)
    for (b, q0, n, k0, m), (want, bound) in zip(spans, _plain(q, k, v, spans, scale)):
        far = (out[b, :, q0:q0 + n].double() - want).abs()
        assert bool((far <= bound).all()), f"span {(b, q0, n, k0, m)}: {(far - bound).max().item()} above its bound, {far.max().item()} off"
        left[b, :, q0:q0 + n] = False
    assert bool((out[left] == 42.0).all())  # rows of no sequence are left as they are


def _tensors(B, nq, nk, hq, hkv, d, dtype, seed, order="head"):
    import torch

    g = torch.Generator(device="cuda:0").manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32

    def make(h, n, lean):
        x = torch.randn((B, h, n, d), generator=g, device="cuda:0") * lean
        return x.to(dt) if order == "head" else x.to(dt).transpose(1, 2).contiguous().transpose(1, 2)

    return make(hq, nq, 1.7), make(hkv, nk, 1.3), make(hkv, nk, 1.0)


KINDS = [("bf16", 64), ("bf16", 128), ("f32", 64), ("f32", 128)]


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("hq,hkv", [(4, 4), (7, 1), (6, 2), (16, 1), (34, 1)])
def test_lengths(dtype, d, hq, hkv):
    """Prompts, pieces and single tokens, one and many, lengths at and around the tiles' borders, none and more rows than keys."""
    import paper_2503_23956_amd as A

    pairs = [(1, 1), (2, 2), (5, 5), (31, 31), (32, 32), (33, 33), (63, 64), (64, 64), (65, 65), (127, 130), (1, 63), (1, 64), (1, 65), (3, 129),
             (4, 700), (130, 257), (0, 9), (9, 0), (7, 3), (200, 150)]
    spans = [(b, 0, n, 0, m) for b, (n, m) in enumerate(pairs)]
    q, k, v = _tensors(len(pairs), 200, 700, hq, hkv, d, dtype, 17 * d + hq)
    _check(q, k, v, spans, _run(A, q, k, v, spans))
    few = [(b, 1, 2, 3, m) for b, m in enumerate((1, 2, 31, 64, 65, 500, 697, 96, 128, 160))]
    _check(q, k, v, few, _run(A, q, k, v, few))


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("n,m", [(1, 5000), (4, 4099), (20, 3000), (150, 2900), (1200, 1200)])
def test_long_axes_are_split_and_joined(dtype, d, n, m):
    import paper_2503_23956_amd as A

    q, k, v = _tensors(1, n, m, 8, 2, d, dtype, n + m, order="token")
    spans = [(0, 0, n, 0, m)]
    call = A.prepare_prompt_attn(q, k, v, q.clone(), spans=spans)
    if n < 1000:
        assert call.workspace_bytes > 0
    _check(q, k, v, spans, _run(A, q, k, v, spans))


# The library chooses tiles of 32, 128 or 256 rows and a number of splits by the work of a call: shapes of every choice
SHAPES = [(128, 28, 4, 1, 9000), (128, 28, 4, 7, 3001), (128, 28, 4, 200, 200), (128, 28, 4, 500, 500), (128, 28, 4, 61, 9001), (128, 28, 4, 1300, 1311),
          (128, 28, 4, 3000, 3000), (128, 20, 5, 700, 5003), (128, 64, 8, 511, 12001), (64, 14, 2, 1, 20000), (64, 14, 2, 900, 900), (64, 14, 2, 130, 9000),
          (64, 14, 2, 3500, 3500), (64, 14, 2, 5000, 6001), (64, 32, 8, 257, 15000)]


F32_SHAPES = [(128, 28, 4, 61, 8001), (128, 28, 4, 700, 701), (128, 28, 4, 1500, 1500), (128, 20, 5, 300, 3001), (128, 3, 3, 1700, 1700),
              (64, 14, 2, 2100, 2100), (64, 14, 2, 3500, 3600), (64, 32, 8, 257, 5000)]


@pytest.mark.parametrize("dtype,d,hq,hkv,n,m", [("bf16", *s) for s in SHAPES] + [("f32", *s) for s in F32_SHAPES])
def test_tiles_and_splits(dtype, d, hq, hkv, n, m):
    """The result, and what is not finite: at a key behind the first rows of a tile and behind the sequence."""
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _tensors(1, n, m + 20, hq, hkv, d, dtype, n + m, order="token")
    spans = [(0, 0, n, 0, m)]
    _check(q, k, v, spans, _run(A, q, k, v, spans))
    at = m - 1 - n // 3  # the first key that is not finite
    v[:, :, at, 3], v[:, :, at, d - 1], v[:, :, m:] = math.inf, -math.inf, math.nan
    k[:, :, m:] = math.nan
    got = _run(A, q, k, v, spans)[0, :, :n].double()
    v[:, :, at, 3], v[:, :, at, d - 1] = 0.0, 0.0
    want, bound = _plain(q, k, v, spans)[0]
    sees = torch.arange(n, device=q.device) + (m - n) >= at
    assert bool((got[:, sees, 3] == math.inf).all()) and bool((got[:, sees, d - 1] == -math.inf).all())
    got[:, sees, 3], got[:, sees, d - 1] = want[:, sees, 3], want[:, sees, d - 1]
    assert bool(((got - want).abs() <= bound).all()), ((got - want).abs() - bound).max().item()


@pytest.mark.parametrize("dtype,d", KINDS)
def test_prompts_pieces_and_tokens_in_one_call(dtype, d):
    import paper_2503_23956_amd as A

    pairs = [(700, 700), (1, 3000), (1, 5), (64, 2000), (0, 50), (33, 33), (1, 1), (3, 2999)]
    spans, at, kt = [], 3, 1
    for n, m in pairs:  # packed, with gaps between the sequences
        spans.append((0, at, n, kt, m))
        at, kt = at + n + 2, kt + m + 3
    q, k, v = _tensors(1, at, kt, 12, 4, d, dtype, 77, order="token")
    _check(q, k, v, spans, _run(A, q, k, v, spans))


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("hq,hkv,pairs", [(16, 1, [(20 + (11 * i) % 37, 20 + (11 * i) % 37 + (i % 4) * (i % 3) * 9) for i in range(33)]),
                                          (28, 4, [(901, 901), (333, 400), (1, 1), (0, 0), (612, 612), (95, 1500), (1100, 800)])])
def test_ragged_prompts(dtype, d, hq, hkv, pairs):
    import paper_2503_23956_amd as A

    spans = [(b, 0, n, 0, m) for b, (n, m) in enumerate(pairs)]
    q, k, v = _tensors(len(pairs), max(n for n, _ in pairs), max(m for _, m in pairs), hq, hkv, d, dtype, hq + d, order="token")
    _check(q, k, v, spans, _run(A, q, k, v, spans))


def test_sixty_four_sequences():
    import paper_2503_23956_amd as A

    spans = [(b, b % 3, 1 + (7 * b) % 40, b % 5, 1 + (7 * b) % 40 + (b % 4) * 150) for b in range(64)]
    q, k, v = _tensors(64, 45, 600, 6, 3, 64, "bf16", 4)
    _check(q, k, v, spans, _run(A, q, k, v, spans))


@pytest.mark.parametrize("dtype,d", KINDS)
def test_packed_sequences_of_a_projection_buffer(dtype, d):
    """Sequences one behind the other, q, k and v views of one [token][head][d] buffer, a scale of the caller's."""
    import torch

    import paper_2503_23956_amd as A

    lens = [40, 1, 129, 77, 3, 260]
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda:0").manual_seed(9)
    x = torch.randn((1, sum(lens) + 5, 10, d), generator=g, device="cuda:0").to(dt).transpose(1, 2)
    q, k, v = x[:, :6], x[:, 6:8], x[:, 8:]
    spans, at = [], 0
    for n in lens:
        spans.append((0, at, n, at, n))
        at += n
    _check(q, k, v, spans, _run(A, q, k, v, spans, scale=0.25), scale=0.25)


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("n,m", [(1, 100), (3, 70), (90, 90), (90, 200)])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_lies_behind_a_row_counts_for_nothing(dtype, d, n, m, bad):
    """Keys and values behind every row, and behind the rows before some token, may hold anything."""
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _tensors(1, n, m + 40, 6, 2, d, dtype, 5)
    spans = [(0, 0, n, 0, m)]
    clean = _run(A, q, k, v, spans)
    _check(q, k, v, spans, clean)
    k2, v2 = k.clone(), v.clone()
    k2[:, :, m:] = bad
    v2[:, :, m:] = bad
    assert torch.equal(_run(A, q, k2, v2, spans), clean)
    if n > 1:  # from the last query's own token on: the rows before it see nothing of it, its own row all of it
        v2[:, :, m - 1:, 5] = bad
        got = _run(A, q, k2, v2, spans)
        want, bound = _plain(q, k, v, spans)[0]
        far = (got[0, :, :n - 1].double() - want[:, :n - 1]).abs()
        assert bool((far <= bound[:, :n - 1]).all())
        last = got[0, :, n - 1, 5].float()
        assert bool(torch.isnan(last).all()) if math.isnan(bad) else bool((last == bad).all())
        others = torch.arange(d, device=v.device) != 5
        assert bool(((got[0, :, n - 1][:, others].double() - want[:, n - 1][:, others]).abs() <= bound[:, n - 1][:, others]).all())
        k2[:, :, m - 1:] = bad
        got = _run(A, q, k2, v2, spans)
        assert bool(((got[0, :, :n - 1].double() - want[:, :n - 1]).abs() <= bound[:, :n - 1]).all())


@pytest.mark.parametrize("dtype,d", KINDS)
def test_extreme_logits(dtype, d):
    """Logits of thousands (one key takes it all), of the type's lowest value, of -inf, and keys of which all weigh nothing."""
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _tensors(1, 70, 300, 4, 2, d, dtype, 8)
    for n, m in ((70, 300), (2, 300)):
        spans = [(0, 0, n, 0, m)]
        big = q * 100
        _check(big, k, v, spans, _run(A, big, k, v, spans))
        one = q.abs()
        k2 = k.clone()
        k2[:, :, 10:200] = -math.inf  # logits of -inf
        got = _run(A, one, k2, v, spans)
        keep = torch.tensor([*range(10), *range(200, m)], device=k.device)
        # the same as without those keys (every query comes behind them)
        if n == 2:
            _check(one, k[:, :, keep], v[:, :, keep], [(0, 0, n, 0, len(keep))], got)
        k2[:] = -math.inf
        got = _run(A, one, k2, v, spans)
        assert bool((got[0, :, :n] == 0).all())
        low = torch.full_like(k, -1e30)
        flat = _run(A, torch.full_like(q, 1e3), low, v, spans)  # equal logits near the lowest number: the mean of the values seen
        want = v[0].double().cumsum(1)[:, m - n:m] / torch.arange(m - n + 1, m + 1, device=v.device)[:, None]
        want = want.repeat_interleave(2, dim=0)
        bound = v.abs().max().item() * (2.0 ** -7 if dtype == "bf16" else (m + 64) * 2.0 ** -23)
        assert float((flat[0, :, :n].double() - want).abs().max()) <= bound
        nan = q.clone()
        nan[:, 1] = math.nan
        got = _run(A, nan, k, v, spans)
        assert bool(torch.isnan(got[0, 1, :n]).all()) and not bool(torch.isnan(got[0, [0, 2, 3], :n]).any())


def test_offsets_beyond_32_bits():
    """A long cache whose token stride is wide: the last keys lie more than 2^32 bytes behind the first."""
    import torch

    import paper_2503_23956_amd as A

    m, wide = 1100, 2 ** 21
    buf = torch.empty(m * wide, dtype=torch.bfloat16, device="cuda:0")  # 4.6 GB
    k = buf.view(1, m, 1, wide)[..., :64].transpose(1, 2)
    v = buf.view(1, m, 1, wide)[..., 64:128].transpose(1, 2)
    k.copy_(torch.randn(k.shape, device="cuda:0"))
    v.copy_(torch.randn(v.shape, device="cuda:0"))
    q = torch.randn((1, 4, 100, 64), device="cuda:0").bfloat16()
    for spans in ([(0, 0, 100, 0, m)], [(0, 3, 1, 0, m)], [(0, 3, 1, 1050, 50)]):
        _check(q, k, v, spans, _run(A, q, k, v, spans))


def test_same_bits_twice_on_streams_and_in_graphs():
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _tensors(2, 300, 2000, 8, 2, 128, "bf16", 21)
    shapes = [[(0, 0, 300, 0, 300), (1, 0, 120, 0, 2000)], [(0, 0, 1, 0, 2000), (1, 4, 1, 0, 1500)]]
    side = torch.cuda.Stream()
    outs, graphs = [], []
    for spans in shapes:
        out = torch.zeros_like(q)
        call = A.prepare_prompt_attn(q, k, v, out, spans=spans)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            A.air_prompt_attn(prepared=call)
        outs.append(out)
        graphs.append(g)
    for step in range(4):
        q.copy_(torch.randn_like(q))
        for g in graphs:
            g.replay()
        side.wait_stream(torch.cuda.current_stream())
        eager = [torch.zeros_like(q) for _ in shapes]
        with torch.cuda.stream(side):
            for spans, out in zip(shapes, eager):
                A.air_prompt_attn(q, k, v, out, spans=spans)
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a, b)
    # a stream handle of the caller's needs the caller's workspace
    call = A.prepare_prompt_attn(q, k, v, torch.zeros_like(q), spans=shapes[1])
    with pytest.raises(A.AirError):
        A.air_prompt_attn(prepared=call, stream=side.cuda_stream)
    ws = torch.empty(call.workspace_bytes, dtype=torch.uint8, device="cuda:0")
    torch.cuda.synchronize()
    A.air_prompt_attn(prepared=call, stream=side.cuda_stream, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(call._keepalive[3], outs[1])


@pytest.mark.parametrize("d,hq,hkv,n,m", [(128, 28, 4, 1300, 600), (128, 28, 4, 3000, 2000), (64, 14, 2, 900, 70), (64, 14, 2, 5000, 4000), (128, 8, 8, 600, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_rows_than_keys(dtype, d, hq, hkv, n, m):
    """Whole tiles of rows that see no key, tiles whose last rows see some."""
    import paper_2503_23956_amd as A

    q, k, v = _tensors(1, n, m, hq, hkv, d, dtype, n, order="token")
    spans = [(0, 0, n, 0, m)]
    out = _run(A, q, k, v, spans)
    _check(q, k, v, spans, out)
    assert bool((out[:, :, :n - m] == 0).all())


@pytest.mark.parametrize("dtype,d", KINDS)
@pytest.mark.parametrize("n,m", [(1, 3000), (40, 40), (700, 700)])
def test_broadcast_keys_and_outputs_inside_a_buffer(dtype, d, n, m):
    """One head's keys and values for all KV heads and batch rows; output rows apart from each other."""
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _tensors(2, n, m, 6, 3, d, dtype, n, order="token")
    k, v = (x[:1, :1].expand(2, 3, m, d) for x in (k, v))
    buf = torch.full((2, n, 7, d + 24), 42.0, dtype=q.dtype, device=q.device)
    out = buf[:, :, :6, 8:d + 8].transpose(1, 2)
    spans = [(b, 0, n, 0, m) for b in range(2)]
    _check(q, k, v, spans, _run(A, q, k, v, spans, out=out))
    out.fill_(42.0)
    assert bool((buf == 42.0).all())


def test_calls_without_work():
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _tensors(2, 5, 9, 4, 2, 64, "bf16", 1)
    assert bool((_run(A, q, k, v, []) == 42.0).all())
    assert bool((_run(A, q, k, v, [(0, 5, 0, 9, 0), (1, 2, 0, 0, 9)]) == 42.0).all())
    assert bool((_run(A, q, k[:, :, :0], v[:, :, :0], None) == 0.0).all())
    _run(A, q[:, :, :0], k, v, None)
    _run(A, q[:0], k[:0], v[:0], None)
    with pytest.raises(A.AirError):
        A.air_prompt_attn(q, k, v, torch.empty_like(q), spans=[(0, 0, 1, 0, 1)] * 65)
    call = A.prepare_prompt_attn(q, k, v, torch.empty_like(q))
    with pytest.raises(A.AirError, match="workspace"):
        A.air_prompt_attn(prepared=call, workspace=torch.empty(1 << 20, dtype=torch.uint8))  # the host's


def test_as_many_rows_as_a_call_takes():
    import torch

    import paper_2503_23956_amd as A

    n, m = 2 ** 26 - 1, 100  # 8.6 GB of queries, 100 of them see keys
    q = torch.empty((1, 1, n, 64), dtype=torch.bfloat16, device="cuda:0")
    out = torch.full_like(q, 42.0)
    q[:, :, n - 1000:] = torch.randn((1, 1, 1000, 64), device="cuda:0").bfloat16()
    _, k, v = _tensors(1, 1, m, 1, 1, 64, "bf16", 8)
    _run(A, q, k, v, [(0, 0, n, 0, m)], out=out)
    assert int(torch.count_nonzero(out[:, :, :n - m])) == 0
    last = (0, 0, 1000, 0, m)
    _check(q[:, :, n - 1000:], k, v, [last], out[:, :, n - 1000:])
    with pytest.raises(A.AirError):
        wide = q.expand(1, 2, n, 64)  # twice the rows
        A.air_prompt_attn(wide, k, v, torch.empty((1, 2, 1, 64), dtype=q.dtype, device="cuda:0").expand(1, 2, n, 64))


def test_two_calls_at_once_and_two_graphs_of_one_workspace():
    import torch

    import paper_2503_23956_amd as A

    q, k, v = _tensors(4, 260, 3000, 14, 2, 128, "bf16", 5)
    jobs = [[(0, 0, 1, 0, 3000), (1, 0, 3, 0, 2900)], [(2, 0, 260, 0, 3000), (3, 0, 7, 0, 1000)]]
    want = [_run(A, q, k, v, spans) for spans in jobs]
    outs = [torch.zeros_like(w) for w in want]
    calls = [A.prepare_prompt_attn(q, k, v, o, spans=spans) for o, spans in zip(outs, jobs)]
    own = [torch.empty(c.workspace_bytes, dtype=torch.uint8, device="cuda:0") for c in calls]
    assert all(c.workspace_bytes > 0 for c in calls)
    sides = [torch.cuda.Stream() for _ in jobs]
    torch.cuda.synchronize()
    for _ in range(10):  # side by side, each with its workspace
        for c, ws, s in zip(calls, own, sides):
            A.air_prompt_attn(prepared=c, workspace=ws, stream=s.cuda_stream)
    torch.cuda.synchronize()
    for o, w, spans in zip(outs, want, jobs):
        for b, q0, n, _, _ in spans:
            assert torch.equal(o[b, :, q0:q0 + n], w[b, :, q0:q0 + n])
    shared = torch.empty(max(c.workspace_bytes for c in calls), dtype=torch.uint8, device="cuda:0")
    graphs = [torch.cuda.CUDAGraph() for _ in calls]
    for g, c in zip(graphs, calls):
        with torch.cuda.graph(g):
            A.air_prompt_attn(prepared=c, workspace=shared)
    for step in range(4):
        for o in outs:
            o.zero_()
        for g in graphs if step % 2 else graphs[::-1]:
            g.replay()
        torch.cuda.synchronize()
        for o, w, spans in zip(outs, want, jobs):
            for b, q0, n, _, _ in spans:
                assert torch.equal(o[b, :, q0:q0 + n], w[b, :, q0:q0 + n])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv", [(16384, 1), (16384, 16384), (16383, 3)])
def test_as_many_heads_as_a_call_takes(dtype, hq, hkv):
    import paper_2503_23956_amd as A

    spans = [(0, 0, 3, 0, 40), (1, 1, 1, 2, 9), (1, 2, 1, 0, 70)]
    q, k, v = _tensors(2, 3, 70, hq, hkv, 64, dtype, hkv)
    _check(q, k, v, spans, _run(A, q, k, v, spans))
