"""air_evict against its rule, stated with sorts and sets on the host; everything it moves is compared bit for bit."""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _ints(x):
    import torch

    return torch.tensor(x, dtype=torch.int32, device="cuda:0")


def _plan(weights, positions, n, keep, first, recent):
    """(slots given up, slots that move in) of one head."""
    w = weights[:n].astype(np.float64)
    safe = np.zeros(n, dtype=bool)
    if positions is not None:
        pos = positions[:n].astype(np.int64)
        safe = (pos < first) | ((pos.max() - pos < recent) if n else False)
    rank = np.where(safe, 0, np.where(np.isnan(w), 1, 2))
    order = np.lexsort((np.arange(n), -np.where(rank == 2, w, 0.0), rank))
    stay = np.sort(order[:keep])
    return np.setdiff1d(np.arange(keep), stay), stay[stay >= keep]


def _check(weights, positions, lens, keep, limit, first=0, recent=0, planes=(), workspace=None):
    """weights (and positions) numpy [B][H][cap]; planes: torch tensors [B][H][cap][n]."""
    import torch

    import paper_2503_23956_amd as A

    B, H, cap = weights.shape
    w = torch.from_numpy(weights.copy()).cuda()
    pos = torch.from_numpy(positions.copy()).cuda() if positions is not None else None
    before = [p.clone() for p in planes]
    out = _ints([-9] * B)
    A.air_evict(list(planes), w, lens=_ints(lens), lens_out=out, keep=keep, limit=limit, positions=pos, first=first, recent=recent, workspace=workspace)
    torch.cuda.synchronize()
    want_w, want_p = weights.copy(), None if positions is None else positions.copy()
    moved, held = 0, [min(max(n, 0), cap) for n in lens]
    for b, n in enumerate(held):
        for h in range(H) if n > limit else ():
            to, come = _plan(weights[b, h], None if positions is None else positions[b, h], n, keep, first, recent)
            assert len(to) == len(come)
            moved += len(to)
            want_w[b, h, to] = weights[b, h, come]
            if positions is not None:
                want_p[b, h, to] = positions[b, h, come]
            i, j = torch.from_numpy(to).cuda(), torch.from_numpy(come).cuda()
            for x in before:
                x[b, h, i] = x[b, h, j]
    assert out.tolist() == [keep if n > limit else n for n in held]
    assert np.array_equal(w.cpu().numpy().view(np.int32), want_w.view(np.int32))
    assert positions is None or np.array_equal(pos.cpu().numpy(), want_p)
    for x, y in zip(before, planes):
        assert torch.equal(x, y)
    return moved


def _planes(B, H, cap, seed=0):
    """Rows of any bytes: wide ones, narrow ones, token-major ones, of 4 and of 1024 bytes."""
    import torch

    g = torch.Generator(device="cuda:0").manual_seed(seed)
    make = lambda *s: torch.randint(0, 256, s, generator=g, device="cuda:0", dtype=torch.int32).to(torch.uint8)  # noqa: E731
    return [make(B, H, cap, 64), make(B, H, cap, 4), make(B, cap, H, 128).transpose(1, 2), make(B, H, cap, 1024 + 16)[..., :1024],
            make(B, H, cap, 36), make(H, B, cap, 72).transpose(0, 1)[..., 4:68]]


@pytest.mark.parametrize("cap,lens,keep,limit", [
    (1, [1, 0, 1], 1, 1), (2, [2, 1, 0], 1, 1), (3, [3, 2, 3], 2, 2), (70, [70, 64, 65], 64, 64), (130, [130, 129, 7], 128, 129),
    (1000, [1000, 999, 500], 100, 600), (1500, [1500, 1499, 1023], 1024, 1024), (300, [300, 1, 299], 299, 299),
    (90, [91, -5, 2 ** 31 - 1], 30, 40),  # lengths outside the capacity are clamped
])
def test_lengths(cap, lens, keep, limit):
    rng = np.random.default_rng(cap + keep)
    B, H = len(lens), 2
    w = np.exp(2 * rng.standard_normal((B, H, cap))).astype(np.float32)
    pos = np.stack([[rng.permutation(cap) for _ in range(H)] for _ in range(B)]).astype(np.int32)
    _check(w, pos, lens, keep, limit, planes=_planes(B, H, cap))
    _check(w, pos, lens, keep, limit, first=min(2, keep), recent=min(8, keep - min(2, keep)), planes=_planes(B, H, cap, 1))
    _check(w, None, lens, keep, limit, planes=_planes(B, H, cap, 2)[:1])


def test_weights_of_every_kind():
    """Ties, zeros of both signs, negative weights, infinities, NaN, the smallest numbers."""
    rng = np.random.default_rng(5)
    kinds = np.array([0.0, -0.0, 1.0, 1.0, -1.0, math.inf, -math.inf, math.nan, 1e-45, -1e-45, 3e38, 1.0000001, -math.nan], dtype=np.float32)
    w = kinds[rng.integers(0, len(kinds), (4, 3, 700))]
    w[1] = 0.0
    w[2] = math.nan
    w[3, 0] = -math.inf
    for keep, limit in ((1, 1), (53, 60), (350, 350), (699, 699)):
        moved = _check(w, None, [700, 700, 700, 650], keep, limit)
        assert moved > 0 or keep == 699
    pos = np.stack([[rng.permutation(700) for _ in range(3)] for _ in range(4)]).astype(np.int32)
    _check(w, pos, [700, 700, 700, 650], 60, 60, first=4, recent=56)


def test_protected_tokens():
    rng = np.random.default_rng(6)
    w = np.arange(600, dtype=np.float32)[None, None].repeat(2, 0).repeat(2, 1)
    pos = rng.permutation(600).astype(np.int32)[None, None].repeat(2, 0).repeat(2, 1)
    _check(w, pos, [600, 600], 100, 100, first=100)
    _check(w, pos, [600, 600], 100, 100, recent=100)
    _check(w, pos, [600, 590], 100, 100, first=50, recent=50)
    # positions that repeat protect more slots than stay: the lower slots first
    _check(w, np.zeros_like(pos), [600, 600], 100, 100, first=1)
    # positions at both ends of their type
    ends = np.where(np.arange(600) % 3 == 0, 2 ** 31 - 1, -2 ** 31).astype(np.int32)[None, None].repeat(2, 0).repeat(2, 1)
    _check(w, ends, [600, 600], 250, 250, recent=250)
    # a negative position lies in front of every other
    _check(w, (pos - 300).astype(np.int32), [600, 600], 100, 100, first=0, recent=30)


@pytest.mark.parametrize("n,keep", [(4000, 3900), (4093, 700), (4094, 4000), (16381, 9000), (16382, 16000), (20001, 9000), (20001, 200), (24573, 12000), (24574, 5000), (70000, 33000)])
def test_many_slots(n, keep):
    """Keys in LDS and formed again, more moves than one workgroup takes, ties by the thousand."""
    rng = np.random.default_rng(n)
    cap = n + 3
    w = np.exp(2 * rng.standard_normal((2, 2, cap))).astype(np.float32)
    w[:, :, ::7] = 0.25
    pos = np.stack([[rng.permutation(cap) for _ in range(2)] for _ in range(2)]).astype(np.int32)
    assert _check(w, pos, [n, n - 5], keep, keep, first=3, recent=100, planes=_planes(2, 2, cap)[:3]) > 0
    w[1] = np.float32(1.5)
    w[1, :, -900:] = 2.0
    assert _check(w, None, [n, n - 5], keep, keep, planes=_planes(2, 2, cap, 1)[:1]) > 0


def test_other_streams_graphs_and_workspaces():
    import torch

    import paper_2503_23956_amd as A

    rng = np.random.default_rng(8)
    cap, keep = 6000, 3000
    w0 = torch.from_numpy(np.exp(rng.standard_normal((2, 2, cap))).astype(np.float32)).cuda()
    rows0 = torch.from_numpy(rng.standard_normal((2, 2, cap, 128)).astype(np.float32)).cuda()
    lens, results = _ints([6000, 4000]), []
    w, rows, out = w0.clone(), rows0.clone(), _ints([0, 0])
    call = A.prepare_evict([rows], w, lens=lens, lens_out=out, keep=keep, limit=3500)
    assert call.workspace_bytes > 0
    space = torch.empty(call.workspace_bytes, dtype=torch.uint8, device="cuda:0")
    call(workspace=space)
    torch.cuda.synchronize()
    results.append((w.clone(), rows.clone(), out.clone()))
    stream = torch.cuda.Stream()
    with pytest.raises(A.AirError):
        call(stream=stream.cuda_stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(workspace=space)
    for turn in range(4):
        w.copy_(w0)
        rows.copy_(rows0)
        out.zero_()
        torch.cuda.synchronize()
        if turn % 2:
            call(stream=stream.cuda_stream, workspace=space)
        else:
            graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(results[0], (w, rows, out)):
            assert torch.equal(x, y)
