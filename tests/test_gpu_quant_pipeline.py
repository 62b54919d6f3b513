"""Long generation as a serving program runs it: a prompt rotated and attended to, its rows in 4 bits, weighed by its last queries and cut down;
then, token by token, rotation, append and attention with weights, and eviction whenever a sequence has grown by a few tokens.  Every step against fp64;
the step recorded into a HIP graph against the eager one, bit for bit."""
import numpy as np
import pytest

from quant_util import attention, unpacked
from test_gpu_evict import _plan

pytestmark = pytest.mark.gpu

HQ, HKV, B = 8, 2, 2
PROMPT, WINDOW, STEPS = [93, 70], 12, 21
KEEP, LIMIT, CAP, FIRST, RECENT = 64, 69, 96, 4, 16


class Generation:
    def __init__(self, A, dtype, d, group):
        import torch

        self.A, self.torch, self.dev = A, torch, torch.device("cuda:0")
        self.dt = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.d, self.group = d, group
        self.cache = A.QuantCache(B, HKV, CAP, d, A.AIR_BF16 if dtype == "bf16" else A.AIR_F32, group=group)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device=self.dev)  # noqa: E731
        self.lens, self.kept, self.next_pos = ints([0] * B), ints([0] * B), ints(PROMPT)
        self.weights = torch.zeros((B, HKV, CAP), device=self.dev)
        self.positions = torch.full((B, HKV, CAP), -1, dtype=torch.int32, device=self.dev)
        freqs, _ = A.air_rope_frequencies(d // 2, 1e6)
        self.freqs = torch.tensor(freqs, device=self.dev)
        # buffers of a step, as a graph needs them
        self.qkv = torch.zeros((B, 1, HQ + 2 * HKV, d), dtype=self.dt, device=self.dev)
        heads = self.qkv.transpose(1, 2)
        self.q, self.k, self.v = (torch.zeros((B, h, 1, d), dtype=self.dt, device=self.dev) for h in (HQ, HKV, HKV))
        self.out = torch.zeros((B, HQ, 1, d), dtype=self.dt, device=self.dev)
        self.rope = A.prepare_rope(heads[:, :HQ], heads[:, HQ:HQ + HKV], heads[:, HQ + HKV:], self.q, self.k, self.v,
                                   positions=self.next_pos.view(1, B, 1), freqs=self.freqs, axis_pairs=(d // 2,))
        self.attn = A.prepare_quant_attn(self.cache, self.q, self.out, lens=self.lens, k=self.k, v=self.v, weights=self.weights, positions=self.positions,
                                         first_positions=self.next_pos)
        self.evict = A.prepare_evict(self.cache.planes, self.weights, positions=self.positions, lens=self.lens, lens_out=self.kept, keep=KEEP,
                                     limit=LIMIT, first=FIRST, recent=RECENT)
        self.spaces = [torch.empty(max(1, c.workspace_bytes or 0), dtype=torch.uint8, device=self.dev) for c in (self.attn, self.evict)]

    def prompt(self, seed):
        torch, A = self.torch, self.A
        gen = torch.Generator(device="cuda:0").manual_seed(seed)
        T, d = max(PROMPT), self.d
        qkv = torch.randn((B, T, HQ + 2 * HKV, d), generator=gen, device=self.dev).to(self.dt).transpose(1, 2)
        pos = torch.arange(T, device=self.dev, dtype=torch.int32).expand(B, T).contiguous()
        q, k, v = (torch.zeros((B, h, T, d), dtype=self.dt, device=self.dev) for h in (HQ, HKV, HKV))
        A.air_rope(qkv[:, :HQ], qkv[:, HQ:HQ + HKV], qkv[:, HQ + HKV:], q, k, v, positions=pos, freqs=self.freqs, axis_pairs=(d // 2,))
        out = torch.zeros_like(q)
        A.air_prompt_attn(q, k, v, out, spans=[(b, 0, n, 0, n) for b, n in enumerate(PROMPT)])
        counts = torch.tensor(PROMPT, dtype=torch.int32, device=self.dev)
        A.air_quant_append(self.cache, k, v, counts=counts, positions=self.positions, first_positions=torch.zeros_like(counts), weights=self.weights)
        self.lens.copy_(counts)
        # the last queries of every prompt weigh its slots
        window = torch.stack([q[b, :, n - WINDOW:n] for b, n in enumerate(PROMPT)])
        A.air_quant_attn(self.cache, window, None, lens=self.lens, weights=self.weights)
        return window

    def grow(self):
        """What is recorded: the step's tokens are in self.qkv."""
        self.rope()
        self.attn(workspace=self.spaces[0])
        self.lens.add_(1)
        self.next_pos.add_(1)

    def shrink(self):
        self.evict(workspace=self.spaces[1])
        self.lens.copy_(self.kept)


@pytest.mark.parametrize("dtype,d,group", [("bf16", 128, 32), ("bf16", 64, 64), ("f32", 64, 32)])
def test_generation(dtype, d, group):
    import torch

    import paper_2503_23956_amd as A

    one, other = Generation(A, dtype, d, group), Generation(A, dtype, d, group)
    window = one.prompt(5)
    other.prompt(5)
    for b, (_, _, w, wb) in enumerate(attention(one.cache, window, PROMPT, [WINDOW] * B, True)):
        n = PROMPT[b]
        assert bool(((one.weights[b, :, :n].double() - w).abs() <= wb + w * 2.0 ** -23).all())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        other.grow()
        other.shrink()
    gen = torch.Generator(device="cuda:0").manual_seed(6)
    held = list(PROMPT)
    seen = [[set(range(n)) for _ in range(HKV)] for n in PROMPT]
    for step in range(STEPS):
        x = torch.randn(one.qkv.shape, generator=gen, device=one.dev).to(one.dt)
        for g in (one, other):
            g.qkv.copy_(x)
        before = one.weights.clone()
        one.grow()
        # ---- the step's attention and weights
        after = [n + 1 for n in held]
        for b, (o, bound, w, wb) in enumerate(attention(one.cache, one.q, after, [1] * B, True)):
            assert bool(((one.out[b].double() - o).abs() <= bound).all())
            was = before[b, :, :after[b]].double()
            was[:, held[b]] = 0.0
            assert bool(((one.weights[b, :, :after[b]].double() - was - w).abs() <= wb + (was + w) * 2.0 ** -23).all())
        # ---- what stays
        weights, positions = one.weights.cpu().numpy().copy(), one.positions.cpu().numpy().copy()
        rows = [lo + up for lo, up, _ in unpacked(one.cache)]
        one.shrink()
        now = [KEEP if n > LIMIT else n for n in after]
        assert one.lens.tolist() == now
        got_w, got_p = one.weights.cpu().numpy(), one.positions.cpu().numpy()
        new_rows = [lo + up for lo, up, _ in unpacked(one.cache)]
        for b, n in enumerate(after):
            for h in range(HKV):
                seen[b][h].add(PROMPT[b] + step)
                if n > LIMIT:
                    to, come = _plan(weights[b, h], positions[b, h], n, KEEP, FIRST, RECENT)
                    weights[b, h, to], positions[b, h, to] = weights[b, h, come], positions[b, h, come]
                    i, j = torch.from_numpy(to).cuda(), torch.from_numpy(come).cuda()
                    for r in rows:
                        r[b, h, i] = r[b, h, j]
                m = now[b]
                assert np.array_equal(got_w[b, h, :m], weights[b, h, :m]) and np.array_equal(got_p[b, h, :m], positions[b, h, :m])
                have = set(got_p[b, h, :m].tolist())
                latest = PROMPT[b] + step
                assert len(have) == m and have <= seen[b][h] and set(range(FIRST)) <= have and set(range(latest - RECENT + 1, latest + 1)) <= have
                seen[b][h] = have
                for r, s in zip(rows, new_rows):
                    assert torch.equal(r[b, h, :m], s[b, h, :m])
        held = now
        # ---- the recorded step does the same
        graph.replay()
        torch.cuda.synchronize()
        for x, y in ((one.out, other.out), (one.weights, other.weights), (one.positions, other.positions), (one.lens, other.lens),
                     (one.next_pos, other.next_pos), *zip(one.cache.planes, other.cache.planes)):
            a, c = x, y
            if x.dim() == 4 and x.shape[2] == CAP or x.dim() == 3 and x.shape[2] == CAP:
                a, c = x[:, :, : min(held)], y[:, :, : min(held)]
            assert torch.equal(a, c)
