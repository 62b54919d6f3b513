"""What air_rope and air_prompt_attn promise at the edges of their arguments, on the GPU."""
import pytest

pytestmark = pytest.mark.gpu


def test_outputs_expanded_over_the_batch_are_refused():
    import torch

    import paper_2503_23956_amd as A

    q = torch.randn((2, 4, 3, 64), device="cuda:0").bfloat16()
    k = torch.randn((2, 2, 3, 64), device="cuda:0").bfloat16()
    out = torch.full((1, 4, 3, 64), 42.0, device="cuda:0").bfloat16()
    with pytest.raises(A.AirError, match="two sequences overlap"):
        A.air_prompt_attn(q, k, k, out.expand(2, 4, 3, 64))
    with pytest.raises(A.AirError, match="two sequences overlap"):
        A.air_prompt_attn(q[:1], k[:1], k[:1], out, spans=[(0, 0, 2, 0, 2), (0, 1, 2, 1, 2)])
    skew = out.as_strided((1, 4, 3, 64), (768, 64, 64, 1))  # head 1 of a token is head 0 of the next
    with pytest.raises(A.AirError, match="output rows overlap"):
        A.air_prompt_attn(q[:1], k[:1], k[:1], skew)
    with pytest.raises(A.AirError, match="rows of a destination overlap"):
        A.air_rope(q[:1], q_out=skew)
    torch.cuda.synchronize()
    assert bool((out == 42.0).all())


def test_prepared_calls_called_directly():
    import torch

    import paper_2503_23956_amd as A

    q = torch.randn((1, 8, 5, 128), device="cuda:0").bfloat16()
    k, v = (torch.randn((1, 2, 5000, 128), device="cuda:0").bfloat16() for _ in range(2))
    for spans in ([(0, 0, 5, 0, 5000)], [(0, 0, 5, 0, 5)]):  # with splits and without
        want, out = torch.zeros_like(q), torch.zeros_like(q)
        A.air_prompt_attn(q, k, v, want, spans=spans)
        call = A.prepare_prompt_attn(q, k, v, out, spans=spans)
        assert (call.workspace_bytes > 0) == (spans[0][4] == 5000)
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        out.zero_()
        ws = torch.empty(max(1, call.workspace_bytes), dtype=torch.uint8, device="cuda:0")
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        call(side.cuda_stream, ws)
        torch.cuda.synchronize()
        assert torch.equal(out, want)
    with pytest.raises(A.AirError, match="needs its workspace"):
        A.prepare_prompt_attn(q, k, v, out)(side.cuda_stream)
    turn = A.prepare_rope(q)
    turn()
    with pytest.raises(A.AirError, match="takes no workspace"):
        turn(workspace=ws)
