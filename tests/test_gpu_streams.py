"""Calls that are given a stream: their results lie in memory that is free in that stream's order, whatever the current stream has
still to do with the blocks it has freed."""
import pytest
import torch

from paper_2506_15545_b200 import binding as R

pytestmark = pytest.mark.gpu


def _calls():
    g = torch.Generator(device="cuda").manual_seed(5)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    B, H, N, d, w, V = 2, 4, 6, 128, 64, 700
    q, k, v = (rnd(B, H, N, d).bfloat16() for _ in range(3))
    kr, vr = (rnd(B, H, w, d).bfloat16() for _ in range(2))
    state = rnd(B, H, d, d)
    par = (torch.arange(N, device="cuda", dtype=torch.int32) - 1).repeat(B, 1)
    at = torch.arange(N, device="cuda", dtype=torch.int32).repeat(1, B, 1)
    p = torch.softmax(rnd(B, N, V), -1)
    u, gain = torch.rand(B, N, device="cuda", generator=g), 1 + 0.1 * rnd(d)
    return {
        "attention": lambda **s: [R.rattn_draft_attention(q, k, v, par, kr, vr, state, 100, scale=0.09, **s)],
        "verify": lambda **s: list(R.rattn_draft_verify(par + 1, par, p, p, u, **s)),
        "axes": lambda **s: list(R.rattn_qk_prologue_axes(q, k, at, [d // 2], q_gain=gain, **s)),
        "axes_backward": lambda **s: list(R.rattn_qk_prologue_axes_backward(q, k, v, v, at, [d // 2], q_gain=gain, k_gain=gain, **s)),
        "prologue": lambda **s: list(R.rattn_qk_prologue(q, k, q_gain=gain, **s)),
        "prologue_backward": lambda **s: list(R.rattn_qk_prologue_backward(q, k, v, v, q_gain=gain, k_gain=gain, **s)),
        "forward": lambda **s: [R.rattn_forward(q, k, v, 3, **s)],
    }


@pytest.mark.parametrize("name", ["attention", "verify", "axes", "axes_backward", "prologue", "prologue_backward", "forward"])
def test_results_are_not_taken_from_the_current_streams_memory(name):
    call = _calls()[name]
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(400_000_000)                               # the current stream is busy for some 0.2 s
    freed = [torch.empty_like(y) for y in want for _ in range(8)]
    for x in freed:
        x.fill_(3)                                               # ... and then writes to what is freed below
    del freed, x
    got = call(stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    assert torch.cuda.current_stream() == torch.cuda.default_stream()


def test_the_current_stream_is_as_it_was_after_an_error():
    q = torch.zeros(1, 2, 3, 128, device="cuda")
    side = torch.cuda.Stream()
    with pytest.raises(ValueError):
        R.rattn_draft_verify(q, q, q, None, q, stream=side)
    with pytest.raises(ValueError):
        R.rattn_forward(q[0], q, q, 3, stream=side)
    assert torch.cuda.current_stream() == torch.cuda.default_stream()
