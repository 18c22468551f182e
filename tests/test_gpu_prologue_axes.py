"""The prologue for tokens with several coordinates against the fp64 oracle.  Tolerances are those of the plain prologue
(test_gpu_prologue): the same arithmetic, fp32 with angles reduced in fp64."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as D
from paper_2506_15545_b200 import binding as R
from test_gpu_parity import np64, rel_fro
from test_gpu_prologue import close, cu, make

pytestmark = pytest.mark.gpu

ORDER = {"runs": R.AXES_RUNS, "own": R.AXES_OWN, "dealt": R.AXES_DEALT}
CASES = [
    # B, Hq, Hkv, T, d, dtype, sections, order, farthest coordinate
    (2, 4, 2, 300, 128, "bf16", [16, 24, 24], "dealt", 100),
    (2, 4, 2, 300, 128, "f32", [16, 24, 24], "runs", 100),
    (1, 3, 1, 77, 64, "f32", [16, 16], "own", 70000),
    (1, 16, 4, 9, 128, "bf16", [64], "runs", 2 ** 31 - 1),        # a tree's nodes: the kernel of few head vectors
    (3, 2, 2, 1, 128, "f32", [3, 5, 7, 1], "dealt", 1000),        # pairs that no axis has
    (2, 16, 4, 1100, 128, "bf16", [10, 20, 30], "own", 5000),
    (2, 8, 8, 700, 64, "bf16", [8, 8, 8, 8], "dealt", 64),
    (1, 1, 1, 5000, 128, "f32", [1, 63], "runs", 4),              # one head
]


def coordinates(B, T, sections, far, seed):
    rng = np.random.default_rng(seed)
    at = rng.integers(-min(far, 2 ** 30), far, (len(sections), B, T), endpoint=True)
    return torch.tensor(at, dtype=torch.int32), at


def lay(x, layout):
    return x.transpose(1, 2).contiguous() if layout == R.LAYOUT_BTHD and x is not None else x


@pytest.mark.parametrize("layout", [R.LAYOUT_BHTD, R.LAYOUT_BTHD])
@pytest.mark.parametrize("case", CASES)
def test_forward_and_backward(case, layout):
    B, Hq, Hkv, T, d, dtype, sections, order, far = case
    q, k, gq, gk = make(B, Hq, Hkv, T, d, dtype, 70 + T)
    dq, dk, _, _ = make(B, Hq, Hkv, T, d, dtype, 71 + T)
    at, at64 = coordinates(B, T, sections, far, T)
    ang = D.axes_angles(at64, sections, order, 5e5, d)
    args = dict(order=ORDER[order], q_gain=cu(gq), k_gain=cu(gk), layout=layout)
    dev = [lay(x, layout).cuda() for x in (q, k, dq, dk)]
    qo, ko = R.rattn_qk_prologue_axes(dev[0], dev[1], at.cuda(), sections, **args)
    grads = R.rattn_qk_prologue_axes_backward(*dev, at.cuda(), sections, **args)
    torch.cuda.synchronize()
    assert R.rattn_qk_prologue_status() == 0
    for got, x, g in ((qo, q, gq), (ko, k, gk)):
        close(lay(got, layout), D.qk_prologue_axes(np64(x), np64(g), ang), dtype, "forward")
    for got, ggot, x, g, dy in ((grads[0], grads[2], q, gq, dq), (grads[1], grads[3], k, gk, dk)):
        want, gwant = D.qk_prologue_axes_bwd(np64(x), np64(g), ang, np64(dy))
        # fp32: a few ulp of values up to |dy| |gain| / rms(x) ~ 10; bf16: half a step on top
        err = np.abs(np64(lay(got, layout)) - want)
        bound = 2.0 ** -8 * np.abs(want) + 1e-4 if dtype == "bf16" else np.full_like(want, 1e-4)
        assert (err <= bound).all(), float((err - bound).max())
        assert np.abs(np64(ggot) - gwant).max() <= 1e-4 * max(1.0, np.abs(gwant).max())
    # in place, and one tensor alone
    q2, k2 = dev[0].clone(), dev[1].clone()
    R.rattn_qk_prologue_axes(q2, k2, at.cuda(), sections, inplace=True, **args)
    assert torch.equal(q2, qo) and torch.equal(k2, ko)
    only, none = R.rattn_qk_prologue_axes(dev[0], None, at.cuda(), sections, **args)
    assert none is None and torch.equal(only, qo)


@pytest.mark.parametrize("T,layout", [(5, R.LAYOUT_BHTD), (900, R.LAYOUT_BHTD), (900, R.LAYOUT_BTHD)])
def test_one_axis_of_consecutive_positions_is_the_plain_prologue(T, layout):
    q, k, gq, gk = make(2, 8, 2, T, 128, "bf16", 5)
    q, k = lay(q, layout).cuda(), lay(k, layout).cuda()
    at = (torch.arange(T, dtype=torch.int32) + 777).repeat(1, 2, 1).cuda()
    kw = dict(q_gain=cu(gq), k_gain=cu(gk), layout=layout)
    for a, b in zip(R.rattn_qk_prologue_axes(q, k, at, [64], **kw), R.rattn_qk_prologue(q, k, pos0=777, **kw)):
        assert torch.equal(a, b)
    for a, b in zip(R.rattn_qk_prologue_axes_backward(q, k, q, k, at, [64], **kw), R.rattn_qk_prologue_backward(q, k, q, k, pos0=777, **kw)):
        assert torch.equal(a, b)


def test_gradient_against_differences():
    """Central differences of the fp32 forward: step 2^-7, error of the quotient ~ 2^-24 / 2^-7 * 2 per output times the size of the
    sum (d outputs of one row, weights ~ 1) and h^2 of third derivatives of x / rms(x), below 1e-3 for rows of unit rms."""
    B, T, d, sections = 1, 2, 64, [10, 12, 6]
    q, _, gq, _ = make(B, 1, 1, T, d, "f32", 3)
    dy = torch.randn(B, 1, T, d, generator=torch.Generator().manual_seed(4))
    at, _ = coordinates(B, T, sections, 30, 1)
    kw = dict(order=R.AXES_DEALT, q_gain=cu(gq))
    f = lambda x: float((R.rattn_qk_prologue_axes(x, None, at.cuda(), sections, **kw)[0].double() * dy.cuda().double()).sum())  # noqa: E731
    grad = R.rattn_qk_prologue_axes_backward(q.cuda(), None, dy.cuda(), None, at.cuda(), sections, gain_grads=False, **kw)[0]
    h = 2.0 ** -7
    for i in ((0, 0, 0, 0), (0, 0, 1, 5), (0, 0, 0, 33), (0, 0, 1, 63)):
        e = torch.zeros_like(q)
        e[i] = h
        assert abs((f((q + e).cuda()) - f((q - e).cuda())) / (2 * h) - grad[i].item()) < 1e-3


def test_replayed_graph_follows_its_coordinates():
    q, k, gq, gk = make(2, 4, 2, 40, 128, "bf16", 8)
    q, k = q.cuda(), k.cuda()
    at, _ = coordinates(2, 40, [20, 44], 99, 2)
    at = at.cuda()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = R.rattn_qk_prologue_axes(q, k, at, [20, 44])
    for _ in range(2):
        at += 5
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, R.rattn_qk_prologue_axes(q, k, at, [20, 44])))


def test_binding_checks():
    q = torch.randn(2, 4, 9, 128, device="cuda")
    at = torch.zeros(2, 2, 9, dtype=torch.int32, device="cuda")
    for bad in ([], [1, 2, 3, 4, 5], [0, 5], [10 ** 12, 1]):
        with pytest.raises(ValueError):
            R.rattn_qk_prologue_axes(q, None, at, bad)
    with pytest.raises(ValueError):
        R.rattn_qk_prologue_axes(q, None, at[:, :, :8].contiguous(), [8, 8])
    with pytest.raises(TypeError):
        R.rattn_qk_prologue_axes(q, None, at.long(), [8, 8])
    with pytest.raises(ValueError):
        R.rattn_qk_prologue_axes(q, None, at, [8])
    with pytest.raises(R.RattnError):
        R.rattn_qk_prologue_axes(q, None, at, [60, 5])
    with pytest.raises(ValueError):
        R.rattn_qk_prologue_axes_backward(q, None, q[:, :, :8].contiguous(), None, at, [8, 8])
