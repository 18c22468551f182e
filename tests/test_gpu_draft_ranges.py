"""Draft attention where the sizes of values, the norms' eps or the gains are far from one, on every kernel and plan, against the
fp64 oracle.

Tolerance: relative to the row.  The output's own rounding, 2^-8 of it (fp32: 2^-24), and for either branch 2^-10 of the rms that it has
in the output, gain included (fp32: 2^-13).  The bf16 kernels keep 16 bits of weights, feature maps and state (2^-16 of a term, and
three such terms to a product), and a branch's terms are at most some 8 times its rms (the root of the 41 keys that average out), which
is 2^-11.  fp32: a score of 64 products is off by 64 * 2^-24 of sums of 8, 2^-15 in the exponent."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as D
from oracle import rattn_oracle as O
from paper_2506_15545_b200 import binding as R
from test_gpu_draft import Setup
from test_gpu_parity import np64

pytestmark = pytest.mark.gpu

PLANS = [  # B, H, d, dtype, flags
    (10, 8, 128, "bf16", 0),                             # a CTA per head
    (1, 4, 128, "bf16", 0),                              # clusters
    (2, 4, 128, "bf16", R.FLAG_FORCE_GENERIC),
    (2, 4, 64, "f32", 0),
]


def run_and_check(s, eps, flags, entries):
    q, k, v = (x.cuda() for x in (s.q, s.k, s.v))
    y = np64(R.rattn_draft_attention(q, k, v, torch.tensor(s.parents, dtype=torch.int32, device="cuda"), s.k_ring, s.v_ring, s.state,
                                     s.pos[0], scale=s.scale, eps=eps, gamma_swa=s.gain(s.gs), gamma_rla=s.gain(s.gr), flags=flags))
    assert R.rattn_draft_status() == 0
    gs, gr = s.gains64()
    for b in entries:
        branch = [D.draft_attention(np64(s.q[b]), np64(s.k[b]), np64(s.v[b]), s.parents[b], np64(s.hist[b][0]), np64(s.hist[b][1]), s.w,
                                    s.scale, eps, g1, g2) for g1, g2 in ((gs, 0 * gr), (0 * gs, gr))]
        ref = branch[0] + branch[1]
        of_branch, of_y = (2.0 ** -10, 2.0 ** -8) if s.dtype == "bf16" else (2.0 ** -13, 2.0 ** -24)
        bound = of_y * np.abs(ref) + of_branch * sum(np.sqrt((x * x).mean(-1, keepdims=True)) for x in branch)
        err = np.abs(y[b] - ref)
        assert (err <= bound).all(), (b, float((err / bound).max()))


@pytest.mark.parametrize("B,H,d,dtype,flags", PLANS)
@pytest.mark.parametrize("size,eps,gain", [(-17, 1e-6, 1.0), (-24, 1e-6, 1.0), (0, 100.0, 1.0), (0, 1e6, 1.0), (0, 1e-6, 2.0 ** 10), (-17, 1e-6, 2.0 ** 10)])
def test_rows_far_below_eps_and_large_gains(B, H, d, dtype, flags, size, eps, gain):
    """Rows whose rms is far below the root of eps are small behind their norm, and as exact as others."""
    s = Setup(B, H, H, 5, d, 40, dtype, 100, "tree", seed=31)
    f = 2.0 ** size
    s.v, s.v_ring, s.state = s.v * f, s.v_ring * f, s.state * f
    s.hist = [[k, v * f] for k, v in s.hist]
    s.gs = s.gs * gain
    run_and_check(s, eps, flags, (0, B - 1))


@pytest.mark.parametrize("B,H,d,dtype,flags", PLANS)
@pytest.mark.parametrize("size", [58, 64, 90, 115])
def test_values_whose_squares_leave_fp32(B, H, d, dtype, flags, size):
    """The norms cancel a factor common to all values, up to where the sums of values themselves leave fp32 (2^128; here they
    are below 2^7 times the factor: the state of 60 tokens times a feature map of at most 1)."""
    s = Setup(B, H, H, 5, d, 40, dtype, 100, "tree", seed=32)
    f = 2.0 ** size
    s.v, s.v_ring, s.state = s.v * f, s.v_ring * f, s.state * f
    s.hist = [[k, v * f] for k, v in s.hist]
    run_and_check(s, 1e-6, flags, (0, B - 1))


@pytest.mark.parametrize("B,H,d,dtype,flags", PLANS)
def test_one_node_of_large_values(B, H, d, dtype, flags):
    """Rows that see the node overflow, their neighbours do not; an eps of that size counts."""
    s = Setup(B, H, H, 6, d, 40, dtype, 100, "star", seed=33)
    s.v[:, :, 2] *= 2.0 ** 70
    run_and_check(s, 1e-6, flags, (0, B - 1))
    run_and_check(s, 2.0 ** 127, flags, (0, B - 1))


@pytest.mark.parametrize("B,H,d,dtype,flags", PLANS)
def test_one_node_at_the_last_position(B, H, d, dtype, flags):
    """At 2^31 - 1 - w: the bits of a small position with the same remainder, from the call and from the commit."""
    w = 100
    s = Setup(B, H, H, 1, d, w, dtype, 2 * w + (2 ** 31 - 1) % w, "chain", seed=34)
    top = 2 ** 31 - 1 - w
    par, one = torch.zeros(B, 1, dtype=torch.int32, device="cuda") - 1, torch.ones(B, dtype=torch.int32, device="cuda")
    q, k, v = (x.cuda() for x in (s.q, s.k, s.v))
    got = []
    for pos in (s.pos[0], top):
        cache = [s.k_ring.clone(), s.v_ring.clone(), s.state.clone()]
        y = R.rattn_draft_attention(q, k, v, par, *cache, pos, scale=s.scale, flags=flags)
        R.rattn_draft_commit(k, v, par + 1, one, *cache, pos)
        got.append([y] + cache)
    assert all(torch.equal(a, b) for a, b in zip(*got))
    with pytest.raises(R.RattnError):
        R.rattn_draft_attention(q, k, v, par, *cache, top + 1, scale=s.scale, flags=flags)
