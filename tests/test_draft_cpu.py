"""Speculative decoding and the several-axes prologue without a GPU: pins of the oracle (tests compare the kernels with it),
and what the entry points refuse before anything is launched."""
import ctypes
import os
import subprocess
from fractions import Fraction

import numpy as np
import pytest
import torch

from oracle import draft_oracle as D
from oracle import prologue_oracle as P
from oracle import rattn_oracle as O

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def R():
    from paper_2506_15545_b200 import binding, build
    build.build()
    binding.lib()
    return binding


# ---------------------------------------------------------------------------- oracle pins

@pytest.mark.parametrize("pos,w,N", [(0, 3, 5), (2, 4, 6), (20, 4, 7), (9, 1, 6)])
def test_chain_of_drafts_is_the_rows_of_one_forward(pos, w, N):
    rng = np.random.default_rng(pos + w)
    q, k, v = rng.standard_normal((4, pos + N, 8)), rng.standard_normal((2, pos + N, 8)), rng.standard_normal((2, pos + N, 8))
    ref = O.forward(q[None], k[None], v[None], w, 0.3)[0]
    got = D.draft_attention(q[:, pos:], k[:, pos:], v[:, pos:], np.arange(N) - 1, k[:, :pos], v[:, :pos], w, 0.3)
    assert np.abs(got - ref[:, pos:]).max() < 1e-12


def test_nodes_off_the_path_and_unused_nodes_have_no_part():
    rng = np.random.default_rng(0)
    q, k, v = (rng.standard_normal((1, 6, 4)) for _ in range(3))
    kh, vh = (rng.standard_normal((1, 7, 4)) for _ in range(2))
    parents = np.array([-1, 0, 0, 1, -2, 4])
    a = D.draft_attention(q, k, v, parents, kh, vh, 3)
    assert np.isnan(a[:, 4:]).all() and np.isfinite(a[:, :4]).all()
    k2 = k.copy()
    k2[:, 2] = np.nan
    b = D.draft_attention(q, k2, v, parents, kh, vh, 3)
    assert np.array_equal(a[:, [0, 1, 3]], b[:, [0, 1, 3]]) and np.isnan(b[:, 2]).all()


def test_commit_is_the_cache_of_the_longer_history():
    rng = np.random.default_rng(1)
    for pos, w, n in ((3, 5, 4), (11, 4, 3), (11, 4, 6), (0, 2, 5)):
        kh, vh = (rng.standard_normal((2, pos + n, 4)) for _ in range(2))
        ring = D.cache_of(kh[:, :pos], vh[:, :pos], w)
        got = D.commit(kh[:, pos:], vh[:, pos:], list(range(n)), n, *ring, pos)
        for x, y in zip(got, D.cache_of(kh, vh, w)):
            assert np.abs(x - y).max() < 1e-12


def _drawn(parents, q, rng):
    """Tokens of the nodes, each from its parent's row of q."""
    return [0] + [int(rng.choice(len(q[0]), p=[float(x) for x in q[parents[i]]])) for i in range(1, len(parents))]


def test_verified_tokens_are_distributed_as_the_target():
    """The first new token (the first accepted child's, or the one drawn) has the target's distribution: 20000 trials of a
    tree with three children; a count is within 5 standard deviations of its mean in all but 6e-7 of cases."""
    rng = np.random.default_rng(5)
    p0, q0 = np.array([0.5, 0.2, 0.2, 0.1]), np.array([0.1, 0.4, 0.2, 0.3])
    parents = [-1, 0, 0, 0]
    p, q = [p0] * 4, [q0] * 4
    n, seen = 20000, np.zeros(4)
    for _ in range(n):
        tokens = _drawn(parents, q, rng)
        line, token = D.verify(tokens, parents, p, q, rng.random(4))
        seen[tokens[line[1]] if len(line) > 1 else token] += 1
    assert (np.abs(seen - n * p0) <= 5 * np.sqrt(n * p0 * (1 - p0))).all(), seen


def test_verification_by_hand():
    F = Fraction
    p = [[F(1, 2), F(1, 4), F(1, 4)], [F(1), F(0), F(0)], [F(0), F(1), F(0)]]
    q = [[F(1, 4), F(1, 2), F(1, 4)]] * 3
    # child 1 (token 1): 0.9 * 1/2 < 1/4 fails; what is left is (1/4, 0, 0); child 2 (token 0): 0.9 * 1/4 * 1/4 < 1/4 holds
    assert D.verify([9, 1, 0], [-1, 0, 0], p, q, [F(0), F(9, 10), F(9, 10)]) == ([0, 2], 1)
    # greedy drafts: token 1 taken out, 3/4 left; token 0: 0.5 * 3/4 < 1/2
    assert D.verify([9, 1, 0], [-1, 0, 0], p, None, [F(0), F(9, 10), F(1, 2)]) == ([0, 2], 1)
    # both rejected: token 2 is all that is left
    assert D.verify([9, 1, 0], [-1, 0, 0], p, None, [F(1, 3), F(9, 10), F(9, 10)]) == ([0], 2)
    assert D.verify([9, 1, 0], [-2, 0, 0], p, None, [F(0)] * 3) == ([], -1)


def test_axes_reduce_to_the_plain_rotation_and_to_complex_products():
    rng = np.random.default_rng(2)
    x = rng.standard_normal((1, 2, 5, 16))
    pos = np.arange(5) + 1000
    for order in ("runs", "own", "dealt"):
        ang = D.axes_angles(pos[None, None], [8], order, 5e5, 16)
        assert np.allclose(D.axes_rotate(x, ang), P.rope(x, pos, 5e5), atol=1e-12)
    ang = D.axes_angles(rng.integers(0, 50, (3, 1, 5)), [2, 3, 2], "dealt", 1e4, 16)
    assert (ang[..., 7] == 0).all()                                # pairs that no axis has are not turned
    z = (torch.complex(torch.tensor(x[..., :8]), torch.tensor(x[..., 8:])) * torch.polar(torch.ones(1, 1, 5, 8, dtype=torch.float64), torch.tensor(ang)[:, None]))
    assert np.allclose(D.axes_rotate(x, ang), torch.cat([z.real, z.imag], -1).numpy(), atol=1e-12)


def test_axes_orders_by_hand():
    at = np.array([[[1]], [[10]], [[100]]])
    theta, d = 16.0, 8
    assert np.allclose(D.axes_angles(at, [1, 2, 1], "runs", theta, d)[0, 0], [1, 10 * 16 ** -.25, 10 * 16 ** -.5, 100 * 16 ** -.75])
    assert np.allclose(D.axes_angles(at, [1, 2, 1], "own", theta, d)[0, 0], [1, 10, 10 * 16 ** -.5, 100])
    assert np.allclose(D.axes_angles(at, [1, 2, 1], "dealt", theta, d)[0, 0], [1, 10 * 16 ** -.25, 100 * 16 ** -.5, 10 * 16 ** -.75])


def test_axes_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(3)
    x, dy, gain = rng.standard_normal((1, 2, 3, 8)), rng.standard_normal((1, 2, 3, 8)), rng.standard_normal(8)
    ang = D.axes_angles(rng.integers(0, 9, (2, 1, 3)), [1, 2], "own", 1e4, 8)
    f = lambda x, g: (D.qk_prologue_axes(x, g, ang) * dy).sum()  # noqa: E731
    dx, dgain = D.qk_prologue_axes_bwd(x, gain, ang, dy)
    h = 1e-6
    for arr, grad, call in ((x, dx, lambda a: f(a, gain)), (gain, dgain, lambda a: f(x, a))):
        for i in np.ndindex(arr.shape):
            up, down = arr.copy(), arr.copy()
            up[i] += h
            down[i] -= h
            assert abs((call(up) - call(down)) / (2 * h) - grad[i]) < 1e-6


# ---------------------------------------------------------------------------- refusals

def test_structs_match_the_binding(R, tmp_path):
    src = tmp_path / "sz.c"
    src.write_text('#include "rattn.h"\n#include <stdio.h>\n#include <stddef.h>\nint main(void){printf("%zu %zu %zu %zu %zu %zu %zu %d\\n",'
                   'sizeof(rattn_draft_params), offsetof(rattn_draft_params, B), offsetof(rattn_draft_params, gamma_swa),'
                   'offsetof(rattn_draft_params, pos), sizeof(rattn_verify_params), offsetof(rattn_verify_params, B),'
                   'sizeof(rattn_qk_axes), RATTN_DRAFT_MAX_NODES);return 0;}\n')
    exe = tmp_path / "sz"
    subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    got = list(map(int, subprocess.check_output([str(exe)]).split()))
    d, v = R.RattnDraftParams, R.RattnVerifyParams
    assert got == [ctypes.sizeof(d), d.B.offset, d.gamma_swa.offset, d.pos.offset, ctypes.sizeof(v), v.B.offset,
                   ctypes.sizeof(R.RattnQkAxes), R.DRAFT_MAX_NODES]


FAKE = 0x10000                                 # non-null, aligned; never dereferenced


def _draft(R, **kw):
    p = R.RattnDraftParams()
    for f in ("q", "k", "v", "out", "parents", "k_ring", "v_ring", "state", "path", "n_accepted"):
        setattr(p, f, FAKE)
    p.B, p.H_q, p.H_kv, p.N, p.d, p.w, p.dtype, p.scale, p.eps = 2, 8, 2, 5, 128, 64, R.RATTN_BF16, 0.1, 1e-6
    for k, v in kw.items():
        setattr(p, k, v)
    return ctypes.byref(p)


_COMMON = [(dict(B=0), -1), (dict(H_kv=0), -1), (dict(N=0), -1), (dict(N=129), -1), (dict(w=0), -1),
           (dict(pos=-1), -1), (dict(pos=2 ** 31 - 64), -1), (dict(B=1 << 20, w=1 << 20), -1), (dict(d=96), -4), (dict(dtype=7), -4),
           (dict(feature_map=3), -4), (dict(layout=2), -4), (dict(k=0), -2), (dict(v=0), -2), (dict(k_ring=0), -2),
           (dict(v_ring=0), -2), (dict(state=0), -2), (dict(k=FAKE + 8), -3), (dict(v_ring=FAKE + 4), -3),
           (dict(state=FAKE + 4), -3), (dict(pos_dev=FAKE + 2), -3)]


@pytest.mark.parametrize("kw,code", _COMMON + [
    (dict(H_q=3), -1), (dict(H_q=0), -1), (dict(eps=0.0), -1), (dict(eps=float("nan")), -1), (dict(eps=float("inf")), -1),
    (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1), (dict(q=0), -2), (dict(out=0), -2), (dict(parents=0), -2),
    (dict(q=FAKE + 8), -3), (dict(out=FAKE + 2), -3), (dict(parents=FAKE + 1), -3), (dict(gamma_swa=FAKE + 4), -3)])
def test_draft_attention_refuses(R, kw, code):
    before = R.rattn_launch_count()
    assert R.lib().rattn_draft_attention(_draft(R, **kw), None) == code
    assert R.rattn_launch_count() == before


@pytest.mark.parametrize("kw,code", _COMMON + [(dict(path=0), -2), (dict(n_accepted=0), -2), (dict(path=FAKE + 2), -3),
                                               (dict(n_accepted=FAKE + 1), -3)])
def test_draft_commit_refuses(R, kw, code):
    before = R.rattn_launch_count()
    assert R.lib().rattn_draft_commit(_draft(R, **kw), None) == code
    assert R.rattn_launch_count() == before
    assert R.lib().rattn_draft_commit(None, None) == R.lib().rattn_draft_attention(None, None) == -2


@pytest.mark.parametrize("w", [1, 64, 1000])
def test_every_position_that_is_documented_is_taken(R, w):
    """2^31 - 1 - w is the last; that a position passes shows in the next check's answer, and nothing is launched."""
    for call in (R.lib().rattn_draft_attention, R.lib().rattn_draft_commit):
        for pos, code in ((2 ** 31 - 1 - w, -3), (2 ** 31 - 1 - w - 128, -3), (2 ** 31 - w, -1)):
            assert call(_draft(R, pos=pos, w=w, k=FAKE + 8), None) == code


@pytest.mark.parametrize("kw,code", [
    (dict(B=0), -1), (dict(N=0), -1), (dict(N=129), -1), (dict(V=0), -1), (dict(V=2 ** 31 - 1), -1), (dict(dtype=2), -4),
    (dict(tokens=0), -2), (dict(parents=0), -2), (dict(target_probs=0), -2), (dict(u=0), -2), (dict(path=0), -2),
    (dict(n_accepted=0), -2), (dict(token=0), -2), (dict(target_probs=FAKE + 8), -3), (dict(draft_probs=FAKE + 2), -3),
    (dict(u=FAKE + 2), -3), (dict(tokens=FAKE + 1), -3)])
def test_draft_verify_refuses(R, kw, code):
    p = R.RattnVerifyParams()
    for f in ("tokens", "parents", "target_probs", "draft_probs", "u", "path", "n_accepted", "token"):
        setattr(p, f, FAKE)
    p.B, p.N, p.V, p.dtype = 2, 4, 100, R.RATTN_F32
    for k, v in kw.items():
        setattr(p, k, v)
    before = R.rattn_launch_count()
    assert R.lib().rattn_draft_verify(ctypes.byref(p), None) == code
    assert R.lib().rattn_draft_verify(None, None) == -2
    assert R.rattn_launch_count() == before


@pytest.mark.parametrize("kw,ax,code", [
    (dict(B=0), {}, -1), (dict(q_out=None), {}, -2), (dict(d=96), {}, -4), (dict(theta=0.0), {}, -1), (dict(theta=-1.0), {}, -1),
    (dict(pos0=3), {}, -1), (dict(pos=FAKE), {}, -1), ({}, dict(n_axes=0), -1), ({}, dict(n_axes=5), -1),
    ({}, dict(sections=(0, 4, 4, 4)), -1), ({}, dict(sections=(40, 25, 0, 0)), -1), ({}, dict(sections=(2 ** 31 - 1, 2 ** 31 - 1, 0, 0)), -1),
    ({}, dict(order=3), -4), ({}, dict(at=None), -2), ({}, dict(at=FAKE + 2), -3)])
def test_prologue_axes_refuses(R, kw, ax, code):
    p, x = R.RattnQkParams(), R.RattnQkAxes()
    p.q = p.k = p.q_out = p.k_out = FAKE
    p.B, p.H_q, p.H_kv, p.T, p.d, p.dtype, p.eps, p.theta = 2, 4, 2, 64, 128, R.RATTN_BF16, 1e-6, 5e5
    x.at, x.n_axes, x.sections, x.order = FAKE, 2, (32, 32, 0, 0), R.AXES_RUNS
    for o, d in ((p, kw), (x, ax)):
        for k, v in d.items():
            setattr(o, k, v)
    L, before = R.lib(), R.rattn_launch_count()
    assert L.rattn_qk_prologue_axes(ctypes.byref(p), ctypes.byref(x), None) == code
    if "q_out" not in kw:
        assert L.rattn_qk_prologue_axes_backward(ctypes.byref(p), ctypes.byref(x), FAKE, FAKE, FAKE, FAKE, None, None, None, 0, None) == code
    assert L.rattn_qk_prologue_axes(ctypes.byref(p), None, None) in (-2, code)
    assert R.rattn_launch_count() == before
