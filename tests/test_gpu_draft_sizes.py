"""Speculative decoding at the sizes that take the kernels' other plans, against the fp64 oracle: vocabularies that reach the
verification's loop of whole vectors, more heads than SMs in the commit, and the portable attention with four rows to a warp."""
import numpy as np
import pytest
import torch

from oracle import draft_oracle as D
from oracle import rattn_oracle as O
from paper_2506_15545_b200 import binding as R
from test_gpu_draft import Setup, _rows, tree
from test_gpu_parity import np64

pytestmark = pytest.mark.gpu


def verify_and_check(tokens, parents, p, q, u):
    path, n, token = R.rattn_draft_verify(tokens.cuda(), torch.tensor(parents, dtype=torch.int32).cuda(), p.cuda(),
                                          None if q is None else q.cuda(), u.cuda())
    for b in range(len(parents)):
        line, x = D.verify(tokens[b].tolist(), parents[b].tolist(), np64(p[b]).tolist(), None if q is None else np64(q[b]).tolist(),
                           np64(u[b]).tolist())
        assert path[b].tolist() == line + [-1] * (len(parents[b]) - len(line)) and n[b].item() == len(line), b
        assert token[b].item() == x, b


# From 49150 (fp32) and 98300 (bf16) tokens on a warp's run has room for the loop; odd ones start rows at every offset from a 16-byte
# boundary, the last two have steps behind the loop.
@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("V,dtype", [(50257, "f32"), (65536, "f32"), (151643, "f32"), (100003, "bf16"), (131073, "bf16"), (200001, "bf16")])
@pytest.mark.parametrize("kind", ["star", "chain"])
def test_verify_large_vocabularies(V, dtype, kind, draft):
    """The drawn token in the first step, in the first and a later CTA's loop, behind it, and at the row's end."""
    B, N = 5, 7
    p, q, u, g = _rows(B, N, V, V + N, dtype, 1.0, 0.9)
    parents = np.stack([tree(N, kind, None) for _ in range(B)])
    tokens = torch.zeros(B, N, dtype=torch.int32)
    for b in range(B):
        for i in range(N):
            if i == 2 and not draft:
                tokens[b, i] = int(p[b, 0].argmax())             # a token with weight is taken out
            else:
                tokens[b, i] = int(torch.multinomial((q if draft else p)[b, max(0, parents[b][i])].double(), 1, generator=g))
    u[:, 0] = torch.tensor([0.0, 3e-3, 6e-3, 0.6, 1 - 2.0 ** -24])
    if kind == "star":
        u[1:, 1:] = u[1:, 1:].clamp(min=0.9)                    # most are rejected, one after the other
    verify_and_check(tokens, parents, p, q if draft else None, u)


@pytest.mark.parametrize("V,dtype", [(151643, "f32"), (131073, "bf16")])
def test_verify_draws_every_step_of_a_run(V, dtype):
    """One token of the row has all the weight: it is drawn, wherever it lies."""
    vec, step = (4, 128) if dtype == "f32" else (8, 256)
    at = [0, 1, vec, step - 1, step, step + 1, 4 * step, 5 * step - 1, 5 * step + 3, 9 * step, 10 * step + 1, V // 2, V - step, V - 2, V - 1]
    p = torch.zeros(len(at), 2, V, dtype=torch.float32 if dtype == "f32" else torch.bfloat16)
    for b, x in enumerate(at):
        p[b, :, x] = 1.0
    q = torch.full_like(p, 1.0 / V)
    par = torch.tensor([[-1, 0]] * len(at), dtype=torch.int32)
    tok = torch.tensor([[0, (x + 1) % V] for x in at], dtype=torch.int32)      # has no weight: rejected
    for u0 in (0.0, 0.5, 1 - 2.0 ** -24):
        for drafts in (None, q):
            _, n, token = R.rattn_draft_verify(tok.cuda(), par.cuda(), p.cuda(), None if drafts is None else drafts.cuda(),
                                               torch.tensor([[u0, 0.5]] * len(at)).cuda())
            assert n.tolist() == [1] * len(at) and token.tolist() == at


@pytest.mark.parametrize("phi", [O.PHI_SOFTMAX, O.PHI_RELU])
@pytest.mark.parametrize("d,dtype", [(128, "bf16"), (64, "bf16"), (128, "f32"), (64, "f32")])
@pytest.mark.parametrize("layout", [R.LAYOUT_BHTD, R.LAYOUT_BTHD])
def test_commit_of_more_heads_than_sms(d, dtype, layout, phi):
    """A CTA per head: positions inside the first window and far beyond it, paths shorter and longer than the window, empty ones."""
    B, H, N, w = 40, 8, 21, 9
    rng = np.random.default_rng(d)
    pos = rng.integers(0, 60, B)
    pos[:6] = 0, 1, w - 1, w, w + 1, 59
    n = rng.integers(0, N + 1, B)
    n[:6] = N, w, w + 1, N, 1, 0
    s = Setup(B, H, H, N, d, w, dtype, pos.tolist(), "chain", phi=phi, seed=d, fill=0.0)
    path = np.stack([rng.permutation(N) for _ in range(B)])
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    lay = (lambda x: x.transpose(1, 2).contiguous()) if layout == R.LAYOUT_BTHD else (lambda x: x)
    kr, vr, st = s.k_ring.clone(), s.v_ring.clone(), s.state.clone()
    R.rattn_draft_commit(lay(s.k).cuda(), lay(s.v).cuda(), dev(path), dev(n), kr, vr, st, pos_dev=dev(pos), phi=phi, layout=layout)
    for b in list(range(8)) + [B - 2, B - 1]:
        ref = D.commit(np64(s.k[b]), np64(s.v[b]), path[b], n[b], np64(s.k_ring[b]), np64(s.v_ring[b]), np64(s.state[b]), pos[b], phi)
        assert np.array_equal(np64(kr[b]), ref[0]) and np.array_equal(np64(vr[b]), ref[1]), b
        # n sums rounded to half a step, 2^-24 of an entry each, and n terms that three fp32 operations and exp (2 ulp, 2^-22) have formed: 2^-20
        top = max(1.0, np.abs(ref[2]).max(), np.abs(np64(s.state[b])).max())
        assert np.abs(np64(st[b]) - ref[2]).max() <= n[b] * (2.0 ** -24 * top + 2.0 ** -20), b


@pytest.mark.parametrize("phi", [O.PHI_SOFTMAX, O.PHI_IDENTITY])
@pytest.mark.parametrize("Hq,d,dtype,N,w,kind", [
    (16, 64, "f32", 13, 33, "padded"),                   # 26 rows a head: a block of 16 and a part of one
    (8, 64, "bf16", 9, 100, "tree"),
    (24, 128, "f32", 11, 5, "chain"),                    # paths longer than the window
    (8, 128, "f32", 16, 64, "star"),
])
def test_portable_attention_with_four_rows_to_a_warp(Hq, d, dtype, N, w, kind, phi):
    """More CTAs of one row to a warp than run at once, each entry at a position of its own; rows against the oracle, for some
    entries."""
    B, Hkv = 80, 8
    pos = np.random.default_rng(N).integers(0, 3 * w, B)
    pos[0], pos[1], pos[-1] = 0, w, 3 * w
    s = Setup(B, Hq, Hkv, N, d, w, dtype, pos.tolist(), kind, phi=phi, seed=N)
    gs, gr = s.gains64()
    for layout in (R.LAYOUT_BHTD, R.LAYOUT_BTHD):
        y = np64(s.run(layout=layout))
        for b in (0, 1, 2, B - 1):
            ref = D.draft_attention(np64(s.q[b]), np64(s.k[b]), np64(s.v[b]), s.parents[b], np64(s.hist[b][0]), np64(s.hist[b][1]), w,
                                    s.scale, gs=gs, gr=gr, phi=phi)
            rows = ~np.isnan(ref)
            assert (y[b][~rows] == 7.0).all()
            # fp32 arithmetic: the framework's bound for fp32 outputs, 1e-4, and the rounding of the output
            bound = 1e-4 + (2.0 ** -8 if dtype == "bf16" else 0.0) * np.abs(ref[rows])
            assert (np.abs(y[b][rows] - ref[rows]) <= bound).all(), b


@pytest.mark.parametrize("heads", [14, 15, 16, 18, 32, 33, 34, 37, 38, 73, 74, 75, 80])
def test_attention_around_the_cluster_sizes(heads):
    """As many heads as clusters of eight, four, two CTAs run at once, and one more: the same rows as the portable kernel's."""
    B, G, N, d, w, pos = heads, 4, 6, 128, 320, 1000
    g = torch.Generator(device="cuda").manual_seed(heads)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    q, k, v, kr, vr = (rnd(*s).bfloat16() for s in ((B, G, N, d), (B, 1, N, d), (B, 1, N, d), (B, 1, w, d), (B, 1, w, d)))
    state = 5 * rnd(B, 1, d, d)
    par = torch.tensor([[-1, 0, 0, 1, 3, 2]] * B, dtype=torch.int32, device="cuda")
    a, b = (R.rattn_draft_attention(q, k, v, par, kr, vr, state, pos, scale=d ** -0.5, flags=f).float() for f in (0, R.FLAG_FORCE_GENERIC))
    assert R.rattn_draft_status() == 0
    # each rounds an output once, to 2^-8 of it at most, from values that are 2^-10 apart at most
    assert ((a - b).abs() <= 2 * (2.0 ** -8 * b.abs() + 2.0 ** -10)).all()


@pytest.mark.parametrize("heads", [141, 142, 143, 147, 148, 149, 300])
def test_commit_around_the_cluster_sizes(heads):
    """Tokens are added in order whatever shares a head: the bits of the same entries in calls of a few."""
    B, N, d, w, pos = heads, 12, 128, 8, 50
    g = torch.Generator(device="cuda").manual_seed(heads)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    k, v, kr, vr = (rnd(*s).bfloat16() for s in ((B, 1, N, d), (B, 1, N, d), (B, 1, w, d), (B, 1, w, d)))
    state = rnd(B, 1, d, d)
    path = torch.stack([torch.randperm(N, device="cuda", generator=g) for _ in range(B)]).int()
    n = torch.randint(0, N + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
    whole, parts = [kr.clone(), vr.clone(), state.clone()], [kr.clone(), vr.clone(), state.clone()]
    R.rattn_draft_commit(k, v, path, n, *whole, pos)
    for i in range(0, B, 50):
        at = slice(i, i + 50)
        R.rattn_draft_commit(k[at], v[at], path[at], n[at], *(x[at] for x in parts), pos)
    assert all(torch.equal(a, b) for a, b in zip(whole, parts))
    assert not torch.equal(whole[2], state)
