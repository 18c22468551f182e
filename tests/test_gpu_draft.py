"""Speculative decoding on the GPU against the fp64 oracle: attention of a tree of drafts (which the oracle evaluates on each
node's whole sequence, without ring, state or tree mask), verification, commit, and a run of them together.

Tolerances.  The arithmetic is fp32, or 16-bit products of operands that are split so that 16 bits of every weight are
kept.  fp32: a score is a sum of d products of unit-norm rows, off by at most d 2^-24 |q||k| scale <= 128 * 2^-24 * 11.3 =
9e-5 and typically by its square root; the framework's bound for fp32 outputs, 1e-4, holds that.  bf16: the output's own
rounding, half a step, 2^-8 |y|, and 2^-9 times the size of a branch (a row of unit rms: |y| <= 4 nearly always) over the
root of the number of terms that the 2^-9 roundings of phi(q), phi(k) and of 16-bit weights average over, for which
2^-10 absolute is allowed.  (The kernels keep 16 bits of each of these, and the window's output waits in fixed point, off by
1.7e-4 times its gain of up to 1.4: together a third of that.)  State after a commit: fp32 sums of n terms, n 2^-23 of the largest entry."""
import math

import numpy as np
import pytest
import torch

from oracle import draft_oracle as D
from oracle import rattn_oracle as O
from paper_2506_15545_b200 import binding as R
from test_gpu_parity import np64

pytestmark = pytest.mark.gpu


def tree(N, kind, rng):
    if kind == "chain":
        return np.arange(N) - 1
    if kind == "star":
        return np.array([-1] + [0] * (N - 1))
    if kind == "roots":
        return np.full(N, -1)
    par = [-1]
    for i in range(1, N):
        par.append(int(rng.integers(max(-1, i - 9), i)))
    par = np.array(par)
    if kind == "padded":                               # an unused tail, one unused node inside, and what hangs from it
        par[N - max(1, N // 4):] = -2
        if N > 4:
            par[N // 2] = -2
    return par


class Setup:
    def __init__(self, B, Hq, Hkv, N, d, w, dtype, pos, kind, phi=O.PHI_SOFTMAX, seed=0, gains=True, fill=math.nan):
        rng = np.random.default_rng(1000 + seed)
        t = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.t, self.dtype, self.w, self.phi, self.d = t, dtype, w, phi, d
        self.scale = 1.0 / math.sqrt(d)
        round_ = lambda x: torch.tensor(x, dtype=torch.float32).to(t)  # noqa: E731
        unit = lambda x: x / np.sqrt((x * x).mean(-1, keepdims=True))  # noqa: E731
        self.pos = list(pos) if not isinstance(pos, int) else [pos] * B
        self.q = round_(unit(rng.standard_normal((B, Hq, N, d))))
        self.k = round_(unit(rng.standard_normal((B, Hkv, N, d))))
        self.v = round_(rng.standard_normal((B, Hkv, N, d)))
        self.hist = [[round_(f(rng.standard_normal((Hkv, p, d)))) for f in (unit, lambda x: x)] for p in self.pos]
        self.parents = np.stack([tree(N, kind, rng) for _ in range(B)])
        self.gs, self.gr = (1.0 + 0.1 * rng.standard_normal((Hq, d)) for _ in range(2)) if gains else (None, None)
        caches = [D.cache_of(np64(k), np64(v), w, phi, fill) for k, v in self.hist]
        self.k_ring, self.v_ring = (torch.tensor(np.stack([c[i] for c in caches]), dtype=torch.float32).to(t).cuda() for i in (0, 1))
        self.state = torch.tensor(np.stack([c[2] for c in caches]), dtype=torch.float32).cuda()

    def gain(self, g):
        return None if g is None else torch.tensor(g, dtype=torch.float32).cuda()

    def gains64(self):
        return [None if g is None else np64(torch.tensor(g, dtype=torch.float32)) for g in (self.gs, self.gr)]

    def run(self, layout=R.LAYOUT_BHTD, flags=0, per_entry=True, out=None, **kw):
        lay = (lambda x: x.transpose(1, 2).contiguous()) if layout == R.LAYOUT_BTHD else (lambda x: x)
        q, k, v = (lay(x).cuda() for x in (self.q, self.k, self.v))
        out = torch.full_like(q, 7.0) if out is None else out
        pos_dev = torch.tensor(self.pos, dtype=torch.int32, device="cuda") if per_entry else None
        y = R.rattn_draft_attention(q, k, v, torch.tensor(self.parents, dtype=torch.int32, device="cuda"), self.k_ring,
                                    self.v_ring, self.state, 0 if per_entry else self.pos[0], scale=self.scale,
                                    gamma_swa=self.gain(self.gs), gamma_rla=self.gain(self.gr), out=out, phi=self.phi,
                                    pos_dev=pos_dev, layout=layout, flags=flags, **kw)
        torch.cuda.synchronize()
        assert R.rattn_draft_status() == 0
        return y.transpose(1, 2) if layout == R.LAYOUT_BTHD else y

    def reference(self):
        gs, gr = self.gains64()
        return np.stack([D.draft_attention(np64(self.q[b]), np64(self.k[b]), np64(self.v[b]), self.parents[b], np64(h[0]),
                                           np64(h[1]), self.w, self.scale, gs=gs, gr=gr, phi=self.phi)
                         for b, h in enumerate(self.hist)])


def check(y, ref, dtype, what=""):
    y = np64(y)
    rows = ~np.isnan(ref)
    assert (y[~rows] == 7.0).all(), (what, "rows of no node were written")
    err = np.abs(y - ref)[rows]
    assert np.isfinite(y[rows]).all(), what
    bound = (2.0 ** -8 * np.abs(ref) + 2.0 ** -10 if dtype == "bf16" else np.full_like(ref, 1e-4))[rows]
    assert (err <= bound).all(), (what, float(err.max()), float((err / bound).max()))


CASES = [
    # B, Hq, Hkv, N, d, w, dtype, pos, tree
    (1, 1, 1, 1, 128, 64, "bf16", 0, "chain"),                 # one token, empty cache
    (2, 4, 2, 1, 128, 128, "bf16", (1, 300), "chain"),         # one token: a decode step
    (2, 8, 2, 6, 128, 64, "bf16", (200, 64), "chain"),         # exactly a window; more
    (3, 4, 4, 7, 128, 100, "bf16", (99, 101, 3), "tree"),      # odd window, around it
    (2, 4, 1, 13, 128, 5, "bf16", (4, 40), "chain"),           # deeper than the window: drafts leave it themselves
    (2, 2, 2, 33, 128, 1, "bf16", (0, 9), "chain"),            # a window of one
    (1, 8, 1, 40, 128, 192, "bf16", 500, "padded"),            # 320 rows of a K/V head
    (2, 5, 1, 48, 128, 130, "bf16", (130, 700), "padded"),     # 240 rows, a group that is no power of two
    (1, 3, 1, 128, 128, 160, "bf16", 170, "tree"),             # the most nodes
    (1, 2, 2, 128, 128, 64, "bf16", 1000, "chain"),            # the deepest tree, twice the window
    (1, 2, 1, 128, 128, 129, "bf16", 1, "chain"),              # a window that does not fill
    (2, 2, 1, 65, 128, 300, "bf16", (290, 310), "roots"),      # many first tokens
    (1, 40, 8, 9, 128, 256, "bf16", 555, "star"),              # the 12B layer's heads
    (1, 64, 1, 5, 128, 70, "bf16", 77, "tree"),                # a group of 64
    (2, 4, 2, 12, 64, 33, "bf16", (20, 90), "padded"),         # heads of 64
    (2, 4, 2, 12, 64, 33, "f32", (20, 90), "padded"),
    (1, 2, 2, 30, 128, 17, "f32", 100, "tree"),
]


@pytest.mark.parametrize("flags", [0, R.FLAG_FORCE_GENERIC])
@pytest.mark.parametrize("case", CASES)
def test_attention(case, flags):
    s = Setup(*case)
    ref = s.reference()
    check(s.run(flags=flags), ref, s.dtype, "heads outside")
    check(s.run(flags=flags, layout=R.LAYOUT_BTHD), ref, s.dtype, "heads inside")


@pytest.mark.parametrize("phi", [O.PHI_RELU, O.PHI_IDENTITY])
@pytest.mark.parametrize("case", [CASES[2], CASES[4], CASES[7], CASES[15]])
def test_attention_other_feature_maps(case, phi):
    s = Setup(*case, phi=phi, gains=False)
    ref = s.reference()
    y = np64(s.run())
    rows = ~np.isnan(ref)
    # signed sums cancel: an element-wise map's products are rounded to 2^-9 of terms larger than their sum, so the bound
    # is the framework's for the linear branch with these maps, 2e-2 absolute (fp32: 1e-4)
    bound = 2.0 ** -8 * np.abs(ref) + (2e-2 if s.dtype == "bf16" else 1e-4)
    assert (np.abs(y - ref)[rows] <= bound[rows]).all()


def test_one_position_for_all_and_one_per_entry_agree():
    s = Setup(2, 4, 2, 9, 128, 64, "bf16", 150, "tree")
    assert torch.equal(s.run(per_entry=False), s.run(per_entry=True))


@pytest.mark.parametrize("flags", [0, R.FLAG_FORCE_GENERIC])
@pytest.mark.parametrize("N,Hq,what", [(9, 4, "inf"), (9, 4, "nan"), (70, 4, "inf"), (70, 4, "nan")])
def test_a_node_that_is_not_finite_reaches_its_descendants_only(N, Hq, what, flags):
    s = Setup(1, Hq, 1, N, 128, 64, "bf16", 100, "tree", seed=4)
    bad = 3
    s.k[0, 0, bad, 5] = s.v[0, 0, bad, 7] = float(what)
    y = np64(s.run(flags=flags))
    ref = s.reference()
    under = np.array([bad in (D.path_of(s.parents[0], i) or []) for i in range(N)])
    assert under.any() and not under.all()
    err = np.abs(y - ref)[0][:, ~under]
    assert np.isfinite(y[0][:, ~under]).all()
    assert (err <= 2.0 ** -8 * np.abs(ref[0][:, ~under]) + 2.0 ** -10).all()
    assert np.isnan(y[0][:, under][:, :, 7]).all()


def test_large_values_are_taken_as_they_are():
    """|v| up to 1e30 (fp16 would not hold it): both norms cancel a common factor."""
    a = Setup(1, 4, 1, 40, 128, 64, "bf16", 200, "tree", seed=6)
    b = Setup(1, 4, 1, 40, 128, 64, "bf16", 200, "tree", seed=6)
    f = 2.0 ** 40
    b.v = b.v * f
    b.hist = [[k, v * f] for k, v in b.hist]
    b.v_ring, b.state = b.v_ring * f, b.state * f
    ref = b.reference()
    check(b.run(), ref, "bf16")
    assert np.abs(np64(a.run()) - np64(b.run())).max() <= 2.0 ** -6 * 4


def test_large_logits_and_the_same_result_twice():
    s = Setup(2, 8, 2, 20, 128, 200, "bf16", (150, 600), "tree", seed=7)
    s.scale = 40.0
    y = s.run()
    assert torch.equal(y, s.run())
    ref = s.reference()
    # a logit of size 40 * 128 is off by 128 * 2^-24 of it in fp32: 4e-2 in the exponent where weights are shared
    rows = ~np.isnan(ref)
    assert (np.abs(np64(y) - ref)[rows] <= 2.0 ** -8 * np.abs(ref[rows]) + 0.2).all()


def test_cache_is_left_alone_and_garbage_parents_are_no_nodes():
    s = Setup(2, 4, 2, 8, 128, 64, "bf16", (30, 90), "chain", seed=8)
    s.parents[0] = [-1, 0, 5, 1, -7, 2 ** 30, 6, -2 ** 31]       # a parent behind its child, none, itself
    s.parents[1] = [0, -1, 1, 2, 2, 127, 3, 8]
    before = [x.clone() for x in (s.k_ring, s.v_ring, s.state)]
    y = s.run()
    check(y, s.reference(), "bf16")
    assert all(torch.equal(a.nan_to_num(3.0), b.nan_to_num(3.0)) for a, b in zip(before, (s.k_ring, s.v_ring, s.state)))


def test_large_cache_offsets():
    """Rings of more than 2^32 bytes: the last entry's slots lie beyond 32-bit offsets."""
    B, Hkv, w, d, N = 5, 8, 1 << 19, 128, 3                      # 5 * 8 * 2^19 * 128 * 2 bytes = 5.4 GB a ring
    g = torch.Generator(device="cuda").manual_seed(9)
    kr = torch.zeros(B, Hkv, w, d, device="cuda", dtype=torch.bfloat16)
    vr = torch.zeros_like(kr)
    pos = [700] * B
    kr[:, :, :700] = torch.randn(B, Hkv, 700, d, device="cuda", generator=g).bfloat16()
    vr[:, :, :700] = torch.randn(B, Hkv, 700, d, device="cuda", generator=g).bfloat16()
    q, k, v = (torch.randn(B, Hkv, N, d, device="cuda", generator=g).bfloat16() for _ in range(3))
    state = torch.zeros(B, Hkv, d, d, device="cuda")
    par = torch.tensor([[-1, 0, 1]] * B, dtype=torch.int32, device="cuda")
    b = B - 1
    ref = D.draft_attention(np64(q[b]), np64(k[b]), np64(v[b]), [-1, 0, 1], np64(kr[b, :, :700]), np64(vr[b, :, :700]), w, 0.1)
    for flags in (0, R.FLAG_FORCE_GENERIC):
        y = R.rattn_draft_attention(q, k, v, par, kr, vr, state, pos[0], scale=0.1, flags=flags)
        err = np.abs(np64(y[b]) - ref)
        assert (err <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -10).all()
    R.rattn_draft_commit(k, v, par.clamp(min=0), torch.full((B,), 2, dtype=torch.int32, device="cuda"), kr, vr, state, 700)
    assert torch.equal(kr[b, :, 700], k[b, :, 0]) and torch.equal(vr[b, :, 701], v[b, :, 0])


# ---------------------------------------------------------------------------- commit

@pytest.mark.parametrize("phi", [O.PHI_SOFTMAX, O.PHI_RELU])
@pytest.mark.parametrize("B,Hkv,N,d,w,dtype,pos,n", [
    (3, 2, 6, 128, 64, "bf16", (200, 63, 0), (3, 6, 6)),
    (4, 2, 9, 64, 5, "f32", (3, 40, 5, 4), (9, 8, 0, 1)),         # more accepted tokens than slots
    (2, 1, 128, 128, 100, "bf16", (99, 1000), (128, 57)),
    (2, 3, 40, 128, 1, "f32", (0, 7), (40, 2)),
    (2, 3, 1, 128, 33, "bf16", (33, 34), (1, 0)),
])
def test_commit(B, Hkv, N, d, w, dtype, pos, n, phi):
    s = Setup(B, Hkv, Hkv, N, d, w, dtype, pos, "chain", phi=phi, seed=N, fill=0.0)
    rng = np.random.default_rng(N)
    path = np.stack([rng.permutation(N) for _ in range(B)])
    if N > 2:
        path[0, 1] = path[0, 0]                                  # the same node twice
    for b in range(B):
        path[b, n[b]:] = -1
    ref = [D.commit(np64(s.k[b]), np64(s.v[b]), path[b], n[b], np64(s.k_ring[b]), np64(s.v_ring[b]), np64(s.state[b]), pos[b], phi)
           for b in range(B)]
    dev = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    for layout in (R.LAYOUT_BHTD, R.LAYOUT_BTHD):
        lay = (lambda x: x.transpose(1, 2).contiguous()) if layout == R.LAYOUT_BTHD else (lambda x: x)
        kr, vr, st = s.k_ring.clone(), s.v_ring.clone(), s.state.clone()
        R.rattn_draft_commit(lay(s.k).cuda(), lay(s.v).cuda(), dev(path), dev(n), kr, vr, st, pos_dev=dev(pos), phi=phi, layout=layout)
        torch.cuda.synchronize()
        for b in range(B):
            assert np.array_equal(np64(kr[b]), ref[b][0]) and np.array_equal(np64(vr[b]), ref[b][1]), b
            err = np.abs(np64(st[b]) - ref[b][2]).max()
            assert err <= (n[b] + 1) * 2.0 ** -23 * max(1.0, np.abs(ref[b][2]).max()) + n[b] * 2.0 ** -20, (b, err)


def test_commit_ends_at_a_bad_path_entry_and_clips_counts():
    s = Setup(3, 2, 2, 5, 128, 64, "bf16", 100, "chain", seed=3)
    path = torch.tensor([[0, 1, 9, 2, 3], [0, -1, 2, 3, 4], [4, 3, 2, 1, 0]], dtype=torch.int32, device="cuda")
    good = torch.tensor([2, 1, 5], dtype=torch.int32, device="cuda")
    wild = torch.tensor([5, 2 ** 31 - 1, 77], dtype=torch.int32, device="cuda")
    out = []
    for n in (good, wild):
        kr, vr, st = s.k_ring.clone(), s.v_ring.clone(), s.state.clone()
        R.rattn_draft_commit(s.k.cuda(), s.v.cuda(), path, n, kr, vr, st, 100)
        out.append((kr, vr, st))
    assert all(torch.equal(a, b) for a, b in zip(*out))
    before = [x.clone() for x in out[0]]
    R.rattn_draft_commit(s.k.cuda(), s.v.cuda(), path, -wild, *out[0], 100)       # nothing accepted
    assert all(torch.equal(a, b) for a, b in zip(before, out[0]))


def test_commit_is_that_many_decode_steps():
    B, H, N, w, d, pos = 2, 2, 7, 64, 128, 90
    s = Setup(B, H, H, N, d, w, "bf16", pos, "chain", seed=11)
    kr, vr, st = s.k_ring.clone(), s.v_ring.clone(), s.state.clone()
    k2, v2, s2 = s.k_ring.clone(), s.v_ring.clone(), s.state.clone()
    y = s.run()
    steps = [R.rattn_decode_step_ex(s.q[:, :, i].contiguous().cuda(), s.k[:, :, i].contiguous().cuda(), s.v[:, :, i].contiguous().cuda(),
                                    kr, vr, st, pos + i, scale=s.scale, gamma_swa=s.gain(s.gs), gamma_rla=s.gain(s.gr)) for i in range(N)]
    path = torch.arange(N, dtype=torch.int32, device="cuda").repeat(B, 1)
    R.rattn_draft_commit(s.k.cuda(), s.v.cuda(), path, torch.full((B,), N, dtype=torch.int32, device="cuda"), k2, v2, s2, pos)
    assert torch.equal(kr, k2) and torch.equal(vr, v2)
    assert (st - s2).abs().max() <= N * 2.0 ** -20 * max(1.0, float(st.abs().max()))
    # both round an output once, to 2^-8 of it at most, from values that are 2^-10 apart at most
    a, b = torch.stack(steps, 2).float(), y.float()
    assert ((a - b).abs() <= 2 * (2.0 ** -8 * a.abs() + 2.0 ** -10)).all()


# ---------------------------------------------------------------------------- verification

def _rows(B, N, V, seed, dtype, sharp=1.0, near=0.7):
    g = torch.Generator().manual_seed(seed)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    x = sharp * torch.randn(B, N, V, generator=g)
    y = x + near * torch.randn(B, N, V, generator=g)
    p, q = torch.softmax(x, -1).to(t), torch.softmax(y, -1).to(t)
    return p, q, torch.rand(B, N, generator=g), g


@pytest.mark.parametrize("draft", [True, False])
@pytest.mark.parametrize("B,N,V,dtype,kind,sharp", [
    (2, 1, 1, "f32", "chain", 1.0),                     # one node, one token
    (3, 6, 7, "f32", "chain", 1.0),
    (4, 8, 100, "bf16", "tree", 2.0),
    (5, 12, 1001, "f32", "star", 1.0),                  # many rejections in one row
    (3, 128, 37, "f32", "tree", 3.0),
    (6, 20, 333, "bf16", "padded", 3.0),
    (2, 5, 40009, "f32", "star", 2.0),
])
def test_verify(B, N, V, dtype, kind, sharp, draft):
    p, q, u, g = _rows(B, N, V, N + V, dtype, sharp)
    rng = np.random.default_rng(N * V)
    parents = np.stack([tree(N, kind, rng) for _ in range(B)])
    tokens = torch.zeros(B, N, dtype=torch.int32)
    for b in range(B):
        for i in range(N):
            row = (q if draft else p)[b, max(0, parents[b][i])].double()
            tokens[b, i] = int(torch.multinomial(row, 1, generator=g))
    if N > 5:
        parents[-1][0] = -2                              # an idle entry
        tokens[0, 2], tokens[0, 3] = -1, V               # no tokens
    path, n, token = R.rattn_draft_verify(tokens.cuda(), torch.tensor(parents, dtype=torch.int32).cuda(), p.cuda(),
                                          q.cuda() if draft else None, u.cuda())
    torch.cuda.synchronize()
    assert R.rattn_draft_status() == 0
    for b in range(B):
        line, x = D.verify(tokens[b].tolist(), parents[b].tolist(), np64(p[b]), np64(q[b]) if draft else None, np64(u[b]))
        assert n[b].item() == len(line) and path[b].tolist() == line + [-1] * (N - len(line)), b
        assert token[b].item() == x, b


def test_verify_in_exact_arithmetic():
    """Probabilities that are sums of powers of two and u on their borders: products and sums are exact in fp64, and the result
    is that of rational arithmetic (ties: u q Z = r is a rejection, a sum equal to the target is passed over)."""
    V, N = 8, 6
    rng = np.random.default_rng(3)
    for trial in range(40):
        p, q = ([[x / 16 for x in rng.multinomial(16, [1 / V] * V)] for _ in range(N)] for _ in range(2))
        parents = tree(N, "tree" if trial % 2 else "star", rng)
        tokens = rng.integers(0, V, N).tolist()
        u = (rng.integers(0, 16, N) / 16).tolist()
        for drafts in (q, None):
            ref = D.verify(tokens, parents.tolist(), [D.rational(r) for r in p], None if drafts is None else [D.rational(r) for r in drafts],
                           D.rational(u))
            t = lambda x, dt: torch.tensor(np.array(x)[None], dtype=dt, device="cuda")  # noqa: E731
            path, n, token = R.rattn_draft_verify(t(tokens, torch.int32), t(parents, torch.int32), t(p, torch.float32),
                                                  None if drafts is None else t(drafts, torch.float32), t(u, torch.float32))
            assert (path[0, :n[0]].tolist(), token.item()) == ref, trial


def test_verify_rows_that_hold_garbage():
    """NaN and negative probabilities count as 0, rows that nothing asks for are not read, an empty row gives -1, u = 1 or
    NaN the last token that has any weight."""
    V = 300
    p = torch.zeros(4, 3, V)
    p[:, 0, 10:14] = torch.tensor([0.5, math.nan, -1.0, 0.5])
    p[:, 1:] = math.nan
    p[2, 0] = 0.0
    tokens = torch.tensor([[0, 11, 12]] * 4, dtype=torch.int32)
    par = torch.tensor([[-1, 0, 0]] * 4, dtype=torch.int32)
    u = torch.tensor([[0.6, 0.0, 0.0], [1.0, 0.0, 0.0], [0.3, 0.0, 0.0], [math.nan, 0.0, 0.0]])
    for q in (None, p.clone()):
        path, n, token = R.rattn_draft_verify(tokens.cuda(), par.cuda(), p.cuda(), None if q is None else q.cuda(), u.cuda())
        assert n.tolist() == [1] * 4 and token.tolist() == [13, 13, -1, 13]
        assert path.tolist() == [[0, -1, -1]] * 4


# ---------------------------------------------------------------------------- together, and around

def test_speculative_steps_follow_plain_decoding():
    """A layer serving two sequences through prologue, draft attention, verification and commit, with drafts that are right or wrong
    at random: the rows of the accepted nodes are those of decoding token by token, and so are ring and state at the end."""
    B, Hq, Hkv, d, w, V, N = 2, 4, 2, 128, 64, 50, 6
    g = torch.Generator(device="cuda").manual_seed(21)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    table = rnd(3, V, (Hq + 2 * Hkv) * d)[0].bfloat16()           # a token's projections
    def project(tok, at):                                          # tok, at [B, n]
        x = table[tok.long()].view(*tok.shape, Hq + 2 * Hkv, d)
        q, k, v = (y.contiguous() for y in x.split([Hq, Hkv, Hkv], 2))
        q, k = R.rattn_qk_prologue_axes(q, k, at[None].contiguous(), [d // 2], layout=R.LAYOUT_BTHD)
        return q, k, v
    T0 = 70
    prompt = torch.randint(0, V, (B, T0), device="cuda", generator=g, dtype=torch.int32)
    q, k, v = project(prompt, torch.arange(T0, device="cuda", dtype=torch.int32).repeat(B, 1))
    state = torch.zeros(B, Hkv, d, d, device="cuda")
    kr, vr = (torch.zeros(B, Hkv, w, d, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    R.rattn_forward_ex(q, k, v, w, scale=0.09, state_out=state, k_ring_out=kr, v_ring_out=vr, layout=R.LAYOUT_BTHD,
                       workspace=R.alloc_workspace(q, k, w, layout=R.LAYOUT_BTHD))
    plain = [x.clone() for x in (kr, vr, state)]
    pos = torch.full((B,), T0, device="cuda", dtype=torch.int32)
    last = torch.randint(0, V, (B,), device="cuda", generator=g, dtype=torch.int32)
    parents = torch.tensor([[-1, 0, 0, 1, 2, 4]] * B, dtype=torch.int32, device="cuda")
    depth = torch.tensor([0, 1, 1, 2, 2, 3], device="cuda", dtype=torch.int32)
    seqs = [[] for _ in range(B)]
    for step in range(8):
        tokens = torch.randint(0, V, (B, N), device="cuda", generator=g, dtype=torch.int32)
        tokens[:, 0] = last
        q, k, v = project(tokens, pos[:, None] + depth)
        y = R.rattn_draft_attention(q, k, v, parents, kr, vr, state, scale=0.09, pos_dev=pos, layout=R.LAYOUT_BTHD)
        probs = torch.softmax(y.float().mean(2)[..., :V] * 3, -1)
        path, n, new = R.rattn_draft_verify(tokens, parents, probs, torch.full_like(probs, 1.0 / V), torch.rand(B, N, device="cuda", generator=g))
        R.rattn_draft_commit(k, v, path, n, kr, vr, state, pos_dev=pos, layout=R.LAYOUT_BTHD)
        for b in range(B):
            for a in range(n[b].item()):
                i = path[b, a].item()
                seqs[b].append((tokens[b, i].item(), y[b, i].float()))
        pos, last = pos + n, new
    for b in range(B):
        cache = [x[b:b + 1].clone() for x in plain]
        for a, (tok, row) in enumerate(seqs[b]):
            at = torch.tensor([[T0 + a]], device="cuda", dtype=torch.int32)
            q, k, v = (x[:, 0].contiguous() for x in project(torch.tensor([[tok]], device="cuda"), at))
            want = R.rattn_decode_step_ex(q, k, v, *cache, T0 + a, scale=0.09)[0].float()
            assert ((want - row).abs() <= 2 * (2.0 ** -8 * want.abs() + 2.0 ** -9)).all(), (b, a)
        assert torch.equal(cache[0][0], kr[b]) and torch.equal(cache[1][0], vr[b])
        assert (cache[2][0] - state[b]).abs().max() <= 2.0 ** -16 * max(1.0, float(state[b].abs().max()))
    assert max(len(s) for s in seqs) > 8


def test_captured_and_replayed_on_another_stream():
    s = Setup(2, 4, 2, 40, 128, 64, "bf16", (150, 70), "tree", seed=13)
    q, k, v = (x.cuda() for x in (s.q, s.k, s.v))
    par, pos = torch.tensor(s.parents, dtype=torch.int32, device="cuda"), torch.tensor(s.pos, dtype=torch.int32, device="cuda")
    p, qq, u, g = _rows(2, 40, 500, 1, "f32")
    p, qq, u = p.cuda(), qq.cuda(), u.cuda()
    tok = torch.randint(0, 500, (2, 40), dtype=torch.int32, generator=g).cuda()
    kr, vr, st = s.k_ring.clone(), s.v_ring.clone(), s.state.clone()
    out = torch.zeros_like(q)

    def call(kr, vr, st):
        y = R.rattn_draft_attention(q, k, v, par, kr, vr, st, scale=s.scale, pos_dev=pos, out=out)
        path, n, token = R.rattn_draft_verify(tok, par, p, qq, u)
        R.rattn_draft_commit(k, v, path, n, kr, vr, st, pos_dev=pos)
        return [y, path, n, token, kr, vr, st]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [x.clone() for x in call(s.k_ring.clone(), s.v_ring.clone(), s.state.clone())]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call(kr, vr, st)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a.nan_to_num(3.0), b.nan_to_num(3.0)) for a, b in zip(want, got))


def test_binding_checks_types_shapes_and_devices():
    s = Setup(1, 4, 2, 3, 64, 8, "f32", 9, "chain")
    q, k, v = (x.cuda() for x in (s.q, s.k, s.v))
    par = torch.tensor(s.parents, dtype=torch.int32, device="cuda")
    good = dict(q=q, k=k, v=v, parents=par, k_ring=s.k_ring, v_ring=s.v_ring, state=s.state)
    for name, bad, err in (("parents", par.long(), TypeError), ("parents", par[:, :2].contiguous(), ValueError), ("q", q.bfloat16(), TypeError),
                           ("v", v[:, :, :2].contiguous(), ValueError), ("v_ring", s.v_ring[:, :, :4].contiguous(), ValueError),
                           ("state", s.state.double(), TypeError), ("k", k.cpu(), ValueError), ("q", q[:, :, ::2], ValueError),
                           ("k", k.half(), TypeError)):
        with pytest.raises(err):
            R.rattn_draft_attention(**{**good, name: bad}, pos=9)
    with pytest.raises(ValueError):
        R.rattn_draft_attention(**good, pos=9, out=q[:, :, :2].contiguous())
    with pytest.raises(R.RattnError):
        R.rattn_draft_attention(**good, pos=-1)
    path = torch.zeros(1, 3, dtype=torch.int32, device="cuda")
    with pytest.raises(TypeError):
        R.rattn_draft_commit(k, v, path, path[0, :1].long(), s.k_ring, s.v_ring, s.state)
    p = torch.ones(1, 3, 5, device="cuda")
    with pytest.raises(TypeError):
        R.rattn_draft_verify(path, path, p, p.bfloat16(), torch.zeros(1, 3, device="cuda"))
    with pytest.raises(ValueError):
        R.rattn_draft_verify(path, path, p, p[:, :2].contiguous(), torch.zeros(1, 3, device="cuda"))


@pytest.mark.parametrize("B,Hq,Hkv,N,w,top,kind,layout", [
    (1, 8, 2, 11, 1000, 5000, "tree", R.LAYOUT_BHTD),         # clusters of eight CTAs, several tiles of keys each
    (4, 16, 8, 20, 700, 2100, "padded", R.LAYOUT_BTHD),       # of four
    (9, 8, 8, 6, 1500, 3000, "chain", R.LAYOUT_BHTD),         # of two, many tiles each
    (25, 32, 8, 20, 448, 1500, "padded", R.LAYOUT_BTHD),      # a CTA per head, more than run at once
    (19, 40, 8, 64, 640, 1300, "tree", R.LAYOUT_BHTD),        # 320 rows a head: three row tiles, two waves
    (20, 8, 8, 100, 576, 600, "chain", R.LAYOUT_BTHD),        # a hundred levels
])
def test_attention_of_a_batch(B, Hq, Hkv, N, w, top, kind, layout):
    """Sizes at which CTAs walk many tiles and share keys in every way, each entry at a position of its own: the oracle on two
    entries, the portable kernel on all."""
    g = torch.Generator(device="cuda").manual_seed(N)
    rng = np.random.default_rng(N)
    d, G = 128, Hq // Hkv
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    unit = lambda x: x / x.square().mean(-1, keepdim=True).sqrt()  # noqa: E731
    pos = rng.integers(1, top, B)
    pos[0], pos[-1] = min(w + 5, top), top
    hist = {b: [unit(rnd(Hkv, int(pos[b]), d)).bfloat16(), rnd(Hkv, int(pos[b]), d).bfloat16()] for b in range(B)}
    kr, vr = (torch.full((B, Hkv, w, d), math.nan, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    state = torch.zeros(B, Hkv, d, d, device="cuda")
    for b in range(B):
        p = int(pos[b])
        slots = torch.arange(max(0, p - w), p, device="cuda") % w
        for r, x in zip((kr, vr), hist[b]):
            r[b][:, slots] = x[:, max(0, p - w):]
        k, v = (x[:, :max(0, p - w)].double() for x in hist[b])
        state[b] = (torch.softmax(k, -1).transpose(1, 2) @ v).float()
    q, k, v = unit(rnd(B, Hq, N, d)).bfloat16(), unit(rnd(B, Hkv, N, d)).bfloat16(), rnd(B, Hkv, N, d).bfloat16()
    parents = np.stack([tree(N, kind, rng) for _ in range(B)])
    gs, gr = 1 + 0.1 * rnd(Hq, d), 1 + 0.1 * rnd(Hq, d)
    lay = (lambda x: x.transpose(1, 2).contiguous()) if layout == R.LAYOUT_BTHD else (lambda x: x)
    out = []
    for flags in (0, R.FLAG_FORCE_GENERIC, 0):
        y = R.rattn_draft_attention(lay(q), lay(k), lay(v), torch.tensor(parents, dtype=torch.int32, device="cuda"), kr, vr, state,
                                    scale=d ** -0.5, gamma_swa=gs, gamma_rla=gr, out=torch.full_like(lay(q), 7.0), layout=layout,
                                    flags=flags, pos_dev=torch.tensor(pos, dtype=torch.int32, device="cuda"))
        out.append(lay(y))
    torch.cuda.synchronize()
    assert R.rattn_draft_status() == 0
    assert torch.equal(out[0], out[2])                            # the same bits again
    a, b = out[0].float(), out[1].float()
    assert ((a - b).abs() <= 2 * (2.0 ** -8 * b.abs() + 2.0 ** -10)).all()
    for i in (0, B - 1):
        heads = [0, Hq - 1]
        hk = [h // G for h in heads]
        ref = D.draft_attention(np64(q[i][heads]), np64(k[i][hk]), np64(v[i][hk]), parents[i], np64(hist[i][0][hk]), np64(hist[i][1][hk]),
                                w, d ** -0.5, gs=np64(gs[heads]), gr=np64(gr[heads]))
        check(out[0][i][heads], ref, "bf16", i)


@pytest.mark.parametrize("Hq,Hkv,B", [(4, 2, 2), (8, 8, 40)])
@pytest.mark.parametrize("flags", [0, R.FLAG_FORCE_GENERIC])
def test_the_largest_positions(Hq, Hkv, B, flags):
    """A position matters by its remainder modulo w once the ring is full: the largest that are taken give the bits of a small one."""
    N, w = 20, 100
    s = Setup(B, Hq, Hkv, N, 128, w, "bf16", 2 * w + 47, "chain", seed=21)
    small = s.run(flags=flags)
    top = 2 ** 31 - 1 - w - R.DRAFT_MAX_NODES
    top -= (top - 47) % w
    s.pos = [top] * B
    assert torch.equal(small, s.run(flags=flags)) and torch.equal(small, s.run(flags=flags, per_entry=False))
    path = torch.arange(N, dtype=torch.int32, device="cuda").repeat(B, 1)
    n = torch.full((B,), N, dtype=torch.int32, device="cuda")
    caches = []
    for pos in (2 * w + 47, top):
        caches.append([s.k_ring.clone(), s.v_ring.clone(), s.state.clone()])
        R.rattn_draft_commit(s.k.cuda(), s.v.cuda(), path, n, *caches[-1], pos)
    assert all(torch.equal(a, b) for a, b in zip(*caches))
    with pytest.raises(ValueError):
        s.pos = [2 ** 32 + 47] * B
        s.run(flags=flags, per_entry=False)
    with pytest.raises(ValueError):
        R.rattn_draft_commit(s.k.cuda(), s.v.cuda(), path, n, *caches[0], 2 ** 32)


def test_two_calls_at_once():
    """Calls on two streams share nothing but what they read: the same bits as one after the other, all operators at work."""
    setups = [Setup(1, 8, 2, 6, 128, 512, "bf16", 700, "chain", seed=1), Setup(24, 8, 8, 30, 128, 192, "bf16", 300, "tree", seed=2)]
    jobs = []
    for s in setups:
        B, N = s.parents.shape
        p, q, u, g = _rows(B, N, 5003, B, "bf16", 2.0)
        jobs.append(dict(q=s.q.cuda(), k=s.k.cuda(), v=s.v.cuda(), par=torch.tensor(s.parents, dtype=torch.int32, device="cuda"),
                         p=p.cuda(), dq=q.cuda(), u=u.cuda(), tok=torch.randint(0, 5003, (B, N), generator=g, dtype=torch.int32).cuda(),
                         cache=[s.k_ring, s.v_ring, s.state], pos=s.pos[0], scale=s.scale))

    def step(j):
        path, n, token = R.rattn_draft_verify(j["tok"], j["par"], j["p"], j["dq"], j["u"])
        cache = [x.clone() for x in j["cache"]]
        y = R.rattn_draft_attention(j["q"], j["k"], j["v"], j["par"], *cache, j["pos"], scale=j["scale"])
        R.rattn_draft_commit(j["k"], j["v"], path, n, *cache, j["pos"])
        rows = torch.tensor([[D.path_of(par, i) is not None for i in range(len(par))] for par in j["par"].tolist()])
        return [path, n, token, y.transpose(1, 2)[rows.cuda()]] + cache

    want = [step(j) for j in jobs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in jobs]
    got = [[], []]
    for _ in range(10):
        for i, j in enumerate(jobs):
            with torch.cuda.stream(streams[i]):
                got[i].append(step(j))
    torch.cuda.synchronize()
    assert R.rattn_draft_status() == 0
    for w_, runs in zip(want, got):
        for r in runs:
            assert all(torch.equal(a, b) for a, b in zip(w_, r))


@pytest.mark.parametrize("how", [1, 2])
@pytest.mark.parametrize("B,Hkv,w,pos", [(1, 2, 256, 900), (40, 8, 256, 300), (9, 8, 1024, 2000), (20, 8, 1024, 2000)])
def test_a_wait_that_runs_out_is_reported(B, Hkv, w, pos, how):
    """In the debug build one arrival of the attention kernel never comes, or a wait counts as run out: the call ends, says so once,
    writes no row, and the next call on the same buffers is right (clusters of CTAs, of which one gives up, and single ones; more
    loads than slots, so that some are still to be asked for)."""
    import ctypes

    from paper_2506_15545_b200 import build
    L = ctypes.CDLL(build.build(debug=True))
    vp = ctypes.c_void_p
    L.rattn_draft_attention.argtypes = [ctypes.POINTER(R.RattnDraftParams), vp]
    L.rattn_draft_status.argtypes = [vp]
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g).bfloat16()  # noqa: E731
    N, d = 6, 128
    q, k, v, kr, vr = rnd(B, Hkv, N, d), rnd(B, Hkv, N, d), rnd(B, Hkv, N, d), rnd(B, Hkv, w, d), rnd(B, Hkv, w, d)
    state, out = torch.randn(B, Hkv, d, d, device="cuda", generator=g), torch.full_like(q, 7.0)
    par = torch.tensor([[-1, 0, 1, 1, 2, 0]] * B, dtype=torch.int32, device="cuda")
    p = R.RattnDraftParams()
    for f, t in (("q", q), ("k", k), ("v", v), ("out", out), ("parents", par), ("k_ring", kr), ("v_ring", vr), ("state", state)):
        setattr(p, f, t.data_ptr())
    p.B, p.H_q, p.H_kv, p.N, p.d, p.w, p.dtype, p.scale, p.eps, p.pos = B, Hkv, Hkv, N, d, w, R.RATTN_BF16, 0.1, 1e-6, pos
    stream = vp(torch.cuda.current_stream().cuda_stream)
    try:
        L.rattn_debug_withhold_arrival(how)
        assert L.rattn_draft_attention(ctypes.byref(p), stream) == 0
        assert L.rattn_draft_status(stream) == -7
        assert (out == 7.0).all()
    finally:
        L.rattn_debug_withhold_arrival(0)
    assert L.rattn_draft_status(stream) == 0
    assert L.rattn_draft_attention(ctypes.byref(p), stream) == 0 and L.rattn_draft_status(stream) == 0
    assert torch.equal(out, R.rattn_draft_attention(q, k, v, par, kr, vr, state, pos, scale=0.1))
