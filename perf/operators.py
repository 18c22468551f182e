"""Speculative decoding on the RAttention cache, and rotary positions with several axes, as measurable cases.

A pass is one call of a layer or of a server's step: attention of a tree of drafted tokens over the
ring and the state, the verification of that tree against the target's probabilities, the accepted
tokens' entry into the cache, and the prologue of tokens whose positions are not consecutive (tree
nodes, images, video).  Head shapes, windows and head sizes are those of the 3B and 12B layers that
the rest of the benchmark uses, and the small fp32 layer that numerics are checked on.
"""
import math

import torch

own = False

# ---- the cases --------------------------------------------------------------------------
# op "attention"  N nodes per sequence (a chain, or a tree of at most `deep` levels) at position `pos`
#                 (per_entry: each sequence at its own); padded: entries use fewer than N nodes
# op "verify"     N nodes, vocabulary V; draft "probs": the drafter's distributions are known,
#                 "none": the drafter took its tokens greedily
# op "commit"     the accepted path goes into ring and state
# op "axes"       the prologue with `axes` positions per token; direction "fwd" or "bwd" (with gains)


def listed():
    return [
        # one user's chat, a chain of five drafts behind the token sampled last: latency only
        _case("draft_chain_single", "attention", B=1, H_q=32, H_kv=8, N=6, w=512, pos=1777, deep=0),
        # a serving batch, a tree of 48 nodes per sequence, tensors as the projections leave them
        _case("draft_tree_batch", "attention", B=16, H_q=32, H_kv=8, N=48, w=512, pos=9000, deep=7, per_entry=True,
              padded=True, bthd=True),
        # a full server with wide trees and a long window
        _case("draft_tree_wide", "attention", B=32, H_q=32, H_kv=8, N=64, w=1024, pos=32768, deep=9, per_entry=True),
        # the small fp32 layer, sequences that have not filled a window of odd size
        _case("draft_fp32_odd", "attention", B=3, H_q=4, H_kv=2, N=13, w=100, pos=131, deep=4, d=64, dtype="f32",
              per_entry=True, padded=True),
        # one user's chain
        _case("verify_chain_single", "verify", B=1, N=6, V=32000, deep=0),
        # a serving batch's trees over a large vocabulary
        _case("verify_tree_batch", "verify", B=32, N=32, V=131072, deep=7, padded=True),
        # drafts taken greedily, probabilities in 16 bits, vocabulary of odd size
        _case("verify_greedy_odd", "verify", B=7, N=24, V=50257, deep=6, draft="none", dtype="bf16"),
        # one user's accepted chain
        _case("commit_single", "commit", B=1, H_q=32, H_kv=8, N=6, w=512, pos=1777, deep=0),
        # a serving batch's accepted paths
        _case("commit_batch", "commit", B=64, H_q=32, H_kv=8, N=48, w=512, pos=9000, deep=7, per_entry=True, bthd=True),
        # the prologue of a batch of trees: a node's position is its depth's
        _case("axes_tree_nodes", "axes", B=16, H_q=32, H_kv=8, T=48, axes=1, order="runs", bthd=True),
        # a video's tokens in a prompt: time, height and width
        _case("axes_video_prompt", "axes", B=2, H_q=32, H_kv=8, T=8191, axes=3, order="dealt"),
        # training on images: height and width with frequencies of their own
        _case("axes_image_train", "axes", B=4, H_q=16, H_kv=16, T=4096, axes=2, order="own", direction="bwd", bthd=True),
    ]


_DEFAULTS = {
    "attention": dict(d=128, dtype="bf16", per_entry=False, padded=False, bthd=False),
    "verify": dict(dtype="f32", draft="probs", padded=False),
    "commit": dict(d=128, dtype="bf16", per_entry=False, padded=False, bthd=False),
    "axes": dict(d=128, dtype="bf16", direction="fwd", bthd=False),
}


def _case(name, op, **sizes):
    case = dict(_DEFAULTS[op], op=op, **sizes)
    return dict(case, name=name) if name else case


# ---- more cases of the same ranges ---------------------------------------------------------
_HEADS = ((16, 16), (16, 4), (32, 8), (40, 8), (8, 8), (8, 1))


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw_once(rng):
    op = rng.choice(("attention", "attention", "verify", "commit", "axes"))
    H_q, H_kv = rng.choice(_HEADS)
    small = rng.random() < 0.15
    kind = dict(d=64, dtype="f32") if small else dict(d=128, dtype="bf16")
    if op in ("attention", "commit"):
        w = rng.choice((_log(rng, 16, 2048), 128 * rng.randint(1, 12)))
        return _case(None, op, B=_log(rng, 1, 4 if small else 48), H_q=H_q, H_kv=H_kv, N=_log(rng, 1, 128), w=w,
                     pos=_log(rng, 8, 40000), deep=rng.choice((0, 3, 6, 10)), per_entry=rng.random() < 0.5,
                     padded=rng.random() < 0.5, bthd=rng.random() < 0.5, **kind)
    if op == "verify":
        return _case(None, op, B=_log(rng, 1, 48), N=_log(rng, 1, 64), V=_log(rng, 500, 140000), deep=rng.choice((0, 3, 6)),
                     draft=rng.choice(("probs", "probs", "none")), dtype=rng.choice(("f32", "f32", "bf16")),
                     padded=rng.random() < 0.5)
    return _case(None, op, B=_log(rng, 1, 8), H_q=H_q, H_kv=H_kv, T=_log(rng, 1, 9000), axes=rng.randint(1, 4),
                 order=rng.choice(("runs", "own", "dealt")), direction=rng.choice(("fwd", "bwd")),
                 bthd=rng.random() < 0.5, **kind)


def draw(rng):
    most = {}
    for c in listed():
        x = most.setdefault(c["op"], [0.0, 0.0])
        for i, n in enumerate(_cost(c)):
            x[i] = max(x[i], n)
    while True:
        c = _draw_once(rng)
        if all(n <= m for n, m in zip(_cost(c), most[c["op"]])):
            return c


def _cost(c):
    """What a pass of the plain form handles: work, and the size of the state that is prepared for it."""
    if c["op"] == "attention":
        return c["B"] * c["H_q"] * c["N"] * (c["w"] + c["N"] + c["d"]), c["B"] * c["H_kv"] * (c["w"] + c["d"])
    if c["op"] == "verify":
        return c["B"] * c["N"] * c["V"], 0.0
    if c["op"] == "commit":
        return c["B"] * c["H_kv"] * (c["w"] + c["N"] + c["d"]), 0.0
    return c["B"] * (c["H_q"] + c["H_kv"]) * c["T"] * c["d"] * (2 if c["dtype"] == "f32" else 1), 0.0


# ---- inputs ----------------------------------------------------------------------------------
_THETA, _EPS = 5.0e5, 1e-6


def _type(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def _heads(x, c):
    """[B, H, T, d] as the case keeps it."""
    return x.transpose(1, 2).contiguous() if c["bthd"] else x


def _unit(x):
    return x / x.square().mean(-1, keepdim=True).sqrt()


def _tree(c, g):
    """Parents [B, N] on the host: node 0 is the token sampled last, a chain (deep = 0) or a tree hangs from
    it, and the nodes that an entry does not use have parent -2."""
    B, N = c["B"], c["N"]
    parents = torch.full((B, N), -2, dtype=torch.int32)
    pick = torch.rand(B, N, generator=g).tolist()
    used = torch.randint(max(1, N // 2), N + 1, (B,), generator=g).tolist()
    for b in range(B):
        depth = []
        row = []
        for i in range(used[b] if c["padded"] else N):
            if i == 0:
                up = -1
            elif c["deep"] == 0:
                up = i - 1
            else:
                open_ = [j for j in range(max(0, i - 12), i) if depth[j] < c["deep"]] or [0]
                up = open_[int(pick[b][i] * len(open_))]
            row.append(up)
            depth.append(0 if up < 0 else depth[up] + 1)
        parents[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
    return parents


def _positions(c, g):
    B = c["B"]
    if not c["per_entry"]:
        return torch.full((B,), c["pos"], dtype=torch.int32)
    return torch.randint(max(1, c["pos"] // 4), c["pos"] + 1, (B,), generator=g).to(torch.int32)


def _cache(c, pos, g):
    """Ring and state of running sequences: unit-norm keys, the state summed over 256 tokens' worth."""
    B, Hkv, w, d, t = c["B"], c["H_kv"], c["w"], c["d"], _type(c)
    held = (torch.arange(w, device="cuda") < pos.cuda()[:, None])[:, None, :, None]
    ring = []
    for unit in (True, False):
        x = torch.randn(B, Hkv, w, d, device="cuda", generator=g)
        ring.append(((_unit(x) if unit else x) * held).to(t))
    k = _unit(torch.randn(B, Hkv, 256, d, device="cuda", generator=g))
    v = torch.randn(B, Hkv, 256, d, device="cuda", generator=g)
    left = (pos.cuda() - w).clamp(min=0).float()
    state = torch.softmax(k, -1).transpose(2, 3) @ v * (left / 256.0).sqrt()[:, None, None, None]
    return ring[0], ring[1], state.contiguous()


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    h = torch.Generator().manual_seed(seed)
    s = {"case": c}
    if c["op"] in ("attention", "commit"):
        B, N, d, t = c["B"], c["N"], c["d"], _type(c)
        parents, pos = _tree(c, h), _positions(c, h)
        s["k_ring"], s["v_ring"], s["state"] = _cache(c, pos, g)
        s["pos"] = pos.cuda() if c["per_entry"] else None
        make = lambda H: torch.randn(B, H, N, d, device="cuda", generator=g)  # noqa: E731
        s["k"], s["v"] = _heads(_unit(make(c["H_kv"])).to(t), c), _heads(make(c["H_kv"]).to(t), c)
        if c["op"] == "attention":
            s["parents"] = parents.cuda()
            s["q"] = _heads(_unit(make(c["H_q"])).to(t), c)
            s["out"] = torch.zeros_like(s["q"])
            s["gains"] = [1.0 + 0.1 * torch.randn(c["H_q"], d, device="cuda", generator=g) for _ in range(2)]
        else:
            s["path"], s["n"] = (x.cuda() for x in _accepted(parents, h))
    elif c["op"] == "verify":
        B, N, V, t = c["B"], c["N"], c["V"], _type(c)
        s["parents"] = _tree(c, h).cuda()
        logits = 2.0 * torch.randn(B, N, V, device="cuda", generator=g)
        other = logits + 0.7 * torch.randn(B, N, V, device="cuda", generator=g)
        s["target"] = torch.softmax(logits, -1).to(t)
        s["draft"] = None
        up = s["parents"].clamp(min=0).long()
        if c["draft"] == "probs":
            s["draft"] = torch.softmax(other, -1).to(t)
            # every node's token is drawn from its parent's distribution
            sums = torch.softmax(other, -1).cumsum(-1)
            rows = torch.gather(sums, 1, up[..., None].expand(-1, -1, V))
            u = torch.rand(B, N, 1, device="cuda", generator=g) * rows[..., -1:]
            tokens = torch.searchsorted(rows, u).squeeze(-1).clamp(max=V - 1)
        else:
            # the parent's most probable tokens, one after the other
            best = other.topk(min(16, V), -1).indices
            nth = (torch.arange(N, device="cuda") - up - 1).clamp(min=0) % best.shape[-1]
            tokens = torch.gather(best[torch.arange(B, device="cuda")[:, None], up], 2, nth[..., None]).squeeze(-1)
        s["tokens"] = tokens.to(torch.int32).contiguous()
        s["u"] = torch.rand(B, N, device="cuda", generator=g)
    else:
        B, T, d, t, A = c["B"], c["T"], c["d"], _type(c), c["axes"]
        make = lambda H: _heads((2.0 * torch.randn(B, H, T, d, device="cuda", generator=g)).to(t), c)  # noqa: E731
        s["q"], s["k"] = make(c["H_q"]), make(c["H_kv"])
        s["gains"] = [1.0 + 0.1 * torch.randn(d, device="cuda", generator=g) for _ in range(2)]
        # one axis: nodes a few levels behind a far position; more: time, and places in a picture
        far = torch.randint(0, 100000, (1, B, 1), device="cuda", generator=g)
        near = torch.randint(0, 10 if A == 1 else 64, (A, B, T), device="cuda", generator=g)
        near[0] += far[0]
        s["at"] = near.to(torch.int32).contiguous()
        s["sections"] = _sections(c)
        if c["direction"] == "bwd":
            s["dq"], s["dk"] = make(c["H_q"]), make(c["H_kv"])
    return s


def _sections(c):
    """Rotated pairs of each axis; with several axes the first has fewer, as time has in video models."""
    half, A = c["d"] // 2, c["axes"]
    if A == 1:
        return [half]
    rest = (half - half // (A + 1)) // (A - 1)
    return [half - rest * (A - 1)] + [rest] * (A - 1)


def _accepted(parents, g):
    """A path from node 0 down each tree (about three in four children accepted), and its length."""
    B, N = parents.shape
    path, n = torch.full((B, N), -1, dtype=torch.int32), torch.zeros(B, dtype=torch.int32)
    for b in range(B):
        row, at, coin = [0], 0, torch.rand(N, generator=g).tolist()
        for i in range(1, N):
            if parents[b, i] == at and coin[i] < 0.75:
                row.append(i)
                at = i
        path[b, :len(row)] = torch.tensor(row, dtype=torch.int32)
        n[b] = len(row)
    return path, n


# ---- one pass --------------------------------------------------------------------------------

def run(state):
    c = state["case"]
    if own:
        return _OWN[c["op"]](state, c)
    return _PLAIN[c["op"]](state, c)


def _own_attention(s, c):
    from paper_2506_15545_b200 import binding as rb
    return rb.rattn_draft_attention(s["q"], s["k"], s["v"], s["parents"], s["k_ring"], s["v_ring"], s["state"], c["pos"],
                                    scale=1.0 / math.sqrt(c["d"]), eps=_EPS, gamma_swa=s["gains"][0],
                                    gamma_rla=s["gains"][1], out=s["out"], pos_dev=s["pos"],
                                    layout=rb.LAYOUT_BTHD if c["bthd"] else rb.LAYOUT_BHTD)


def _own_verify(s, c):
    from paper_2506_15545_b200 import binding as rb
    return rb.rattn_draft_verify(s["tokens"], s["parents"], s["target"], s["draft"], s["u"])


def _own_commit(s, c):
    from paper_2506_15545_b200 import binding as rb
    rb.rattn_draft_commit(s["k"], s["v"], s["path"], s["n"], s["k_ring"], s["v_ring"], s["state"], c["pos"],
                          pos_dev=s["pos"], layout=rb.LAYOUT_BTHD if c["bthd"] else rb.LAYOUT_BHTD)
    return s["k_ring"], s["v_ring"], s["state"]


def _own_axes(s, c):
    from paper_2506_15545_b200 import binding as rb
    kw = dict(order={"runs": rb.AXES_RUNS, "own": rb.AXES_OWN, "dealt": rb.AXES_DEALT}[c["order"]], q_gain=s["gains"][0],
              k_gain=s["gains"][1], theta=_THETA, eps=_EPS, layout=rb.LAYOUT_BTHD if c["bthd"] else rb.LAYOUT_BHTD)
    if c["direction"] == "fwd":
        return rb.rattn_qk_prologue_axes(s["q"], s["k"], s["at"], s["sections"], **kw)
    return rb.rattn_qk_prologue_axes_backward(s["q"], s["k"], s["dq"], s["dk"], s["at"], s["sections"], **kw)


# ---- the plain forms -------------------------------------------------------------------------

def _reach(parents):
    """[B, N, N]: whether column j is row i itself or one of its ancestors (seven doublings reach 128 levels)."""
    N = parents.shape[1]
    at = torch.arange(N, device=parents.device)
    r = ((parents[..., None] == at) | (at[:, None] == at)).float()
    for _ in range(7):
        r = ((r @ r) > 0).float()
    return r > 0


def _phi(x):
    e = torch.exp(x - x.max(-1, keepdim=True).values)
    return e / e.sum(-1, keepdim=True)


def _rms(x, gain):
    return x / (x.square().mean(-1, keepdim=True) + _EPS).sqrt() * gain


def _dense(x, c):
    return (x.transpose(1, 2) if c["bthd"] else x).float()


def _pos(s, c):
    return s["pos"].long() if s["pos"] is not None else torch.full((c["B"],), c["pos"], device="cuda")


def _plain_attention(s, c):
    B, Hkv, N, w, d, G = c["B"], c["H_kv"], c["N"], c["w"], c["d"], c["H_q"] // c["H_kv"]
    pos, reach = _pos(s, c), _reach(s["parents"])
    depth = reach.sum(-1) - 1
    # distances in tokens: ring slot -> how many tokens before `pos`, nodes -> their depth
    back = w - (torch.arange(w, device="cuda") - pos[:, None]) % w
    key_at = torch.cat([-back, depth], 1)
    seen = torch.cat([(back <= pos[:, None])[:, None].expand(B, N, w), reach], 2)
    near = seen & (depth[..., None] - key_at[:, None] <= w)
    q = _dense(s["q"], c).reshape(B, Hkv, G, N, d)
    k = torch.cat([s["k_ring"].float(), _dense(s["k"], c)], 2)[:, :, None]
    v = torch.cat([s["v_ring"].float(), _dense(s["v"], c)], 2)[:, :, None]
    near, far = near[:, None, None], (seen & ~near)[:, None, None]
    x = (q @ k.transpose(-1, -2) / math.sqrt(d)).masked_fill(~near, -math.inf)
    x = torch.exp(x - x.max(-1, keepdim=True).values)
    o_swa = (x @ v) / x.sum(-1, keepdim=True)
    fq = _phi(q)
    o_rla = fq @ s["state"][:, :, None] + ((fq @ _phi(k).transpose(-1, -2)) * far) @ v
    gs, gr = (g.reshape(1, Hkv, G, 1, d) for g in s["gains"])
    y = (_rms(o_swa, gs) + _rms(o_rla, gr)).reshape(B, c["H_q"], N, d).to(s["q"].dtype)
    y = y.transpose(1, 2) if c["bthd"] else y
    used = s["parents"] >= -1
    used = used[:, :, None, None] if c["bthd"] else used[:, None, :, None]
    return torch.where(used, y, s["out"])


def _plain_verify(s, c):
    """One look at each node in index order: a node is tested when its parent is the node accepted last.  The
    loop is the operator's own: what a test compares with depends on the tests before it."""
    B, N = s["parents"].shape
    V = s["target"].shape[2]
    b = torch.arange(B, device="cuda")
    u, parents, tokens = s["u"].double(), s["parents"].long(), s["tokens"].long()
    tiny = 2.0 ** -40
    used = parents[:, 0] == -1
    now = torch.where(used, 0, -1)                                  # the node accepted last
    n = used.long()
    path = torch.full((B, N), -1, device="cuda", dtype=torch.long)
    path[:, 0] = now
    row = s["target"][:, 0].double()                                # its row, and what the rejections have left of it
    left, total = row, torch.ones(B, device="cuda", dtype=torch.float64)
    for i in range(1, N):
        asked = used & (parents[:, i] == now)
        x = tokens[:, i, None]
        if s["draft"] is not None:
            q = s["draft"][b, now.clamp(min=0)].double()
        else:
            q = torch.zeros(B, V, device="cuda", dtype=torch.float64).scatter(1, x, 1.0)
        took = asked & (u[:, i] * q.gather(1, x)[:, 0] * total < left.gather(1, x)[:, 0])
        missed = asked & ~took
        less = (left - total[:, None] * q).clamp(min=0)
        if s["draft"] is None:
            less = torch.where(q > 0, 0.0, left)
            rest = total - left.gather(1, x)[:, 0]
        else:
            rest = less.sum(-1)
            missed = missed & (rest > tiny * total)
        here = s["target"][:, i].double()
        row = torch.where(took[:, None], here, row)
        left = torch.where(took[:, None], here, torch.where(missed[:, None], less, left))
        total = torch.where(took, 1.0, torch.where(missed, rest, total))
        now = torch.where(took, i, now)
        path.scatter_(1, n.clamp(max=N - 1)[:, None], torch.where(took, i, path.gather(1, n.clamp(max=N - 1)[:, None])[:, 0])[:, None])
        n = n + took
    left = torch.where((left.sum(-1) > 0)[:, None], left, row)
    sums = left.cumsum(-1)
    token = (sums <= (u[:, 0] * sums[:, -1])[:, None]).sum(-1)
    token = torch.where(used & (sums[:, -1] > 0), token, -1)
    return path.to(torch.int32), n.to(torch.int32), token.to(torch.int32)


def _plain_commit(s, c):
    B, Hkv, N, w, d = c["B"], c["H_kv"], c["N"], c["w"], c["d"]
    pos, n = _pos(s, c), s["n"].long()
    a = torch.arange(N, device="cuda")
    path = s["path"].long().clamp(min=0)
    pick = lambda x, i: torch.gather(x, 2, i[:, None, :, None].expand(B, Hkv, i.shape[1], d))  # noqa: E731
    new = [pick(x.transpose(1, 2) if c["bthd"] else x, path) for x in (s["k"], s["v"])]
    # the token that leaves the window as accepted token a enters: from the ring, or accepted itself
    slot = (pos[:, None] + a) % w
    inside = (a < w)[:, None]
    gone = [torch.where(inside, pick(r, slot), x[:, :, (a - w).clamp(min=0)]) for r, x in zip((s["k_ring"], s["v_ring"]), new)]
    leaves = ((a < n[:, None]) & (pos[:, None] + a >= w))[:, None, :, None]
    s["state"] += (_phi(gone[0].float()) * leaves).transpose(2, 3) @ gone[1].float()
    # a slot takes the last accepted token that falls on it
    first = (torch.arange(w, device="cuda") - pos[:, None]) % w
    last = first + w * ((n[:, None] - 1 - first).clamp(min=0) // w)
    hit = (first < n[:, None])[:, None, :, None]
    for r, x in zip((s["k_ring"], s["v_ring"]), new):
        r.copy_(torch.where(hit, pick(x, last.clamp(max=N - 1)), r))
    return s["k_ring"], s["v_ring"], s["state"]


def _angles(s, c):
    """cos and sin [B, T, d/2] of every pair, from angles in 64 bits."""
    half, sizes = c["d"] // 2, s["sections"]
    A = len(sizes)
    axis, power = [], []
    if c["order"] == "dealt":
        room, a = list(sizes), 0
        while len(axis) < sum(sizes):
            if room[a] > 0:
                room[a] -= 1
                axis.append(a)
            a = (a + 1) % A
        power = [i / half for i in range(len(axis))]
    else:
        axis = [a for a in range(A) for _ in range(sizes[a])]
        power = [j / sizes[a] for a in range(A) for j in range(sizes[a])] if c["order"] == "own" else [i / half for i in range(len(axis))]
    f = torch.tensor([_THETA ** -p for p in power], device="cuda", dtype=torch.float64)
    ang = s["at"].double()[torch.tensor(axis, device="cuda")].permute(1, 2, 0) * f
    return ang.cos().float(), ang.sin().float()


def _plain_axes(s, c):
    cos, sin = (x[:, :, None] if c["bthd"] else x[:, None] for x in _angles(s, c))
    half, d = c["d"] // 2, c["d"]

    def turned(x, sign):
        lo, hi = x[..., :half], x[..., half:]
        return torch.cat([lo * cos - sign * hi * sin, hi * cos + sign * lo * sin], -1)

    if c["direction"] == "fwd":
        return tuple(turned(_rms(x.float(), g), 1.0).to(x.dtype) for x, g in zip((s["q"], s["k"]), s["gains"]))
    grads, gains = [], []
    for x, dy, g in zip((s["q"], s["k"]), (s["dq"], s["dk"]), s["gains"]):
        x, dn, t = x.float(), turned(dy.float(), -1.0), x.dtype
        r = 1.0 / (x.square().mean(-1, keepdim=True) + _EPS).sqrt()
        gains.append((dn * x * r).sum((0, 1, 2)))
        dn = dn * g
        grads.append((r * dn - x * r ** 3 * (dn * x).sum(-1, keepdim=True) / d).to(t))
    return (*grads, *gains)


# ---- bytes and operations that a pass cannot do without -----------------------------------------

def work(case):
    c = case
    e = 4 if c["dtype"] == "f32" else 2
    if c["op"] == "attention":
        B, Hq, Hkv, N, w, d = (c[x] for x in ("B", "H_q", "H_kv", "N", "w", "d"))
        return {"bytes": e * d * B * (2 * Hq * N + 2 * Hkv * (N + w)) + 4 * d * d * B * Hkv,
                "flops": 4.0 * d * B * Hq * N * (w + 1) + 2.0 * d * d * B * Hq * N}
    if c["op"] == "verify":
        # the row that the last token is drawn from, of the target and (where there is one) of the drafter
        rows = 2 if c["draft"] == "probs" else 1
        return {"bytes": c["B"] * (rows * e * (c["V"] + c["N"]) + 16 * c["N"]), "flops": float(c["B"] * c["V"] * (rows + 1))}
    if c["op"] == "commit":
        B, Hkv, d = c["B"], c["H_kv"], c["d"]
        n = 1 if c["N"] == 1 else 3                                   # tokens that a step accepts, or more
        return {"bytes": B * Hkv * (8 * d * d + n * 6 * d * e), "flops": 2.0 * n * B * Hkv * d * d}
    rows = c["B"] * (c["H_q"] + c["H_kv"]) * c["T"]
    n = 2 if c["direction"] == "fwd" else 3
    return {"bytes": n * e * rows * c["d"] + 4 * c["axes"] * c["B"] * c["T"], "flops": 10.0 * rows * c["d"]}


# ---- the definitions, in 64 bits ------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "verify": _exact_verify, "commit": _exact_commit, "axes": _exact_axes}[case["op"]](s, case)


def _norm64(x, gain):
    return gain.double() * x / torch.sqrt((x * x).sum(-1, keepdim=True) / x.shape[-1] + _EPS)


def _exact_attention(s, c):
    """Every node on its own: the tokens before it in order (the cache's, then its path), the last w + 1 by
    softmax, the earlier ones and the state by the feature map."""
    w, d, G = c["w"], c["d"], c["H_q"] // c["H_kv"]
    bhtd = lambda x: (x.permute(0, 2, 1, 3) if c["bthd"] else x).double()  # noqa: E731
    q, k, v = bhtd(s["q"]), bhtd(s["k"]), bhtd(s["v"])
    out = bhtd(s["out"]).clone()
    parents = s["parents"].tolist()
    pos = s["pos"].tolist() if s["pos"] is not None else [c["pos"]] * c["B"]
    for b in range(c["B"]):
        slots = torch.tensor([j % w for j in range(max(0, pos[b] - w), pos[b])], device="cuda", dtype=torch.long)
        past = [r[b].double()[:, slots] for r in (s["k_ring"], s["v_ring"])]
        S = s["state"][b].double().repeat_interleave(G, 0)
        for i in range(c["N"]):
            if parents[b][i] < -1:
                continue
            line = [i]
            while parents[b][line[0]] >= 0:
                line.insert(0, parents[b][line[0]])
            keys, values = (torch.cat([p, x[b][:, line]], 1).repeat_interleave(G, 0) for p, x in zip(past, (k, v)))
            cut = max(0, keys.shape[1] - (w + 1))
            qi = q[b, :, i]
            weight = torch.softmax((keys[:, cut:] * qi[:, None]).sum(-1) / math.sqrt(d), -1)
            o_swa = (weight[..., None] * values[:, cut:]).sum(1)
            f = torch.softmax(qi, -1)
            o_rla = (f[..., None] * S).sum(1)
            if cut:
                o_rla = o_rla + ((torch.softmax(keys[:, :cut], -1) * f[:, None]).sum(-1, keepdim=True) * values[:, :cut]).sum(1)
            out[b, :, i] = _norm64(o_swa, s["gains"][0]) + _norm64(o_rla, s["gains"][1])
    return out.permute(0, 2, 1, 3) if c["bthd"] else out


def _exact_verify(s, c):
    parents, tokens, u = s["parents"].tolist(), s["tokens"].tolist(), s["u"].double().tolist()
    B, N = len(parents), len(parents[0])
    path, count, last = torch.full((B, N), -1, dtype=torch.int32), [], []
    for b in range(B):
        if parents[b][0] != -1:
            count.append(0)
            last.append(-1)
            continue
        line, node = [0], 0
        weights, norm = s["target"][b, 0].double(), 1.0
        while True:
            kids = [i for i in range(node + 1, N) if parents[b][i] == node]
            q = None if s["draft"] is None else s["draft"][b, node].double()
            for i in kids:
                x = tokens[b][i]
                p = weights[x].item()
                if u[b][i] * (1.0 if q is None else q[x].item()) * norm < p:
                    line.append(i)
                    break
                if q is None:
                    weights = weights.clone()
                    weights[x] = 0.0
                    norm -= p
                else:
                    less = torch.relu(weights - norm * q)
                    if less.sum().item() > 2.0 ** -40 * norm:
                        weights, norm = less, less.sum().item()
            else:
                break
            node = line[-1]
            weights, norm = s["target"][b, node].double(), 1.0
        if not weights.sum().item() > 0:
            weights = s["target"][b, node].double()
        sums = weights.cumsum(0)
        ahead = torch.nonzero(sums > u[b][0] * sums[-1])
        path[b, :len(line)] = torch.tensor(line, dtype=torch.int32)
        count.append(len(line))
        last.append(int(ahead[0]) if len(ahead) else -1)
    return path, torch.tensor(count, dtype=torch.int32), torch.tensor(last, dtype=torch.int32)


def _exact_commit(s, c):
    """One accepted token after the other, as so many single steps would enter them."""
    w = c["w"]
    bhtd = lambda x: x.permute(0, 2, 1, 3) if c["bthd"] else x  # noqa: E731
    k, v = bhtd(s["k"]), bhtd(s["v"])
    kr, vr, S = s["k_ring"].double(), s["v_ring"].double(), s["state"].double()
    pos = s["pos"].tolist() if s["pos"] is not None else [c["pos"]] * c["B"]
    for b, (line, n) in enumerate(zip(s["path"].tolist(), s["n"].tolist())):
        for a in range(n):
            at = (pos[b] + a) % w
            if pos[b] + a >= w:
                S[b] += torch.softmax(kr[b, :, at], -1)[:, :, None] * vr[b, :, at][:, None, :]
            kr[b, :, at], vr[b, :, at] = k[b, :, line[a]].double(), v[b, :, line[a]].double()
    return kr, vr, S


def _exact_axes(s, c):
    """Norm and gain, then every pair as a complex number times exp(i angle); gradients by differentiation."""
    half, A, sizes = c["d"] // 2, c["axes"], s["sections"]
    phase = torch.zeros(c["B"], c["T"], half, device="cuda", dtype=torch.float64)
    if c["order"] == "dealt":
        turn, i = [0] * A, 0
        while i < sum(sizes):
            for a in range(A):
                if turn[a] < sizes[a]:
                    phase[..., i] = s["at"][a].double() * _THETA ** (-i / half)
                    turn[a], i = turn[a] + 1, i + 1
    else:
        i = 0
        for a in range(A):
            for j in range(sizes[a]):
                phase[..., i] = s["at"][a].double() * _THETA ** (-(j / sizes[a] if c["order"] == "own" else i / half))
                i += 1
    spin = torch.polar(torch.ones_like(phase), phase)
    spin = spin[:, :, None] if c["bthd"] else spin[:, None]

    def apply(x, gain):
        n = _norm64(x, gain)
        z = torch.complex(n[..., :half], n[..., half:]) * spin
        return torch.cat([z.real, z.imag], -1)

    if c["direction"] == "fwd":
        return tuple(apply(x.double(), g) for x, g in zip((s["q"], s["k"]), s["gains"]))
    out = []
    for x, dy, g in zip((s["q"], s["k"]), (s["dq"], s["dk"]), s["gains"]):
        x, g = x.double().requires_grad_(), g.double().requires_grad_()
        with torch.enable_grad():
            out.append(torch.autograd.grad(apply(x, g), (x, g), dy.double()))
    return out[0][0], out[1][0], out[0][1], out[1][1]


_OWN = {"attention": _own_attention, "verify": _own_verify, "commit": _own_commit, "axes": _own_axes}
_PLAIN = {"attention": _plain_attention, "verify": _plain_verify, "commit": _plain_commit, "axes": _plain_axes}
