"""The scored attention, drafted-token attention and cache operators, case by case:
their calls, the same mathematics in plain torch operations, and in 64 bits.

A case is a dict; "kind" selects the operator:

  forward   keyless_scored_forward: attention over projected routed queries and
            values with a tanh cap, a distance bias, a document or prefix mask
  train     the same with its log-sum-exp and fp32 output kept, then
            keyless_scored_backward: one layer's attention in a training step
  tree      keyless_tree_decode: T drafted tokens per sequence (a tree or a
            chain; T = 1 is one serving step) over a value-only cache
  keep      value_cache_keep: the accepted drafted rows move up in the cache
"""

import math

import numpy as np
import torch

own = False  # True: run() calls the library; False: the plain form

BF16, F32 = "bf16", "f32"
DTYPES = {BF16: torch.bfloat16, F32: torch.float32}
DEV = "cuda"

# (query heads, value groups, d_head)
TESTBED = (12, 2, 128)    # the paper's decode testbed: 12 heads over 2 value heads
LARGE = (32, 32, 128)     # the prefill workload's layer
LARGE_GQA = (32, 8, 128)  # the paged workload's heads
MEDIUM = (8, 8, 128)      # the paper's GPT-2 heads
TINY = (4, 4, 64)         # the small fp32 layer
SMALL = (8, 8, 64)


def _case(kind, dtype, dims, **more):
    H, G, d = dims
    return dict(kind=kind, dtype=dtype, H=H, G=G, d=d, **more)


def _attend(kind, dtype, dims, B, N, cap=0.0, slopes=False, docs=1, prefix=0.0, pad=0, causal=True):
    return _case(kind, dtype, dims, B=B, N=N, cap=cap, slopes=slopes, docs=docs, prefix=prefix,
                 pad=pad, causal=causal)


def _drafts(dtype, dims, B, T, lo, hi, cap=0.0, slopes=False, branch=True, paged=False):
    return _case("tree", dtype, dims, B=B, T=T, lo=lo, hi=hi, cap=cap, slopes=slopes, branch=branch,
                 paged=paged)


def _keep(dtype, dims, B, T, lo, hi, paged=False):
    return _case("keep", dtype, dims, B=B, T=T, lo=lo, hi=hi, paged=paged)


def listed():
    return [
        # The small fp32 layer's prompt with a distance bias: the shortest attention call.
        dict(_attend("forward", F32, TINY, 1, 128, slopes=True), name="fwd_f32_128"),
        # A prompt of odd length whose first part is seen by every token (prefix mask), capped.
        dict(_attend("forward", BF16, TESTBED, 1, 517, cap=30.0, prefix=0.4), name="fwd_prefix_517"),
        # A long prompt through a large grouped layer with capped scores.
        dict(_attend("forward", BF16, LARGE_GQA, 1, 8192, cap=50.0), name="fwd_8k"),
        # An fp32 training step of the paper's 12-layer size: three packed documents, cap and bias.
        dict(_attend("train", F32, MEDIUM, 1, 512, cap=20.0, slopes=True, docs=3), name="train_f32"),
        # Two packed, padded sequences of a grouped layer in training, capped scores.
        dict(_attend("train", BF16, TESTBED, 2, 1000, cap=30.0, docs=5, pad=37), name="train_docs"),
        # Long-context training on one sequence of a few packed documents, capped.
        dict(_attend("train", BF16, LARGE_GQA, 1, 8192, cap=50.0, docs=2), name="train_8k"),
        # One token of one sequence, capped and biased: the smallest serving call.
        dict(_drafts(BF16, TESTBED, 1, 1, 2040, 2040, cap=30.0, slopes=True, branch=False),
             name="tree_b1"),
        # fp32 serving of a small model: chains of five drafted tokens, uneven lengths.
        dict(_drafts(F32, SMALL, 6, 5, 5, 1500, slopes=True, branch=False), name="tree_f32"),
        # A serving batch of trees of 16 drafted tokens over a paged cache, capped.
        dict(_drafts(BF16, LARGE_GQA, 16, 16, 1024, 32000, cap=50.0, paged=True), name="tree_paged"),
        # Wide trees of 64 tokens, one head per value group, long caches.
        dict(_drafts(BF16, LARGE, 8, 64, 2000, 4030), name="tree_wide"),
        # The end of a draft step of one sequence.
        dict(_keep(BF16, TESTBED, 1, 8, 500, 500), name="keep_b1"),
        # The same for a serving batch with 64 drafted tokens each, paged.
        dict(_keep(BF16, LARGE_GQA, 64, 64, 64, 500, paged=True), name="keep_b64"),
    ]


def _log(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi], odd ones included."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("forward", "train", "train", "tree", "tree", "keep"))
    cap = rng.choice((0.0, 15.0, 30.0, 50.0))
    slopes = rng.random() < 0.4
    fp32 = rng.random() < 0.3
    bf16_dims = (TESTBED, LARGE_GQA, LARGE, MEDIUM, (16, 4, 64))
    fp32_dims = (TINY, SMALL, MEDIUM, (16, 4, 64))
    dtype, dims = (F32, rng.choice(fp32_dims)) if fp32 else (BF16, rng.choice(bf16_dims))
    if kind in ("forward", "train"):
        B, causal = rng.choice((1, 1, 2, 4)), rng.random() < 0.85
        most = (8192 if causal else 5800) if kind == "forward" else (5800 if causal else 4000)
        N = _log(rng, 1 if kind == "forward" else 16, 1000 if fp32 else most // B)
        docs = 1 if N < 64 else rng.choice((1, 1, 2, 5, 9))
        return _attend(kind, dtype, dims, B, N, cap, slopes, docs, rng.choice((0.0, 0.0, 0.3)),
                       rng.choice((0, 0, N // 20)), causal)
    paged = rng.random() < 0.5
    if kind == "keep":
        hi = _log(rng, 16, 1000)
        return _keep(dtype, dims, _log(rng, 1, 64), _log(rng, 1, 64), max(1, hi // 4), hi, paged)
    B, T = _log(rng, 1, 32), _log(rng, 1, 64)
    most = min(32000, (1 << 21) // (B * max(1, dims[1] // 4)), (1 << 28) // (B * T * dims[0]))
    hi = _log(rng, 16, max(64, min(most, 3000) if fp32 else most))
    return _drafts(dtype, dims, B, T, max(1, hi // rng.choice((1, 2, 8, 32))), hi, cap, slopes,
                   rng.random() < 0.6, paged)


def _doc_lengths(c):
    """The documents of one sequence, from the case alone: lengths that rise evenly."""
    n, k = c["N"] - c["pad"], c["docs"]
    ends = np.floor(n * np.cumsum(np.arange(1, k + 1)) / (k * (k + 1) / 2)).astype(np.int64)
    return np.diff(ends, prepend=0)


def _cached(c):
    """Rows cached per sequence, from the case alone: from lo to hi in even ratios."""
    return np.round(np.geomspace(c["lo"], c["hi"], c["B"])).astype(np.int64)


def _kept(c):
    """Accepted tokens per sequence: a few of the T drafted ones, none for some."""
    return np.arange(c["B"]) * 7 % (c["T"] // 4 + 2) if c["B"] > 1 else np.array([(c["T"] + 1) // 2])


class _Draw:
    """Normal tensors in the case's dtype, made on the GPU from the seed."""

    def __init__(self, seed, dtype):
        self.gen = torch.Generator(device=DEV)
        self.gen.manual_seed(int(seed))
        self.dtype = dtype

    def normal(self, *shape, std=1.0):
        t = torch.empty(shape, dtype=self.dtype, device=DEV)
        t.normal_(0.0, std, generator=self.gen)
        return t


def _int32(a):
    return torch.as_tensor(a, dtype=torch.int32).to(DEV)


def prepare(case, seed):
    c = case
    r, rs = _Draw(seed, DTYPES[c["dtype"]]), np.random.RandomState(int(seed) % (1 << 32))
    B, H, G, d = c["B"], c["H"], c["G"], c["d"]
    s = dict(kind=c["kind"], cap=c.get("cap", 0.0), causal=c.get("causal", True), slopes=None)
    if c.get("slopes"):  # the usual geometric series over the heads
        s["slopes"] = (2.0 ** (-8.0 * torch.arange(1, H + 1) / H)).to(DEV)
    if c["kind"] in ("forward", "train"):
        N = c["N"]
        # Routed queries that give scores of a spread of three: the cap bends the far ones.
        s["q"], s["v"] = r.normal(B, N, H, d, std=3.0), r.normal(B, N, G, d)
        if c["kind"] == "train":
            s["dout"] = r.normal(B, N, H, d)
        s["first"] = s["last"] = None
        if c["docs"] > 1 or c["prefix"] > 0 or c["pad"] > 0:
            # What the data loader hands over: where each token's document starts, and
            # the end of what it sees.
            first, last = np.zeros((B, N), np.int64), np.zeros((B, N), np.int64)
            for b in range(B):
                lens = rs.permutation(_doc_lengths(c))
                start = np.repeat(np.cumsum(lens) - lens, lens)
                size, i = np.repeat(lens, lens), np.arange(len(start))
                upto = start + np.ceil(c["prefix"] * size).astype(np.int64)
                first[b, :len(start)] = start
                last[b, :len(start)] = np.maximum(i + 1, upto) if c["causal"] else start + size
            s["first"], s["last"] = _int32(first), _int32(last)
        if own:
            from paper_2606_21848_amd import binding as kb
            s["scoring"] = kb.Scoring(cap=s["cap"], slopes=s["slopes"], first=s["first"],
                                      last=s["last"], causal=s["causal"])
            if c["kind"] == "train":
                s["ws"] = torch.empty(kb.scored_backward_workspace_bytes(B, N, H, G, d, s["q"].dtype),
                                      dtype=torch.uint8, device=DEV)
        return s
    T = c["T"]
    n = rs.permutation(_cached(c))
    s["before"] = _int32(n)
    room = int(n.max()) + T
    if c["paged"]:
        bs = 16
        width = -(-room // bs)
        order = rs.permutation(B * width)  # blocks in no order, as a serving program has them
        s["cache"] = r.normal(B * width, G, bs, d)
        s["table"] = _int32(order.reshape(B, width))
    else:
        s["cache"], s["table"] = r.normal(B, G, room, d), None
    if c["kind"] == "tree":
        s["q"] = r.normal(B, T, H, d, std=3.0)
        s["tree"] = None
        if c["branch"]:
            # Each token's parent is any earlier one; a token sees its ancestors and itself.
            sees = np.zeros((B, T, T), bool)
            for t in range(T):
                if t:
                    sees[:, t] = sees[np.arange(B), rs.randint(0, t, B)]
                sees[:, t, t] = True
            words = (sees.astype(np.uint64) << np.arange(T, dtype=np.uint64)).sum(2, dtype=np.uint64)
            s["tree"] = torch.from_numpy(words.view(np.int64)).to(DEV)
    else:
        kept = rs.permutation(_kept(c))
        path = np.zeros((B, T), np.int64)
        for b in range(B):
            path[b, :kept[b]] = np.sort(rs.permutation(T)[:kept[b]])
        s["path"], s["kept"] = _int32(path), _int32(kept)
    if own:
        from paper_2606_21848_amd import binding as kb
        s["vc"] = kb.ValueCache(s["cache"], s["table"])
        if c["kind"] == "tree":
            s["out"] = torch.empty_like(s["q"])
            s["ws"] = torch.empty(max(kb.tree_decode_workspace_bytes(s["vc"], B, T, H), 256),
                                  dtype=torch.uint8, device=DEV)
    return s


# ---------------------------------------------------------------------------
# The library's calls
# ---------------------------------------------------------------------------

def _own(s):
    from paper_2606_21848_amd import binding as kb
    kind = s["kind"]
    if kind == "forward":
        out, lse = kb.keyless_scored_forward(s["q"], s["v"], s["scoring"])
        return dict(out=out, lse=lse)
    if kind == "train":
        o32 = torch.empty(s["q"].shape, dtype=torch.float32, device=DEV)
        out, lse = kb.keyless_scored_forward(s["q"], s["v"], s["scoring"], out_f32=o32)
        dq, dv = kb.keyless_scored_backward(s["q"], s["v"], out, s["dout"], lse, s["scoring"],
                                            out_f32=o32, workspace=s["ws"])
        return dict(out=out, lse=lse, dq=dq, dv=dv)
    if kind == "tree":
        return dict(out=kb.keyless_tree_decode(s["q"], s["vc"], s["before"], tree=s["tree"],
                                               cap=s["cap"], slopes=s["slopes"], out=s["out"],
                                               workspace=s["ws"]))
    kb.value_cache_keep(s["vc"], s["before"], s["path"], s["kept"])
    return dict(cache=s["cache"])


# ---------------------------------------------------------------------------
# The plain form: elementary operations in 32 bits
# ---------------------------------------------------------------------------

def _grouped(x, G):
    """[B, N, H, d] -> fp32 [B, G, H / G * N, d], the heads of a group one after another."""
    B, N, H, d = x.shape
    return x.float().reshape(B, N, G, H // G, d).permute(0, 2, 3, 1, 4).reshape(B, G, -1, d)


def _heads(x, N):
    """The inverse of _grouped."""
    B, G, RN, d = x.shape
    return x.reshape(B, G, RN // N, N, d).permute(0, 3, 1, 2, 4).reshape(B, N, -1, d)


def _plain_weights(q, v, cap, slopes, distance, seen):
    """Weights, tanh values and log-sum-exp of grouped queries [B, G, R N, d] over rows
    [B, G, L, d]; distance [B or 1, N, L], seen likewise."""
    B, G, RN, d = q.shape
    N, L = distance.shape[1:]
    x = torch.matmul(q, v.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    t = None
    if cap > 0:
        t = torch.tanh(x / cap)
        x = t * cap
    x = x.reshape(B, G, RN // N, N, L)
    if slopes is not None:
        x = x - slopes.reshape(1, G, -1, 1, 1) * distance[:, None, None].float()
    x = torch.where(seen[:, None, None], x, torch.full((), float("-inf"), device=x.device))
    m = x.amax(-1, keepdim=True)
    m = torch.where(m == float("-inf"), torch.zeros_like(m), m)
    p = torch.exp(x - m)
    total = p.sum(-1, keepdim=True)
    lse = torch.log(total) + m
    p = p / torch.where(total > 0, total, torch.ones_like(total))
    return p.reshape(B, G, RN, L), t, lse.reshape(B, G, RN // N, N)


def _plain_mask(s, N):
    i = torch.arange(N, device=DEV)
    distance = (i[:, None] - i[None, :]).abs()[None]
    if s["first"] is not None:
        seen = (i >= s["first"][:, :, None]) & (i < s["last"][:, :, None])
    elif s["causal"]:
        seen = (i[None, :] <= i[:, None])[None]
    else:
        seen = torch.ones((1, N, N), dtype=torch.bool, device=DEV)
    return distance, seen


def _plain_attend(s):
    q, v, dt = s["q"], s["v"], s["q"].dtype
    B, N, H, d = q.shape
    G = v.shape[2]
    qg, vg = _grouped(q, G), v.float().permute(0, 2, 1, 3).contiguous()
    distance, seen = _plain_mask(s, N)
    p, t, lse = _plain_weights(qg, vg, s["cap"], s["slopes"], distance, seen)
    o = torch.matmul(p, vg)
    got = dict(out=_heads(o, N).to(dt), lse=lse.reshape(B, H, N))
    if s["kind"] == "forward":
        return got
    g = _grouped(s["dout"], G)
    dz = torch.matmul(g, vg.transpose(2, 3).contiguous())
    dz = p * (dz - (g * o).sum(-1, keepdim=True))
    if t is not None:
        dz = dz * (1.0 - t * t)
    dz = dz * (1.0 / math.sqrt(d))
    dv = torch.matmul(p.transpose(2, 3), g) + torch.matmul(dz.transpose(2, 3), qg)
    got["dq"] = _heads(torch.matmul(dz, vg), N).to(dt)
    got["dv"] = dv.permute(0, 2, 1, 3).contiguous().to(dt)
    return got


def _dense(s, room):
    """The cache as [B, G, room, d], blocks of a paged one in order."""
    if s["table"] is None:
        return s["cache"][:, :, :room]
    rows = s["cache"][s["table"].long()]  # [B, width, G, 16, d]
    B, width, G, bs, d = rows.shape
    return rows.permute(0, 2, 1, 3, 4).reshape(B, G, width * bs, d)[:, :, :room]


def _plain_tree(s):
    q, n = s["q"], s["before"].long()
    B, T, H, d = q.shape
    G = s["cache"].shape[1]
    room = s["cache"].shape[2] if s["table"] is None else s["table"].shape[1] * 16
    rows = _dense(s, room).float()
    u, j = torch.arange(T, device=DEV), torch.arange(room, device=DEV)
    words = s["tree"]
    if words is None:
        sees = (u[None, :] <= u[:, None]).expand(B, T, T)
    else:
        sees = (words[:, :, None] >> u) & 1 == 1
    depth = sees.sum(-1) - torch.diagonal(sees, dim1=1, dim2=2).long()
    draft = (j[None, :] - n[:, None])  # [B, room]
    inside = (draft >= 0) & (draft < T)
    at = draft.clamp(0, T - 1)[:, None].expand(B, T, room)
    seen = (draft < 0)[:, None] | (inside[:, None] & torch.gather(sees, 2, at))
    place = torch.where(inside, n[:, None] + torch.gather(depth, 1, draft.clamp(0, T - 1)), j[None, :])
    distance = ((n[:, None] + depth)[:, :, None] - place[:, None]).abs()
    p, _, _ = _plain_weights(_grouped(q, G), rows.contiguous(), s["cap"], s["slopes"], distance, seen)
    p = torch.where(seen[:, None, None], p.reshape(B, G, -1, T, room), torch.zeros((), device=DEV))
    return dict(out=_heads(torch.matmul(p.reshape(B, G, -1, room), rows), T).to(q.dtype))


def _plain_keep(s):
    cache, n, path = s["cache"], s["before"].long(), s["path"].long()
    k = torch.arange(path.shape[1], device=DEV)
    b, k = torch.nonzero(k[None, :] < s["kept"][:, None], as_tuple=True)
    src, dst = n[b] + path[b, k], n[b] + k
    if s["table"] is None:
        cache[b, :, dst] = cache[b, :, src]
    else:
        table, bs = s["table"].long(), cache.shape[2]
        cache[table[b, dst // bs], :, dst % bs] = cache[table[b, src // bs], :, src % bs]
    return dict(cache=cache)


def run(state):
    if own:
        return _own(state)
    if state["kind"] in ("forward", "train"):
        return _plain_attend(state)
    return _plain_tree(state) if state["kind"] == "tree" else _plain_keep(state)


def work(case):
    c = case
    e = 2 if c["dtype"] == BF16 else 4
    B, H, G, d = c["B"], c["H"], c["G"], c["d"]
    if c["kind"] == "keep":
        return dict(bytes=2 * int(_kept(c).sum()) * G * d * e + 8 * B, flops=0)
    if c["kind"] == "tree":
        rows = int(_cached(c).sum()) + B * c["T"]
        return dict(bytes=e * (rows * G * d + 2 * B * c["T"] * H * d), flops=4 * rows * c["T"] * H * d)
    # Seen pairs: a document's prefix rows see the whole prefix, the others what came before.
    n = _doc_lengths(c).astype(np.float64)
    pre = np.ceil(c["prefix"] * n)
    pairs = float((n * n if not c["causal"] else n * (n + 1) / 2 + pre * (pre - 1) / 2).sum())
    qo, vv = B * c["N"] * H * d, B * c["N"] * G * d
    flops = 4 * B * H * d * pairs
    if c["kind"] == "forward":
        return dict(bytes=e * (2 * qo + vv) + 4 * B * H * c["N"], flops=flops)
    # dP, dQ~ and both terms of dV beside the forward's two products.
    return dict(bytes=e * (4 * qo + 2 * vv) + 4 * B * H * c["N"], flops=3 * flops)


# ---------------------------------------------------------------------------
# The definition in 64 bits, head by head
# ---------------------------------------------------------------------------

def _scores64(q, v, cap, slope, dist, mask):
    z = (q @ v.T) / math.sqrt(q.shape[1])
    bend = None
    if cap > 0:
        z = cap * torch.tanh(z / cap)
        bend = 1 - (z / cap) ** 2
    if slope is not None:
        z = z - slope * dist
    return z.masked_fill_(~mask, -math.inf), bend


def exact(case, seed):
    c, f = case, torch.float64
    s = prepare(case, seed)
    B, H, G, d = c["B"], c["H"], c["G"], c["d"]
    R, cap = H // G, c.get("cap", 0.0)
    slopes = None if s["slopes"] is None else s["slopes"].to(f)
    slope = lambda h: None if slopes is None else slopes[h]  # noqa: E731
    if c["kind"] in ("forward", "train"):
        N = c["N"]
        pos = torch.arange(N, device=DEV)
        dist = (pos[:, None] - pos[None]).abs().to(f)
        q, v = s["q"].to(f), s["v"].to(f)
        out, lse = torch.zeros_like(q), torch.zeros((B, H, N), dtype=f, device=DEV)
        got = dict(out=out, lse=lse)
        if c["kind"] == "train":
            dout = s["dout"].to(f)
            got["dq"], got["dv"] = torch.zeros_like(q), torch.zeros_like(v)
        for b in range(B):
            mask = torch.zeros((N, N), dtype=torch.bool, device=DEV)
            if s["first"] is None:
                mask = ~mask.logical_not().triu(1) if c["causal"] else ~mask
            else:
                mask = (pos[None] - s["first"][b][:, None] >= 0) & (s["last"][b][:, None] - pos[None] > 0)
            some = mask.any(1)
            for h in range(H):
                qh, vh = q[b, :, h].contiguous(), v[b, :, h // R].contiguous()
                x, bend = _scores64(qh, vh, cap, slope(h), dist, mask)
                lse[b, h] = torch.logsumexp(x, 1)
                p = x.sub_(torch.where(some, lse[b, h], 0.0)[:, None]).exp_()
                out[b, :, h] = p @ vh
                if c["kind"] == "train":
                    g = dout[b, :, h].contiguous()
                    ds = (g @ vh.T - (g * out[b, :, h]).sum(1)[:, None]) * p / math.sqrt(d)
                    if bend is not None:
                        ds *= bend
                    got["dq"][b, :, h] = ds @ vh
                    got["dv"][b, :, h // R] += p.T @ g + ds.T @ qh
        return got
    T, n = c["T"], [int(x) for x in s["before"].tolist()]
    if c["kind"] == "keep":
        cache = s["cache"].clone()
        for b in range(B):
            for k in range(int(s["kept"][b])):
                a, z = n[b] + k, n[b] + int(s["path"][b, k])
                if s["table"] is None:
                    cache[b, :, a] = s["cache"][b, :, z]
                else:
                    t = s["table"][b]
                    cache[t[a // 16], :, a % 16] = s["cache"][t[z // 16], :, z % 16]
        return dict(cache=cache)
    out = torch.zeros((B, T, H, d), dtype=f, device=DEV)
    for b in range(B):
        L = n[b] + T
        if s["table"] is None:
            rows = s["cache"][b, :, :L].to(f)
        else:
            used = s["table"][b, :-(-L // 16)].long()
            rows = s["cache"][used].transpose(0, 1).reshape(G, -1, d)[:, :L].to(f)
        sees = np.tril(np.ones((T, T), bool))
        if s["tree"] is not None:
            words = s["tree"][b].cpu().numpy().view(np.uint64)
            sees = np.array([[bool(int(w) >> k & 1) for k in range(T)] for w in words])
        depth = np.array([sees[t].sum() - sees[t, t] for t in range(T)])
        place = np.concatenate([np.arange(n[b]), n[b] + depth])
        dist = torch.from_numpy(np.abs(n[b] + depth[:, None] - place[None])).to(DEV, f)
        mask = torch.from_numpy(np.concatenate([np.ones((T, n[b]), bool), sees], 1)).to(DEV)
        for h in range(H):
            v = rows[h // R].contiguous()
            x, _ = _scores64(s["q"][b, :, h].to(f), v, cap, slope(h), dist, mask)
            out[b, :, h] = torch.softmax(x, 1) @ v
    return dict(out=out)
