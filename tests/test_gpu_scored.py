"""The scored attention (tanh cap, distance bias, document, prefix and padding masks),
forward and backward, against the 64-bit oracle, with bounds from the roundings."""

import numpy as np
import pytest
import torch

from oracle import keyless as K
from oracle import scored as S
from paper_2606_21848_amd import binding as kb
from tests.parity import assert_parity, say, to64
from tests.scored_tol import bounds, check
from workloads import synth

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = [torch.float32, torch.bfloat16]
# (cap, bias): none, the cap bending scores of a spread of three, the bias, both.
SCORES = [(0.0, False), (4.0, False), (0.0, True), (15.0, True)]
MASKS = ["causal", "full", "docs", "prefix", "padded", "ranges"]
# One token; a ragged tail of a 16-row, a 32-row, a 64-row tile; several 128-row tiles;
# one, two, three, four and six heads per group.
SHAPES = [(2, 1, 4, 1, 128), (1, 17, 6, 2, 64), (2, 64, 2, 2, 128), (1, 77, 3, 1, 64),
          (2, 200, 4, 2, 128), (1, 300, 8, 2, 64), (1, 449, 4, 4, 128)]


def ranges(mask, B, N, seed=5):
    """(first, last, causal) of a mask, as int arrays or None."""
    rs, i = np.random.RandomState(seed + N), np.arange(N)
    if mask in ("causal", "full"):
        return None, None, mask == "causal"
    first, last = np.zeros((B, N), np.int32), np.zeros((B, N), np.int32)
    for b in range(B):
        if mask == "ranges":  # anything: windows, empty rows, ends out of order and out of range
            first[b] = rs.randint(-3, N + 1, N)
            last[b] = first[b] + rs.randint(-2, N + 4, N)
            first[b, rs.randint(0, N)] = -(2 ** 31)
            last[b, rs.randint(0, N)] = 2 ** 31 - 1
            continue
        n = N - N // 5 if mask == "padded" else N
        cuts = np.sort(rs.choice(np.arange(1, n), min(3, n - 1), replace=False)) if n > 1 else []
        starts = np.concatenate([[0], cuts]).astype(int)
        ends = np.concatenate([starts[1:], [n]])
        for s, e in zip(starts, ends):
            first[b, s:e] = s
            last[b, s:e] = np.maximum(i[s:e] + 1, s + (e - s + 1) // 2 if mask == "prefix" else 0)
    return first, last, True


def case(dtype, B, N, H, G, d, seed, std=3.0):
    return (synth.normal((B, N, H, d), seed, 1, std, dtype), synth.normal((B, N, G, d), seed, 2, 1.0, dtype),
            synth.normal((B, N, H, d), seed, 3, 1.0, dtype))


def slopes_of(H):
    s = 2.0 ** (-8.0 * np.arange(1, H + 1) / H)
    s[-1] *= -0.25  # a bias may also favour the far rows
    return s.astype(np.float32)


def gpu(a, dtype=None):
    return None if a is None else torch.as_tensor(a, dtype=dtype).to(DEV)


def scoring(mask, B, N, H, cap, bias):
    first, last, causal = ranges(mask, B, N)
    sl = slopes_of(H) if bias else None
    sc = kb.Scoring(cap=cap, slopes=gpu(sl), first=gpu(first), last=gpu(last), causal=causal)
    return sc, sl, S.row_ranges(B, N, first, last, causal)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("B,N,H,G,d", SHAPES)
def test_matches_oracle(lib, dtype, mask, B, N, H, G, d):
    q, v, g = case(dtype, B, N, H, G, d, 301)
    qs, vs, gs = q.to(DEV), v.to(DEV), g.to(DEV)
    q64, v64, g64 = to64(q), to64(v), to64(g)
    for k, (cap, bias) in enumerate(SCORES):
        say(f"scored {dtype} {mask} B={B} N={N} H={H} G={G} d={d} cap={cap} bias={bias}")
        sc, sl, seen = scoring(mask, B, N, H, cap, bias)
        ref, ref_lse = S.scored_attention(q64, v64, cap, sl, seen)
        ref_dq, ref_dv = S.scored_attention_backward(q64, v64, g64, cap, sl, seen)
        tol = bounds(q64, v64, g64, cap, sl, seen, dtype == torch.bfloat16)
        # With the fp32 output kept (one way of forming rowsum(P dP)) and without.
        o32 = torch.empty(q.shape, dtype=torch.float32, device=DEV) if k % 2 == 0 else None
        out, lse = kb.keyless_scored_forward(qs, vs, sc, out_f32=o32)
        dq, dv = kb.keyless_scored_backward(qs, vs, out, gs, lse, sc, out_f32=o32)
        torch.cuda.synchronize()
        check("out", to64(out), ref, tol["out"])
        check("lse", to64(lse), ref_lse, tol["lse"])
        check("dq", to64(dq), ref_dq, tol["dq"])
        check("dv", to64(dv), ref_dv, tol["dv"])
        if o32 is not None:
            assert torch.equal(o32.to(dtype), out)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [0.0, 0.25])
def test_scale_and_outputs_given(lib, dtype, scale):
    B, N, H, G, d = 2, 130, 4, 2, 64
    say(f"scored, scale {scale}, {dtype}")
    q, v, g = case(dtype, B, N, H, G, d, 302, 1.0)
    sc, sl, seen = scoring("docs", B, N, H, 2.0, True)
    tau = scale or None
    args = [to64(x) for x in (q, v, g)]
    tol = bounds(*args, 2.0, sl, seen, dtype == torch.bfloat16, tau)
    q, v, g = q.to(DEV), v.to(DEV), g.to(DEV)
    out, lse = torch.full_like(q, float("nan")), torch.full((B, H, N), float("nan"), device=DEV)
    dq, dv = torch.full_like(q, float("nan")), torch.full_like(v, float("nan"))
    n = kb.scored_backward_workspace_bytes(B, N, H, G, d, dtype)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device=DEV)
    kb.keyless_scored_forward(q, v, sc, scale=scale, out=out, lse=lse)
    kb.keyless_scored_backward(q, v, out, g, lse, sc, scale=scale, dq=dq, dv=dv, workspace=ws)
    torch.cuda.synchronize()
    ref, ref_lse = S.scored_attention(*args[:2], 2.0, sl, seen, tau)
    check("out", to64(out), ref, tol["out"])
    check("lse", to64(lse), ref_lse, tol["lse"])
    for got, r, k in zip((dq, dv), S.scored_attention_backward(*args, 2.0, sl, seen, tau), ("dq", "dv")):
        check(k, to64(got), r, tol[k])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cap", [0.0, 8.0])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("N,H,G,d", [(140, 4, 2, 128), (70, 2, 2, 64)])
def test_what_a_row_does_not_see_never_reaches_it(lib, dtype, cap, bad, N, H, G, d):
    """A document of rows that are not finite (queries, values and output gradients)
    between two others, its ends inside tiles: the others' results are as if it were
    zeros, its own are not finite."""
    say(f"scored, {bad} in another document, {dtype}, cap {cap}, d {d}")
    a, z = 21, 50  # the bad document
    first = np.concatenate([np.zeros(a), np.full(z - a, a), np.full(N - z, z)]).astype(np.int32)[None]
    last = (np.arange(N, dtype=np.int32) + 1)[None]
    last[0, :7] = 9       # a prefix
    first[0, -3:] = last[0, -3:]  # rows that see nothing
    q, v, g = (x.to(DEV) for x in case(dtype, 1, N, H, G, d, 303))
    sc = kb.Scoring(cap=cap, first=gpu(first), last=gpu(last))
    good, bads = [x.clone() for x in (q, v, g)], [x.clone() for x in (q, v, g)]
    for x in good:
        x[:, a:z] = 0
    for x in bads:
        x[:, a:z, :, 3:5] = bad
    clean = torch.ones(N, dtype=torch.bool, device=DEV)
    clean[a:z] = False
    got = []
    for qq, vv, gg in (good, bads):
        for keep in (True, False):
            o32 = torch.empty(q.shape, dtype=torch.float32, device=DEV) if keep else None
            out, lse = kb.keyless_scored_forward(qq, vv, sc, out_f32=o32)
            dq, dv = kb.keyless_scored_backward(qq, vv, out, gg, lse, sc, out_f32=o32)
            torch.cuda.synchronize()
            got.append((out, lse.transpose(1, 2), dq, dv))
    for r in (0, 1):
        for x, y in zip(got[r], got[2 + r]):
            assert torch.equal(x[:, clean], y[:, clean])
            assert torch.isfinite(x[:, clean][torch.isfinite(y[:, clean])]).all()
        assert not torch.isfinite(got[2 + r][0][:, a:z, :, 3:5]).any()
    # A query row that is not finite spoils its own results only.
    only_q = good[0].clone()
    only_q[:, -3:] = bad
    out, lse = kb.keyless_scored_forward(only_q, good[1], sc)
    dq, dv = kb.keyless_scored_backward(only_q, good[1], out, good[2], lse, sc)
    torch.cuda.synchronize()
    assert torch.equal(dv, got[1][3]) and torch.equal(out, got[1][0])


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_of_any_size(lib, dtype):
    """Scores far above and below the exponential's range, with and without the cap:
    the softmax statistics hold them, one row wins."""
    B, N, H, G, d = 1, 150, 2, 1, 64
    say(f"scored, large scores, {dtype}")
    q, v, g = case(dtype, B, N, H, G, d, 304, 300.0)
    sl = np.array([0.5, -2.0], np.float32)
    for cap in (0.0, 500.0):
        sc = kb.Scoring(cap=cap, slopes=gpu(sl))
        out, lse = kb.keyless_scored_forward(q.to(DEV), v.to(DEV), sc)
        dq, dv = kb.keyless_scored_backward(q.to(DEV), v.to(DEV), out, g.to(DEV), lse, sc)
        torch.cuda.synchronize()
        args = [to64(x) for x in (q, v, g)]
        seen = S.row_ranges(B, N)
        tol = bounds(*args, cap, sl, seen, dtype == torch.bfloat16)
        ref, ref_lse = S.scored_attention(*args[:2], cap, sl, seen)
        rdq, rdv = S.scored_attention_backward(*args, cap, sl, seen)
        for what, x, r in (("out", out, ref), ("lse", lse, ref_lse), ("dq", dq, rdq), ("dv", dv, rdv)):
            check(what, to64(x), r, tol[what])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("causal", [True, False])
def test_without_changes_it_is_the_attention(lib, dtype, causal):
    """No cap, bias or mask: the gradients of keyless_attention_forward / _backward."""
    B, N, H, G, d = 2, 333, 6, 3, 128
    say(f"scored against the unscored attention {dtype} causal={causal}")
    q, v, g = (x.to(DEV) for x in case(dtype, B, N, H, G, d, 305, 1.0))
    sc = kb.Scoring(causal=causal)
    out, lse = kb.keyless_scored_forward(q, v, sc)
    dq, dv = kb.keyless_scored_backward(q, v, out, g, lse, sc)
    o2, l2 = kb.keyless_attention_forward(q, v, causal=causal)
    dq2, dv2 = kb.keyless_attention_backward(q, v, o2, g, l2, causal=causal)
    torch.cuda.synchronize()
    for a, b in ((out, o2), (dq, dq2), (dv, dv2)):
        assert_parity(a, to64(b), dtype, "scored", 1e-2)
    assert (lse - l2).abs().max() < 2e-2


def test_explicit_ranges_equal_the_defaults(lib):
    B, N, H, G, d = 2, 210, 4, 2, 128
    q, v, g = (x.to(DEV) for x in case(torch.bfloat16, B, N, H, G, d, 306))
    i = torch.arange(N, dtype=torch.int32, device=DEV).expand(B, N).contiguous()
    zero = torch.zeros_like(i)
    for a, b in ((kb.Scoring(5.0), kb.Scoring(5.0, first=zero, last=i + 1, causal=False)),
                 (kb.Scoring(5.0, causal=False), kb.Scoring(5.0, last=zero + N)),
                 (kb.Scoring(5.0), kb.Scoring(5.0, first=zero - 9))):
        got = []
        for sc in (a, b):
            out, lse = kb.keyless_scored_forward(q, v, sc)
            got.append((out, lse, *kb.keyless_scored_backward(q, v, out, g, lse, sc)))
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(*got))


@pytest.mark.parametrize("dtype,B,N,H,G,d", [(torch.bfloat16, 1, 700, 8, 2, 128), (torch.float32, 2, 90, 4, 1, 64)])
def test_is_deterministic(lib, dtype, B, N, H, G, d):
    say("scored determinism")
    q, v, g = (x.to(DEV) for x in case(dtype, B, N, H, G, d, 307))
    sc, _, _ = scoring("docs", B, N, H, 10.0, True)
    got = []
    for _ in range(3):
        out, lse = kb.keyless_scored_forward(q, v, sc)
        got.append((out, lse, *kb.keyless_scored_backward(q, v, out, g, lse, sc)))
        torch.cuda.synchronize()
    for other in got[1:]:
        assert all(torch.equal(x, y) for x, y in zip(got[0], other))


def test_a_whole_layer_of_training(lib):
    """x -> routed queries and values -> scored attention -> its gradients -> the weight
    gradients: the calls in the order a training step makes them, on packed documents."""
    B, N, dm, H, G, d = 2, 150, 256, 4, 2, 64
    say("scored layer")
    x = synth.normal((B, N, dm), 308, 1, 1.0, torch.float32)
    wq = synth.normal((dm, H * d), 308, 2, dm ** -0.5, torch.float32)
    wr = synth.normal((H, d, d), 308, 3, d ** -0.5, torch.float32)
    wv = synth.normal((dm, G * d), 308, 4, dm ** -0.5, torch.float32)
    g = synth.normal((B, N, H, d), 308, 5, 1.0, torch.float32)
    sc, sl, seen = scoring("docs", B, N, H, 3.0, True)
    xs, a, r, b, gs = (t.to(DEV) for t in (x, wq, wr, wv, g))
    _, q, v = kb.keyless_prefill(xs, a, r, b, H, G, return_qv=True)
    out, lse = kb.keyless_scored_forward(q, v, sc)
    dq, dv = kb.keyless_scored_backward(q, v, out, gs, lse, sc)
    grads = kb.keyless_weight_gradients(xs, a, r, b, dq, dv, H, G)
    torch.cuda.synchronize()
    x64, wq64, wr64, wv64 = (to64(t) for t in (x, wq, wr, wv))
    q64 = np.stack([x64 @ wq64[:, h * d:(h + 1) * d] @ wr64[h] for h in range(H)], 2)
    v64 = (x64 @ wv64).reshape(B, N, G, d)
    assert_parity(out, S.scored_attention(q64, v64, 3.0, sl, seen)[0], torch.float32, "out")
    rq, rv = S.scored_attention_backward(q64, v64, to64(g), 3.0, sl, seen)
    ref = K.keyless_projection_gradients(x64, wq64, wr64, wv64, rq, rv, H, G, d)
    for k in ("dW_Q", "dW_R", "dW_V", "dX"):
        assert_parity(grads[k], ref[k], torch.float32, k, 1e-2)


@pytest.mark.parametrize("dtype", TYPES)
def test_on_another_stream_and_in_a_graph(lib, dtype):
    """The calls run on the caller's stream; captured, every replay equals the eager
    calls on the same inputs, with eager work between the replays."""
    B, N, H, G, d = 2, 260, 4, 2, 128
    say(f"scored, streams and graphs {dtype}")
    q, v, g = (x.to(DEV) for x in case(dtype, B, N, H, G, d, 309))
    sc, _, _ = scoring("padded", B, N, H, 10.0, True)
    ws = torch.empty(kb.scored_backward_workspace_bytes(B, N, H, G, d, dtype), dtype=torch.uint8, device=DEV)
    bufs = [torch.empty_like(q), torch.empty((B, H, N), device=DEV), torch.empty_like(q), torch.empty_like(v)]
    o32 = torch.empty(q.shape, device=DEV)

    def step():
        kb.keyless_scored_forward(q, v, sc, out=bufs[0], lse=bufs[1], out_f32=o32)
        kb.keyless_scored_backward(q, v, bufs[0], g, bufs[1], sc, dq=bufs[2], dv=bufs[3], workspace=ws,
                                   out_f32=o32)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for rep in range(3):
        for t, k in ((q, 1), (v, 2), (g, 3)):
            t.copy_(synth.normal(tuple(t.shape), 310 + rep, k, 1.0, dtype))
        ref32 = torch.empty_like(o32)
        out, lse = kb.keyless_scored_forward(q, v, sc, out_f32=ref32)
        dq, dv = kb.keyless_scored_backward(q, v, out, g, lse, sc, out_f32=ref32)
        torch.cuda.synchronize()
        ws.fill_(0xFF)
        graph.replay()
        torch.cuda.synchronize()
        same = [bool(torch.equal(a, b)) for a, b in zip(bufs, (out, lse, dq, dv))]
        assert all(same), f"replay {rep}"


def test_a_long_sequence_by_rows(lib):
    """Rows of a long sequence (more than one tile everywhere, few documents) against
    the oracle's softmax of those rows; bf16, grouped heads."""
    B, N, H, G, d, cap = 1, 9001, 6, 2, 128, 30.0
    say("scored, long sequence")
    q, v, g = case(torch.bfloat16, B, N, H, G, d, 320)
    first = np.where(np.arange(N) < 5003, 0, 5003).astype(np.int32)[None]
    last = np.maximum(np.arange(N) + 1, 700).astype(np.int32)[None]
    sl = slopes_of(H) * 0.05
    sc = kb.Scoring(cap=cap, slopes=gpu(sl), first=gpu(first), last=gpu(last))
    qs, vs, gs = q.to(DEV), v.to(DEV), g.to(DEV)
    o32 = torch.empty(q.shape, dtype=torch.float32, device=DEV)
    out, lse = kb.keyless_scored_forward(qs, vs, sc, out_f32=o32)
    dq, dv = kb.keyless_scored_backward(qs, vs, out, gs, lse, sc, out_f32=o32)
    torch.cuda.synchronize()
    q64, v64, g64 = to64(q)[0], to64(v)[0], to64(g)[0]
    tau = d ** -0.5
    for i in (0, 699, 700, 5002, 5003, 7777, 9000):
        for h in (0, 5):
            V = v64[first[0, i]:last[0, i], h // 3]
            pos = np.arange(first[0, i], last[0, i])
            x, bend = S.scores(q64[i, h][None], V, tau, cap, sl[h], np.abs(i - pos)[None])
            P, l = S.masked_softmax(x, np.ones_like(x, bool))
            # Weights rounded by 2^-8 each; scores off by 2^-21 cap and (2 D + 8) 2^-24 S < 1e-3.
            o = (P @ V)[0]
            tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -8 + 3e-3) * (P @ np.abs(V))[0]
            assert (np.abs(to64(out)[0, i, h] - o) <= tol).all(), (i, h)
            assert abs(float(lse[0, h, i]) - l[0]) <= 2e-3
            dP = g64[i, h] @ V.T
            dz = P[0] * bend[0] * (dP - P[0] @ dP)
            C = np.abs(g64[i, h]) @ np.abs(V).T
            ez = P[0] * (2.0 ** -8 + 3e-3) * (P[0] @ C) + (2.0 ** -8 + 3e-3) * np.abs(dz)
            ref = tau * (dz @ V)
            assert (np.abs(to64(dq)[0, i, h] - ref) <= 2.0 ** -8 * np.abs(ref) + tau * (ez @ np.abs(V))).all()
    # dV by differences of a random direction: the loss along it, from the fp32 output.
    # (The forward's own rounding of the weights, 2^-8 of each, is noise of less than
    # 2^-8 sqrt(sum of squares); the check is of the sum over all rows and heads.)
    ref_dv = np.zeros((2, d))
    rows = (5003 + 64, 650)
    for k, j in enumerate(rows):
        for h in range(3):
            sees = np.nonzero((first[0] <= j) & (j < last[0]))[0]
            zj = tau * (q64[sees, h] @ v64[j, 0])
            t = np.tanh(zj / cap)
            p = np.exp(cap * t - sl[h] * np.abs(sees - j) - to64(lse)[0, h, sees])
            dd = np.sum(to64(o32)[0, sees, h] * g64[sees, h], 1)
            dz = p * (1 - t * t) * (g64[sees, h] @ v64[j, 0] - dd)
            ref_dv[k] += p @ g64[sees, h] + tau * (dz @ q64[sees, h])
    got = to64(dv)[0, list(rows), 0]
    assert np.linalg.norm(got - ref_dv) <= 3 * 2.0 ** -8 * np.linalg.norm(ref_dv)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("bias", [False, True])
def test_the_largest_cap(lib, dtype, bias):
    """A cap of 1024, the most that bf16 takes: nearly straight scores, formed as a small
    difference of large numbers."""
    B, N, H, G, d = 1, 210, 4, 2, 128
    say(f"scored, cap 1024, bias {bias}, {dtype}")
    q, v, g = case(dtype, B, N, H, G, d, 331)
    sc, sl, seen = scoring("docs", B, N, H, 1024.0, bias)
    args = [to64(x) for x in (q, v, g)]
    tol = bounds(*args, 1024.0, sl, seen, dtype == torch.bfloat16)
    q, v, g = q.to(DEV), v.to(DEV), g.to(DEV)
    out, lse = kb.keyless_scored_forward(q, v, sc)
    dq, dv = kb.keyless_scored_backward(q, v, out, g, lse, sc)
    torch.cuda.synchronize()
    ref, ref_lse = S.scored_attention(*args[:2], 1024.0, sl, seen)
    check("out", to64(out), ref, tol["out"])
    check("lse", to64(lse), ref_lse, tol["lse"])
    for got, r, k in zip((dq, dv), S.scored_attention_backward(*args, 1024.0, sl, seen), ("dq", "dv")):
        check(k, to64(got), r, tol[k])


def test_the_kept_fp32_output_changes_nothing_in_bf16(lib):
    """The row sums of the bf16 backward start from the output alone, and what its rounding
    takes from them is added on the way: dQ~ is about as exact as its own rounding, sqrt(2)
    of it with that of dz, and so below 1.6 of it."""
    B, N, H, G, d = 1, 700, 4, 2, 128
    say("scored, fp32 output kept and not")
    q, v, g = case(torch.bfloat16, B, N, H, G, d, 332)
    args = [to64(x) for x in (q, v, g)]
    q, v, g = q.to(DEV), v.to(DEV), g.to(DEV)
    for cap in (0.0, 5.0, 50.0):
        sc, sl, seen = scoring("causal", B, N, H, cap, False)
        o32 = torch.empty(q.shape, dtype=torch.float32, device=DEV)
        out, lse = kb.keyless_scored_forward(q, v, sc, out_f32=o32)
        a = kb.keyless_scored_backward(q, v, out, g, lse, sc)
        b = kb.keyless_scored_backward(q, v, out, g, lse, sc, out_f32=o32)
        torch.cuda.synchronize()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
        ref = S.scored_attention_backward(*args, cap, sl, seen)[0]
        own = torch.from_numpy(ref).to(torch.bfloat16).double().numpy()
        assert np.linalg.norm(to64(a[0]) - ref) <= 1.6 * np.linalg.norm(own - ref)
