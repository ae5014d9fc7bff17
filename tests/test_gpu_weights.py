"""Accumulated attention weights against 64 bits: prompt queries over a cache,
decode steps; and what the calls must leave alone."""
import math

import numpy as np
import pytest
import torch

import op_refs as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def P():
    from paper_2310_08152_amd import path
    return path


def B():
    from paper_2310_08152_amd import binding
    return binding


class Held:
    """A cache of one layer whose rows hold given tokens."""

    def __init__(self, b, H, cap, d, dt, T, spans, rows, seed, nq, scale_q=1.0):
        self.spans, self.rows, self.T = spans, rows, T
        self.meta = P().SpanMeta(spans, T, DEV)
        self.cache = c = P().KVCache(1, b, H, cap, d, dt, DEV)
        c.kv.copy_(R.rand(c.kv.shape, seed, dt))
        c.kv_len.copy_(torch.tensor([len(r) for r in rows]))
        for s, r in enumerate(rows):
            c.tok_idx[s, :len(r)] = torch.as_tensor(np.asarray(r), dtype=torch.int32)
        c.track_weights()
        self.ws = P().Workspace(b, H, 1, cap, d, DEV, weights=max(nq, 1))
        self.q = R.rand((b, H, nq, d), seed + 1, dt, scale_q, DEV)

    def check(self, got, w_in, tok0, scale=None):
        """got[s, :, r] against w_in + the sums, within the derived bound."""
        c, nq, d = self.cache, self.q.shape[2], self.q.shape[3]
        for s, r in enumerate(self.rows):
            vu = R.vu_pos(self.spans[s], self.T)[0]
            want, rel = R.prompt_weights(self.q[s].cpu(), c.k(0)[s, :, :len(r)].cpu(), r,
                                         range(tok0, tok0 + nq), vu, scale or d ** -0.5)
            base = w_in[s, :, :len(r)].double().cpu()
            err = (got[s, :, :len(r)].double().cpu() - base - want).abs()
            tol = want * rel + (want + base.abs()) * 2 * R.U + nq * 2.0 ** -126
            assert not (err > tol).any(), (s, float(err.max()), float((err - tol).max()), rel)


def kept(spans, T, upto):
    vu = R.vu_pos(spans, T)[0]
    return [t for t in range(upto) if vu[t] != t and vu[t] >= upto]


CASES = [
    # b, H, d, dtype, prompt, queries (last), compacted, spans' ratio
    (1, 1, 64, "bf16", 1, 1, False, 0.0),
    (1, 2, 80, "f32", 2, 2, False, 0.0),
    (2, 3, 64, "bf16", 31, 31, False, 0.5),
    (2, 2, 80, "bf16", 64, 33, False, 0.3),
    (1, 3, 80, "bf16", 130, 130, False, 0.7),
    (3, 2, 64, "f32", 97, 97, False, 0.5),
    (2, 2, 64, "bf16", 300, 1, True, 0.5),
    (2, 3, 80, "bf16", 517, 32, True, 0.6),
    (1, 2, 64, "bf16", 1025, 1025, False, 0.4),
    (2, 1, 80, "f32", 700, 65, True, 0.5),
    (1, 1, 64, "bf16", 3000, 129, True, 0.1),
    (4, 64, 64, "bf16", 530, 530, False, 0.5),    # two tiles of queries and of rows a wave
    (4, 64, 80, "bf16", 300, 131, True, 0.4),
    (1, 64, 64, "bf16", 4100, 2100, False, 0.6),  # staged
    (1, 110, 80, "f32", 4100, 1030, True, 0.2),
    (1, 64, 64, "bf16", 4091, 2100, False, 0.4),  # ... one tile of rows a wave
    (1, 205, 64, "bf16", 4100, 1025, True, 0.4),  # ... two of queries
    (1, 205, 80, "bf16", 4100, 1025, False, 0.5),
    (1, 110, 80, "bf16", 4100, 1250, False, 0.3),
    (40, 13, 64, "bf16", 520, 5, False, 0.3),     # two tiles of rows, one of queries
    (3, 100, 80, "f32", 260, 45, False, 0.5),
]


@pytest.mark.parametrize("b,H,d,dtype,L,nq,compacted,ratio", CASES)
def test_prompt_weights(b, H, d, dtype, L, nq, compacted, ratio):
    print("weights", b, H, d, dtype, L, nq, compacted, ratio, flush=True)
    spans = [R.some_spans(L, 5 + s, ratio) if ratio else [] for s in range(b)]
    rows = [kept(spans[s], L, L) if compacted else list(range(L)) for s in range(b)]
    cap = L + 5
    h = Held(b, H, cap, d, DT[dtype], L, spans, rows, 21, nq)
    w_in = R.rand((b, H, cap), 9, torch.float32, device=DEV).abs() * (nq / L)
    out = torch.full_like(w_in, 5.0)
    P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, L - nq, w_in, out)
    h.check(out, w_in, L - nq)
    for s, r in enumerate(rows):
        assert bool((out[s, :, len(r):] == 5.0).all())
    again = torch.zeros_like(out)
    P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, L - nq, w_in, again)
    for s, r in enumerate(rows):
        assert torch.equal(again[s, :, :len(r)], out[s, :, :len(r)])  # equal bits
    # in place, and from zeros
    P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, L - nq, w_in, w_in)
    for s, r in enumerate(rows):
        assert torch.equal(w_in[s, :, :len(r)], out[s, :, :len(r)])
    P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, L - nq, None, again)
    h.check(again, torch.zeros_like(again), L - nq)


def test_queries_in_the_middle_and_row_order():
    """Rows later than a query give and get nothing; rows in any order, rows of
    no token, unequal lengths, an empty cache, a length beyond the capacity."""
    print("weights middle", flush=True)
    b, H, d, T, nq, tok0, cap = 4, 2, 64, 400, 70, 100, 300
    spans = [R.some_spans(T, 3 + s) for s in range(b)]
    rng = np.random.default_rng(1)
    rows = [list(rng.permutation(T)[:cap]), list(range(150, 290)), [], list(range(0, 60))]
    rows[3][7], rows[3][9], rows[3][11] = -1, T, 2 ** 31 - 1
    h = Held(b, H, cap, d, torch.bfloat16, T, spans, rows, 4, nq)
    h.cache.kv_len[0] = cap + 50  # clamped to the capacity
    out = torch.full((b, H, cap), 2.0, device=DEV)
    P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, tok0, None, out)
    h.check(out, torch.zeros_like(out), tok0)
    assert bool((out[2] == 2.0).all())
    h.cache.kv_len[2] = -5
    P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, tok0, None, out)
    assert bool((out[2] == 2.0).all())


def test_no_visible_row_gives_nothing():
    """Every query's rows are masked: all keys later, or all enclosed and closed."""
    print("weights empty rows", flush=True)
    b, H, d, T = 2, 2, 80, 100
    spans = [[], [(2, 50)]]
    rows = [list(range(60, 90)), list(range(3, 40))]
    h = Held(b, H, 40, d, torch.bfloat16, T, spans, rows, 4, 5)
    out = torch.full((b, H, 40), 2.0, device=DEV)
    P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, 55, None, out)
    assert bool((out[0, :, :30] == 0).all()) and bool((out[1, :, :37] == 0).all())
    none = h.q[:, :, :0]
    w = torch.ones_like(out)
    P().prompt_weights(none, h.cache, 0, h.meta, h.ws, 55, w, out)
    assert bool((out[0, :, :30] == 1).all()) and bool((out[0, :, 30:] == 2).all())


def test_large_scores_and_masked_infinities():
    """Scores over hundreds of powers of two; infinities and NaN in rows that no
    query sees do not reach the others."""
    print("weights range", flush=True)
    b, H, d, L = 1, 2, 64, 200
    spans = [[(20, 60), (100, 140)]]
    h = Held(b, H, L, d, torch.float32, L, spans, [list(range(L))], 8, 50, scale_q=20.0)
    hidden = list(range(21, 60)) + list(range(101, 140)) + [20, 100]
    h.cache.kv[0, 0, 0, :, hidden[:30]] = float("inf")
    h.cache.kv[0, 0, 0, :, hidden[30:]] = float("nan")
    out = torch.zeros(b, H, L, device=DEV)
    P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, L - 50, None, out)
    assert bool((out[0, :, hidden] == 0).all())
    h.cache.kv[0, 0, 0, :, hidden] = 0
    h.check(out, torch.zeros_like(out), L - 50)


def test_strided_queries_other_scale_and_sharp_ties():
    print("weights strides", flush=True)
    b, H, d, L, nq = 2, 3, 80, 150, 40
    spans = [R.some_spans(L, s) for s in range(b)]
    h = Held(b, H, L, d, torch.bfloat16, L, spans, [list(range(L))] * b, 8, nq)
    wide = torch.zeros(b, H, L, d, dtype=torch.bfloat16, device=DEV)
    wide[:, :, L - nq:] = h.q
    out = torch.zeros(b, H, L, device=DEV)
    P().prompt_weights(wide[:, :, L - nq:], h.cache, 0, h.meta, h.ws, L - nq, None, out, scale=0.7)
    h.check(out, torch.zeros_like(out), L - nq, scale=0.7)
    h.cache.kv.zero_()  # all scores equal
    P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, L - nq, None, out)
    h.check(out, torch.zeros_like(out), L - nq)


@pytest.mark.parametrize("nq,H,L", [(5, 2, 300), (90, 3, 300), (64, 90, 700)])
def test_prompt_weights_graph_and_stream(nq, H, L):
    """A side stream and replays of a graph give the eager bits; another call on
    the same workspace runs between the replays."""
    print("weights graph", nq, H, L, flush=True)
    b, d = 2, 64
    spans = [R.some_spans(L, s) for s in range(b)]
    h = Held(b, H, L, d, torch.bfloat16, L, spans, [list(range(L))] * b, 8, nq)
    w_in = R.rand((b, H, L), 3, torch.float32, device=DEV)
    outs = [torch.zeros_like(w_in) for _ in range(3)]
    call = lambda o, q=h.q: P().prompt_weights(q, h.cache, 0, h.meta, h.ws, L - nq, w_in, o)
    call(outs[0])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        call(outs[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], outs[1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(outs[2])
    for _ in range(3):
        outs[2].zero_()
        call(outs[1], -h.q)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2])


# ---------------------------------------------------------------------------
# decode steps
# ---------------------------------------------------------------------------

def decode_state(b, H, d, dt, cap, lens, seed, T=None, spans=None):
    T = T or cap + 20
    spans = spans or [[] for _ in range(b)]
    meta = P().SpanMeta(spans, T, DEV)
    cache = P().KVCache(2, b, H, cap, d, dt, DEV)
    cache.kv.copy_(R.rand(cache.kv.shape, seed, dt))
    cache.kv_len.copy_(torch.tensor(lens))
    cache.cur_tok.copy_(torch.tensor([max(0, min(n + 3, T - 1)) for n in lens]))
    cache.track_weights()
    cache.w.copy_(R.rand(cache.w.shape, seed + 1, torch.float32).abs())
    ws = P().Workspace(b, H, 1, cap, d, DEV, weights=1)
    qkv = [R.rand((b, H, d), seed + 2 + i, dt, device=DEV) for i in range(3)]
    return meta, cache, ws, qkv, T, spans


def check_decode(cache, before, w_before, qkv, o, w, s, meta_pos, theta, dt, split_q):
    """Sequence s of layer 1 against 64 bits."""
    d = cache.d
    n, t = int(cache.kv_len[s]), int(cache.cur_tok[s])
    q, k, v = (x[s].cpu().double() for x in qkv)
    pos = meta_pos[t:t + 1]
    q, kr = (R.rotate(x[:, None], pos, theta)[:, 0] for x in (q, k))
    row = cache.k(1)[s, :, n].cpu().double()
    # the stored key: angle, sine and cosine, two products, one rounding
    tol = 16 * R.U * k.abs().amax(-1, keepdim=True) * 2
    assert bool(((row - kr).abs() <= tol + R.half_step(dt) * (kr.abs() + tol)).all())
    assert torch.equal(cache.v(1)[s, :, n].cpu(), qkv[2][s].cpu())
    kk = torch.cat([before[0][s, :, :n].double(), row[:, None]], 1)
    vv = torch.cat([before[1][s, :, :n].double(), v[:, None]], 1)
    ow, p, A, pv = R.attend(q, kk, vv, d ** -0.5)
    # scores: d products in fp32, the query's own rounding (16 U from the
    # rotation, and its two bf16 terms' 2^-17), distance from the maximum; sums
    rel = 2 * A * ((d + 24) * R.U + split_q) + (n + 32) * R.U
    err = (o[s].double().cpu() - ow).abs()
    assert bool((err <= pv * rel + R.half_step(dt) * (ow.abs() + pv * rel)).all()), float(err.max())
    base = torch.cat([w_before[s, :, :n].double(), torch.zeros(cache.H, 1, dtype=torch.float64)], 1)
    err = (w[s, :, :n + 1].double().cpu() - base - p).abs()
    tol = p * rel + (base + p) * 2 * R.U + 2.0 ** -126
    assert not (err > tol).any(), (float(err.max()), float((err - tol).max()))


DECODE = [
    # b, H, d, dtype, capacity, lengths, theta
    (1, 1, 64, "bf16", 1, [0], 1e4),
    (1, 2, 80, "f32", 4, [3], 1e4),
    (3, 4, 64, "bf16", 70, [0, 69, 33], 0.0),
    (2, 3, 80, "bf16", 1700, [1699, 40], 1e4),     # few slices, split
    (1, 5, 64, "bf16", 3300, [2900], 1e4),         # split, several chunks of each wave
    (2, 40, 80, "bf16", 600, [599, 0], 1e4),       # one workgroup a slice
    (18, 32, 80, "bf16", 260, None, 1e4),          # 576 slices
    (70, 32, 64, "bf16", 90, None, 1e4),           # one wave a slice
    (2, 2, 64, "f32", 2500, [2499, 1200], 1e4),    # fp32, split
    (20, 32, 80, "f32", 130, None, 0.0),           # fp32, one workgroup a slice
    (40, 32, 64, "f32", 50, None, 1e4),            # fp32, narrow
    (1, 520, 64, "bf16", 16384, [16000], 1e4),     # the most scores kept in LDS
    (1, 520, 64, "bf16", 16500, [16400], 0.0),     # one workgroup a slice, scores in memory
]


@pytest.mark.parametrize("b,H,d,dtype,cap,lens,theta", DECODE)
def test_decode_weights(b, H, d, dtype, cap, lens, theta):
    print("decode weights", b, H, d, dtype, cap, lens, theta, flush=True)
    dt = DT[dtype]
    if lens is None:
        lens = np.random.default_rng(b).integers(0, cap, size=b).tolist()
    meta, cache, ws, qkv, T, spans = decode_state(b, H, d, dt, cap, lens, 31)
    before, w_before = cache.kv[1].cpu(), cache.w[1].cpu()
    ref = P().KVCache(2, b, H, cap, d, dt, DEV, kv=cache.kv.clone())
    ref.kv_len.copy_(cache.kv_len)
    ref.cur_tok.copy_(cache.cur_tok)
    o, o_ref = (torch.empty(b, H, d, dtype=dt, device=DEV) for _ in range(2))
    out = torch.full_like(cache.w[1], -3.0)
    P().decode_weights_layer(*qkv, cache, 1, meta, ws, o, cache.w[1], out, theta=theta)
    P().decode_layer(*qkv, ref, 1, meta, ws, o_ref, theta=theta)
    pos = meta.pos.cpu().numpy()
    some = range(b) if b < 8 else [0, 1, b // 2, b - 1]
    for s in some:
        check_decode(cache, before, w_before, qkv, o, out, s, pos[s], theta, dt,
                     2.0 ** -17 if dtype == "bf16" else 0.0)
    for s in range(b):
        assert bool((out[s, :, lens[s] + 1:] == -3.0).all())
    # the other rows are left alone, and the new ones are decode_layer's to one
    # rounding (its rotation is in 32 bits)
    other = ref.kv.clone()
    for s in range(b):
        a, c = (x[1, 0, s, :, lens[s]].double() for x in (cache.kv, ref.kv))
        assert bool(((a - c).abs() <= 2.5 * R.half_step(dt) * c.abs() + 64 * R.U).all())
        other[1, 0, s, :, lens[s]] = cache.kv[1, 0, s, :, lens[s]]
    assert torch.equal(cache.kv, other)
    assert int(cache.status[0]) == 0
    assert torch.equal(cache.w[1].cpu(), w_before)
    # in place on the cache's sums
    P().decode_weights_layer(*qkv, cache, 1, meta, ws, o_ref, theta=theta)
    assert torch.equal(o, o_ref)
    for s in range(b):
        assert torch.equal(cache.w[1, s, :, :lens[s] + 1], out[s, :, :lens[s] + 1])


@pytest.mark.parametrize("cap,b,H", [(80, 4, 3), (2000, 4, 3), (80, 4, 150)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_decode_weights_special_steps(cap, b, H, dtype):
    """A <CL> step and failed ones add nothing; the others go on."""
    print("decode weights special", cap, b, H, dtype, flush=True)
    dt, d = DT[dtype], 64
    lens = [20, cap, 30, 40]
    spans = [[(23, 30)], [], [], []]
    meta, cache, ws, qkv, T, _ = decode_state(b, H, d, dt, cap, lens, 3, spans=spans)
    cache.cur_tok[2] = T
    before, w_before = cache.kv[1].cpu(), cache.w[1].cpu()
    o = torch.empty(b, H, d, dtype=dt, device=DEV)
    out = torch.full_like(cache.w[1], -3.0)
    P().decode_weights_layer(*qkv, cache, 1, meta, ws, o, cache.w[1], out, theta=1e4)
    assert int(cache.status[0]) == B().STATUS_CAP | B().STATUS_TOKEN
    assert torch.equal(o[0], qkv[2][0]) and bool(o[1:3].isnan().all())
    for s in range(3):
        n = min(lens[s], cap)
        assert torch.equal(out[s, :, :n].cpu(), w_before[s, :, :n])
        assert bool((out[s, :, n:] == -3.0).all())
        assert torch.equal(cache.kv[1, :, s].cpu(), before[:, s])
    check_decode(cache, before, w_before, qkv, o, out, 3, meta.pos[3].cpu().numpy(), 1e4, dt,
                 2.0 ** -17 if dtype == "bf16" else 0.0)
    P().decode_weights_layer(*qkv, cache, 1, meta, ws, o, None, out, theta=1e4)
    assert bool((out[0, :, :20] == 0).all())


def test_offsets_beyond_32_bits():
    """A cache of more than 2^31 elements: the last slices' rows and sums."""
    print("decode weights far offsets", flush=True)
    b, H, cap, d, n = 1, 33, 1 << 20, 64, 150
    meta = P().SpanMeta([[]], 200, DEV)
    kv = torch.empty(1, 2, b, H, cap, d, dtype=torch.bfloat16, device=DEV)
    cache = P().KVCache(1, b, H, cap, d, torch.bfloat16, DEV, kv=kv)
    kv[:, :, :, :, :n + 2] = R.rand((1, 2, b, H, n + 2, d), 3, torch.bfloat16, device=DEV)
    before = kv[0, :, :, :, :n + 2].cpu()
    cache.kv_len.fill_(n)
    cache.cur_tok.fill_(n)
    w_in = torch.ones(b, H, cap, device=DEV)
    out = torch.empty(b, H, cap, device=DEV)
    ws = P().Workspace(b, H, 1, cap, d, DEV, weights=1)
    qkv = [R.rand((b, H, d), i, torch.bfloat16, device=DEV) for i in range(3)]
    o = torch.empty(b, H, d, dtype=torch.bfloat16, device=DEV)
    P().decode_weights_layer(*qkv, cache, 0, meta, ws, o, w_in, out)
    k, v = before[0, 0, :, :n + 1].clone(), before[1, 0, :, :n + 1].clone()
    k[:, n], v[:, n] = qkv[1][0].cpu(), qkv[2][0].cpu()
    want, p, _, _ = R.attend(qkv[0][0].cpu(), k, v, d ** -0.5)
    assert float((o[0].cpu().double() - want).abs().max()) < 2e-2
    p[:, :n] += 1
    assert float((out[0, :, :n + 1].cpu().double() - p).abs().max()) < 1e-5
    assert torch.equal(kv[0, :, 0, :, n + 1].cpu(), before[:, 0, :, n + 1])


@pytest.mark.parametrize("b,H,cap", [(2, 3, 1500), (3, 200, 100)])
def test_decode_weights_in_a_graph(b, H, cap):
    """Captured steps that share a workspace add up like eager ones."""
    print("decode weights graph", b, H, cap, flush=True)
    d, dt = 80, torch.bfloat16
    lens = [cap // 2, 7, cap - 10][:b]
    states = [decode_state(b, H, d, dt, cap, lens, 3) for _ in range(2)]
    outs = []
    for i, (meta, cache, ws, qkv, _, _) in enumerate(states):
        o = torch.empty(2, b, H, d, dtype=dt, device=DEV)

        def step():
            for m in range(2):
                P().decode_weights_layer(*qkv, cache, m, meta, ws, o[m], theta=1e4)
            cache.commit(meta)

        if i == 0:
            for _ in range(3):
                step()
        else:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                step()
            for _ in range(3):
                g.replay()
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        outs.append((o, cache.w.clone(), cache.kv_len.clone()))
    for a, c in zip(*outs):
        assert torch.equal(a, c)


def test_workspace_of_more_queries():
    """Calls of fewer queries than the workspace was made for."""
    print("weights workspace", flush=True)
    b, H, d, L = 1, 4, 64, 3000
    spans = [R.some_spans(L, 3)]
    h = Held(b, H, L, d, torch.bfloat16, L, spans, [list(range(L))], 8, 33)
    for n in (33, 32, 5, 1):
        out = torch.zeros(b, H, L, device=DEV)
        h.q = h.q[:, :, -n:]
        P().prompt_weights(h.q, h.cache, 0, h.meta, h.ws, L - n, None, out)
        h.check(out, torch.zeros_like(out), L - n)


@pytest.mark.parametrize("d", (64, 80))
def test_stored_key_is_plain_arithmetic(d):
    """The new bf16 key: sine and cosine in 64 bits, rounded once; products and
    sum in fp32, each rounded; the same bits, at far positions too."""
    print("weights key", d, flush=True)
    b, H, T = 9, 32, 9000
    toks = [0, 1, 7, 100, 1023, 2048, 5000, 8191, 8999]
    h = Held(b, H, 64, d, torch.bfloat16, T, [[] for _ in range(b)], [[0]] * b, 3, 1)
    c = h.cache
    c.cur_tok.copy_(torch.tensor(toks))
    q, k, v = (R.rand((b, H, d), 5 + i, torch.bfloat16, 1.0, DEV) for i in range(3))
    o = torch.empty_like(q)
    P().decode_weights_layer(q, k, v, c, 0, h.meta, h.ws, o, theta=1e4)
    a = torch.tensor(toks, dtype=torch.float64)[:, None, None] * \
        1e4 ** (-torch.arange(d // 2, dtype=torch.float64) / (d // 2))
    cs, sn, x = a.cos().float(), a.sin().float(), k.cpu().float()
    x1, x2 = x[..., :d // 2], x[..., d // 2:]
    want = torch.cat([x1 * cs - x2 * sn, x2 * cs + x1 * sn], -1).bfloat16()
    assert torch.equal(c.k(0)[:, :, 1].cpu(), want)
