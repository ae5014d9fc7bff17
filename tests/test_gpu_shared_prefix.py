"""shared_prefix_decode_attn against 64 bits, and a run of the operators beside
the cache together."""
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


class Shared:
    def __init__(self, G, per, H, d, dt, P_cap, pre, cap, lens, seed, spans=None, scale=1.0):
        b = G * per
        self.T = P_cap + cap + 8
        self.spans = spans or [[] for _ in range(b)]
        self.meta = P().SpanMeta(self.spans, self.T, DEV)
        self.pre = P().KVCache(2, G, H, P_cap, d, dt, DEV)
        self.pre.kv.copy_(R.rand(self.pre.kv.shape, seed, dt))
        self.pre.kv_len.copy_(torch.tensor(pre))
        self.c = c = P().KVCache(2, b, H, cap, d, dt, DEV)
        c.kv.copy_(R.rand(c.kv.shape, seed + 1, dt))
        c.start_behind(P_cap)
        c.kv_len.copy_(torch.tensor(lens))
        c.cur_tok.add_(c.kv_len.clamp(0, cap))
        self.ws = P().Workspace(b, H, 1, cap, d, DEV, prefixes=G, prefix_rows=P_cap)
        self.qkv = [R.rand((b, H, d), seed + 2 + i, dt, scale if i == 0 else 1.0, DEV)
                    for i in range(3)]
        self.o = torch.full((b, H, d), 9.0, dtype=dt, device=DEV)
        self.before = c.kv[1].cpu()
        self.per, self.dt, self.d = per, dt, d

    def run(self, theta):
        P().shared_decode_layer(*self.qkv, self.pre, self.c, 1, self.meta, self.ws, self.o,
                                theta=theta)

    def check(self, s, theta):
        c, dt, d = self.c, self.dt, self.d
        n, t = int(c.kv_len[s]), int(c.cur_tok[s])
        g = s // self.per
        m = min(max(int(self.pre.kv_len[g]), 0), self.pre.L_cap)
        q, k, v = (x[s].cpu().double() for x in self.qkv)
        pos = self.meta.pos[s].cpu().numpy()[t:t + 1]
        q, kr = (R.rotate(x[:, None], pos, theta)[:, 0] for x in (q, k))
        row = c.k(1)[s, :, n].cpu().double()
        tol = 32 * R.U * k.abs().amax(-1, keepdim=True)
        assert bool(((row - kr).abs() <= tol + R.half_step(dt) * (kr.abs() + tol)).all())
        assert torch.equal(c.v(1)[s, :, n].cpu(), self.qkv[2][s].cpu())
        ks = torch.cat([self.pre.k(1)[g, :, :m].cpu().double(), self.before[0][s, :, :n].double(),
                        row[:, None]], 1)
        vs = torch.cat([self.pre.v(1)[g, :, :m].cpu().double(), self.before[1][s, :, :n].double(),
                        v[:, None]], 1)
        ow, _, A, pv = R.attend(q, ks, vs, d ** -0.5)
        # scores as in a decode step; bf16: the prefix's softmax weights are
        # two bf16 terms in the value product (2^-17 of a weight at most)
        bf = dt == torch.bfloat16
        rel = 2 * A * ((d + 24) * R.U + (2.0 ** -17 if bf else 0)) + (m + n + 64) * R.U
        rel += 2.0 ** -17 if bf else 0
        err = (self.o[s].double().cpu() - ow).abs()
        assert bool((err <= pv * rel + R.half_step(dt) * (ow.abs() + pv * rel)).all()), \
            (s, float(err.max()), float(err.max() / pv.max()))


CASES = [
    # G, sequences a prefix, H, d, dtype, prefix capacity and lengths, own capacity, own lengths
    (1, 1, 1, 64, "bf16", 1, [1], 1, [0]),
    (1, 2, 1, 80, "f32", 5, [3], 4, [3, 0]),
    (2, 3, 2, 64, "bf16", 130, [130, 63], 20, None),
    (1, 17, 3, 80, "bf16", 300, [297], 40, None),
    (3, 1, 4, 80, "bf16", 257, [0, 1, 257], 9, None),
    (1, 33, 2, 64, "bf16", 1100, [1031], 70, None),
    (1, 64, 2, 80, "bf16", 513, [513], 65, None),
    (1, 70, 8, 64, "bf16", 900, [900], 30, None),    # more than one tile of queries
    (4, 8, 32, 80, "bf16", 600, [600, 599, 1, 64], 50, None),
    (1, 130, 5, 80, "bf16", 200, [190], 12, None),
    (2, 2, 3, 64, "bf16", 5000, [5000, 4097], 1800, [1799, 3, 900, 0]),
    (2, 5, 3, 64, "f32", 700, [700, 33], 40, None),
    (1, 40, 16, 80, "f32", 150, [150], 20, None),
]


@pytest.mark.parametrize("G,per,H,d,dtype,P_cap,pre,cap,lens", CASES)
@pytest.mark.parametrize("theta", [1e4, 0.0])
def test_shared(G, per, H, d, dtype, P_cap, pre, cap, lens, theta):
    print("shared", G, per, H, d, dtype, P_cap, pre, cap, theta, flush=True)
    if lens is None:
        lens = np.random.default_rng(per).integers(0, cap, size=G * per).tolist()
    x = Shared(G, per, H, d, DT[dtype], P_cap, pre, cap, lens, 40)
    p0 = x.pre.kv.cpu()
    x.run(theta)
    b = G * per
    for s in (range(b) if b < 10 else [0, 1, 15, 16, b // 2, b - 2, b - 1]):
        if s < b:
            x.check(s, theta)
    assert torch.equal(x.pre.kv.cpu(), p0) and int(x.c.status[0]) == 0
    after = x.c.kv[1].cpu()  # only the new rows were written
    for s in range(b):
        after[:, s, :, lens[s]] = x.before[:, s, :, lens[s]]
    assert torch.equal(after, x.before)
    first = x.o.clone()
    x.run(theta)
    assert torch.equal(first, x.o)


def test_special_steps_and_clamped_lengths():
    """<CL> steps, a full cache, a token outside the metadata; prefix lengths
    outside the capacity."""
    print("shared special", flush=True)
    for H, dtype in ((3, "bf16"), (3, "f32"), (130, "bf16")):
        spans = [[(102, 110)], [], [], []]
        x = Shared(2, 2, H, 64, DT[dtype], 100, [150, -3], 10, [2, 10, 3, 4], 7, spans=spans)
        x.c.cur_tok[2] = -1
        x.run(1e4)
        assert int(x.c.status[0]) == B().STATUS_CAP | B().STATUS_TOKEN
        assert torch.equal(x.o[0], x.qkv[2][0])
        assert bool(x.o[1:3].isnan().all())
        for s in range(3):
            assert torch.equal(x.c.kv[1, :, s].cpu(), x.before[:, s])
        x.check(3, 1e4)


def test_large_scores_and_unwritten_rows():
    """Scores over hundreds of powers of two; what lies behind the last row,
    infinities and NaN included, does not count."""
    print("shared range", flush=True)
    for dtype in ("bf16", "f32"):
        x = Shared(1, 20, 2, 80, DT[dtype], 400, [333], 50, [20] * 20, 9, scale=15.0)
        x.pre.kv[:, :, :, :, 333:] = float("nan")
        x.c.kv[:, :, :, :, 21:] = float("inf")
        x.before = x.c.kv[1].cpu()
        x.run(1e4)
        for s in (0, 19):
            x.check(s, 1e4)


def test_prefix_offsets_beyond_32_bits():
    """A prefix cache of more than 2^31 elements: the last heads."""
    print("shared far offsets", flush=True)
    H, P_cap, d, m, per = 33, 1 << 20, 64, 300, 3
    kv = torch.empty(2, 2, 1, H, P_cap, d, dtype=torch.bfloat16, device=DEV)[1:]
    pre = P().KVCache(1, 1, H, P_cap, d, torch.bfloat16, DEV, kv=kv)
    kv[:, :, :, :, :m] = R.rand((1, 2, 1, H, m, d), 3, torch.bfloat16, device=DEV)
    kv[:, :, :, :, m:m + 8] = float("nan")
    pre.kv_len.fill_(m)
    meta = P().SpanMeta([[]] * per, m + 8, DEV)
    c = P().KVCache(1, per, H, 4, d, torch.bfloat16, DEV)
    c.start_behind(m)
    ws = P().Workspace(per, H, 1, 4, d, DEV, prefixes=1, prefix_rows=P_cap)
    qkv = [R.rand((per, H, d), i, torch.bfloat16, device=DEV) for i in range(3)]
    o = torch.empty(per, H, d, dtype=torch.bfloat16, device=DEV)
    P().shared_decode_layer(*qkv, pre, c, 0, meta, ws, o)
    for s in range(per):
        k, v = (torch.cat([kv[0, i, 0, :, :m].cpu(), qkv[1 + i][s].cpu()[:, None]], 1)
                for i in range(2))
        want = R.attend(qkv[0][s].cpu(), k, v, d ** -0.5)[0]
        assert float((o[s].cpu().double() - want).abs().max()) < 2e-2


def test_equals_one_cache_holding_both():
    """The same rows in one cache: decode_layer gives the same step (to the
    rounding of the two)."""
    print("shared against one cache", flush=True)
    G, per, H, d, dt, pre, n = 1, 6, 4, 64, torch.float32, 200, 30
    x = Shared(G, per, H, d, dt, pre, [pre], n + 1, [n] * per, 5)
    x.run(1e4)
    one = P().KVCache(2, per, H, pre + n + 1, d, dt, DEV)
    one.kv[:, :, :, :, :pre] = x.pre.kv.expand(2, 2, per, H, pre, d)
    one.kv[:, :, :, :, pre:] = x.c.kv
    one.kv_len.fill_(pre + n)
    one.cur_tok.copy_(x.c.cur_tok)
    o = torch.empty_like(x.o)
    P().decode_layer(*x.qkv, one, 1, x.meta, P().Workspace(per, H, 1, pre + n + 1, d, DEV), o,
                     theta=1e4)
    assert float((o - x.o).abs().max()) < 1e-5
    assert torch.equal(one.kv[1, :, :, :, pre + n], x.c.kv[1, :, :, :, n])


def test_graph_and_side_stream():
    print("shared graph", flush=True)
    x = Shared(2, 9, 4, 80, torch.bfloat16, 700, [700, 650], 60, list(range(18)), 5)
    x.run(1e4)
    want = x.o.clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        x.run(1e4)
    torch.cuda.synchronize()
    assert torch.equal(x.o, want)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        x.run(1e4)
    for _ in range(3):
        x.o.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(x.o, want)


def test_run_together():
    """A document with head norms is prefilled in blocks under a budget (rows
    leave by accumulated weight), then several samples continue it: every
    output against 64 bits over the rows that each step had."""
    print("run together", flush=True)
    M, H, d, L, block, dt = 2, 3, 64, 260, 64, torch.float32
    heavy, recent, per, steps, theta, eps = 60, 20, 3, 4, 1e4, 1e-6
    T = L + steps
    spans = [(10, 30), (100, 150), (255, 300)]
    vu, pos = R.vu_pos(spans, T)
    meta1 = P().SpanMeta([spans], T, DEV)
    nm = P().QKNorm(*[(1 + 0.2 * R.rand((d,), i, dt)).to(DEV) for i in range(2)], eps)
    q, k, v = (R.rand((M, 1, H, L, d), 10 + i, dt, device=DEV) for i in range(3))
    o = torch.empty_like(q)
    cap = heavy + recent + block + 8
    pre = P().KVCache(M, 1, H, cap, d, dt, DEV)
    pre.track_weights()
    ws = P().Workspace(1, H, 1, cap, d, DEV, block=block, weights=block)
    seen = []
    P().prefill_progressive(q, k, v, o, pre, meta1, ws, L, block, theta=theta, norm=nm,
                            evict=(heavy, recent),
                            on_block=lambda e: seen.append(pre.tok_idx[0, :int(pre.kv_len[0])].cpu().tolist()))
    assert int(pre.status[0]) == 0
    f = lambda x, w: R.norm_rope(x.cpu(), w.cpu(), eps, pos[:x.shape[-2]], theta)
    held, w = [], torch.zeros(M, H, T, dtype=torch.float64)
    for bi, B0 in enumerate(range(0, L, block)):
        toks = list(range(B0, min(L, B0 + block)))
        rows = held + toks
        see = torch.as_tensor(R.see(rows, toks, vu))
        for m in range(M):
            qq, kk = f(q[m, 0], nm.q_weight)[:, toks], f(k[m, 0], nm.k_weight)[:, rows]
            x = torch.matmul(qq, kk.transpose(1, 2)) * d ** -0.5
            p = torch.nan_to_num(torch.softmax(x.masked_fill(~see, -np.inf), -1), nan=0.0)
            got = o[m, 0, :, toks].cpu().double()
            assert float((got - torch.matmul(p, v[m, 0].cpu().double()[:, rows])).abs().max()) < 1e-5
            w[m, :, rows] += p.sum(1)
        end = toks[-1] + 1
        held = [t for t in rows if vu[t] != t and vu[t] >= end]
        if len(held) > heavy + recent:
            old = held[:len(held) - recent]
            total = w.sum((0, 1)).numpy()
            held = sorted(sorted(old, key=lambda t: -total[t])[:heavy]) + held[len(held) - recent:]
        assert held == seen[bi], bi
    # samples behind what is left of the document
    meta = P().SpanMeta([spans] * per, T, DEV)
    c = P().KVCache(M, per, H, steps, d, dt, DEV)
    c.start_behind(L)
    ws2 = P().Workspace(per, H, 1, steps, d, DEV, prefixes=1, prefix_rows=cap)
    qn, kn, vn = (R.rand((steps, M, per, H, d), 20 + i, dt, device=DEV) for i in range(3))
    on = torch.empty_like(qn)
    for t in range(steps):
        for m in range(M):
            P().shared_decode_layer(qn[t, m], kn[t, m], vn[t, m], pre, c, m, meta, ws2, on[t, m],
                                    theta=theta, norm=nm)
        c.commit(meta)
    assert int(c.status[0]) == 0 and c.kv_len.tolist() == [steps] * per
    g = lambda x, w, t: R.norm_rope(x.cpu()[:, None], w.cpu(), eps, pos[t:t + 1], theta)
    for m in range(M):
        kp, vp = f(k[m, 0], nm.k_weight)[:, held], v[m, 0].cpu().double()[:, held]
        for s in range(per):
            kk, vv = kp, vp
            for t in range(steps):
                kk = torch.cat([kk, g(kn[t, m, s], nm.k_weight, L + t)], 1)
                vv = torch.cat([vv, vn[t, m, s].cpu().double()[:, None]], 1)
                want = R.attend(g(qn[t, m, s], nm.q_weight, L + t)[:, 0], kk, vv, d ** -0.5)[0]
                assert float((on[t, m, s].cpu().double() - want).abs().max()) < 1e-5
