"""qk_norm_rope against the formula in 64 bits: a prompt into the cache, blocks
behind a sequence's rows, single tokens; strides, odd sizes, what must stay
untouched."""
import pytest
import torch

import op_refs as R

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
EPS = 1e-5


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


def close(got, want, tol, dtype, what):
    got, tol = got.double().cpu(), tol + R.half_step(dtype) * (want.abs() + tol)
    bad = (got - want).abs() > tol
    assert not bad.any(), (what, float((got - want).abs().max()))


def weights(d, dtype, seed):
    return [(1 + 0.3 * R.rand((d,), seed + i, torch.float32)).to(dtype) for i in range(2)]


def views(b, H, n, d, dtype, layout, seed):
    """q, k, v (b, H, n, d) on the host, all of one stride pattern."""
    if layout == "tokens":
        x = R.rand((b, n, 3, H, d), seed, dtype)
        return [x[:, :, i].transpose(1, 2) for i in range(3)]
    if layout == "fused-heads":  # (b, n, H, 3, d)
        x = R.rand((b, n, H, 3, d), seed, dtype)
        return [x[:, :, :, i].transpose(1, 2) for i in range(3)]
    return [R.rand((b, H, n, d), seed + i, dtype) for i in range(3)]


def to_dev(xs):
    """The same views of one device copy of their storage."""
    out = []
    for x in xs:
        base = torch.empty(0, dtype=x.dtype).set_(x.untyped_storage()).to(DEV)
        out.append(base.as_strided(x.shape, x.stride(), x.storage_offset()))
    return out


CASES = [
    # b, H, n, d, dtype, layout, theta
    (1, 1, 1, 64, "bf16", "heads", 1e4),
    (1, 1, 1, 80, "f32", "tokens", 1e4),
    (2, 3, 5, 80, "bf16", "tokens", 1e4),
    (2, 3, 64, 64, "bf16", "heads", 1e4),
    (1, 5, 63, 80, "bf16", "fused-heads", 1e4),
    (3, 7, 65, 64, "f32", "tokens", 1e4),
    (3, 2, 130, 80, "f32", "heads", 500000.0),
    (2, 33, 257, 80, "bf16", "tokens", 1e4),
    (2, 9, 101, 64, "bf16", "tokens", 0.0),
    (1, 4, 1000, 64, "bf16", "fused-heads", 1e4),
]


@pytest.mark.parametrize("b,H,n,d,dtype,layout,theta", CASES)
def test_prompt(b, H, n, d, dtype, layout, theta):
    print("norm prompt", b, H, n, d, dtype, layout, theta, flush=True)
    dt, tok0, cap = DT[dtype], 3, n + 7
    spans = [R.some_spans(n + 5, 11 + s) for s in range(b)]
    meta = P().SpanMeta(spans, n + 5, DEV)
    xs = views(b, H, n, d, dt, layout, 5)
    qw, kw = weights(d, dt, 70)
    qd, kd, vd = to_dev(xs)
    qr = torch.full((b, H, n, d), 9.0, dtype=dt, device=DEV)
    kv = torch.full((2, b, H, cap, d), 7.0, dtype=dt, device=DEV)
    P().norm_rope_rows(qd, kd, vd, qr, kv[0], kv[1], P().QKNorm(qw.to(DEV), kw.to(DEV), EPS), meta,
                       n, tok0, theta)
    for s in range(b):
        pos = R.vu_pos(spans[s], n + 5)[1][tok0:tok0 + n]
        for x, w, got in ((xs[0], qw, qr), (xs[1], kw, kv[0])):
            want = R.norm_rope(x[s], w, EPS, pos, theta)
            close(got[s, :, :n], want, R.norm_rope_tol(x[s], w, EPS, dt), dt, (s, "qk"))
        assert torch.equal(kv[1, s, :, :n].cpu(), xs[2][s])
    assert bool((kv[:, :, :, n:] == 7.0).all())


@pytest.mark.parametrize("b,H,n,d,dtype,layout", [
    (2, 33, 500, 80, "bf16", "tokens"),      # four heads a thread, a tensor a workgroup
    (3, 6, 800, 64, "f32", "fused-heads"),
    (2, 33, 8000, 64, "bf16", "tokens"),     # four heads of q, k and v a thread
    (1, 35, 5700, 80, "f32", "tokens"),      # two
])
def test_large_launches(b, H, n, d, dtype, layout):
    print("norm large", b, H, n, d, dtype, layout, flush=True)
    dt, spans = DT[dtype], [R.some_spans(n, 3)] * b
    meta = P().SpanMeta(spans, n, DEV)
    pos = R.vu_pos(spans[0], n)[1]
    q, k, v = to_dev(views(b, H, n, d, dt, layout, 5))
    nm = P().QKNorm(*[w.to(DEV) for w in weights(d, dt, 4)], EPS)
    qr = torch.empty(b, H, n, d, dtype=dt, device=DEV)
    kv = torch.empty(2, b, H, n, d, dtype=dt, device=DEV)
    P().norm_rope_rows(q, k, v, qr, kv[0], kv[1], nm, meta, n, 0, 1e4)
    assert torch.equal(kv[1], v)
    for x, w, got in ((q, nm.q_weight, qr), (k, nm.k_weight, kv[0])):
        for s in range(b):
            want = R.norm_rope(x[s], w, EPS, pos, 1e4)
            tol = R.norm_rope_tol(x[s], w, EPS, dt)
            tol = tol + R.half_step(dt) * (want.abs() + tol)
            assert not ((got[s].double() - want).abs() > tol).any(), s


def test_forms_of_one_operand_and_without_weights():
    b, H, n, d, dt = 2, 3, 21, 80, torch.bfloat16
    print("norm single operands", flush=True)
    x, = to_dev([R.rand((b, H, n, d), 1, dt)])
    meta = P().SpanMeta([[], [(2, 9)]], n, DEV)
    s = H * n * d, n * d, d
    nan = float("nan")
    outs = []
    for i in range(3):
        t, o = [None] * 3, [None] * 3
        t[i], o[i] = x, torch.full_like(x, nan)
        B().qk_norm_rope(*t, *o, None, None, EPS, b, H, n, *s, n * d, n * d, n, d, meta.pos, n, 0,
                         None, None, 1e4)
        outs.append(o[i])
    assert torch.equal(outs[0], outs[1])
    assert torch.equal(outs[2], x)
    for i in range(b):
        pos = R.vu_pos([[], [(2, 9)]][i], n)[1]
        close(outs[0][i], R.norm_rope(x[i].cpu(), None, EPS, pos, 1e4),
              R.norm_rope_tol(x[i].cpu(), None, EPS, dt), dt, i)
    y = x.clone()  # in place
    B().qk_norm_rope(y, None, None, y, None, None, None, None, EPS, b, H, n, *s, n * d, 0, 0, d,
                     meta.pos, n, 0, None, None, 1e4)
    assert torch.equal(y, outs[0])


def test_mixed_strides_take_three_launches():
    b, H, n, d, dt = 2, 3, 40, 64, torch.float32
    print("norm mixed strides", flush=True)
    q = R.rand((b, H, n, d), 1, dt, device=DEV)
    k = R.rand((b, n, H, d), 2, dt, device=DEV).transpose(1, 2)
    v = R.rand((b, H, 2 * n, d), 3, dt, device=DEV)[:, :, :n]
    meta = P().SpanMeta([[], []], n, DEV)
    out = [torch.empty(b, H, n, d, device=DEV) for _ in range(6)]
    nm = P().QKNorm(None, None, EPS)
    P().norm_rope_rows(q, k, v, out[0], out[1], out[2], nm, meta, n, 0, 1e4)
    P().norm_rope_rows(q, k.contiguous(), v.contiguous(), out[3], out[4], out[5], nm, meta, n, 0,
                       1e4)
    for a, c in zip(out[:3], out[3:]):
        assert torch.equal(a, c)


@pytest.mark.parametrize("d,dtype", [(64, "f32"), (80, "bf16")])
def test_block_behind_rows_and_without_room(d, dtype):
    """Rows go behind row0[s]; a sequence without room is left alone and says so."""
    print("norm block", d, dtype, flush=True)
    dt, b, H, n, cap = DT[dtype], 4, 3, 33, 60
    meta = P().SpanMeta([[(1, 4)]] * b, 90, DEV)
    q, k, v = (R.rand((b, H, n, d), i, dt, device=DEV) for i in range(3))
    row0 = torch.tensor([0, 27, 28, -1], dtype=torch.int32, device=DEV)
    cache = P().KVCache(1, b, H, cap, d, dt, DEV)
    cache.kv.fill_(3.0)
    qr = torch.empty_like(q)
    P().norm_rope_rows(q, k, v, qr, cache.k(0), cache.v(0), P().QKNorm(None, None, EPS), meta, n, 50,
                       1e4, row0=row0, status=cache.status)
    assert int(cache.status[0]) == B().STATUS_CAP
    pos = R.vu_pos([(1, 4)], 90)[1][50:50 + n]
    for s in range(b):
        close(qr[s], R.norm_rope(q[s].cpu(), None, EPS, pos, 1e4),
              R.norm_rope_tol(q[s].cpu(), None, EPS, dt), dt, ("q", s))
        held = torch.full((2, H, cap, d), 3.0, dtype=dt)
        if s < 2:
            r = int(row0[s])
            close(cache.k(0)[s, :, r:r + n], R.norm_rope(k[s].cpu(), None, EPS, pos, 1e4),
                  R.norm_rope_tol(k[s].cpu(), None, EPS, dt), dt, ("k", s))
            held[0, :, r:r + n] = cache.k(0)[s, :, r:r + n].cpu()
            held[1, :, r:r + n] = v[s].cpu()
        assert torch.equal(cache.kv[0, :, s].cpu(), held), s


@pytest.mark.parametrize("d,dtype,b,H", [(64, "bf16", 1, 32), (80, "bf16", 5, 7), (80, "f32", 70, 3)])
def test_step(d, dtype, b, H):
    """One token a sequence at its own place; a token outside the metadata is
    written as NaN and reported."""
    print("norm step", d, dtype, b, H, flush=True)
    dt, T = DT[dtype], 300
    spans = [R.some_spans(T, s) for s in range(b)]
    meta = P().SpanMeta(spans, T, DEV)
    cache = P().KVCache(1, b, H, 4, d, dt, DEV)
    tok = torch.randint(0, T, (b,), generator=torch.Generator().manual_seed(b))
    if b > 1:
        tok[0], tok[1] = -1, T
    cache.cur_tok.copy_(tok)
    q, k = (R.rand((b, H, d), 30 + i, dt) for i in range(2))
    qw, kw = weights(d, dt, 9)
    qo, ko = torch.empty_like(q, device=DEV), torch.empty_like(k, device=DEV)
    P().norm_rope_step(q.to(DEV), k.to(DEV), qo, ko, P().QKNorm(qw.to(DEV), kw.to(DEV), EPS), cache,
                       meta, 1e4)
    assert int(cache.status[0]) == (B().STATUS_TOKEN if b > 1 else 0)
    for s in range(b):
        t = int(tok[s])
        if not 0 <= t < T:
            assert bool(qo[s].isnan().all()) and bool(ko[s].isnan().all())
            continue
        pos = R.vu_pos(spans[s], T)[1][t:t + 1]
        for x, w, got in ((q, qw, qo), (k, kw, ko)):
            close(got[s][:, None], R.norm_rope(x[s][:, None], w, EPS, pos, 1e4),
                  R.norm_rope_tol(x[s][:, None], w, EPS, dt), dt, s)


def test_far_positions_small_and_special_rows():
    """Positions in the millions, rows of zeros and of tiny numbers, infinity
    and NaN stay in their row."""
    print("norm special rows", flush=True)
    d, n, dt = 64, 6, torch.float32
    pos = torch.tensor([[0, 1, 2 ** 24 + 1, 10 ** 9, 2 ** 31 - 1, 5]], dtype=torch.int32, device=DEV)
    x = R.rand((1, 1, n, d), 4, dt)
    x[0, 0, 0] = 0
    x[0, 0, 1] *= 1e-12
    x[0, 0, 5, 3] = float("inf")
    y = torch.empty(1, 1, n, d, device=DEV)
    B().qk_norm_rope(x.to(DEV), None, None, y, None, None, None, None, EPS, 1, 1, n, n * d, n * d, d,
                     n * d, 0, 0, d, pos, n, 0, None, None, 1e4)
    want = R.norm_rope(x, None, EPS, pos[0].cpu().double(), 1e4)
    # at 2^31 the two 64-bit angles, their frequencies, products and multiples
    # of 2 pi each rounded by up to 2^31 * 2^-53 = 4 U, differ by up to 16 U
    tol = R.norm_rope_tol(x, None, EPS, dt) * 1.5
    close(y[:, :, :5], want[:, :, :5], tol[:, :, :5], dt, "rows")
    assert not y[0, 0, 5].isfinite().all() and bool(y[0, 0, :5].isfinite().all())


def test_side_stream_and_graph_give_the_same_bits():
    print("norm stream and graph", flush=True)
    b, H, d, dt, T = 3, 5, 80, torch.bfloat16, 40
    meta = P().SpanMeta([[(3, 8)]] * b, T, DEV)
    cache = P().KVCache(1, b, H, 4, d, dt, DEV)
    cache.cur_tok.copy_(torch.tensor([5, 9, 30]))
    q, k = (R.rand((b, H, d), i, dt, device=DEV) for i in range(2))
    nm = P().QKNorm(None, None, EPS)
    out = [torch.empty_like(q) for _ in range(6)]
    P().norm_rope_step(q, k, out[0], out[1], nm, cache, meta, 1e4)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        P().norm_rope_step(q, k, out[2], out[3], nm, cache, meta, 1e4)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        P().norm_rope_step(q, k, out[4], out[5], nm, cache, meta, 1e4)
    for turn in range(3):
        cache.cur_tok.add_(turn)
        P().norm_rope_step(q, k, out[0], out[1], nm, cache, meta, 1e4)
        out[4].zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[4], out[0]) and torch.equal(out[5], out[1]), turn
        if turn == 0:
            assert torch.equal(out[2], out[0]) and torch.equal(out[3], out[1])
