"""Operators next to the compacted cache, with their sizes and plain forms.

Kinds
    norm     the RMS norm of each head's queries and keys and the rotation at
             the tied positions in one pass: a prompt or a block of it into the
             cache, or one token a sequence
    weights  the attention weight that queries of a prompt give each cache row
    decode   one generated token's attention, which also adds the weight that
             it gives each cache row
    evict    the rows of least accumulated weight leave the cache
    shared   one generated token for sequences that continue shared prefixes

Where ``own`` is true a pass makes the package's calls; otherwise it computes
the same with elementary torch operations in 32 bits.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

THETA = 10000.0
EPS = 1e-6
DEV = "cuda"


# ---------------------------------------------------------------------------
# the cases
# ---------------------------------------------------------------------------

def _case(kind, **kw):
    c = dict(kind=kind, dtype="bf16", M=1, b=1, H=32, d=64, L=2048, rotary=True, ratio=0.5, lo=16,
             hi=64, nq=0, layout="tokens", offset=0, compacted=False, heavy=0, recent=0, G=1,
             own_rows=0)
    c.update(kw)
    return c


def listed():
    def c(name, kind, **kw):
        return dict(_case(kind, **kw), name=name)

    return [
        # one user's next token: the q and k of one layer of a 3B rotary model
        c("norm-step-one-user", "norm", d=80, nq=0, L=2000),
        # one layer of the 3B rotary model's prompt batch, as the fused
        # projection leaves it (token-major q, k and v)
        c("norm-prompt-3b", "norm", b=16, d=80, L=4096, nq=4096),
        # a ragged block of three prompts in fp32, each behind its own rows
        c("norm-block-ragged-f32", "norm", dtype="f32", b=3, H=12, L=1500, nq=777, offset=400,
          layout="heads"),
        # a short fp32 prompt's weights, all of its queries
        c("weights-tiny-f32", "weights", dtype="f32", H=4, L=256, nq=256, lo=16, hi=16),
        # the last 32 queries of a 3B-rotary prompt batch vote on its compacted cache
        c("weights-window-3b", "weights", b=16, d=80, L=4096, nq=32, compacted=True),
        # all queries of two OPT-1.3B-sized prompts, before compaction
        c("weights-prompt-opt1.3b", "weights", b=2, L=4096, nq=4096),
        # one user's next token with weights: 8 layers of the 3B rotary model
        c("decode-weights-one-user", "decode", M=8, d=80, L=2000),
        # a token for a batch of 16, half the prompt freed
        c("decode-weights-3b", "decode", M=2, b=16, d=80, L=4096),
        # one user's cache brought back to 960 rows
        c("evict-one-user", "evict", M=8, d=80, L=1024, heavy=704, recent=256),
        # half of a batch's cache leaves
        c("evict-opt1.3b", "evict", M=8, b=8, L=2048, heavy=768, recent=256),
        # eight samples for each of four compressed documents
        c("shared-samples", "shared", G=4, b=32, d=80, L=4096, own_rows=64),
        # 64 sequences behind one long system prompt
        c("shared-long", "shared", G=1, b=64, L=16384, ratio=0.25, own_rows=300),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    kind = rng.choice(["norm", "norm", "weights", "weights", "decode", "decode", "evict", "shared",
                       "shared"])
    lo, hi = rng.choice([(2, 25), (16, 64), (32, 32)])
    c = _case(kind, H=rng.choice([8, 12, 20, 32, 32, 40]), d=rng.choice([64, 80]), lo=lo, hi=hi,
              rotary=rng.random() < 0.7, ratio=round(rng.uniform(0.1, 0.8), 3))
    if rng.random() < 0.2:
        c["dtype"] = "f32"
    e = 2 if c["dtype"] == "bf16" else 4
    if kind == "norm":
        c["layout"] = rng.choice(["tokens", "tokens", "heads"])
        if rng.random() < 0.3:
            c.update(L=2000, nq=0, b=_log(rng, 1, 256))
        else:
            c["nq"] = _log(rng, 1, 4096)
            row = c["H"] * c["d"] * e  # at most about the listed prompt's bytes
            c["b"] = _log(rng, 1, max(1, min(64, 65536 * 32 * 80 * 2 // (c["nq"] * row))))
            c["offset"] = rng.choice([0, 0, 100, 333])
            c["L"] = c["nq"] + c["offset"]
    elif kind == "weights":
        c["L"] = _log(rng, 64, 16384 if e == 2 else 2048)
        c["nq"] = rng.choice([1, 16, 32, 64, c["L"], c["L"] // 2])
        most = max(1, min(16, int(2 * 4096 ** 2 * 32 / (c["L"] * c["nq"] * c["H"] * e / 2))))
        if c["nq"] * c["L"] * c["H"] > 2 * 4096 ** 2 * 32:
            c["nq"] = 64
            most = max(1, 65536 // c["L"])
        c["b"] = _log(rng, 1, most)
        c["compacted"] = rng.random() < 0.5
    elif kind == "decode":
        c["L"] = _log(rng, 128, 16000)
        c["b"] = _log(rng, 1, max(1, min(64, 65536 // c["L"])))
        row = 2 * c["b"] * c["H"] * c["L"] * c["d"] * e
        c["M"] = max(1, min(8, 500_000_000 // row))
    elif kind == "evict":
        c.update(M=rng.choice([1, 4, 8]), b=_log(rng, 1, 8), L=_log(rng, 100, 2048))
        c["recent"] = _log(rng, 1, max(2, c["L"] // 2))
        c["heavy"] = rng.randrange(0, c["L"])
    else:
        c["G"] = rng.choice([1, 1, 2, 4, 7])
        c["b"] = c["G"] * _log(rng, 1, 64 // c["G"])
        c["L"] = _log(rng, 64, 16384 // c["G"])
        c["own_rows"] = _log(rng, 1, 400)
    return c


# ---------------------------------------------------------------------------
# spans and what follows from them (host, plain numpy)
# ---------------------------------------------------------------------------

def _dt(case):
    return {"bf16": torch.bfloat16, "f32": torch.float32}[case["dtype"]]


def _spans_uniform(rng, L, ratio, lo, hi):
    """Non-overlapping spans with lengths U[lo, hi] that free about `ratio`
    of L tokens, spread with sorted uniform gaps."""
    lengths, total = [], 0
    while total < ratio * L:
        x = int(rng.integers(lo, hi + 1))
        if total + x + len(lengths) + 1 > L:
            break
        lengths.append(x)
        total += x
    free = L - total - len(lengths)
    cuts = np.sort(rng.integers(0, free + 1, size=len(lengths)))
    gaps = np.diff(np.concatenate([[0], cuts]))
    out, at = [], 0
    for g, x in zip(gaps, lengths):
        c = at + int(g)
        out.append((c, c + x))
        at = c + x + 1
    return out


def _spans(case, seed):
    """Spans of every sequence; those that share a prefix share its spans."""
    rng = np.random.default_rng(seed)
    n = case["G"] if case["kind"] == "shared" else case["b"]
    out = []
    for _ in range(n):
        # serving batches are ragged: each decode sequence has its own ratio
        r = case["ratio"] + (rng.uniform(-0.1, 0.1) if case["kind"] == "decode" else 0.0)
        out.append(_spans_uniform(rng, case["L"], min(max(r, 0.0), 0.85), case["lo"], case["hi"]))
    if case["kind"] == "shared":
        out = [out[i // (case["b"] // n)] for i in range(case["b"])]
    return out


def _meta_len(case):
    return case["L"] + case["own_rows"] + 1


def _vu_pos(spans, T):
    """Per token: the last index that may see it, and its tied position."""
    inf = 2 ** 31 - 1
    vu, pos, sentinel = np.full(T, inf, np.int64), np.zeros(T, np.int64), np.zeros(T, bool)
    for c, r in spans:
        vu[c + 1:min(r, T)] = r
        for t in (c, r):
            if t < T:
                sentinel[t] = True
        if c < T:
            vu[c] = c
    before = np.concatenate([[0], np.cumsum(~sentinel)[:-1]])
    pos[:] = np.where(sentinel, np.maximum(before - 1, 0), before)
    return vu, pos


def _kept(vu, P_next):
    """Indices of tokens [0, P_next) that tokens from P_next on may see."""
    t = np.arange(P_next)
    return t[(vu[:P_next] != t) & (vu[:P_next] >= P_next)]


def _rows(case, spans):
    """Tokens of each sequence's cache rows (shared: of each prefix's)."""
    if case["kind"] == "shared":
        spans = spans[::case["b"] // case["G"]]
    T = _meta_len(case)
    gone = case["compacted"] or case["kind"] in ("decode", "shared")
    return [_kept(_vu_pos(x, T)[0], case["L"]) if gone else np.arange(case["L"]) for x in spans]


def _own_len(case, seed):
    """Rows that each sequence has written behind its shared prefix."""
    rng = np.random.default_rng(seed + 1)
    n = rng.integers(0, case["own_rows"] + 1, size=case["b"])
    n[0] = case["own_rows"]
    return n


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _randn(shape, g, dt):
    # drawn in pieces, so that the 32-bit draw of a large tensor is not held
    x = torch.empty(shape, dtype=dt, device=DEV)
    flat = x.view(-1)
    for i in range(0, flat.numel(), 1 << 26):
        n = min(1 << 26, flat.numel() - i)
        flat[i:i + n] = torch.randn(n, generator=g, device=DEV, dtype=torch.float32)
    return x


def _inputs(case, seed):
    """The seed's tensors, by name (the same for prepare and exact)."""
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    dt, kind = _dt(case), case["kind"]
    M, b, H, d, L, n = (case[k] for k in ("M", "b", "H", "d", "L", "nq"))
    t = {}
    if kind == "norm":
        if case["layout"] == "tokens":
            x = _randn((b, max(n, 1), 3, H, d), g, dt)
            t["q"], t["k"], t["v"] = (x[:, :, i].transpose(1, 2) for i in range(3))
        else:
            t["q"], t["k"], t["v"] = (_randn((b, H, max(n, 1), d), g, dt) for _ in range(3))
        t["qw"], t["kw"] = ((1 + 0.2 * _randn((d,), g, torch.float32)).to(dt) for _ in range(2))
    elif kind == "weights":
        t["q"], t["rows"] = _randn((b, H, n, d), g, dt), _randn((b, H, L, d), g, dt)
        # sums of earlier queries, of the size that this pass adds
        t["w"] = torch.rand((b, H, L), generator=g, device=DEV) * (n / L)
    elif kind == "decode":
        t["rows"] = _randn((M, 2, b, H, L, d), g, dt)
        t["qn"], t["kn"], t["vn"] = (_randn((M, b, H, d), g, dt) for _ in range(3))
        t["w"] = torch.rand((M, b, H, L + 1), generator=g, device=DEV) * (4 / L)
    elif kind == "evict":
        t["rows"] = _randn((M, 2, b, H, L, d), g, dt)
        # sums of attention weights are skewed: a few rows hold most
        t["w"] = torch.rand((M, b, H, L), generator=g, device=DEV).pow_(8)
    else:
        t["prefix"] = _randn((2, case["G"], H, L, d), g, dt)
        t["rows"] = _randn((2, b, H, case["own_rows"], d), g, dt)
        t["qn"], t["kn"], t["vn"] = (_randn((b, H, d), g, dt) for _ in range(3))
    return t


def _i32(x):
    return torch.as_tensor(np.asarray(x), dtype=torch.int32).to(DEV)


def prepare(case, seed):
    dt, kind = _dt(case), case["kind"]
    M, b, H, d, L, n = (case[k] for k in ("M", "b", "H", "d", "L", "nq"))
    spans = _spans(case, seed)
    T = _meta_len(case)
    vp = [_vu_pos(x, T) for x in spans]
    held = _rows(case, spans)
    s = dict(case=case, theta=THETA if case["rotary"] else 0.0)
    s.update(_inputs(case, seed))
    s["vu"], s["pos"] = (_i32(np.stack([x[i] for x in vp])) for i in range(2))
    s["len"] = [len(x) for x in held]
    if kind == "norm":
        s["step"] = n == 0
        if s["step"]:  # every sequence is at a token of its own
            rng = np.random.default_rng(seed)
            s["tok"] = _i32(rng.integers(L // 2, L, size=b))
            s["q"], s["k"] = (s[x][:, :, 0].contiguous() for x in "qk")
            s["qr"], s["kr"] = torch.empty_like(s["q"]), torch.empty_like(s["k"])
        else:
            s["tok0"] = case["offset"]
            s["row0"] = _i32([case["offset"] // (i + 1) for i in range(b)])
            s["qr"] = torch.empty((b, H, n, d), dtype=dt, device=DEV)
            s["kv"] = torch.zeros((1, 2, b, H, L, d), dtype=dt, device=DEV)
    elif kind == "weights":
        s["tok_idx"] = _i32(np.stack([np.pad(x, (0, L - len(x))) for x in held]))
        s["k"] = s.pop("rows")
        s["out"] = torch.zeros_like(s["w"])
    elif kind == "decode":
        s["kv"] = torch.zeros((M, 2, b, H, L + 1, d), dtype=dt, device=DEV)
        s["kv"][:, :, :, :, :L] = s.pop("rows")
        s["out"], s["on"] = torch.zeros_like(s["w"]), torch.empty_like(s["qn"])
    elif kind == "evict":
        s["kv"] = s.pop("rows")
        s["kv_out"], s["out"] = torch.zeros_like(s["kv"]), torch.zeros_like(s["w"])
    else:
        s["own_len"] = _own_len(case, seed)
        s["kv"] = torch.zeros((1, 2, b, H, case["own_rows"] + 1, d), dtype=dt, device=DEV)
        s["kv"][0, :, :, :, :-1] = s.pop("rows")
        s["on"] = torch.empty_like(s["qn"])
    if own:
        _prepare_own(s, spans, held)
    return s


def _prepare_own(s, spans, held):
    """The package's metadata, caches and workspaces around the same tensors."""
    from paper_2310_08152_amd import path as P
    case, kind, dt = s["case"], s["case"]["kind"], _dt(s["case"])
    M, b, H, d, L, n = (case[k] for k in ("M", "b", "H", "d", "L", "nq"))
    dev = torch.device(DEV, torch.cuda.current_device())
    s["P"] = P
    s["meta"] = P.SpanMeta(spans, _meta_len(case), dev)

    def cache(kv, M, b, rows):
        c = P.KVCache(M, b, H, rows, d, dt, dev, kv=kv)
        c.kept_src.fill_(-1)
        return c

    if kind == "norm":
        s["norm"] = P.QKNorm(s["qw"], s["kw"], EPS)
        if s["step"]:
            s["cache"] = P.KVCache(1, b, H, 1, d, dt, dev)
            s["cache"].cur_tok.copy_(s["tok"])
        else:
            s["cache"] = cache(s["kv"], 1, b, L)
    elif kind == "weights":
        s["cache"] = c = P.KVCache(1, b, H, L, d, dt, dev)
        c.k(0).copy_(s["k"])
        c.kv_len.copy_(_i32(s["len"]))
        c.tok_idx.copy_(s["tok_idx"])
        s["ws"] = P.Workspace(b, H, 1, L, d, dev, weights=n)
    elif kind == "decode":
        s["cache"] = c = cache(s["kv"], M, b, L + 1)
        c.kv_len.copy_(_i32(s["len"]))
        c.cur_tok.fill_(L)
        s["ws"] = P.Workspace(b, H, 1, L + 1, d, dev, weights=1)
    elif kind == "evict":
        s["cache"] = c = cache(s["kv"], M, b, L)
        c.track_weights(w=s["w"])
    else:
        G = case["G"]
        s["prefix"] = pre = P.KVCache(1, G, H, L, d, dt, dev, kv=s["prefix"][None])
        pre.kv_len.copy_(_i32(s["len"]))
        s["cache"] = c = cache(s["kv"], 1, b, case["own_rows"] + 1)
        c.kv_len.copy_(_i32(s["own_len"]))
        c.cur_tok.copy_(_i32(L + s["own_len"]))
        s["ws"] = P.Workspace(b, H, 1, c.L_cap, d, dev, prefixes=G, prefix_rows=L)


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    return (_OWN if own else _PLAIN)[s["case"]["kind"]](s)


def _norm_own(s):
    P = s["P"]
    if s["step"]:
        P.norm_rope_step(s["q"], s["k"], s["qr"], s["kr"], s["norm"], s["cache"], s["meta"],
                         theta=s["theta"])
        return {"q": s["qr"], "k": s["kr"]}
    c = s["case"]
    P.norm_rope_rows(s["q"], s["k"], s["v"], s["qr"], s["cache"].k(0), s["cache"].v(0), s["norm"],
                     s["meta"], c["nq"], s["tok0"], s["theta"], row0=s["row0"])
    return {"q": s["qr"], "kv": s["kv"]}


def _weights_own(s):
    c = s["case"]
    s["P"].prompt_weights(s["q"], s["cache"], 0, s["meta"], s["ws"], c["L"] - c["nq"], s["w"],
                          s["out"])
    return {"w": s["out"]}


def _decode_own(s):
    for m in range(s["case"]["M"]):
        s["P"].decode_weights_layer(s["qn"][m], s["kn"][m], s["vn"][m], s["cache"], m, s["meta"],
                                    s["ws"], s["on"][m], s["w"][m], s["out"][m], theta=s["theta"])
    return {"o": s["on"], "w": s["out"], "kv": s["kv"]}


def _evict_own(s):
    case, c = s["case"], s["cache"]
    c.start_prompt(case["L"], s["meta"])
    c.evict(case["heavy"], case["recent"], kv_out=s["kv_out"], w_out=s["out"])
    return {"kv": s["kv_out"], "w": s["out"], "total": c.total, "kv_len": c.kv_len,
            "tok_idx": c.tok_idx, "pos_ids": c.pos_ids, "kept_src": c.kept_src}


def _shared_own(s):
    s["P"].shared_decode_layer(s["qn"], s["kn"], s["vn"], s["prefix"], s["cache"], 0, s["meta"],
                               s["ws"], s["on"], theta=s["theta"])
    return {"o": s["on"], "kv": s["kv"]}


_OWN = {"norm": _norm_own, "weights": _weights_own, "decode": _decode_own, "evict": _evict_own,
        "shared": _shared_own}


def _turn(x, pos, theta):
    """Rotate-half of x (..., n, d), 32 bits, at positions (..., n); the
    angles of far positions are taken in 64."""
    if theta == 0:
        return x
    h = x.shape[-1] // 2
    w = theta ** (-torch.arange(h, dtype=torch.float64, device=x.device) / h)
    a = pos.double()[..., None] * w
    c, s = a.cos().float(), a.sin().float()
    return torch.cat([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], -1)


def _norm_turn(x, w, pos, theta, dt):
    x = x.float()
    x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + EPS) * w.float()
    return _turn(x, pos, theta).to(dt)


def _norm_plain(s):
    c, dt = s["case"], _dt(s["case"])
    if s["step"]:
        at = s["pos"].gather(1, s["tok"].long()[:, None])  # (b, 1): one position for all heads
        s["qr"].copy_(_norm_turn(s["q"], s["qw"], at, s["theta"], dt))
        s["kr"].copy_(_norm_turn(s["k"], s["kw"], at, s["theta"], dt))
        return {"q": s["qr"], "k": s["kr"]}
    n, t0 = c["nq"], s["tok0"]
    at = s["pos"][:, None, t0:t0 + n]
    s["qr"].copy_(_norm_turn(s["q"], s["qw"], at, s["theta"], dt))
    k = _norm_turn(s["k"], s["kw"], at, s["theta"], dt)
    rows = (s["row0"].long()[:, None] + torch.arange(n, device=DEV))[:, None, :, None].expand_as(k)
    s["kv"][0, 0].scatter_(2, rows, k)
    s["kv"][0, 1].scatter_(2, rows, s["v"])
    return {"q": s["qr"], "kv": s["kv"]}


def _see(i, tok, vu):
    """Which of the rows' tokens each token i sees."""
    t = tok.long()
    j, i = t[None, :], i[:, None]
    return (j <= i) & (i <= vu[t][None, :]) & ((vu[i] != i) | (j == i))


def _weights_plain(s):
    c = s["case"]
    nq, L, d, H = c["nq"], c["L"], c["d"], c["H"]
    i = torch.arange(L - nq, L, device=DEV)
    s["out"].copy_(s["w"])
    hs = max(1, (1 << 28) // (nq * L))
    for r in range(c["b"]):
        n = s["len"][r]
        see = _see(i, s["tok_idx"][r, :n], s["vu"][r].long())
        for h in range(0, H, hs):
            k = s["k"][r, h:h + hs, :n].float()
            x = torch.matmul(s["q"][r, h:h + hs].float(), k.transpose(1, 2)) / math.sqrt(d)
            x.masked_fill_(~see, -math.inf)
            m = x.amax(-1, keepdim=True)
            x = torch.exp(x - m.masked_fill(m == -math.inf, 0.0))
            total = x.sum(-1, keepdim=True)
            x /= total.masked_fill(total == 0, 1.0)
            s["out"][r, h:h + hs, :n] += x.sum(1)
        s["out"][r, :, n:] = 0.0  # rows behind the last one are not the operator's
    return {"w": s["out"]}


def _append(s, m, q, k, v, lens):
    """The rotated query and the new row, written behind each sequence's rows."""
    case, kv = s["case"], s["kv"]
    b = case["b"]
    n = torch.as_tensor(np.asarray(lens), device=DEV)
    tok = case["L"] + (n if case["kind"] == "shared" else torch.zeros_like(n))
    at = s["pos"].gather(1, tok[:, None])
    q = _turn(q.float(), at, s["theta"])
    i = torch.arange(b, device=DEV)
    kv[m, 0, i, :, n] = _turn(k.float(), at, s["theta"]).to(kv.dtype)
    kv[m, 1, i, :, n] = v
    return q, n + 1


def _decode_plain(s):
    c = s["case"]
    for m in range(c["M"]):
        q, n = _append(s, m, s["qn"][m], s["kn"][m], s["vn"][m], s["len"])
        k, v = s["kv"][m, 0].float(), s["kv"][m, 1].float()
        r = torch.arange(k.shape[2], device=DEV)
        x = torch.matmul(k, q[..., None])[..., 0] / math.sqrt(c["d"])
        x.masked_fill_(r >= n[:, None, None], -math.inf)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        x /= x.sum(-1, keepdim=True)
        s["on"][m] = torch.matmul(x[:, :, None], v)[:, :, 0].to(s["on"].dtype)
        old = s["w"][m].masked_fill(r >= (n - 1)[:, None, None], 0.0)
        s["out"][m] = old + x
    return {"o": s["on"], "w": s["out"], "kv": s["kv"]}


def _evict_plain(s):
    c = s["case"]
    b, L, heavy, recent = (c[k] for k in ("b", "L", "heavy", "recent"))
    dev = s["kv"].device
    total = s["w"].sum((0, 2), dtype=torch.float64).float()  # near ties decide which rows stay
    tok_idx = torch.arange(L, dtype=torch.int32, device=dev).repeat(b, 1)
    pos_ids = s["pos"][:, :L].clone()
    kept_src = torch.full((b, L), -1, dtype=torch.int32, device=dev)
    n = min(L, heavy + recent)
    if n < L:
        # a stable descending sort puts the lower index of a tie first
        by = total[:, :L - recent].sort(dim=1, descending=True, stable=True).indices[:, :heavy]
        last = torch.arange(L - recent, L, device=dev).expand(b, -1)
        rows = torch.cat([by, last], 1).sort(dim=1).values
    else:
        rows = torch.arange(L, device=dev).expand(b, -1)
    tok_idx[:, :n] = tok_idx.gather(1, rows)
    pos_ids[:, :n] = pos_ids.gather(1, rows)
    kept_src[:, :n] = rows
    s["out"].zero_()
    for i in range(b):
        s["kv_out"][:, :, i, :, :n] = s["kv"][:, :, i].index_select(3, rows[i])
        s["out"][:, i, :, :n] = s["w"][:, i].index_select(2, rows[i])
    return {"kv": s["kv_out"], "w": s["out"], "total": total,
            "kv_len": torch.full((b,), n, dtype=torch.int32, device=dev),
            "tok_idx": tok_idx, "pos_ids": pos_ids, "kept_src": kept_src}


def _shared_plain(s):
    c = s["case"]
    G, b, H, d = c["G"], c["b"], c["H"], c["d"]
    per = b // G
    q, n = _append(s, 0, s["qn"], s["kn"], s["vn"], s["own_len"])
    for g in range(G):
        seqs = slice(g * per, (g + 1) * per)
        kp, vp = (s["prefix"][i, g, :, :s["len"][g]].float() for i in range(2))
        k, v = (s["kv"][0, i, seqs].float() for i in range(2))
        qg = q[seqs]
        xp = torch.matmul(kp, qg.permute(1, 2, 0).contiguous()).permute(2, 0, 1)  # (per, H, P)
        xo = torch.matmul(k, qg[..., None])[..., 0]
        r = torch.arange(k.shape[2], device=DEV)
        xo.masked_fill_(r >= n[seqs, None, None], -math.inf)
        x = torch.cat([xp, xo], -1) / math.sqrt(d)
        x = torch.exp(x - x.amax(-1, keepdim=True))
        x /= x.sum(-1, keepdim=True)
        P = kp.shape[1]
        o = torch.matmul(x[..., :P].transpose(0, 1).contiguous(), vp).transpose(0, 1)
        o = o + torch.matmul(x[..., None, P:], v)[:, :, 0]
        s["on"][seqs] = o.to(s["on"].dtype)
    return {"o": s["on"], "kv": s["kv"]}


_PLAIN = {"norm": _norm_plain, "weights": _weights_plain, "decode": _decode_plain,
          "evict": _evict_plain, "shared": _shared_plain}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def _pairs(vu, L, nq, rows):
    """Visible (query, row) pairs of the last nq tokens."""
    i = np.arange(L - nq, L)
    seen = np.zeros(L + 1, np.int64)
    end = np.minimum(vu[rows], L - 1)
    np.add.at(seen, rows, 1)
    np.add.at(seen, end + 1, -1)
    return int(np.where(vu[i] == i, 1, np.cumsum(seen)[i]).sum())


def work(case):
    kind = case["kind"]
    M, b, H, d, L, n = (case[k] for k in ("M", "b", "H", "d", "L", "nq"))
    e = 4 if case["dtype"] == "f32" else 2
    row = H * d * e
    spans = _spans(case, 1)
    held = _rows(case, spans)
    if kind == "norm":
        nb = b * (2 * 2 if n == 0 else 3 * 2 * n) * row
        return {"bytes": nb, "flops": b * max(n, 1) * 2 * H * d * 7}
    if kind == "weights":
        vu = [_vu_pos(x, _meta_len(case))[0] for x in spans]
        pairs = sum(_pairs(v, L, n, r) for v, r in zip(vu, held))
        rows = sum(len(r) for r in held)
        return {"bytes": (b * n + rows) * row + rows * H * 8, "flops": 2 * d * H * pairs}
    if kind == "decode":
        rows = sum(len(r) for r in held)
        return {"bytes": M * ((2 * rows + 6 * b) * row + (2 * rows + b) * H * 4),
                "flops": M * 4 * d * H * (rows + b)}
    if kind == "evict":
        left = min(L, case["heavy"] + case["recent"])
        moved = M * b * left * (2 * 2 * row + 4 * H)
        return {"bytes": moved + M * b * L * H * 4, "flops": M * b * L * H}
    per = b // case["G"]
    pre = sum(len(r) for r in held)
    mine = int(_own_len(case, 1).sum())
    return {"bytes": (2 * (pre + mine) + 6 * b) * row,
            "flops": 4 * d * H * (per * pre + mine + b)}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions
# ---------------------------------------------------------------------------

def _rotated64(x, pos, rotary):
    """Pair (i, i + d/2) as a complex number times exp(1j pos theta^(-2i/d))."""
    if not rotary:
        return x
    h = x.shape[-1] // 2
    ang = pos.double()[..., None] * torch.pow(
        torch.tensor(THETA, dtype=torch.float64, device=x.device),
        -2.0 * torch.arange(h, device=x.device).double() / (2 * h))
    z = torch.complex(x[..., :h].contiguous(), x[..., h:].contiguous()) * torch.polar(
        torch.ones_like(ang), ang)
    return torch.cat([z.real, z.imag], -1)


def exact(case, seed):
    kind, dt = case["kind"], _dt(case)
    M, b, H, d, L, n = (case[k] for k in ("M", "b", "H", "d", "L", "nq"))
    spans = _spans(case, seed)
    vp = [_vu_pos(x, _meta_len(case)) for x in spans]
    pos = torch.as_tensor(np.stack([p for _, p in vp]), device=DEV)
    held = _rows(case, spans)
    t = _inputs(case, seed)
    if kind == "norm":
        rms = lambda x, w: x / (x.pow(2).sum(-1, keepdim=True) / d + EPS).sqrt() * w.double()
        if n == 0:
            tok = np.random.default_rng(seed).integers(L // 2, L, size=b)
            at = pos[torch.arange(b, device=DEV), torch.as_tensor(tok, device=DEV)][:, None]
            return {x: _rotated64(rms(t[x][:, :, 0].double(), t[x + "w"]), at, case["rotary"])
                    for x in "qk"}
        o = case["offset"]
        out = {"q": torch.empty((b, H, n, d), dtype=torch.float64, device=DEV),
               "kv": torch.zeros((1, 2, b, H, L, d), dtype=torch.float64, device=DEV)}
        for i in range(b):
            q, k = (_rotated64(rms(t[x][i].double(), t[x + "w"]), pos[i, o:o + n], case["rotary"])
                    for x in "qk")
            r0 = o // (i + 1)
            out["q"][i] = q
            out["kv"][0, 0, i, :, r0:r0 + n] = k
            out["kv"][0, 1, i, :, r0:r0 + n] = t["v"][i].double()
        return out
    if kind == "weights":
        w = torch.zeros((b, H, L), dtype=torch.float64, device=DEV)
        for i in range(b):
            vu = vp[i][0]
            rows = torch.as_tensor(held[i], device=DEV)
            vis = torch.as_tensor(vu[held[i]], device=DEV)
            w[i, :, :len(rows)] = t["w"][i, :, :len(rows)].double()
            for h in range(H):
                k = t["rows"][i, h, :len(rows)].double()
                for a in range(0, n, 2048):  # queries by the block
                    tok = torch.arange(L - n + a, min(L, L - n + a + 2048), device=DEV)[:, None]
                    x = torch.mm(t["q"][i, h, a:a + 2048].double(), k.t().contiguous()) / d ** 0.5
                    alone = torch.as_tensor(vu, device=DEV)[tok] == tok
                    hid = (rows > tok) | (vis < tok) | (alone & (rows != tok))
                    x[hid] = -math.inf
                    w[i, h, :len(rows)] += torch.nan_to_num(torch.softmax(x, -1)).sum(0)
        return {"w": w}
    if kind == "evict":
        return {"kv": None, "w": None, "total": t["w"].double().sum((0, 2)), "kv_len": None,
                "tok_idx": None, "pos_ids": None, "kept_src": None}
    # decode and shared: one sequence at a time, the rows it sees put together
    lens = [len(r) for r in held] if kind == "decode" else _own_len(case, seed)
    cap = (L if kind == "decode" else case["own_rows"]) + 1
    o = torch.empty((M, b, H, d), dtype=torch.float64, device=DEV)
    kv = torch.zeros((M, 2, b, H, cap, d), dtype=torch.float64, device=DEV)
    w = torch.zeros((M, b, H, cap), dtype=torch.float64, device=DEV)
    for m in range(M):
        for i in range(b):
            rows = t["rows"][m] if kind == "decode" else t["rows"]
            qn, kn, vn = (t[x][m, i] if kind == "decode" else t[x][i] for x in ("qn", "kn", "vn"))
            ln = int(lens[i])
            at = pos[i, L + (0 if kind == "decode" else ln)].expand(H)
            q = _rotated64(qn.double(), at, case["rotary"])
            kv[m, :, i, :, :cap - 1] = rows[:, i].double()
            kv[m, 0, i, :, ln] = _rotated64(kn.double(), at, case["rotary"]).to(dt).double()
            kv[m, 1, i, :, ln] = vn.double()
            k, v = kv[m, 0, i, :, :ln + 1], kv[m, 1, i, :, :ln + 1]
            if kind == "shared":
                g = i // (b // case["G"])
                k, v = (torch.cat([t["prefix"][j, g, :, :len(held[g])].double(), x], 1)
                        for j, x in enumerate((k, v)))
            p = torch.softmax(torch.matmul(k, q[:, :, None])[:, :, 0] / d ** 0.5, -1)
            o[m, i] = torch.matmul(p[:, None], v)[:, 0]
            if kind == "decode":
                w[m, i, :, :ln + 1] = p
                w[m, i, :, :ln] += t["w"][m, i, :, :ln].double()
    return {"o": o, "w": w, "kv": kv} if kind == "decode" else {"o": o[0], "kv": kv}
