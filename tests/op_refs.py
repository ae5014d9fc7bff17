"""Plain 64-bit forms of the operators beside the cache, and how far fp32
arithmetic may take a result from them (test infrastructure)."""
import math

import numpy as np
import torch

U = 2.0 ** -24  # half a step of fp32, relative
INF = 0x7fffffff


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def rand(shape, seed, dtype, scale=1.0, device="cpu"):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype).to(device)


def vu_pos(spans, T):
    """Span metadata and tied positions of one sequence, from the rules."""
    vu, pos = np.full(T, INF, np.int64), np.zeros(T, np.int64)
    kind = np.zeros(T, np.int64)
    for c, r in spans:
        vu[c + 1:min(r, T)] = r
        vu[c] = c
        kind[c] = 1
        if r < T:
            kind[r] = 1
    at = 0
    for t in range(T):
        if kind[t]:
            pos[t] = pos[t - 1] if t else 0
        else:
            pos[t] = at
            at += 1
    return vu, pos


def some_spans(T, seed, ratio=0.5, lo=2, hi=25):
    rng = np.random.default_rng(seed)
    out, at = [], 0
    while True:
        c = at + int(rng.integers(0, int((lo + hi) / 2 * (1 - ratio) / max(ratio, 0.05)) * 2 + 1))
        r = c + int(rng.integers(lo, hi + 1))
        if r >= T:
            return out
        out.append((c, r))
        at = r + 1


def rotate(x, pos, theta):
    """Rotate-half of x (..., n, d) at positions pos (n,), 64 bits."""
    if theta == 0:
        return x
    h = x.shape[-1] // 2
    a = torch.as_tensor(pos, dtype=torch.float64, device=x.device)[:, None] * theta ** (
        -torch.arange(h, dtype=torch.float64, device=x.device) / h)
    c, s = a.cos(), a.sin()
    return torch.cat([x[..., :h] * c - x[..., h:] * s, x[..., h:] * c + x[..., :h] * s], -1)


def norm(x, w, eps):
    x = x.double()
    y = x / (x.square().mean(-1, keepdim=True) + eps).sqrt()
    return y if w is None else y * w.double()


def norm_rope(x, w, eps, pos, theta):
    return rotate(norm(x, w, eps), pos, theta)


def norm_rope_tol(x, w, eps, dtype):
    """Half a step of the result's type (added by the caller, relative to the
    result) and, relative to the pair's size: the squares' sum of d terms in
    chains of at most 21 (half of 21 U on the root), root, quotient, two
    products, angle (pi U) and sine/cosine (2 U each), two fused products:
    together below 32 U."""
    y = norm(x, w, eps).abs()
    h = y.shape[-1] // 2
    pair = y[..., :h] + y[..., h:]
    return 32 * U * torch.cat([pair, pair], -1)


def see(tok_rows, toks, vu):
    """(queries, rows): which rows' tokens each token sees."""
    j, i = np.asarray(tok_rows, np.int64)[None, :], np.asarray(toks, np.int64)[:, None]
    ok = (j >= 0) & (j < len(vu))
    jj = np.where(ok, j, 0)
    return ok & (j <= i) & (i <= vu[jj]) & ((vu[i] != i) | (j == i))


def prompt_weights(q, k, tok_rows, toks, vu, scale):
    """Weights that q (H, nq, d) give rows k (H, n, d): (sums, relative bound)."""
    m = torch.as_tensor(see(tok_rows, toks, vu), device=q.device)
    q, k = q.double(), k.double()
    x = torch.matmul(q, k.transpose(1, 2)) * scale
    x = x.masked_fill(~m, -math.inf)
    p = torch.nan_to_num(torch.softmax(x, -1), nan=0.0)
    # a score's error: d products summed in fp32, of size at most A; its
    # distance from the normaliser is rounded once more; exponential and
    # quotient a few U; the sums over rows and over queries
    A = float((torch.matmul(q.abs(), k.abs().transpose(1, 2)) * scale).max()) if k.shape[1] and \
        q.shape[1] else 0.0
    d, n, nq = q.shape[2], k.shape[1], q.shape[1]
    rel = 2 * (d + 8) * U * A + (n + nq + 16) * U
    return p.sum(1), rel


def attend(q, k, v, scale):
    """One query a head: q (H, d), k, v (H, n, d) -> (o, p, error scale of the
    scores A, sum of p |v|)."""
    q, k, v = q.double(), k.double(), v.double()
    p = torch.softmax(torch.matmul(k, q[:, :, None])[..., 0] * scale, -1)
    o = torch.matmul(p[:, None], v)[:, 0]
    A = float((torch.matmul(k.abs(), q.abs()[:, :, None]) * scale).max())
    return o, p, A, torch.matmul(p[:, None], v.abs())[:, 0]
