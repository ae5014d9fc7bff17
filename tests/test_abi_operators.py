"""Refusals of the operators beside the cache: every bad argument is turned
down on the host, before any HIP call (so these run without a GPU)."""
import ctypes
import math
import os
import re
import shutil
import subprocess

import pytest
import torch

from paper_2310_08152_amd import build

FAKE = ctypes.c_void_p(4096)   # never dereferenced: every call below fails a host check first
FAKE2 = ctypes.c_void_p(8192)
ODD = ctypes.c_void_p(4098)
NULL = None


@pytest.fixture(scope="module")
def B():
    from paper_2310_08152_amd import binding
    return binding


def caller(f, ok):
    """f with the arguments of `ok` (in order), some of them replaced."""
    def call(**kw):
        assert set(kw) <= set(ok), kw
        return f(*dict(ok, **kw).values())
    return call


def test_norm_rope_refuses(B):
    ok = dict(q=FAKE, k=FAKE, v=FAKE, qo=FAKE2, ko=FAKE2, vo=FAKE2, qw=FAKE, kw=FAKE, eps=1e-6, b=2,
              H=4, n=8, xb=4 * 8 * 64, xh=8 * 64, xr=64, qs=8 * 64, ks=10 * 64, rows=10, d=64,
              dt=B.BF16, pos=FAKE, L_meta=20, tok0=12, cur=NULL, row0=NULL, theta=1e4, st=NULL,
              stream=NULL)
    call = caller(B.lib.qk_norm_rope, ok)
    assert call(q=NULL) == B.EINVAL and call(qo=NULL) == B.EINVAL
    assert call(k=NULL) == B.EINVAL and call(vo=NULL) == B.EINVAL
    assert call(q=NULL, k=NULL, v=NULL, qo=NULL, ko=NULL, vo=NULL) == B.EINVAL
    assert call(dt=3) == B.EINVAL and call(d=72) == B.EUNSUP
    assert call(b=0) == B.EINVAL and call(H=-1) == B.EINVAL and call(n=-1) == B.EINVAL
    for eps in (0.0, -1.0, math.inf, math.nan):
        assert call(eps=eps) == B.EINVAL
    assert call(xb=-64) == B.EINVAL and call(xr=60) == B.EINVAL and call(xh=-1) == B.EINVAL
    assert call(qs=8 * 64 - 8) == B.EINVAL and call(ks=10 * 64 - 8) == B.EINVAL
    assert call(rows=7) == B.EINVAL
    assert call(tok0=13) == B.EINVAL and call(tok0=-1) == B.EINVAL and call(pos=NULL) == B.EINVAL
    assert call(theta=-1.0) == B.EINVAL and call(theta=math.nan) == B.EINVAL
    assert call(cur=FAKE, L_meta=0) == B.EINVAL
    assert call(cur=FAKE, L_meta=0, theta=0.0, pos=NULL) == B.EINVAL
    for x in ("q", "k", "v", "qo", "ko", "vo", "qw", "kw"):
        assert call(**{x: ODD}) == B.EINVAL, x
    assert "aligned" in B.last_error()
    assert call(b=2 ** 20, H=2 ** 11, n=8) == B.EUNSUP
    assert call(n=0) == B.OK  # nothing to do


def test_attn_weights_refuses(B):
    ws = B.sckv_attn_weights_workspace_bytes(2, 3, 40, 100)
    assert ws > 0 and B.sckv_attn_weights_workspace_bytes(0, 3, 40, 100) == 0
    assert B.sckv_attn_weights_workspace_bytes(2, 3, 0, 100) > 0
    ok = dict(q=FAKE, k=FAKE, wi=FAKE, wo=FAKE2, b=2, H=3, nq=40, d=80, qs=40 * 80, ks=100 * 80,
              dt=B.F32, scale=0.1, vu=FAKE, L_meta=90, tok0=50, len=FAKE, tok=FAKE, cap=100,
              ws=FAKE, wsb=ws, stream=NULL)
    call = caller(B.lib.cached_attn_weights, ok)
    for x in ("q", "k", "wo", "vu", "len", "tok", "ws"):
        assert call(**{x: NULL}) == B.EINVAL, x
    for x in ("q", "k", "wi", "wo", "ws"):
        assert call(**{x: ODD}) == B.EINVAL, x
    assert call(dt=2) == B.EINVAL and call(d=128) == B.EUNSUP
    for x in ("b", "H", "cap", "L_meta"):
        assert call(**{x: 0}) == B.EINVAL, x
    assert call(nq=-1) == B.EINVAL
    assert call(tok0=51) == B.EINVAL and call(tok0=-1) == B.EINVAL
    assert call(qs=40 * 80 - 4) == B.EINVAL and call(ks=99 * 80) == B.EINVAL
    assert call(qs=40 * 80 + 2) == B.EINVAL
    for s in (0.0, -1.0, math.inf, math.nan):
        assert call(scale=s) == B.EINVAL
    assert call(wsb=ws - 1) == B.EINVAL and "workspace" in B.last_error()
    assert call(cap=65537, ks=65537 * 80) == B.EUNSUP
    assert call(nq=65537, qs=65537 * 80, L_meta=70000, tok0=0) == B.EUNSUP


STEP = dict(q=FAKE, kn=FAKE, vn=FAKE, kc=FAKE2, vc=FAKE2, len=FAKE, cur=FAKE, vu=FAKE, pos=FAKE,
            L_meta=100)


def step_refusals(B, call, arrays, aligned, ws):
    for x in arrays:
        assert call(**{x: NULL}) == B.EINVAL, x
    for x in aligned:
        assert call(**{x: ODD}) == B.EINVAL, x
    assert call(dt=9) == B.EINVAL and call(d=96) == B.EUNSUP
    for x in ("b", "H", "cap", "L_meta"):
        assert call(**{x: 0}) == B.EINVAL, x
    assert call(scale=0.0) == B.EINVAL and call(scale=math.nan) == B.EINVAL
    assert call(theta=-1.0) == B.EINVAL and call(theta=math.inf) == B.EINVAL
    assert call(pos=NULL) == B.EINVAL
    assert call(wsb=ws - 1) == B.EINVAL and "workspace" in B.last_error()


def test_decode_weights_refuses(B):
    ws = B.sckv_decode_weights_workspace_bytes(2, 4, 128, 64)
    assert ws > 0 and B.sckv_decode_weights_workspace_bytes(2, 4, 0, 64) == 0
    ok = dict(STEP, o=FAKE2, wi=FAKE, wo=FAKE, b=2, H=4, cap=128, d=64, dt=B.BF16, scale=0.1,
              theta=1e4, ws=FAKE, wsb=ws, st=NULL, stream=NULL)
    call = caller(B.lib.compacted_decode_attn_weights, ok)
    step_refusals(B, call, ("q", "kn", "vn", "kc", "vc", "len", "cur", "vu", "o", "wo", "ws"),
                  ("q", "kn", "vn", "kc", "vc", "o", "wi", "wo", "ws"), ws)


def test_shared_prefix_refuses(B):
    ws = B.sckv_shared_decode_workspace_bytes(6, 4, 3, 200, 128, 64)
    assert ws > 0 and B.sckv_shared_decode_workspace_bytes(6, 4, 0, 200, 128, 64) == 0
    ok = dict(q=FAKE, kn=FAKE, vn=FAKE, kp=FAKE, vp=FAKE, plen=FAKE, G=3, P=200, kc=FAKE2, vc=FAKE2,
              len=FAKE, cur=FAKE, vu=FAKE, pos=FAKE, L_meta=100, o=FAKE2, b=6, H=4, cap=128, d=64,
              dt=B.BF16, scale=0.1, theta=1e4, ws=FAKE, wsb=ws, st=NULL, stream=NULL)
    call = caller(B.lib.shared_prefix_decode_attn, ok)
    step_refusals(B, call, ("q", "kn", "vn", "kp", "vp", "plen", "kc", "vc", "len", "cur", "vu", "o",
                            "ws"),
                  ("q", "kn", "vn", "kp", "vp", "kc", "vc", "o", "ws"), ws)
    assert call(G=4) == B.EINVAL and call(G=0) == B.EINVAL and call(P=0) == B.EINVAL
    assert call(G=12) == B.EINVAL


def test_evict_refuses(B):
    ok = dict(kv=FAKE, out=NULL, w=FAKE, wo=NULL, M=2, b=3, H=4, cap=100, d=64, dt=B.BF16, len=FAKE,
              tok=FAKE, pos=FAKE, heavy=5, recent=5, total=FAKE, src=FAKE, stream=NULL)
    call = caller(B.lib.kv_evict, ok)
    for x in ("kv", "w", "len", "tok", "pos", "total", "src"):
        assert call(**{x: NULL}) == B.EINVAL, x
    for x in ("kv", "out", "w", "wo"):
        assert call(**{x: ODD}) == B.EINVAL, x
    assert call(out=FAKE) == B.EINVAL and call(wo=FAKE) == B.EINVAL
    for x in ("M", "b", "H", "cap"):
        assert call(**{x: 0}) == B.EINVAL, x
    assert call(dt=5) == B.EINVAL and call(d=96) == B.EUNSUP and call(cap=65537) == B.EUNSUP
    assert call(heavy=-1) == B.EINVAL and call(recent=-1) == B.EINVAL
    assert call(heavy=0, recent=0) == B.EINVAL
    assert call(M=2 ** 15, b=2 ** 15, H=4) == B.EUNSUP
    ok = dict(w=FAKE, wo=NULL, M=2, b=3, H=4, cap=100, len=FAKE, src=FAKE, stream=NULL)
    call = caller(B.lib.kv_compact_weights, ok)
    for x in ("w", "len", "src"):
        assert call(**{x: NULL}) == B.EINVAL, x
    assert call(w=ODD) == B.EINVAL and call(wo=ODD) == B.EINVAL
    assert call(M=0) == B.EINVAL and call(cap=65537) == B.EUNSUP
    assert call(M=2 ** 15, b=2 ** 15, H=4) == B.EUNSUP


def test_binding_refuses_what_is_not_on_a_gpu(B):
    x = torch.zeros(2, 4, 8, 64)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(B.SckvError):
        B.qk_norm_rope(x, None, None, x, None, None, None, None, 1e-6, 2, 4, 8, 2048, 512, 64, 512,
                       0, 0, 64, i, 1, 0, None, None, 0.0)
    with pytest.raises(B.SckvError):  # an output without its input
        B.qk_norm_rope(x, None, None, x, x, None, None, None, 1e-6, 2, 4, 8, 2048, 512, 64, 512, 0,
                       0, 64, i, 1, 0, None, None, 0.0)
    with pytest.raises(B.SckvError):
        B.cached_attn_weights(x, x, None, x, 2, 4, 8, 64, 512, 512, 0.1, i, 1, 0, i, i, 8, x)
    with pytest.raises(B.SckvError):
        B.kv_compact_weights(x, None, 1, 2, 4, 8, i, i)


def test_path_refuses(B):
    from paper_2310_08152_amd import path as P
    with pytest.raises(ValueError):
        P.KVCache(1, 1, 2, 8, 64, torch.float32, "cpu", kv=torch.zeros(1, 2, 1, 2, 8, 80))
    with pytest.raises(ValueError):
        P.KVCache(1, 1, 2, 8, 64, torch.bfloat16, "cpu", kv=torch.zeros(1, 2, 1, 2, 8, 64))
    c = P.KVCache(1, 1, 2, 8, 64, torch.float32, "cpu")
    with pytest.raises(ValueError):
        c.evict(1, 1)
    with pytest.raises(ValueError):
        c.track_weights(torch.zeros(1, 1, 2, 9))
    meta, x = None, torch.zeros(1, 2, 1, 64)
    with pytest.raises(ValueError):
        P.prompt_weights(x, c, 0, meta, None, 0)
    with pytest.raises(ValueError):
        P.decode_weights_layer(x[:, :, 0], x[:, :, 0], x[:, :, 0], c, 0, meta, None, x)
    c.track_weights()
    assert c.w.shape == (1, 1, 2, 8)
    c.kv_len.fill_(3)
    with pytest.raises(ValueError):  # no workspace for weights: refused before anything changes
        P.prefill_progressive(x[None], x[None], x[None], x[None], c, meta,
                              type("Ws", (), {"weights": None}), 1, 1, evict=(1, 1))
    assert int(c.kv_len[0]) == 3


@pytest.mark.parametrize("source", ("norm_rope", "evict", "weights", "shared"))
def test_no_kernel_spills(source, tmp_path):
    if not (shutil.which("hipcc") or os.path.exists("/opt/rocm/bin/hipcc")):
        pytest.skip("no hipcc")
    r = subprocess.run([build._hipcc(), *build.HIPCC_FLAGS, "-Rpass-analysis=kernel-resource-usage",
                        "--cuda-device-only", "-c", os.path.join(build.CSRC, source + ".hip"),
                        "-o", str(tmp_path / "k.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    names = re.findall(r"Function Name: (\S+)", r.stderr)
    scratch = [int(x) for x in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", r.stderr)]
    spilled = [int(x) for x in re.findall(r"VGPRs Spill: (\d+)", r.stderr)]
    assert names and len(names) == len(scratch) == len(spilled)
    assert not [n for n, s, v in zip(names, scratch, spilled) if s or v]


@pytest.mark.parametrize("b,H,L_cap", [(1, 4, 256), (1, 32, 2000), (16, 32, 4096), (3, 7, 65536)])
def test_weights_workspace_serves_fewer_queries(B, b, H, L_cap):
    """A workspace for the most queries of a call holds every smaller call (a
    prompt's ragged last block)."""
    most = 0
    for nq in [*range(1, 300), 511, 512, 513, 1023, 1024, 1025, 2047, 2049, 4096, 65535, 65536]:
        n = B.sckv_attn_weights_workspace_bytes(b, H, nq, L_cap)
        assert n >= most, (nq, n, most)
        most = n
