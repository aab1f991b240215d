"""GPU parity of the norms of queries and keys with the position rotation, forward
and backward, against plain 64-bit runs, differences and torch's autograd.

What is allowed beyond the outputs' own rounding (see _serve_ref.close): a row's sum of
squares, its root, weight, turn and scale are about ten fp32 roundings of values up to
six RMS, and the reduced angle is held to 2^-24 of a half turn: 10 6 2^-24 + 6 pi 2^-24
= 5e-6.  Without a norm or with a row's own size the scale is that of the row.  A weight
gradient sums n terms in chains of at most a few hundred: |error| <= 300 2^-24 sum |terms|.
"""
import numpy as np
import pytest
import torch

import paper_2608_06838_amd as sf

import _serve_ref as ref
from _serve_ref import close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DELTA = 1e-5
IO = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(B, L, Hq, Hk, D, io="bf16", seed=0, weight=True, R=0, far=4096, given_pos=True):
    gen = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    t = [rnd(B, L, H, D).to(IO[io]).to(DEV) for H in (Hq, Hk, Hq, Hk)]
    kw = dict(q_weight=(1 + 0.3 * rnd(D)).to(DEV), k_weight=(1 + 0.3 * rnd(D)).to(DEV)) if weight else {}
    if R:
        kw["inv_freq"] = (10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).to(DEV)
        if given_pos:
            kw["pos"] = torch.randint(0, far, (B, L), generator=gen).to(DEV)
    return t, kw


def check(t, kw, out_f=None, out_b=None):
    q, k, dyq, dyk = t
    yq, yk = sf.qk_norm_fwd(q, k, **kw, out=out_f)
    dq, dk, dwq, dwk = sf.qk_norm_bwd(q, k, dyq, dyk, **kw, out=out_b)
    torch.cuda.synchronize()
    wq, wk = ref.qk(q, k, **kw)
    close("yq", yq, wq, DELTA)
    close("yk", yk, wk, DELTA)
    (rq, rwq, aq), (rk, rwk, ak) = ref.qk(q, k, **kw, dyq=dyq, dyk=dyk)
    close("dq", dq, rq, DELTA)
    close("dk", dk, rk, DELTA)
    if kw.get("q_weight") is None:
        assert dwq is None and dwk is None
    else:
        for name, x, r, a in (("dwq", dwq, rwq, aq), ("dwk", dwk, rwk, ak)):
            off = np.abs(ref.f64(x) - r) / (300 * 2.0 ** -24 * a + 1e-30)
            print(f"  {name}: {off.max():.3f} of its bound", flush=True)
            assert off.max() <= 1, name
    return yq, yk, dq, dk, dwq, dwk


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("norm", ["l2", "rms", "none"])
@pytest.mark.parametrize("R,inter", [(0, False), (128, False), (128, True), (48, False), (16, True)])
def test_qk_parity(io, norm, R, inter):
    print(f"[qk] {io} {norm} R={R} interleaved={inter}", flush=True)
    for weight in (True, False):
        t, kw = make(2, 37, 6, 3, 128, io, seed=R, weight=weight, R=R)
        check(t, dict(kw, norm=norm, interleaved=inter, q_scale=0.3))


@pytest.mark.parametrize("D", [16, 32, 48, 64, 96, 112, 144, 192, 256])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_qk_head_dims(D, io):
    print(f"[qk] {io} D={D}", flush=True)
    for R in sorted({16, D // 32 * 16, D} - {0}):
        t, kw = make(1, 21, 5, 2, D, io, seed=D, R=R)
        check(t, dict(kw, norm="rms"))


@pytest.mark.parametrize("B,L,Hq,Hk", [(1, 1, 1, 1), (1, 1, 40, 8), (3, 1, 2, 2), (1, 5, 17, 1), (1, 700, 40, 40),
                                       (2, 4099, 3, 1)])
def test_qk_sizes(B, L, Hq, Hk):
    """One token and many, heads that leave a wave's rows half empty, more tokens than
    the launch has waves."""
    print(f"[qk] B={B} L={L} heads {Hq}/{Hk}", flush=True)
    t, kw = make(B, L, Hq, Hk, 64, seed=L, R=64)
    check(t, dict(kw, norm="rms"))


def test_qk_positions():
    """Far positions keep their angles; pos0 + l; one row of positions for all batches;
    negative positions."""
    print("[qk] positions", flush=True)
    t, kw = make(2, 33, 2, 2, 128, "f32", seed=3, R=128, far=2 ** 31)
    check(t, dict(kw, norm="l2"))
    kw.pop("pos")
    check(t, dict(kw, norm="l2", pos0=262144))
    check(t, dict(kw, norm="l2", pos=(torch.arange(33, device=DEV) - 17)[None].expand(2, 33)))
    a = sf.qk_norm_fwd(t[0], t[1], norm="l2", **{n: kw[n] for n in ("q_weight", "k_weight", "inv_freq")}, pos0=1000)
    b = sf.qk_norm_fwd(t[0][:, 13:], t[1][:, 13:], norm="l2",
                       **{n: kw[n] for n in ("q_weight", "k_weight", "inv_freq")}, pos0=1013)
    assert torch.equal(a[0][:, 13:], b[0]) and torch.equal(a[1][:, 13:], b[1])


def test_qk_strides_and_slices():
    """q and k as slices of one projection; outputs and gradients into slices of one
    buffer, whose other columns stay; a gradient broadcast over the tokens."""
    B, L, Hq, Hk, D = 2, 19, 4, 2, 64
    print("[qk] slices", flush=True)
    t, kw = make(B, L, Hq, Hk, D, seed=4, R=32)
    wide = torch.full((B, L + 1, (Hq + Hk) * D + 32), 3.0, dtype=torch.bfloat16, device=DEV)[:, :L]
    views = lambda w: (w[..., :Hq * D].unflatten(2, (Hq, D)),  # noqa: E731
                       w[..., Hq * D:(Hq + Hk) * D].unflatten(2, (Hk, D)))
    for dst, src in zip(views(wide), t):
        dst.copy_(src)
    dyk = t[3][:, :1].expand(B, L, Hk, D)
    y, d = torch.full_like(wide, 7.0), torch.full_like(wide, 7.0)
    ws = torch.empty(sf.qk_norm_bwd_workspace_bytes(*views(wide), t[2], dyk), dtype=torch.uint8, device=DEV)
    dw = [torch.empty(D, device=DEV) for _ in range(2)]
    check([*views(wide), t[2], dyk], dict(kw, norm="rms"), out_f=views(y), out_b=(*views(d), *dw, ws))
    assert bool((y[..., (Hq + Hk) * D:] == 7).all()) and bool((d[..., (Hq + Hk) * D:] == 7).all())
    # heads outermost: [B, H, L, D] tensors seen as [B, L, H, D]
    turned = [x.transpose(1, 2).contiguous().transpose(1, 2) for x in t]
    check(turned, dict(kw, norm="l2"))


def test_qk_zero_and_odd_rows():
    """A zero row stays zero (its gradient is finite), a row of NaN or infinity spoils
    only itself, tiny and large rows are normalised."""
    print("[qk] odd rows", flush=True)
    t, kw = make(1, 8, 2, 1, 64, "f32", seed=5, R=64)
    q = t[0]
    q[0, 1] = 0
    q[0, 2, 0] = float("nan")
    q[0, 3, 1, 5] = float("inf")
    q[0, 4] *= 1e-3
    q[0, 5] *= 1e15
    yq, yk = sf.qk_norm_fwd(q, t[1], norm="rms", **kw)
    dq, dk, dwq, dwk = sf.qk_norm_bwd(q, t[1], t[2], t[3], norm="rms", **kw)
    torch.cuda.synchronize()
    assert not yq[0, 1].any() and bool(dq[0, 1].isfinite().all())
    bad = [(2, 0), (3, 1)]
    for tok in range(8):
        for h in range(2):
            assert bool(yq[0, tok, h].isfinite().all()) == ((tok, h) not in bad)
    assert bool(yk.isfinite().all()) and bool(dwk.isfinite().all())
    want, _ = ref.qk(q[:, 4:6], t[1][:, 4:6], norm="rms", **{**kw, "pos": kw["pos"][:, 4:6]})
    close("yq", yq[:, 4:6], want, DELTA)


def test_qk_gradient_against_differences():
    """Central differences of the 64-bit formula's loss agree with the kernel's gradient."""
    print("[qk] differences", flush=True)
    t, kw = make(1, 3, 2, 1, 32, "f32", seed=6, R=16)
    kw = dict(kw, norm="l2", q_scale=0.7, interleaved=True)
    dq, dk, dwq, dwk = sf.qk_norm_bwd(*t, **kw)
    loss = lambda q, k, kw: sum(float((a * ref.f64(b)).sum()) for a, b in zip(ref.qk(q, k, **kw), t[2:]))  # noqa: E731
    rng, h = np.random.RandomState(0), 1e-5
    for name, x, d in (("q", t[0], dq), ("k", t[1], dk), ("q_weight", kw["q_weight"], dwq),
                       ("k_weight", kw["k_weight"], dwk)):
        for _ in range(6):
            at = tuple(rng.randint(n) for n in x.shape)
            vals = []
            for s in (h, -h):
                y = x.double().cpu().clone()
                y[at] += s
                a = dict(q=t[0], k=t[1])
                b = dict(kw)
                (a if name in a else b)[name] = y
                vals.append(loss(a["q"], a["k"], b))
            want = (vals[0] - vals[1]) / (2 * h)
            assert abs(float(d[at]) - want) <= 1e-4 * max(1.0, abs(want)), (name, at)


def test_qk_graph_streams_repeat():
    """Captured with its workspace, replayed with eager calls between: always the same bits."""
    print("[qk] graph", flush=True)
    t, kw = make(2, 300, 8, 2, 128, seed=7, R=64)
    kw["norm"] = "rms"
    y0, g0 = sf.qk_norm_fwd(*t[:2], **kw), sf.qk_norm_bwd(*t, **kw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y1, g1 = sf.qk_norm_fwd(*t[:2], **kw, stream=side), sf.qk_norm_bwd(*t, **kw, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*y0, *g0), (*y1, *g1)))
    out_f, out_b = tuple(torch.empty_like(x) for x in y0), [torch.empty_like(x) for x in g0]
    ws = torch.empty(sf.qk_norm_bwd_workspace_bytes(*t), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sf.qk_norm_fwd(*t[:2], **kw, out=out_f)
        sf.qk_norm_bwd(*t, **kw, out=(*out_b, ws))
    for _ in range(3):
        for x in (*out_f, *out_b):
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((*y0, *g0), (*out_f, *out_b)))
        assert torch.equal(sf.qk_norm_bwd(*t, **kw)[2], g0[2])


def test_qk_far_rows():
    """Rows more than 2^32 bytes from the first."""
    print("[qk] far rows", flush=True)
    t, kw = make(1, 60, 1, 1, 64, seed=8, R=64)
    wide = torch.empty(1, 60, 1, 50000000, dtype=torch.bfloat16, device=DEV)  # 100 MB rows, 6 GB
    q, k = wide[..., :64], wide[..., 64:128]
    q.copy_(t[0])
    k.copy_(t[1])
    check([q, k, t[2], t[3]], dict(kw, norm="l2"))


def test_qk_empty():
    t, kw = make(1, 4, 2, 1, 64, seed=9)
    dq, dk, dwq, dwk = sf.qk_norm_bwd(*[x[:, :0] for x in t], norm="rms", **kw)
    yq, yk = sf.qk_norm_fwd(t[0][:, :0], t[1][:, :0], norm="rms", **kw)
    torch.cuda.synchronize()
    assert yq.numel() == dk.numel() == 0 and not dwq.any() and not dwk.any()
