"""GPU parity of the ragged-batch calls (gated delta rule and short convolution over
packed sequences, states and tails in a pool of slots) against plain 64-bit runs.

What is allowed beyond the outputs' own rounding: the arithmetic is fp32.  A token of
the delta rule rounds a state element about three times (2^-24 each); the transition
contracts, so the errors of the last n_eff ~ 100 tokens remain, sqrt(100) 3 2^-24 =
2e-6 of the RMS, and the largest of 10^6 elements lies about five deviations out: 1e-5.
DELTA allows five times that.  The convolution rounds five times, then the activation
(exp2, a division): 20 2^-24 at most of values up to six RMS, 1e-5.
"""
import numpy as np
import pytest
import torch

import paper_2608_06838_amd as sf
from paper_2608_06838_amd import synth

import _serve_ref as ref
from _serve_ref import close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DELTA, DELTA_CONV = 5e-5, 1e-5
IO = {"bf16": torch.bfloat16, "f32": torch.float32}


def gdn_inputs(T, Hk, Hv, Dk, Dv, n_slots, io="bf16", seed=0, g_mu=3.0):
    gen = torch.Generator().manual_seed(seed)
    q, k = torch.randn(T, Hk, Dk, generator=gen), torch.randn(T, Hk, Dk, generator=gen)
    k = k / k.norm(dim=-1, keepdim=True).clamp_min(1e-9)
    v = torch.randn(T, Hv, Dv, generator=gen)
    g = torch.nn.functional.logsigmoid(torch.randn(T, Hv, generator=gen) + g_mu)
    beta = torch.sigmoid(torch.randn(T, Hv, generator=gen))
    state = 0.1 * torch.randn(n_slots, Hv, Dk, Dv, generator=gen)
    return [x.to(IO[io]).to(DEV) for x in (q, k, v)] + [x.to(DEV) for x in (g, beta, state)]


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=DEV)


def run_gdn(args, cu, slots=None, fresh=None, max_len=None, delta=DELTA, **kw):
    """The call against the plain run; rows of no sequence and slots of none keep their bits."""
    q, k, v, g, beta, state = args
    want_o, written, want_S = ref.gdn(q, k, v, g, beta, state, cu, slots, fresh)
    before = state.clone()
    o = torch.full(v.shape, 7.0, dtype=v.dtype, device=DEV)
    cu_d, sl = i32(cu), None if slots is None else i32(slots)
    fr = None if fresh is None else torch.tensor(fresh, dtype=torch.uint8, device=DEV)
    ws = torch.empty(sf.gdn_ragged_workspace_bytes(*args, cu_d, sl, max_len=max_len), dtype=torch.uint8, device=DEV)
    got = sf.gdn_ragged_fwd(*args, cu_d, sl, fresh=fr, max_len=max_len, out=(o, ws), **kw)
    torch.cuda.synchronize()
    assert got is o
    w = torch.tensor(written, device=DEV)
    assert bool((o[~w] == 7).all()), "rows of no sequence were written"
    close("o", o[w], want_o[written], delta)
    used = sorted({(i if slots is None else int(slots[i])) for i in range(len(cu) - 1)
                   if min(max(cu[i + 1], 0), v.shape[0]) > min(max(cu[i], 0), v.shape[0])
                   and 0 <= (i if slots is None else int(slots[i])) < len(state)})
    rest = [s for s in range(len(state)) if s not in used]
    assert torch.equal(state[rest], before[rest]), "a slot of no sequence was written"
    if used:
        close("state", state[used], want_S[used], delta)
    return o


LENS = {"one": [1], "decode": [1] * 9, "drafts": [3, 1, 0, 5, 2], "mixed": [1, 70, 1, 0, 129, 2],
        "edges": [63, 64, 65, 127, 128, 15, 16, 17], "long": [300, 1, 515]}


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("name", list(LENS))
def test_gdn_lengths(io, name):
    lens = LENS[name]
    print(f"[gdn ragged] {io} {lens}", flush=True)
    cu, T = ref.sequences(lens)
    slots = np.random.RandomState(1).permutation(len(lens) + 3)[:len(lens)]
    run_gdn(gdn_inputs(T, 2, 4, 128, 128, len(lens) + 3, io, seed=len(lens)), cu, slots, max_len=max(lens))


@pytest.mark.parametrize("Hk,Hv,Dk,Dv", [(1, 1, 64, 64), (3, 3, 64, 128), (2, 6, 128, 64), (1, 5, 128, 256),
                                         (2, 2, 64, 256)])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_gdn_heads(Hk, Hv, Dk, Dv, io):
    print(f"[gdn ragged] {io} heads {Hk}/{Hv} of {Dk}, {Dv}", flush=True)
    cu, T = ref.sequences([5, 150, 1, 64])
    run_gdn(gdn_inputs(T, Hk, Hv, Dk, Dv, 4, io, seed=Hv), cu, max_len=150)


def test_gdn_fresh_and_skipped_slots():
    """fresh starts from zero whatever the slot holds (NaN here); slots out of range skip
    their sequence; an empty sequence's slot stays, fresh or not."""
    lens, slots, fresh = [3, 100, 2, 90, 0, 4], [4, 1, -1, 99, 0, 2], [1, 1, 0, 1, 1, 0]
    print("[gdn ragged] fresh and skipped", flush=True)
    cu, T = ref.sequences(lens)
    args = gdn_inputs(T, 1, 2, 64, 64, 6, seed=5)
    args[5][4] = float("nan")
    args[5][1] = float("inf")
    args[5][5] = float("nan")
    keep = args[5].clone()
    state = args[5]
    want_o, written, want_S = ref.gdn(*args[:5], torch.nan_to_num(state, 0, 0, 0), cu, slots, fresh)
    o = torch.full(args[2].shape, 7.0, dtype=torch.bfloat16, device=DEV)
    sf.gdn_ragged_fwd(*args, i32(cu), i32(slots), fresh=torch.tensor(fresh, dtype=torch.bool, device=DEV),
                      out=(o, torch.empty(1 << 24, dtype=torch.uint8, device=DEV)))
    torch.cuda.synchronize()
    w = torch.tensor(written, device=DEV)
    assert bool((o[~w] == 7).all())
    close("o", o[w], want_o[written], DELTA)
    close("state", state[[4, 1, 2]], want_S[[4, 1, 2]], DELTA)
    assert torch.equal(state[[0, 3]], keep[[0, 3]]) and bool(state[5].isnan().all())


@pytest.mark.parametrize("max_len", [None, 1, 5000])
def test_gdn_rows_outside(max_len):
    """Rows before the first sequence and behind the last hold NaN and are not read;
    max_len never changes what is computed."""
    lens = [70, 1, 33]
    print(f"[gdn ragged] rows outside, max_len {max_len}", flush=True)
    cu, T = ref.sequences(lens, T=5 + sum(lens) + 66, before=5)
    args = gdn_inputs(T, 2, 2, 128, 64, 3, seed=8)
    for x in args[:5]:
        x[:5] = float("nan")
        x[cu[-1]:] = float("nan")
    run_gdn(args, cu, max_len=max_len)


@pytest.mark.parametrize("cu", [[-7, 40, 40, 1000], [400, 500, 600, 700], [-90, -80, 30, 150]])
def test_gdn_bounds_outside(cu):
    """Entries outside [0, T] count as the nearer end."""
    print(f"[gdn ragged] bounds {cu}", flush=True)
    for max_len in (1, 150):
        run_gdn(gdn_inputs(150, 1, 1, 64, 64, 3, seed=9), cu, max_len=max_len)


@pytest.mark.parametrize("cu", [[0, 200, 90, 150], [150, 100, 50, 0], [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0],
                                [130, 0, 150, 20, 70]])
def test_gdn_decreasing_bounds(cu):
    """Entries that decrease: rows and slots no sequence names are left alone."""
    T, N = 150, len(cu) - 1
    print(f"[gdn ragged] bounds {cu}", flush=True)
    args = gdn_inputs(T, 1, 2, 64, 64, N + 1, seed=9)
    at = [min(max(c, 0), T) for c in cu]
    named = np.zeros(T, bool)
    for b, e in zip(at, at[1:]):
        named[b:e] = True
    for max_len in (1, 150):
        S, o = args[5].clone(), torch.full(args[2].shape, 7.0, dtype=torch.bfloat16, device=DEV)
        ws = torch.zeros(1 << 24, dtype=torch.uint8, device=DEV)
        sf.gdn_ragged_fwd(*args[:5], S, i32(cu), max_len=max_len, out=(o, ws))
        torch.cuda.synchronize()
        assert bool((o[torch.tensor(~named, device=DEV)] == 7).all())
        idle = [i for i in range(N + 1) if i == N or at[i + 1] <= at[i]]
        assert torch.equal(S[idle], args[5][idle])


def test_gdn_strides_and_broadcast():
    """q, k, v as slices of wider rows, o into one, g and beta transposed, beta the same
    for all heads (stride 0), slots wider than a state."""
    lens, Hk, Hv, Dk, Dv = [130, 2, 1, 66], 2, 4, 64, 128
    cu, T = ref.sequences(lens)
    print("[gdn ragged] strides", flush=True)
    q, k, v, g, beta, state = gdn_inputs(T, Hk, Hv, Dk, Dv, 4, seed=10)
    row = torch.full((T, 2 * Hk * Dk + Hv * Dv + 8), float("nan"), dtype=torch.bfloat16, device=DEV)
    row[:, :Hk * Dk], row[:, Hk * Dk:2 * Hk * Dk], row[:, 2 * Hk * Dk:-8] = (x.flatten(1) for x in (q, k, v))
    qs, ks, vs = (row[:, a:b].unflatten(1, (-1, D)) for a, b, D in
                  ((0, Hk * Dk, Dk), (Hk * Dk, 2 * Hk * Dk, Dk), (2 * Hk * Dk, 2 * Hk * Dk + Hv * Dv, Dv)))
    gs = g.t().contiguous().t()
    bs = beta[:, :1].t().contiguous().t().expand(T, Hv)
    pool = torch.zeros(4, 3, Hv, Dk, Dv, device=DEV)
    pool[:, 1] = state
    want_o, _, want_S = ref.gdn(q, k, v, g, bs, state, cu, None)
    out = torch.full((T, Hv, Dv + 16), 7.0, dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(1 << 24, dtype=torch.uint8, device=DEV)
    with pytest.raises(ValueError):  # g and beta share strides
        sf.gdn_ragged_fwd(qs, ks, vs, gs, bs, pool[:, 1], i32(cu))
    ge = gs[:, :1].expand(T, Hv)
    want_o, _, want_S = ref.gdn(q, k, v, ge, bs, state, cu, None)
    sf.gdn_ragged_fwd(qs, ks, vs, ge, bs, pool[:, 1], i32(cu), out=(out[..., :Dv], ws))
    torch.cuda.synchronize()
    close("o", out[..., :Dv], want_o, DELTA)
    close("state", pool[:, 1], want_S, DELTA)
    assert bool((out[..., Dv:] == 7).all()) and not pool[:, [0, 2]].any()


@pytest.mark.parametrize("g_mu", [-40.0, 0.0, 12.0])
def test_gdn_gates(g_mu):
    """Near-memoryless, medium and nearly lossless decay."""
    print(f"[gdn ragged] gate mean {g_mu}", flush=True)
    cu, T = ref.sequences([200, 7])
    run_gdn(gdn_inputs(T, 1, 2, 128, 128, 2, seed=12, g_mu=g_mu), cu, max_len=200)


def test_gdn_gate_of_minus_infinity():
    """g = -inf forgets the state; the tokens behind it are as after a zero state."""
    cu, T = ref.sequences([150, 3])
    print("[gdn ragged] g = -inf", flush=True)
    for io in ("bf16", "f32"):
        args = gdn_inputs(T, 1, 1, 64, 64, 2, io, seed=13)
        args[3][40] = args[3][100] = args[3][151] = float("-inf")
        run_gdn(args, cu, max_len=150)


def test_gdn_parallel_keys():
    """Nearly parallel keys, beta near 1: the triangular system is far from diagonal."""
    print("[gdn ragged] parallel keys", flush=True)
    inp = synth.make_gdn_inputs(1, 192, 2, 128, seed=14, key_spread=0.2, beta_min=0.9, g_mu=8.0)
    args = [inp[n][0].to(DEV) for n in ("q", "k", "v", "g", "beta")] + [inp["S_in"].to(DEV)]
    run_gdn(args, [0, 192], max_len=192)


def test_gdn_is_the_training_recurrence():
    """Prompts through the ragged call, split anywhere, then decoded token by token:
    the segment call's outputs and state."""
    L, H, D = 256, 2, 128
    print("[gdn ragged] against gdn_fwd", flush=True)
    inp = synth.make_gdn_inputs(2, L, H, D, seed=15)
    q, k, v, g, beta, S0 = (inp[n].to(DEV) for n in ("q", "k", "v", "g", "beta", "S_in"))
    want_o, want_S = sf.gdn_fwd(q, k, v, g, beta, S0)
    state, o = S0.clone(), torch.empty_like(v)
    done = [0, 0]
    while min(done) < L:
        lens = [min(n, L - d) for n, d in zip(((100, 201), (1, 3), (1, 1), (150, 2), (4, 1), (1, 60))[
            min(5, sum(done) // 60)], done)]
        take = [torch.cat([x[i, d:d + n] for i, (d, n) in enumerate(zip(done, lens))]) for x in (q, k, v, g, beta)]
        out = sf.gdn_ragged_fwd(*take, state, i32(np.cumsum([0] + lens)), max_len=max(lens))
        o[0, done[0]:done[0] + lens[0]], o[1, done[1]:done[1] + lens[1]] = out[:lens[0]], out[lens[0]:]
        done = [d + n for d, n in zip(done, lens)]
    torch.cuda.synchronize()
    # both sides round o to bf16, and the segment call carries bf16 pairs (2^-17)
    d = (o.float() - want_o.float()).abs()
    assert bool((d <= 2 * 2.0 ** -8 * want_o.float().abs() + 2e-3 * want_o.float().square().mean().sqrt()).all())
    close("state", state, ref.f64(want_S), 2e-4)


def test_gdn_far_slots_and_rows():
    """Slots and rows more than 2^32 bytes from the first."""
    print("[gdn ragged] far offsets", flush=True)
    cu, T = ref.sequences([2, 70, 1])
    q, k, v, g, beta, state = gdn_inputs(T, 1, 1, 64, 64, 3, seed=16)
    pool = torch.empty(3, 1, 300000, 64, 64, device=DEV)[:, :, 0]  # 4.9 GB from slot to slot
    pool.copy_(state)
    wide = torch.empty(T, 40000000, dtype=torch.bfloat16, device=DEV)  # 80 MB rows, 5.8 GB
    qs, ks, vs = (wide[:, a:a + 64].unflatten(1, (1, 64)) for a in (0, 64, 128))
    for a, b in ((qs, q), (ks, k), (vs, v)):
        a.copy_(b)
    want_o, _, want_S = ref.gdn(q, k, v, g, beta, state, cu, None)
    for max_len in (1, 70):
        pool.copy_(state)
        o = sf.gdn_ragged_fwd(qs, ks, vs, g, beta, pool, i32(cu), max_len=max_len)
        torch.cuda.synchronize()
        close("o", o, want_o, DELTA)
        close("state", pool, want_S, DELTA)


def test_gdn_far_rows_in_chunks():
    """A long sequence whose slot and rows lie more than 2^32 bytes in, in chunks."""
    print("[gdn ragged] far offsets, chunks", flush=True)
    lens = [500, 1, 99]
    cu, T = ref.sequences(lens)
    q, k, v, g, beta, state = gdn_inputs(T, 1, 1, 64, 64, 3, seed=19)
    pool = torch.empty(3, 1, 300000, 64, 64, device=DEV)[:, :, 0]
    pool.copy_(state)
    wide = torch.empty(T, 4000000, dtype=torch.bfloat16, device=DEV)  # 8 MB rows, 4.8 GB
    qs, ks, vs = (wide[:, a:a + 64].unflatten(1, (1, 64)) for a in (0, 64, 128))
    for a, b in ((qs, q), (ks, k), (vs, v)):
        a.copy_(b)
    slots = [0, -1, 2]
    want_o, written, want_S = ref.gdn(q, k, v, g, beta, state, cu, slots)
    out = torch.empty(T, 1, 4000000, dtype=torch.bfloat16, device=DEV)[..., :64]
    ws = torch.empty(sf.gdn_ragged_workspace_bytes(qs, ks, vs, g, beta, pool, i32(cu), i32(slots), max_len=500),
                     dtype=torch.uint8, device=DEV)
    assert ws.numel() > 0  # the chunks' systems: this call takes them
    sf.gdn_ragged_fwd(qs, ks, vs, g, beta, pool, i32(cu), i32(slots), max_len=500, out=(out, ws))
    torch.cuda.synchronize()
    w = torch.tensor(written, device=DEV)
    close("o", out[w], want_o[written], DELTA)
    close("state", pool[[0, 2]], want_S[[0, 2]], DELTA)
    assert torch.equal(pool[1], state[1])


def test_gdn_nan_stays_in_its_sequence():
    """A NaN gate or value reaches its own sequence's state and no other's."""
    lens = [70, 90, 3, 2]
    cu, T = ref.sequences(lens)
    print("[gdn ragged] NaN", flush=True)
    args = gdn_inputs(T, 1, 2, 64, 64, 4, seed=20)
    args[3][30] = float("nan")
    args[2][161] = float("nan")
    for max_len in (1, 90):
        S = args[5].clone()
        o = sf.gdn_ragged_fwd(*args[:5], S, i32(cu), max_len=max_len)
        torch.cuda.synchronize()
        assert bool(S[0].isnan().all()) and bool(S[2].isnan().all())
        assert bool(o[69].isnan().all()) and bool(o[162].isnan().all())
        assert bool(S[[1, 3]].isfinite().all()) and bool(o[70:160].isfinite().all()) and bool(o[163:].isfinite().all())


def test_gdn_many_sequences_of_all_lengths():
    """Sequences over every bucket of the plan up to 40 chunks, more items than workgroups
    at once, in an order of their own; the longest in single column tiles."""
    rng = np.random.RandomState(5)
    lens = [int(n) for n in rng.randint(0, 200, 60)] + [2500, 0, 1, 24, 25, 12, 13, 640]
    rng.shuffle(lens)
    cu, T = ref.sequences(lens)
    print(f"[gdn ragged] {len(lens)} sequences, {T} tokens", flush=True)
    run_gdn(gdn_inputs(T, 1, 2, 64, 64, len(lens), seed=21), cu, max_len=2500)


def test_gdn_streams_graph_and_repeat():
    """Runs on another stream, captured with its workspace and replayed, with eager calls
    between the replays; every run of one input gives the same bits."""
    print("[gdn ragged] graph", flush=True)
    lens = [1, 130, 1, 66]
    cu, T = ref.sequences(lens)
    args = gdn_inputs(T, 2, 4, 128, 128, 4, seed=17)
    start = args[5].clone()
    cu_d = i32(cu)
    o0 = sf.gdn_ragged_fwd(*args, cu_d, max_len=130)
    S0 = args[5].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    args[5].copy_(start)
    side.wait_stream(torch.cuda.current_stream())
    o1 = sf.gdn_ragged_fwd(*args, cu_d, max_len=130, stream=side)
    side.synchronize()
    assert torch.equal(o0, o1) and torch.equal(args[5], S0)
    graph, o2 = torch.cuda.CUDAGraph(), torch.empty_like(o0)
    ws = torch.empty(sf.gdn_ragged_workspace_bytes(*args, cu_d, max_len=130), dtype=torch.uint8, device=DEV)
    with torch.cuda.graph(graph):
        sf.gdn_ragged_fwd(*args, cu_d, max_len=130, out=(o2, ws))
    for _ in range(3):
        args[5].copy_(start)
        o2.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o2, o0) and torch.equal(args[5], S0)
        args[5].copy_(start)
        assert torch.equal(sf.gdn_ragged_fwd(*args, cu_d, max_len=130), o0)
    # the captured call reads the lengths and the slots where they lie: another batch, same graph
    cu_d.copy_(i32([0, 40, 41, 41, 108]))
    want_o, written, want_S = ref.gdn(*args[:5], start, [0, 40, 41, 41, 108], None)
    args[5].copy_(start)
    graph.replay()
    torch.cuda.synchronize()
    close("o", o2[:108], want_o[:108], DELTA)
    close("state", args[5], want_S, DELTA)


def test_stream_of_the_tensors_device():
    """Two streams at once, each on slots of its own in one pool; the bounds and slots are
    let go of right after the call and their memory taken again."""
    cu, T = ref.sequences([70, 3])
    print("[gdn ragged] two streams", flush=True)
    args = gdn_inputs(T, 1, 2, 128, 64, 4, seed=22)
    want = [ref.gdn(*args, cu, s) for s in ([0, 3], [2, 1])]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    outs = [sf.gdn_ragged_fwd(*args, i32(cu), i32(sl), max_len=70, stream=st)
            for sl, st in zip(([0, 3], [2, 1]), streams)]
    again = [i32([7, 7, 7]) for _ in range(64)] + [i32([9, 9]) for _ in range(64)]
    torch.cuda.synchronize()
    assert len(again) == 128
    for o, w in zip(outs, want):
        close("o", o, w[0], DELTA)
    close("state", args[5][[0, 3]], want[0][2][[0, 3]], DELTA)
    close("state", args[5][[2, 1]], want[1][2][[2, 1]], DELTA)


def test_gdn_empty_calls():
    args = gdn_inputs(4, 1, 1, 64, 64, 2, seed=18)
    before = args[5].clone()
    sf.gdn_ragged_fwd(*args, i32([0]))
    sf.gdn_ragged_fwd(*[x[:0] for x in args[:5]], args[5], i32([0, 0, 0]))
    sf.gdn_ragged_fwd(*args, i32([2, 2, 2]))
    sf.gdn_ragged_fwd(*args[:5], args[5][:0], i32([0, 2]), i32([0]))
    torch.cuda.synchronize()
    assert torch.equal(args[5], before)


# ------------------------------------------------------------------ short convolution

def run_conv(x, w, tails, cu, slots=None, fresh=None, act="silu", **kw):
    want_y, written, want_t = ref.conv(x, w, tails, cu, slots, fresh, act)
    y = torch.full(x.shape, 7.0, dtype=x.dtype, device=DEV)
    before = None if tails is None else tails.clone()
    fr = None if fresh is None else torch.tensor(fresh, dtype=torch.uint8, device=DEV)
    sf.conv_ragged_fwd(x, w, tails, i32(cu), None if slots is None else i32(slots), fresh=fr, act=act, out=y, **kw)
    torch.cuda.synchronize()
    m = torch.tensor(written, device=DEV)
    assert bool((y[~m] == 7).all()), "rows of no sequence were written"
    close("y", y[m], want_y[written], DELTA_CONV)
    if before is not None:  # tails hold inputs: exact
        assert torch.equal(tails.cpu(), torch.tensor(want_t).float())
    return y


def conv_inputs(T, C, W, n_slots, io="bf16", seed=0):
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(T, C, generator=gen).to(IO[io]).to(DEV)
    w = (torch.randn(C, W, generator=gen) / W ** 0.5).to(DEV)
    tails = torch.randn(n_slots, W - 1, C, generator=gen).to(IO[io]).float().to(DEV) if W > 1 else None
    return x, w, tails


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("W", [1, 2, 3, 4])
@pytest.mark.parametrize("act", ["none", "silu"])
def test_conv_ragged(io, W, act):
    lens = [1, 300, 2, 0, 3, 8, 7, 9, 65]
    print(f"[conv ragged] {io} W={W} {act}", flush=True)
    cu, T = ref.sequences(lens)
    n = len(lens)
    slots = np.random.RandomState(W).permutation(n + 2)[:n]
    run_conv(*conv_inputs(T, 72, W, n + 2, io, seed=W), cu, slots, act=act)


@pytest.mark.parametrize("C,N", [(8, 700), (2056, 5), (15360, 3)])
def test_conv_ragged_sizes(C, N):
    """Many single tokens (more than 64 sequences, more than 64 x 64 / 8 runs) and wide rows."""
    print(f"[conv ragged] C={C} N={N}", flush=True)
    lens = [1] * N if C == 8 else [40, 1, 23, 2, 5][:N]
    cu, T = ref.sequences(lens)
    run_conv(*conv_inputs(T, C, 4, N, seed=C), cu)


def test_conv_ragged_many_sequences():
    lens = list(np.random.RandomState(3).randint(0, 20, 5000))
    print("[conv ragged] 5000 sequences", flush=True)
    cu, T = ref.sequences(lens)
    run_conv(*conv_inputs(T, 16, 4, 5000, seed=21), cu, np.random.RandomState(4).permutation(5000))


def test_conv_ragged_fresh_skipped_outside():
    lens, slots, fresh = [3, 100, 2, 90, 0, 1], [4, 1, -1, 9, 0, 2], [1, 1, 0, 1, 1, 0]
    print("[conv ragged] fresh and skipped", flush=True)
    cu, T = ref.sequences(lens, T=7 + sum(lens) + 30, before=7)
    x, w, tails = conv_inputs(T, 64, 4, 6, seed=22)
    x[:7] = x[cu[-1]:] = float("nan")
    tails[4] = tails[1] = float("nan")
    tails = tails.nan_to_num(3e38)  # a fresh sequence must not let it through
    run_conv(x, w, tails, cu, slots, fresh)


@pytest.mark.parametrize("cu", [[0, 200, 90, 150], [-7, 40, 40, 1000], [150, 100, 50, 0], [400, 500, 600, 700],
                                [2 ** 31 - 1, -2 ** 31, 2 ** 31 - 1, 0]])
def test_conv_ragged_bad_bounds(cu):
    print(f"[conv ragged] bounds {cu}", flush=True)
    x, w, tails = conv_inputs(150, 64, 3, 3, seed=23)
    before = tails.clone()
    y = sf.conv_ragged_fwd(x, w, tails, i32(cu))
    torch.cuda.synchronize()
    assert bool(y.isfinite().any())
    for i in range(3):  # only slots of sequences with tokens change
        b, e = (min(max(c, 0), 150) for c in cu[i:i + 2])
        assert e > b or torch.equal(tails[i], before[i])


def test_conv_ragged_strides():
    lens = [20, 1, 33]
    cu, T = ref.sequences(lens)
    x, w, tails = conv_inputs(T, 64, 4, 3, seed=24)
    print("[conv ragged] strides", flush=True)
    wide = torch.full((T, 200), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 8:72] = x
    out = torch.full((T, 96), 7.0, dtype=torch.bfloat16, device=DEV)
    pool = torch.full((3, 2, 3, 64), 5.0, device=DEV)
    pool[:, 1] = tails
    want_y, _, want_t = ref.conv(x, w, tails, cu, None)
    sf.conv_ragged_fwd(wide[:, 8:72], w, pool[:, 1], i32(cu), out=out[:, 16:80])
    torch.cuda.synchronize()
    close("y", out[:, 16:80], want_y, DELTA_CONV)
    assert torch.equal(pool[:, 1].cpu(), torch.tensor(want_t).float()) and bool((pool[:, 0] == 5).all())
    assert bool((out[:, :16] == 7).all()) and bool((out[:, 80:] == 7).all())


def test_conv_ragged_is_the_training_convolution():
    """One sequence cut anywhere equals conv_fwd over the whole of it, to the bit."""
    inp = synth.make_conv_inputs(1, 100, 128, 4, seed=25)
    x, w, tail = (inp[n].to(DEV) for n in ("x", "w", "tail_in"))
    print("[conv ragged] against conv_fwd", flush=True)
    want_y, want_t = sf.conv_fwd(x, w, tail)
    pool, ys, t = tail.clone(), [], 0
    for n in (1, 2, 1, 60, 3, 1, 32):
        ys.append(sf.conv_ragged_fwd(x[0, t:t + n], w, pool, i32([0, n])))
        t += n
    torch.cuda.synchronize()
    y = torch.cat(ys)
    assert torch.equal(pool, want_t)
    d = (y.float() - want_y[0].float()).abs()  # one step of bf16 where the roundings part
    assert bool((d <= 2.0 ** -7 * want_y[0].float().abs() + 1e-6).all())


def test_conv_ragged_graph():
    lens = [1, 30, 1]
    cu, T = ref.sequences(lens)
    x, w, tails = conv_inputs(T, 128, 4, 3, seed=26)
    print("[conv ragged] graph", flush=True)
    start, y = tails.clone(), torch.empty_like(x)
    cu_d = i32(cu)
    want = sf.conv_ragged_fwd(x, w, tails, cu_d)
    after = tails.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sf.conv_ragged_fwd(x, w, tails, cu_d, out=y)
    for _ in range(3):
        tails.copy_(start)
        y.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(tails, after)


def test_layer_prefill_then_decode():
    """The operators as a layer runs them: convolution, norms of q and k, delta rule;
    two prompts packed, then single tokens, against one run of the training calls."""
    B, L, H, D, P = 2, 128, 2, 128, (90, 61)
    print("[ragged] a layer's prefill and decode", flush=True)
    gen = torch.Generator().manual_seed(27)
    x = torch.randn(B, L, 3 * H * D, generator=gen).to(torch.bfloat16).to(DEV)
    w = (torch.randn(3 * H * D, 4, generator=gen) / 2).to(DEV)
    g = torch.nn.functional.logsigmoid(torch.randn(B, L, H, generator=gen) + 3).to(DEV)
    beta = torch.sigmoid(torch.randn(B, L, H, generator=gen)).to(DEV)
    inv_freq = (10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64) / D)).to(DEV)

    def heads(y):
        return [t.unflatten(-1, (H, D)) for t in y.split(H * D, dim=-1)]

    yc, tail = sf.conv_fwd(x, w)
    q, k, v = heads(yc)
    qn, kn = sf.qk_norm_fwd(q, k, norm="l2", q_scale=D ** -0.5, inv_freq=inv_freq)
    want_o, want_S = sf.gdn_fwd(qn, kn, v.contiguous(), g, beta)

    state = torch.full((4, H, D, D), float("nan"), device=DEV)
    tails = torch.full((4, 3, 3 * H * D), float("nan"), device=DEV)
    slots, o = i32([3, 1]), torch.empty(B, L, H, D, dtype=torch.bfloat16, device=DEV)

    def step(at, lens, fresh):
        cu = i32(np.cumsum([0] + list(lens)))
        pick = lambda t: torch.cat([t[i, a:a + n] for i, (a, n) in enumerate(zip(at, lens))])  # noqa: E731
        y = sf.conv_ragged_fwd(pick(x), w, tails, cu, slots, fresh=fresh)
        q, k, v = heads(y)
        pos = torch.cat([torch.arange(a, a + n) for a, n in zip(at, lens)])[None].to(DEV)
        qn, kn = sf.qk_norm_fwd(q[None], k[None], norm="l2", q_scale=D ** -0.5, inv_freq=inv_freq, pos=pos)
        out = sf.gdn_ragged_fwd(qn[0], kn[0], v, pick(g), pick(beta), state, cu, slots, fresh=fresh, max_len=max(lens))
        for i, (a, n) in enumerate(zip(at, lens)):
            o[i, a:a + n] = out[sum(lens[:i]):sum(lens[:i]) + n]

    step((0, 0), P, torch.ones(2, dtype=torch.bool, device=DEV))
    at = list(P)
    while min(at) < L:
        lens = [1 if a < L else 0 for a in at]
        step(at, lens, None)
        at = [a + n for a, n in zip(at, lens)]
    torch.cuda.synchronize()
    rms = want_o.float().square().mean().sqrt()
    assert bool(((o.float() - want_o.float()).abs() <= 2 * 2.0 ** -8 * want_o.float().abs() + 5e-3 * rms).all())
    assert torch.equal(tails[[3, 1]], tail)
    d = (state[[3, 1]] - want_S).norm() / want_S.norm()
    assert float(d) < 2e-3, float(d)  # k and q come out of bf16 roundings that may part by a step
