"""Timed calls of the operators that serve a recurrence layer token by token and
prepare its queries and keys, beside their plain forms:

  gdn   the gated delta rule over a ragged batch of sequences, each with a state
        of its own in a pool of slots, updated in place (sf.gdn_ragged_fwd)
  conv  the short convolution over such a batch, its tails in a pool of slots
        (sf.conv_ragged_fwd)
  qk    norms of queries and keys for each head and the position rotation, one
        pass (sf.qk_norm_fwd)
  qkb   the gradients of that pass (sf.qk_norm_bwd)

A case is a dict of plain values:
  lens    tokens of each sequence of a ragged batch, comma separated; "n*c" stands
          for c sequences of n tokens
  fresh   "none", "all" or "some": which sequences start from a zero state
  Hk, Hv  heads of queries and keys, heads of values (gdn); Hq, Hk (qk, qkb)
  Dk, Dv  channels of a key head and of a value head
  norm    "l2", "rms" or "none"; weight: whether the norm has weights
  R       rotated channels (0: none); inter: pairs are neighbours, not halves apart
  far     the positions lie anywhere below this number
"""
import math

import torch

own = False

_IO = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


def listed():
    return [
        # One user's next token on one tensor-parallel rank (10 of 40 heads): latency.
        dict(name="gdn_decode_one", op="gdn", lens="1", Hk=10, Hv=10, Dk=128, Dv=128, io="bf16", fresh="none"),
        # The decode step of a busy server, all 40 heads of a hidden-5120 layer: the
        # states are what is read and written.
        dict(name="gdn_decode_batch", op="gdn", lens="1*256", Hk=40, Hv=40, Dk=128, Dv=128, io="bf16", fresh="none"),
        # A few drafted tokens for each of 48 sequences in fp32, two value heads to a
        # key head; two sequences have nothing to do in this step.
        dict(name="gdn_draft_f32", op="gdn", lens="3*20,1*7,5*13,0*2,6*6", Hk=8, Hv=16, Dk=64, Dv=64, io="f32",
             fresh="none"),
        # A scheduler's mixed step: a prompt chunk beside 63 sequences that decode.
        dict(name="gdn_mixed", op="gdn", lens="1*30,2048,1*33", Hk=20, Hv=40, Dk=128, Dv=128, io="bf16",
             fresh="some"),
        # Prompts of many lengths, packed: 20 heads, all starting afresh.
        dict(name="gdn_prefill", op="gdn", lens="517,64,2048,1,33,1200,300,4096", Hk=20, Hv=20, Dk=128, Dv=128,
             io="bf16", fresh="all"),
        # The convolution's decode step in front of q, k and v of 40 heads.
        dict(name="conv_decode", op="conv", lens="1*256", C=15360, W=4, io="bf16", act="silu", fresh="none"),
        # The convolution over the packed prompts above.
        dict(name="conv_prefill", op="conv", lens="517,64,2048,1,33,1200,300,4096", C=15360, W=4, io="bf16",
             act="silu", fresh="some"),
        # Queries and keys of one decode step of a softmax layer far into a 256K
        # context, 40 heads over 8 key heads: latency.
        dict(name="qk_decode", op="qk", B=1, L=64, Hq=40, Hk=8, D=128, io="bf16", norm="rms", weight=True, R=128,
             inter=False, far=262144),
        # The L2 norm in front of the delta rule, 32K tokens of 40 heads.
        dict(name="qk_l2_train", op="qk", B=1, L=32768, Hq=40, Hk=40, D=128, io="bf16", norm="l2", weight=False, R=0,
             inter=False, far=0),
        # Its gradient.
        dict(name="qkb_l2_train", op="qkb", B=1, L=32768, Hq=40, Hk=40, D=128, io="bf16", norm="l2", weight=False,
             R=0, inter=False, far=0),
        # The gradient of the softmax layer's norm and rotation, with the weights'.
        dict(name="qkb_rope_train", op="qkb", B=2, L=8192, Hq=40, Hk=8, D=128, io="bf16", norm="rms", weight=True,
             R=128, inter=False, far=16384),
        # A small fp32 model, ragged length, half of the channels rotated in
        # neighbouring pairs.
        dict(name="qkb_f32_small", op="qkb", B=2, L=1037, Hq=6, Hk=3, D=64, io="f32", norm="rms", weight=True, R=32,
             inter=True, far=4096),
    ]


def _log(rng, lo, hi):
    return math.exp(rng.uniform(math.log(lo), math.log(hi)))


def _draw_lens(rng, T):
    """A decode step, a step of drafts, packed prompts or both, of about T tokens."""
    kind = rng.choice(("decode", "draft", "prefill", "prefill", "mixed"))
    n = max(1, min(256, int(T)))
    if kind == "decode":
        return f"1*{n}"
    if kind == "draft":
        return ",".join(str(rng.randint(0, 9)) for _ in range(max(1, n // 4))) + ",2"
    lens = [max(1, int(T * rng.random() ** 2)) for _ in range(rng.randint(1, 6))]
    if kind == "mixed":
        lens = lens[:2] + [1] * rng.randint(1, 64)
        rng.shuffle(lens)
    return ",".join(map(str, lens))


def draw(rng):
    op = rng.choice(("gdn", "gdn", "gdn", "conv", "qk", "qkb"))
    io = rng.choice(("bf16", "bf16", "f32"))
    if op == "gdn":
        Hk = int(_log(rng, 1, 41))
        group = rng.choice((1, 1, 2, 3, 4))
        Hv = Hk * group if Hk * group <= 40 else Hk
        return dict(op=op, lens=_draw_lens(rng, _log(rng, 1, 1500)), Hk=Hk, Hv=Hv, Dk=rng.choice((64, 128, 128)),
                    Dv=rng.choice((64, 128, 128)), io=io, fresh=rng.choice(("none", "all", "some")))
    if op == "conv":
        return dict(op=op, lens=_draw_lens(rng, _log(rng, 1, 4096)), C=8 * int(_log(rng, 8, 1920)),
                    W=rng.choice((2, 3, 4, 4)), io=io, act=rng.choice(("silu", "none")),
                    fresh=rng.choice(("none", "all", "some")))
    D = rng.choice((64, 96, 128, 128, 256))
    Hk = int(_log(rng, 1, 17))
    Hq = Hk * rng.choice((1, 1, 2, 5)) if Hk <= 8 else Hk
    R = rng.choice((0, 32, 64, D))
    return dict(op=op, B=rng.choice((1, 1, 2, 3)), L=int(_log(rng, 1, 8192)), Hq=Hq, Hk=Hk, D=D, io=io,
                norm=rng.choice(("l2", "rms", "none")) if R else rng.choice(("l2", "rms")),
                weight=rng.random() < 0.5, R=R, inter=rng.random() < 0.5, far=rng.choice((4096, 262144)))


def _lens(case):
    out = []
    for part in case["lens"].split(","):
        n, _, c = part.partition("*")
        out += [int(n)] * int(c or 1)
    return out


def prepare(case, seed):
    dev = torch.device("cuda:0")
    gen = torch.Generator(device=dev).manual_seed(int(seed))
    io, f32 = _IO[case["io"]], dict(dtype=torch.float32, device=dev, generator=gen)
    st = dict(case=case)
    if case["op"] in ("gdn", "conv"):
        lens = _lens(case)
        N, T = len(lens), sum(lens)
        cu = [0]
        for n in lens:
            cu.append(cu[-1] + n)
        n_slots = N + 1 + N // 8  # a pool has slots to spare, handed out in any order
        host = torch.Generator().manual_seed(int(seed))
        slots = torch.randperm(n_slots, generator=host)[:N]
        fresh = {"none": torch.zeros(N), "all": torch.ones(N),
                 "some": (torch.rand(N, generator=host) < 0.3)}[case["fresh"]].to(torch.uint8)
        # what a scheduler knows of its step: the lengths, longest first
        order = sorted(range(N), key=lambda i: -lens[i])
        st.update(lens=lens, T=T, N=N, longest=max(lens), cu=torch.tensor(cu, dtype=torch.int32, device=dev),
                  slots=slots.to(torch.int32).to(dev), fresh=fresh.to(dev) if case["fresh"] != "none" else None,
                  order=torch.tensor(order, device=dev), counts=[lens[i] for i in order])
    if case["op"] == "gdn":
        Hk, Hv, Dk, Dv = case["Hk"], case["Hv"], case["Dk"], case["Dv"]
        k = torch.randn(T, Hk, Dk, **f32)
        st["k"] = (k / k.norm(dim=-1, keepdim=True)).to(io)
        st["q"] = torch.randn(T, Hk, Dk, **f32).to(io)
        # the values as they lie in the convolution's output, beside its q and k
        width = 2 * Hk * Dk + Hv * Dv
        st["v"] = torch.randn(T, width, **f32).to(io)[:, 2 * Hk * Dk:].unflatten(1, (Hv, Dv))
        st["g"] = torch.nn.functional.logsigmoid(torch.randn(T, Hv, **f32) + 3.0)
        st["beta"] = torch.sigmoid(torch.randn(T, Hv, **f32))
        st["state"] = torch.randn(n_slots, Hv, Dk, Dv, **f32) * 0.1
    elif case["op"] == "conv":
        C, W = case["C"], case["W"]
        st["x"] = torch.randn(T, C, **f32).to(io)
        st["w"] = torch.randn(C, W, **f32) / W ** 0.5
        st["tails"] = torch.randn(n_slots, W - 1, C, **f32).to(io).float()
    else:
        B, L, Hq, Hk, D, R = (case[n] for n in ("B", "L", "Hq", "Hk", "D", "R"))
        x = torch.randn(B, L, (Hq + Hk) * D, **f32).to(io)  # the projection's output: q, then k
        st["q"], st["k"] = x[..., :Hq * D].unflatten(2, (Hq, D)), x[..., Hq * D:].unflatten(2, (Hk, D))
        st["wq"] = 1 + 0.2 * torch.randn(D, **f32) if case["weight"] else None
        st["wk"] = 1 + 0.2 * torch.randn(D, **f32) if case["weight"] else None
        st["inv_freq"], st["pos"] = None, None
        if R:
            st["inv_freq"] = (10000.0 ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)).to(dev)
            st["pos"] = torch.randint(0, case["far"], (B, L), device=dev, generator=gen)
        if case["op"] == "qkb":
            st["dq"] = torch.randn(B, L, Hq, D, **f32).to(io)
            st["dk"] = torch.randn(B, L, Hk, D, **f32).to(io)
    return st


# --- plain forms ---------------------------------------------------------------------------

def _gdn_plain(st):
    """Chunk by chunk over the sequences that still have tokens (the longest come
    first), in 32 bits.  With b the running sum of g in the chunk, A the strictly lower
    triangle of beta_i e^(b_i - b_j) k_i.k_j and U = (I + A)^-1 beta (v - e^b k S):
        o = e^b q S + tril(e^(b_i - b_j) q_i.k_j) U,   S' = e^(b_C) S + (k e^(b_C - b))^T U"""
    case, T, longest = st["case"], st["T"], st["longest"]
    Hk, Hv, Dk, Dv = case["Hk"], case["Hv"], case["Dk"], case["Dv"]
    state, order, cu = st["state"], st["order"], st["cu"].long()
    o = torch.empty(T + 1, Hv, Dv, dtype=st["v"].dtype, device=state.device)  # the last row: rows past an end
    if longest == 0:
        return dict(o=o[:T], state=state)
    C = min(64, longest)
    slots = st["slots"].long()[order]
    S = state[slots]
    if st["fresh"] is not None:
        S = S * (1 - st["fresh"][order].float())[:, None, None, None]
    ones = torch.ones(C, C, device=state.device)
    eye, low, at = torch.eye(C, device=state.device), ones.tril(-1) > 0, torch.arange(C, device=state.device)
    kept = sum(n > 0 for n in st["counts"])
    for c0 in range(0, longest, C):
        n = sum(m > c0 for m in st["counts"])
        rows = cu[order[:n], None] + c0 + at
        live = rows < cu[order[:n] + 1, None]
        row = rows.clamp(max=T - 1)

        def take(x, heads):  # [n Hv, C, ...] in 32 bits, zero past the end
            x = x[row].float() * live.view(n, C, *[1] * (x.dim() - 1))
            x = x.repeat_interleave(Hv // heads, 2) if heads != Hv else x
            return x.transpose(1, 2).flatten(0, 1)

        q, k, v = take(st["q"], Hk), take(st["k"], Hk), take(st["v"], Hv)
        b, beta = take(st["g"], Hv).cumsum(1), take(st["beta"], Hv)[..., None]
        M = (b[:, :, None] - b[:, None]).masked_fill(ones.triu(1) > 0, float("-inf")).exp()
        kt = k.transpose(1, 2).contiguous()
        A = (k @ kt) * M * low * beta
        inv, P, width = eye - A, A, 2
        while width < C:  # (I + A)^-1 = (I - A)(I + A^2)(I + A^4)...
            P = P @ P
            inv, width = inv + inv @ P, 2 * width
        Sn = S[:n].flatten(0, 1)
        eb, end = b.exp()[..., None], b[:, -1:]
        U = inv @ (beta * (v - eb * (k @ Sn)))
        out = eb * (q @ Sn) + ((q @ kt) * M) @ U
        Sn = end.exp()[..., None] * Sn + (kt * (end - b).exp()[:, None]) @ U
        S[:n] = Sn.unflatten(0, (n, Hv))
        o[torch.where(live, rows, T)] = out.unflatten(0, (n, Hv)).transpose(1, 2).to(o.dtype)
    state[slots[:kept]] = S[:kept]
    return dict(o=o[:T], state=state)


def _conv_plain(st):
    case, x, w, tails, T, N = st["case"], st["x"], st["w"], st["tails"], st["T"], st["N"]
    W, cu, slots = case["W"], st["cu"].long(), st["slots"].long()
    old = tails[slots]
    if st["fresh"] is not None:
        old = old * (1 - st["fresh"].float())[:, None, None]
    n = cu[1:] - cu[:-1]
    seq = torch.repeat_interleave(torch.arange(N, device=x.device), n, output_size=T)
    at = torch.arange(T, device=x.device) - cu[seq]

    def rows(i, s):  # row s of sequence i, counted from its first token: the tail below zero
        here = x[(cu[i] + s).clamp(0, max(T - 1, 0))].float()
        return torch.where((s >= 0)[:, None], here, old[i, (s + W - 1).clamp(0, W - 2)])

    u = torch.zeros(T, case["C"], device=x.device)
    for j in range(W):
        u += w[:, j] * rows(seq, at - (W - 1) + j)
    y = (u * (1 / (1 + (-u).exp())) if case["act"] == "silu" else u).to(x.dtype)
    every = torch.arange(N, device=x.device)
    new = torch.stack([rows(every, n - (W - 1) + i) for i in range(W - 1)], 1)
    tails[slots] = torch.where((n > 0)[:, None, None], new, tails[slots])
    return dict(y=y, tails=tails)


def _turn(x, cos, sin, inter):
    """The first 2 n channels rotated in pairs by n angles."""
    n = cos.shape[-1]
    a, b = (x[..., 0:2 * n:2], x[..., 1:2 * n:2]) if inter else (x[..., :n], x[..., n:2 * n])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack((a, b), -1).flatten(-2) if inter else torch.cat((a, b), -1)
    return torch.cat((turned, x[..., 2 * n:]), -1)


def _angles(st):
    if st["inv_freq"] is None:
        return None, None
    a = st["pos"].double()[..., None, None] * st["inv_freq"]
    return a.cos().float(), a.sin().float()


def _scale(x, case):
    """What a row is multiplied by, and the factor of its sum of squares."""
    if case["norm"] == "none":
        return torch.ones_like(x[..., :1]), 0.0
    c = 1.0 if case["norm"] == "l2" else 1.0 / case["D"]
    return (c * x.square().sum(-1, keepdim=True) + EPS).rsqrt(), c


def _qk_plain(st):
    case, (cos, sin), out = st["case"], _angles(st), {}
    for name, w, s in (("q", st["wq"], case["D"] ** -0.5), ("k", st["wk"], 1.0)):
        x = st[name].float()
        y = x * _scale(x, case)[0]
        y = y if w is None else y * w
        y = y if cos is None else _turn(y, cos, sin, case["inter"])
        out[name] = (y * s).to(st[name].dtype)
    return out


def _qkb_plain(st):
    case, (cos, sin), out = st["case"], _angles(st), {}
    for name, w, s in (("q", st["wq"], case["D"] ** -0.5), ("k", st["wk"], 1.0)):
        x, dy = st[name].float(), st["d" + name].float() * s
        dz = dy if cos is None else _turn(dy, cos, -sin, case["inter"])
        r, c = _scale(x, case)
        if w is not None:
            out["dw" + name] = (dz * x * r).sum((0, 1, 2))
            dz = dz * w
        dx = dz * r - x * (c * r * r * r * (dz * x).sum(-1, keepdim=True))
        out["d" + name] = dx.to(st[name].dtype)
    return out


# --- the framework's calls -----------------------------------------------------------------

def _own(st):
    import paper_2608_06838_amd as sf
    case = st["case"]
    if case["op"] == "gdn":
        o = sf.gdn_ragged_fwd(st["q"], st["k"], st["v"], st["g"], st["beta"], st["state"], st["cu"], st["slots"],
                              fresh=st["fresh"], max_len=st["longest"])
        return dict(o=o, state=st["state"])
    if case["op"] == "conv":
        y = sf.conv_ragged_fwd(st["x"], st["w"], st["tails"], st["cu"], st["slots"], fresh=st["fresh"],
                               act=case["act"])
        return dict(y=y, tails=st["tails"])
    how = dict(norm=case["norm"], q_weight=st["wq"], k_weight=st["wk"], eps=EPS, q_scale=case["D"] ** -0.5,
               inv_freq=st["inv_freq"], pos=st["pos"], interleaved=case["inter"])
    if case["op"] == "qk":
        q, k = sf.qk_norm_fwd(st["q"], st["k"], **how)
        return dict(q=q, k=k)
    dq, dk, dwq, dwk = sf.qk_norm_bwd(st["q"], st["k"], st["dq"], st["dk"], **how)
    out = dict(dq=dq, dk=dk)
    return dict(out, dwq=dwq, dwk=dwk) if case["weight"] else out


def run(st):
    if own:
        return _own(st)
    return {"gdn": _gdn_plain, "conv": _conv_plain, "qk": _qk_plain, "qkb": _qkb_plain}[st["case"]["op"]](st)


def work(case):
    io = 2 if case["io"] == "bf16" else 4
    if case["op"] in ("gdn", "conv"):
        lens = _lens(case)
        T, some = sum(lens), sum(n > 0 for n in lens)
        read = 0 if case["fresh"] == "all" else 1  # a fresh state is written, not read
    if case["op"] == "gdn":
        Hk, Hv, Dk, Dv = case["Hk"], case["Hv"], case["Dk"], case["Dv"]
        nbytes = T * io * (2 * Hk * Dk + 2 * Hv * Dv) + 8 * T * Hv + 4 * some * Hv * Dk * Dv * (1 + read)
        return dict(bytes=nbytes, flops=T * Hv * 6 * Dk * Dv)  # S^T k, S^T q and k u^T of every token
    if case["op"] == "conv":
        C, W = case["C"], case["W"]
        return dict(bytes=2 * T * C * io + 4 * C * W + 4 * some * (W - 1) * C * (1 + read), flops=T * C * (2 * W + 4))
    n = case["B"] * case["L"] * (case["Hq"] + case["Hk"]) * case["D"]
    nbytes = n * io * (2 if case["op"] == "qk" else 3) + (8 * case["B"] * case["L"] if case["R"] else 0)
    return dict(bytes=nbytes, flops=n * (8 if case["op"] == "qk" else 16))


# --- the same outputs in 64 bits, from the definitions -------------------------------------

def _exact_gdn(st):
    """Token by token: S <- e^g S, u = beta (v - S^T k), S <- S + k u^T, o = S^T q."""
    case, T = st["case"], st["T"]
    group = case["Hv"] // case["Hk"]
    state, cu, order = st["state"].double(), st["cu"].long(), st["order"]
    o = torch.zeros(T, case["Hv"], case["Dv"], dtype=torch.float64, device=state.device)
    slots = st["slots"].long()[order]
    S = state[slots]
    if st["fresh"] is not None:
        S[st["fresh"][order] > 0] = 0.0
    for t in range(st["longest"]):
        n = sum(m > t for m in st["counts"])
        row = cu[order[:n]] + t
        q, k = (st[x][row].double().repeat_interleave(group, 1) for x in ("q", "k"))
        v, g, beta = st["v"][row].double(), st["g"][row].double(), st["beta"][row].double()
        Sn = S[:n].mul_(g.exp()[..., None, None])
        u = beta[..., None] * (v - (Sn * k[..., None]).sum(-2))
        Sn.addcmul_(k[..., None], u[..., None, :])
        o[row] = (Sn * q[..., None]).sum(-2)
    state[slots] = torch.where(torch.tensor([m > 0 for m in st["counts"]], device=S.device)[:, None, None, None], S,
                               state[slots])
    return dict(o=o, state=state)


def _exact_conv(st):
    case, x, w, tails = st["case"], st["x"].double(), st["w"].double(), st["tails"].double()
    W, y, t = case["W"], torch.empty_like(x), 0
    fresh = [0] * st["N"] if st["fresh"] is None else st["fresh"].tolist()
    for i, (n, slot) in enumerate(zip(st["lens"], st["slots"].tolist())):
        if n == 0:
            continue
        old = torch.zeros_like(tails[slot]) if fresh[i] else tails[slot]
        xe = torch.cat((old, x[t:t + n]))
        y[t:t + n] = (xe.unfold(0, W, 1) * w).sum(-1)
        tails[slot] = xe[n:].clone()
        t += n
    return dict(y=y * torch.sigmoid(y) if case["act"] == "silu" else y, tails=tails)


def _exact_qk(st, grads):
    """The pass in 64 bits, head by head; the gradients through torch's autograd."""
    case, out = st["case"], {}
    ang = None if st["inv_freq"] is None else st["pos"].double()[..., None] * st["inv_freq"]
    turn = None if ang is None else torch.polar(torch.ones_like(ang), ang)
    for name, scale in (("q", case["D"] ** -0.5), ("k", 1.0)):
        w = st["w" + name]
        w = None if w is None else w.double().requires_grad_(grads)
        total = torch.empty(st[name].shape, dtype=torch.float64, device=st[name].device)
        dw = 0.0
        for h in range(total.shape[2]):
            x = st[name][:, :, h].double().requires_grad_(grads)
            y = x
            if case["norm"] != "none":
                ss = x.pow(2).sum(-1) if case["norm"] == "l2" else x.pow(2).mean(-1)
                y = x / (ss + EPS).sqrt()[..., None]
            y = y if w is None else y * w
            if turn is not None:
                R = case["R"]
                head = y[..., :R]
                z = head.unflatten(-1, (R // 2, 2)) if case["inter"] else head.unflatten(-1, (2, R // 2)).mT
                z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
                y = torch.cat(((z if case["inter"] else z.mT).flatten(-2), y[..., R:]), -1)
            y = y * scale
            if not grads:
                total[:, :, h] = y
                continue
            dx, *more = torch.autograd.grad((y * st["d" + name][:, :, h].double()).sum(),
                                            [x] if w is None else [x, w])
            total[:, :, h] = dx
            dw = dw + more[0] if more else dw
        out["d" + name if grads else name] = total
        if grads and w is not None:
            out["dw" + name] = dw
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "gdn":
        return _exact_gdn(st)
    return _exact_conv(st) if case["op"] == "conv" else _exact_qk(st, case["op"] == "qkb")
