"""Performance cases of the attention layers over frames: the work that a
recogniser whose network attends to earlier frames has them do, in training and
in serving, through the public Python entry points
(``paper_2110_02848_amd.gpu.Composer``).

Kinds of case:

* ``norm``          queries and keys normalised head by head and rotated by position;
* ``norm-train``    the same and its gradients;
* ``linear``        linear attention with a decay for each head, whole sequences;
* ``linear-train``  the same and its gradients;
* ``linear-step``   its recurrent form, one frame of many streams;
* ``window``        attention to a window of frames and a sequence's first ones;
* ``window-train``  the same and its gradients;
* ``window-step``   one frame of many streams, keys and values in a ring.

``run`` makes the calls where ``own`` is true; where it is not, it computes
the same by elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = dict(f32=torch.float32, f16=torch.float16, bf16=torch.bfloat16)
EPS = 1e-6
CHUNK = 128  # rows that the plain form of linear attention takes at once


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # streaming recognition: queries and keys of eight callers' next frame,
        # an hour into their streams (latency)
        dict(name="norm-8x8+2x64", kind="norm", type="bf16", N=8, H=8, G=2, D=64, R=64,
             pairs=False, far=360000),
        # a training step's queries and keys: 32 utterances of 500 frames
        dict(name="norm-train-16000x16+4x64", kind="norm-train", type="bf16", N=16000, H=16, G=4,
             D=64, R=64, pairs=False, far=500),
        # the same for a small odd model in full precision, part of a head
        # rotated, pairs side by side
        dict(name="norm-train-1266x5+5x43", kind="norm-train", type="f32", N=1266, H=5, G=5, D=43,
             R=26, pairs=True, far=1266),
        # a full server: the next frame of 1,024 streams
        dict(name="linear-step-1024x8x64x64", kind="linear-step", type="f16", n=1024, H=8, K=64,
             V=64),
        # an hour-long recording's frames in one sequence, read backwards
        dict(name="linear-1x40000x8x64x64", kind="linear", type="bf16", n=1, T=40000, H=8, K=64,
             V=64, empty=False, reverse=True),
        # a small minibatch of unequal utterances (one of them empty), odd
        # widths, full precision
        dict(name="linear-train-6x211x5x41x57", kind="linear-train", type="f32", n=6, T=211, H=5,
             K=41, V=57, empty=True, reverse=False),
        # a large minibatch of long utterances, wide heads
        dict(name="linear-train-64x2000x8x128x128", kind="linear-train", type="bf16", n=64,
             T=2000, H=8, K=128, V=128, empty=False, reverse=False),
        # streaming recognition: the next frame of four callers (latency)
        dict(name="window-step-4x8+2x64", kind="window-step", type="bf16", n=4, H=8, G=2, D=64,
             window=512, sinks=4),
        # a full server: the next frame of 256 streams
        dict(name="window-step-256x16+4x128", kind="window-step", type="f16", n=256, H=16, G=4,
             D=128, window=1000, sinks=4),
        # an hour-long recording in one sequence
        dict(name="window-1x40000x8+8x64", kind="window", type="bf16", n=1, T=40000, H=8, G=8,
             D=64, window=512, sinks=4, empty=False),
        # a small minibatch in full precision, no size a round number
        dict(name="window-train-6x211x6+2x43", kind="window-train", type="f32", n=6, T=211, H=6,
             G=2, D=43, window=50, sinks=3, empty=True),
        # the largest: a minibatch of long utterances, four query heads to a
        # key head
        dict(name="window-train-16x2000x16+4x128", kind="window-train", type="bf16", n=16, T=2000,
             H=16, G=4, D=128, window=1000, sinks=4, empty=False),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A head's width: most often 64 or 128, else any number."""
    return rng.choice([64, 64, 128]) if rng.random() < 0.6 else rng.randint(lo, hi)


def _heads(rng):
    """Query heads and key heads: one, two or four queries to a key."""
    G = rng.choice([1, 2, 3, 4, 5, 8])
    return G * rng.choice([1, 1, 2, 4] if G <= 4 else [1, 2]), G


def draw(rng):
    kind = rng.choice(["norm", "norm-train", "linear", "linear-train", "linear-train",
                       "linear-step", "window", "window-train", "window-train", "window-step"])
    typ = rng.choice(["bf16", "bf16", "f16", "f32"])
    case = dict(kind=kind, type=typ)
    if kind.startswith("norm"):
        H, G = _heads(rng)
        D = _width(rng, 8, 128)
        R = D // 2 * 2 if rng.random() < 0.7 else rng.randint(0, D // 2) * 2
        return dict(case, N=_log_int(rng, 1, 16000), H=H, G=G, D=D, R=R,
                    pairs=rng.random() < 0.3, far=_log_int(rng, 100, 1000000))
    if kind == "linear-step":
        return dict(case, n=_log_int(rng, 1, 512), H=rng.randint(1, 8), K=_width(rng, 16, 128),
                    V=_width(rng, 16, 128))
    if kind == "window-step":
        H, G = _heads(rng)
        return dict(case, n=_log_int(rng, 1, 128), H=H, G=G, D=_width(rng, 16, 128),
                    window=_log_int(rng, 1, 2000), sinks=rng.choice([0, 1, 4, rng.randint(0, 64)]))
    small = typ == "f32"
    whole = kind in ("linear", "window")
    T = _log_int(rng, 1, 40000 if whole and not small else 2000)
    rows = 40000 if kind.startswith("linear") else 20000
    n = _log_int(rng, 1, max(1, min(64, rows // (2 * T if small else T))))
    case.update(n=n, T=T, empty=n > 1 and rng.random() < 0.3)
    if kind.startswith("linear"):
        return dict(case, H=rng.randint(1, 8), K=_width(rng, 16, 128), V=_width(rng, 16, 128),
                    reverse=rng.random() < 0.5)
    H, G = _heads(rng)
    return dict(case, H=H if H <= 8 else G, G=G, D=_width(rng, 16, 128),
                window=_log_int(rng, 1, min(1000, 20000000 // max(T, 1000))),
                sinks=rng.choice([0, 1, 4, rng.randint(0, 64)]))


def _lengths(case):
    """Frames of each sequence: unequal, from T down to half of it."""
    n, T = case["n"], case["T"]
    out = [max(1, T - (i * T) // (2 * n)) for i in range(n)]
    if case["empty"]:
        out[n // 2] = 0
    return out


def _positions(case):
    """The position of each stream's next frame: from a stream's first frame to
    well past the window."""
    n, far = case["n"], 3 * (case["window"] + case["sinks"])
    return [(i * far) // max(1, n - 1) if n > 1 else far for i in range(n)]


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

_composer = None


def _context():
    """The program's context: made once and used for every call."""
    global _composer
    if _composer is None:
        from paper_2110_02848_amd import gpu
        _composer = gpu.Composer(0)
    return _composer


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE)
    gen.manual_seed(1000003 * int(seed) + sum(ord(c) for c in case["kind"]))
    f32, i32, dt = torch.float32, torch.int32, TYPES[case["type"]]

    def normal(*shape, mean=0.0, std=1.0, dtype=dt):
        t = torch.randn(*shape, generator=gen, device=DEVICE, dtype=f32)
        return (mean + std * t).to(dtype)

    s = dict(case=case, comp=_context() if own else None)
    kind = case["kind"]
    if kind.startswith("norm"):
        N, H, G, D, R = (case[c] for c in "NHGDR")
        pos = torch.randint(0, case["far"], (N,), generator=gen, device=DEVICE, dtype=i32)
        freq = 10000.0 ** (-torch.arange(R // 2, dtype=torch.float64) * 2 / max(R, 1))
        s.update(q=normal(N, H * D, std=2.0), k=normal(N, G * D, std=0.7), pos=pos,
                 freq=freq.to(f32).to(DEVICE), q_weight=normal(D, mean=1.0, std=0.2, dtype=f32),
                 k_weight=normal(D, mean=1.0, std=0.2, dtype=f32))
        if kind == "norm-train":
            s.update(grad_q=normal(N, H * D, std=0.1), grad_k=normal(N, G * D, std=0.1))
        return s
    if kind.startswith("linear"):
        n, H, K, V = case["n"], case["H"], case["K"], case["V"]
        # memories from 8 frames (the first head) to 1,000 (the last)
        keep = 1 - 2.0 ** (-3 - 7 * torch.arange(H, dtype=torch.float64) / max(H - 1, 1))
        s.update(log_decay=torch.log(keep).to(f32).to(DEVICE),
                 state=normal(n, H, K, V, std=2.0, dtype=f32))
        N = n
        if kind != "linear-step":
            N = _offsets(s, _lengths(case))
        s.update(q=normal(N, H * K), k=normal(N, H * K), v=normal(N, H * V))
        if kind == "linear-train":
            s.update(grad_y=normal(N, H * V, std=0.1),
                     grad_last=normal(n, H, K, V, std=0.1, dtype=f32))
        return s
    n, H, G, D = (case[c] for c in "nHGD")
    N = n
    if kind == "window-step":
        L = case["window"] + case["sinks"]
        s.update(pos=torch.tensor(_positions(case), dtype=i32, device=DEVICE),
                 k_cache=normal(n * L, G * D), v_cache=normal(n * L, G * D))
    else:
        N = _offsets(s, _lengths(case))
    s.update(q=normal(N, H * D), k=normal(N, G * D), v=normal(N, G * D))
    if kind == "window-train":
        s.update(grad_y=normal(N, H * D, std=0.1))
    return s


def _offsets(s, lens):
    off = [0]
    for k in lens:
        off.append(off[-1] + k)
    s.update(offset=torch.tensor(off, dtype=torch.int32, device=DEVICE), T=max(lens))
    return off[-1]


# ---------------------------------------------------------------------------
# one pass: the framework's operators
# ---------------------------------------------------------------------------

def _run_own(s):
    comp, case = s["comp"], s["case"]
    kind = case["kind"]
    train = kind.endswith("train")
    if kind.startswith("norm"):
        args = (s["q"], s["k"], s["q_weight"], s["k_weight"], s["freq"], s["pos"])
        q, k = comp.head_norms(*args, eps=EPS, pairs=case["pairs"])
        out = dict(q=q, k=k)
        if train:
            g = comp.head_norms_grads(*args, s["grad_q"], s["grad_k"], eps=EPS,
                                      pairs=case["pairs"])
            out.update({"grad_" + c: g[c] for c in ("q", "k", "q_weight", "k_weight")})
        return out
    qkv = (s["q"], s["k"], s["v"])
    if kind == "linear-step":
        y, state = comp.linear_attention_step(*qkv, s["log_decay"], s["state"])
        return dict(y=y, state=state)
    if kind.startswith("linear"):
        r = comp.linear_attention(*qkv, s["log_decay"], s["offset"], state=s["state"],
                                  reverse=case["reverse"])
        if train:
            g = comp.linear_attention_grads(*qkv, s["log_decay"], s["offset"], s["grad_y"],
                                            state=s["state"], grad_last=s["grad_last"],
                                            reverse=case["reverse"])
            r.update({"grad_" + c: g[c] for c in ("q", "k", "v", "state")})
        return r
    how = dict(heads=case["H"], kv_heads=case["G"], window=case["window"], sinks=case["sinks"])
    if kind == "window-step":
        y = comp.window_attention_step(*qkv, s["pos"], s["k_cache"], s["v_cache"], **how)
        return dict(y=y, k_cache=s["k_cache"], v_cache=s["v_cache"])
    r = comp.window_attention(*qkv, s["offset"], **how)
    if train:
        g = comp.window_attention_grads(*qkv, s["offset"], r["y"], r["lse"], s["grad_y"], **how)
        r.update({"grad_" + c: g[c] for c in "qkv"})
    return r


# ---------------------------------------------------------------------------
# one pass: the plain forms
# ---------------------------------------------------------------------------

def _turn(z, cos, sin, pairs):
    """The first 2 P values of each head turned by P angles; the rest as it is."""
    P = cos.shape[-1]
    if P == 0:
        return z
    a, b = (z[..., 0:2 * P:2], z[..., 1:2 * P:2]) if pairs else (z[..., :P], z[..., P:2 * P])
    u, v = a * cos - b * sin, b * cos + a * sin
    both = torch.stack([u, v], -1).flatten(-2) if pairs else torch.cat([u, v], -1)
    return torch.cat([both, z[..., 2 * P:]], -1)


def _plain_norm(s):
    case = s["case"]
    N, D, pairs = case["N"], case["D"], case["pairs"]
    angle = s["pos"].double()[:, None, None] * s["freq"].double()
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()

    def forward(x, w):
        z = x.float().view(N, -1, D)
        r = torch.rsqrt((z * z).mean(-1, keepdim=True) + EPS)
        return z * r, r, _turn(z * r * w, cos, sin, pairs).reshape(N, -1).to(x.dtype)

    def back(x, w, g, z, r):
        g = _turn(g.float().view(N, -1, D), cos, -sin, pairs)
        h = g * w
        gx = r * (h - z * (h * z).mean(-1, keepdim=True))
        return gx.reshape(N, -1).to(x.dtype), (g * z).sum((0, 1))

    zq, rq, q = forward(s["q"], s["q_weight"])
    zk, rk, k = forward(s["k"], s["k_weight"])
    out = dict(q=q, k=k)
    if case["kind"] == "norm-train":
        gq, gwq = back(s["q"], s["q_weight"], s["grad_q"], zq, rq)
        gk, gwk = back(s["k"], s["k_weight"], s["grad_k"], zk, rk)
        out.update(grad_q=gq, grad_k=gk, grad_q_weight=gwq, grad_k_weight=gwk)
    return out


def _padded(s):
    """(rows of [N, ..] tensors as [n, T], which of them there are, lengths)."""
    off, T = s["offset"].long(), s["T"]
    length = off[1:] - off[:-1]
    pos = torch.arange(T, device=DEVICE)[None, :]
    there = pos < length[:, None]
    row = off[:-1, None] + (length[:, None] - 1 - pos if s["case"].get("reverse") else pos)
    return torch.where(there, row, torch.zeros_like(row)), there, length


def _linear(q, k, v, g, S0, first):
    """y[t] = sum over j <= t of e^(g (t - j)) (q[t] . k[j]) v[j], and
    e^(g (t + first)) q[t] S0; all [n, H, T, .], a chunk's rows at once and the
    chunks' states by one product."""
    n, H, T, _ = q.shape
    C = min(CHUNK, T)
    m = (T + C - 1) // C

    def cut(t):
        t = torch.nn.functional.pad(t, (0, 0, 0, m * C - T))
        return t.view(n, H, m, C, t.shape[-1])

    q, k, v = cut(q), cut(k), cut(v)
    i = torch.arange(C, device=DEVICE, dtype=torch.float32)
    c = torch.arange(m, device=DEVICE, dtype=torch.float32)
    g = g[:, None, None]
    d = i[:, None] - i[None, :]
    inside = torch.where(d >= 0, torch.exp(g * d.clamp(min=0)), torch.zeros_like(d))
    y = ((q @ k.transpose(-1, -2).contiguous()) * inside[:, None]) @ v
    add = (k * torch.exp(g * (C - 1 - i)[:, None])[:, None]).transpose(-1, -2).contiguous() @ v
    d = c[:, None] - 1 - c[None, :]
    between = torch.where(d >= 0, torch.exp(g * C * d.clamp(min=0)), torch.zeros_like(d))
    state = (between @ add.flatten(-2)).view_as(add)
    y = y + (q * torch.exp(g * (i + 1)[:, None])[:, None]) @ state
    from0 = torch.exp(g[..., None] * (c[:, None] * C + i)[..., None] + first * g[..., None])
    y = y + (q * from0) @ S0[:, :, None]
    return y.view(n, H, m * C, -1)[:, :, :T]


def _plain_linear(s):
    case, dt = s["case"], s["q"].dtype
    H, K, V = case["H"], case["K"], case["V"]
    g, scale, S0 = s["log_decay"], case["K"] ** -0.5, s["state"]
    if case["kind"] == "linear-step":
        q, k, v = (s[c].float().view(-1, H, w) for c, w in (("q", K), ("k", K), ("v", V)))
        S = torch.exp(g)[:, None, None] * S0 + k[..., None] * v[..., None, :]
        y = scale * (q[..., None, :] @ S)[..., 0, :]
        return dict(y=y.reshape(-1, H * V).to(dt), state=S)
    row, there, length = _padded(s)
    m = there[:, :, None, None].float()

    def spread(t, w):
        return (t.float().view(-1, H, w)[row] * m).transpose(1, 2).contiguous()

    to = torch.where(there, row, torch.full_like(row, s["q"].shape[0])).reshape(-1)

    def rows(t):
        t = t.transpose(1, 2).reshape(to.shape[0], -1)
        out = torch.empty(s["q"].shape[0] + 1, t.shape[1], device=DEVICE)
        return out.index_copy_(0, to, t)[:-1].to(dt)

    q, k, v = spread(s["q"], K), spread(s["k"], K), spread(s["v"], V)
    t = torch.arange(s["T"], device=DEVICE)
    left = (length[:, None] - 1 - t).clamp(min=0).float()[:, None]
    decay = torch.exp(g[:, None] * left)  # [n, H, T], to the sequence's end
    whole = torch.exp(g * length[:, None])[..., None, None]
    last = (k * decay[..., None]).transpose(-1, -2).contiguous() @ v + whole * S0
    out = dict(y=rows(scale * _linear(q, k, v, g, S0, 1.0)), last=last)
    if case["kind"] == "linear":
        return out
    # the gradients are linear attention too: of (grad_y, v, k) forward, and
    # of (v, grad_y, q) and (k, q, grad_y) from each sequence's end back
    gy = spread(s["grad_y"], V) * scale
    back = torch.where(there, length[:, None] - 1 - t, t)[:, None, :, None]

    def flip(x):
        return x.gather(2, back.expand(x.shape))

    gl = s["grad_last"]
    gq = _linear(gy, v, k, g, S0.transpose(-1, -2), 1.0)
    qf, kf, vf, yf = flip(q), flip(k), flip(v), flip(gy)
    gk = flip(_linear(vf, yf, qf, g, gl.transpose(-1, -2), 0.0))
    gv = flip(_linear(kf, qf, yf, g, gl, 0.0))
    from0 = torch.exp(g[:, None] * (t + 1).float())
    gs = (q * from0[..., None]).transpose(-1, -2).contiguous() @ gy + whole * gl
    return dict(out, grad_q=rows(gq), grad_k=rows(gk), grad_v=rows(gv), grad_state=gs)


def _softmax(z):
    """Weights and log-sums of rows that have one finite score at least."""
    m = z.max(-1, keepdim=True).values
    e = torch.exp(z - m)
    t = e.sum(-1, keepdim=True)
    return e / t, m + torch.log(t)


def _plain_window_step(s):
    case, dt = s["case"], s["q"].dtype
    H, G, D, W, S = (case[c] for c in ("H", "G", "D", "window", "sinks"))
    n, L, pos = case["n"], W + S, s["pos"].long()
    base = torch.arange(n, device=DEVICE) * L
    row = base + torch.where(pos < S, pos, S + (pos - S) % W)
    s["k_cache"][row] = s["k"]
    s["v_cache"][row] = s["v"]
    k = s["k_cache"].view(n, L, G, 1, D).permute(0, 2, 3, 4, 1)
    v = s["v_cache"].view(n, L, G, D).transpose(1, 2)
    q = s["q"].float().view(n, G, H // G, D)
    z = D ** -0.5 * (q @ k.float()[:, :, 0].contiguous())
    z = z.masked_fill((torch.arange(L, device=DEVICE) > pos[:, None])[:, None, None], -math.inf)
    y = _softmax(z)[0] @ v.float().contiguous()
    return dict(y=y.reshape(n, H * D).to(dt), k_cache=s["k_cache"], v_cache=s["v_cache"])


def _plain_window(s):
    """Blocks of queries against the frames that any of a block sees: the
    window before it, itself, and the first ones."""
    case, dt = s["case"], s["q"].dtype
    H, G, D, W, S = (case[c] for c in ("H", "G", "D", "window", "sinks"))
    scale, E = D ** -0.5, H // G
    row, there, length = _padded(s)
    n, T = row.shape
    B = min(T, max(W, 64))
    m, W, S = (T + B - 1) // B, min(W, T), min(S, T)
    t = torch.arange(m * B, device=DEVICE).view(m, B)
    key = torch.cat([torch.arange(S, device=DEVICE).expand(m, S),
                     t[:, :1] + torch.arange(1 - W, B, device=DEVICE)], 1)
    ahead = t[:, :, None] - key[:, None, :]
    first = torch.arange(key.shape[1], device=DEVICE) < S
    see = (ahead >= 0) & (key[:, None, :] >= 0) & torch.where(first, ahead >= W, ahead < W)
    kt, qt = key.clamp(0, T - 1), t.clamp(max=T - 1)
    kthere = there[:, kt] & (key < T) & (key >= 0)
    qthere = there[:, qt] & (t < T)

    def take(x, at, real, heads):
        x = x.float().view(-1, heads, D)[row[:, at]] * real[..., None, None]
        return x.permute(0, 3, 1, 2, 4)  # [n, heads, m, ., D]

    q = take(s["q"], qt, qthere, H).reshape(n, G, E, m, B, D).transpose(2, 3)
    q = q.reshape(n, G, m, E * B, D)
    k, v = take(s["k"], kt, kthere, G), take(s["v"], kt, kthere, G)
    seen = see.repeat(1, E, 1)
    z = scale * (q @ k.transpose(-1, -2).contiguous())
    p, lse = _softmax(z.masked_fill(~seen, -math.inf))
    del z

    def rows(x, heads):  # of queries' blocks
        x = x.view(n, G, m, E, B, -1).permute(0, 2, 4, 1, 3, 5).reshape(n * m * B, -1)
        to = torch.where(qthere, row[:, qt], torch.full_like(qt, s["q"].shape[0])).reshape(-1)
        out = torch.empty(s["q"].shape[0] + 1, x.shape[1], device=DEVICE)
        return out.index_copy_(0, to, x)[:-1]

    y = p @ v.contiguous()
    out = dict(y=rows(y, H).to(dt), lse=rows(lse, H))
    if case["kind"] == "window":
        return out
    gy = take(s["grad_y"], qt, qthere, H).reshape(n, G, E, m, B, D).transpose(2, 3)
    gy = gy.reshape(n, G, m, E * B, D)
    d = gy @ v.transpose(-1, -2).contiguous()
    d = scale * p * (d - (d * p).sum(-1, keepdim=True))

    def sums(x):  # of keys' blocks, every block's share
        x = x.permute(0, 2, 3, 1, 4).reshape(-1, G * D)
        to = torch.where(kthere, row[:, kt], torch.full_like(kt, s["q"].shape[0])).reshape(-1)
        out = torch.zeros(s["q"].shape[0] + 1, G * D, device=DEVICE)
        return out.index_add_(0, to, x)[:-1].to(dt)

    gv = p.transpose(-1, -2).contiguous() @ gy
    gk = d.transpose(-1, -2).contiguous() @ q
    return dict(out, grad_q=rows(d @ k.contiguous(), H).to(dt), grad_k=sums(gk), grad_v=sums(gv))


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind.startswith("norm"):
        return _plain_norm(s)
    if kind.startswith("linear"):
        return _plain_linear(s)
    return _plain_window_step(s) if kind == "window-step" else _plain_window(s)


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# the least work of one pass
# ---------------------------------------------------------------------------

def _seen(W, S, T):
    """Pairs of a frame and one that it sees, in a sequence of T."""
    w = min(W, T)
    near = w * (w + 1) // 2 + (T - w) * w
    # first frames outside the window: frame t has min(S, t - W + 1) of them
    b = max(0, T - W)
    s = min(S, b)
    return near + s * (s + 1) // 2 + (b - s) * S


def work(case):
    """Every input read once, every output written once.  A row of linear
    attention takes two products with the K x V state forward and five for its
    gradients (one state again, one back, and one for each of the three); a
    pair of the window attention two dot products forward and five more."""
    kind, e = case["kind"], 4 if case["type"] == "f32" else 2
    if kind.startswith("norm"):
        m = case["N"] * (case["H"] + case["G"]) * case["D"]
        small = 4 * case["N"] + 8 * case["D"] + 2 * case["R"]
        if kind == "norm":
            return dict(bytes=2 * m * e + small, flops=8 * m)
        return dict(bytes=4 * m * e + small + 8 * case["D"], flops=24 * m)
    if kind.startswith("linear"):
        n, H, K, V = case["n"], case["H"], case["K"], case["V"]
        N = n if kind == "linear-step" else sum(_lengths(case))
        ends = 8 * n * H * K * V
        if kind != "linear-train":
            return dict(bytes=2 * N * H * (K + V) * e + ends, flops=4 * N * H * K * V)
        return dict(bytes=N * H * e * (4 * K + 4 * V) + 2 * ends, flops=14 * N * H * K * V)
    H, G, D, W, S = (case[c] for c in ("H", "G", "D", "window", "sinks"))
    if kind == "window-step":
        seen = sum(min(p + 1, W + S) for p in _positions(case))
        return dict(bytes=e * (2 * seen * G * D + case["n"] * (2 * H + 4 * G) * D),
                    flops=4 * seen * H * D)
    lens = _lengths(case)
    N, pairs = sum(lens), sum(_seen(W, S, T) for T in lens) * H
    if kind == "window":
        return dict(bytes=N * (2 * H + 2 * G) * D * e + 4 * N * H, flops=4 * pairs * D)
    return dict(bytes=N * (4 * H + 4 * G) * D * e + 4 * N * H, flops=14 * pairs * D)


# ---------------------------------------------------------------------------
# values in 64 bits
# ---------------------------------------------------------------------------

def _starts(lens):
    out = [0]
    for k in lens:
        out.append(out[-1] + k)
    return out


def _exact_norm(s):
    case, f64 = s["case"], torch.float64
    N, D, R = case["N"], case["D"], case["R"]
    angle = s["pos"].to(f64)[:, None] * s["freq"].to(f64)[None]
    # a rotation as complex numbers
    turn = torch.complex(torch.cos(angle), torch.sin(angle))[:, None]
    at = torch.arange(R, device=DEVICE).view(R // 2, 2) if case["pairs"] else \
        torch.arange(R, device=DEVICE).view(2, R // 2).t()

    def rotate(z, by):
        z = z.clone()
        if R:
            c = torch.complex(z[..., at[:, 0]], z[..., at[:, 1]]) * by
            z[..., at[:, 0]], z[..., at[:, 1]] = c.real, c.imag
        return z

    out = {}
    for c in "qk":
        x, w = s[c].to(f64).view(N, -1, D), s[c + "_weight"].to(f64)
        size = torch.sqrt((x ** 2).sum(-1, keepdim=True) / D + EPS)
        out[c] = rotate(x / size * w, turn).reshape(N, -1)
        if case["kind"] == "norm-train":
            g = rotate(s["grad_" + c].to(f64).view(N, -1, D), turn.conj())
            inner = (g * w * x).sum(-1, keepdim=True) / D
            out["grad_" + c] = (g * w / size - x * inner / size ** 3).reshape(N, -1)
            out["grad_" + c + "_weight"] = (g * x / size).reshape(-1, D).sum(0)
    if case["kind"] == "norm":
        return dict(q=out["q"], k=out["k"])
    return {c: out[c] for c in ("q", "k", "grad_q", "grad_k", "grad_q_weight", "grad_k_weight")}


def _exact_linear(s):
    """Frame by frame, as the recurrent form is defined."""
    case, f64 = s["case"], torch.float64
    n, H, K, V, step = case["n"], case["H"], case["K"], case["V"], case["kind"] == "linear-step"
    lens = [1] * n if step else _lengths(case)
    T, start = max(lens), _starts(lens)
    rows = torch.full((T, n), -1, dtype=torch.int64)
    for i, k in enumerate(lens):
        order = torch.arange(start[i], start[i + 1])
        rows[:k, i] = order.flip(0) if case.get("reverse") else order
    live = [torch.nonzero(r >= 0).reshape(-1).to(DEVICE) for r in rows]
    all_there = [len(a) == n for a in live]
    rows = rows.to(DEVICE)
    scale, keep = K ** -0.5, torch.exp(s["log_decay"].to(f64))[:, None, None]
    q, k = s["q"].to(f64).view(-1, H, K), s["k"].to(f64).view(-1, H, K)
    v = s["v"].to(f64).view(-1, H, V)
    train = case["kind"] == "linear-train"
    gy = s["grad_y"].to(f64).view(-1, H, V) * scale if train else None
    y, gq, gk, gv = torch.zeros_like(v), torch.zeros_like(q), torch.zeros_like(q), \
        torch.zeros_like(v)
    S = s["state"].to(f64).clone()
    for t in range(T):
        a = slice(None) if all_there[t] else live[t]
        r = rows[t][a]
        now = keep * S[a] + k[r][..., None] * v[r][:, :, None]
        S[a] = now
        y[r] = scale * (q[r][:, :, None] @ now)[:, :, 0]
        if train:
            gq[r] = (now @ gy[r][..., None])[..., 0]
    out = dict(y=y.reshape(-1, H * V), last=S)
    if step:
        return dict(y=out["y"], state=S)
    if not train:
        return out
    dS = s["grad_last"].to(f64).clone()
    for t in range(T - 1, -1, -1):
        a = slice(None) if all_there[t] else live[t]
        r = rows[t][a]
        now = dS[a] + q[r][..., None] * gy[r][:, :, None]
        gk[r] = (now @ v[r][..., None])[..., 0]
        gv[r] = (k[r][:, :, None] @ now)[:, :, 0]
        dS[a] = keep * now
    return dict(out, grad_q=gq.reshape(-1, H * K), grad_k=gk.reshape(-1, H * K),
                grad_v=gv.reshape(-1, H * V), grad_state=dS)


def _exact_window_step(s):
    """Each stream by itself, its frames in their order."""
    case, f64 = s["case"], torch.float64
    H, G, D, W, S = (case[c] for c in ("H", "G", "D", "window", "sinks"))
    n, L = case["n"], W + S
    kc, vc = s["k_cache"].to(f64).view(n, L, G, D), s["v_cache"].to(f64).view(n, L, G, D)
    y = torch.zeros(n, H, D, dtype=f64, device=DEVICE)
    for i, p in enumerate(_positions(case)):
        at = p if p < S else S + (p - S) % W
        kc[i, at], vc[i, at] = s["k"][i].to(f64).view(G, D), s["v"][i].to(f64).view(G, D)
        frames = [f for f in range(min(S, p + 1))]
        frames += [f for f in range(max(S, p - W + 1), p + 1)]
        at = torch.tensor([f if f < S else S + (f - S) % W for f in frames], device=DEVICE)
        q = s["q"][i].to(f64).view(G, H // G, D)
        z = torch.bmm(q, kc[i, at].permute(1, 2, 0).contiguous()) / math.sqrt(D)
        w = torch.softmax(z, -1)
        y[i] = torch.bmm(w, vc[i, at].transpose(0, 1).contiguous()).reshape(H, D)
    return dict(y=y.reshape(n, H * D), k_cache=kc.reshape(n * L, G * D),
                v_cache=vc.reshape(n * L, G * D))


def _exact_window(s):
    """Sequence by sequence, some queries at a time against all frames from the
    window's first on and the first frames before it."""
    case, f64 = s["case"], torch.float64
    H, G, D, W, S = (case[c] for c in ("H", "G", "D", "window", "sinks"))
    lens = _lengths(case)
    start = _starts(lens)
    train = case["kind"] == "window-train"
    q = s["q"].to(f64).view(-1, H, D).transpose(0, 1)
    k, v = (s[c].to(f64).view(-1, G, D).transpose(0, 1) for c in "kv")
    y, lse = torch.zeros_like(q), torch.zeros(H, q.shape[1], dtype=f64, device=DEVICE)
    if train:
        gy = s["grad_y"].to(f64).view(-1, H, D).transpose(0, 1)
        gq, gk, gv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    share = torch.arange(H, device=DEVICE) // (H // G)
    for i, T in enumerate(lens):
        for t0 in range(0, T, 512):
            t = torch.arange(t0, min(T, t0 + 512), device=DEVICE)
            lo = max(0, t0 - W + 1)
            f = torch.cat([torch.arange(min(S, lo), device=DEVICE),
                           torch.arange(lo, int(t[-1]) + 1, device=DEVICE)])
            hidden = (f > t[:, None]) | ((t[:, None] - f >= W) & (f >= S))
            a, b = start[i] + t, start[i] + f
            kb, vb = k[:, b][share], v[:, b][share]
            z = torch.bmm(q[:, a].contiguous(), kb.transpose(1, 2).contiguous()) / math.sqrt(D)
            z[:, hidden] = -math.inf
            lse[:, a] = torch.logsumexp(z, -1)
            w = torch.exp(z - lse[:, a][..., None])
            yb = torch.bmm(w, vb)
            y[:, a] = yb
            if train:
                g = gy[:, a].contiguous()
                dw = torch.bmm(g, vb.transpose(1, 2).contiguous())
                dz = w * (dw - (g * yb).sum(-1, keepdim=True)) / math.sqrt(D)
                gq[:, a] = torch.bmm(dz, kb)
                one = torch.bmm(dz.transpose(1, 2).contiguous(), q[:, a].contiguous())
                gk[:, b] += one.view(G, H // G, -1, D).sum(1)
                one = torch.bmm(w.transpose(1, 2).contiguous(), g)
                gv[:, b] += one.view(G, H // G, -1, D).sum(1)

    def flat(x):
        return x.transpose(0, 1).reshape(x.shape[1], -1)

    out = dict(y=flat(y), lse=lse.t().contiguous())
    if train:
        out.update(grad_q=flat(gq), grad_k=flat(gk), grad_v=flat(gv))
    return out


def exact(case, seed):
    """What run() returns, in 64 bits."""
    s = prepare(case, seed)
    kind = case["kind"]
    if kind.startswith("norm"):
        return _exact_norm(s)
    if kind.startswith("linear"):
        return _exact_linear(s)
    return _exact_window_step(s) if kind == "window-step" else _exact_window(s)
