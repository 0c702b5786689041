"""Performance cases of the operators between a network and its graphs: the
work that a recogniser's training and serving have them do, through the public
Python entry points (``paper_2110_02848_amd.gpu.Composer``).

Kinds of case:

* ``step``        one frame of many streams through the gated recurrence;
* ``scan``        the recurrence over whole sequences, forward only;
* ``scan-train``  the same and its gradients;
* ``emit``        log-softmax of a linear head: weights of emission graphs;
* ``emit-train``  the same and its gradients;
* ``loss``        cross entropy over a vocabulary of words, forward only;
* ``loss-train``  the same and its gradients.

``run`` makes the calls where ``own`` is true; where it is not, it computes
the same by elementary torch operations in 32 bits.
"""
import math

import torch

own = False

DEVICE = "cuda:0"
TYPES = dict(f32=torch.float32, f16=torch.float16, bf16=torch.bfloat16)


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def listed():
    return [
        # streaming recognition: the next frame of eight callers (latency)
        dict(name="step-8x256", kind="step", type="bf16", n=8, D=256),
        # streaming on a full server: every stream's next frame
        dict(name="step-4096x1024", kind="step", type="f16", n=4096, D=1024),
        # an hour-long recording's frames in one sequence, read backwards
        dict(name="scan-1x40000x512", kind="scan", type="bf16", n=1, T=40000, D=512, empty=False,
             reverse=True),
        # a small minibatch of unequal utterances (one of them empty), odd
        # width, full precision
        dict(name="train-6x211x333", kind="scan-train", type="f32", n=6, T=211, D=333,
             empty=True, reverse=False),
        # a large minibatch of long utterances
        dict(name="train-64x2000x1024", kind="scan-train", type="bf16", n=64, T=2000, D=1024,
             empty=False, reverse=False),
        # emission weights of a short stream's frames, 28 tokens
        dict(name="emit-16x28x256", kind="emit", type="f16", N=16, C=28, H=256),
        # a training step's emissions: 32 utterances of 500 frames, 69 phonemes
        dict(name="emit-train-16000x69x512", kind="emit-train", type="bf16", N=16000, C=69,
             H=512),
        # the same for a small odd model in full precision
        dict(name="emit-train-1266x41x333", kind="emit-train", type="f32", N=1266, C=41, H=333),
        # scores of the next word of four hypotheses over 10,000 words
        dict(name="loss-4x10000x512", kind="loss", type="bf16", N=4, V=10000, H=512),
        # training on words, no size a round number
        dict(name="loss-train-1053x7919x509", kind="loss-train", type="f16", N=1053, V=7919,
             H=509),
        # a small model's step in full precision
        dict(name="loss-train-1000x1000x256", kind="loss-train", type="f32", N=1000, V=1000,
             H=256),
        # the largest: every frame of a minibatch against 32,000 words
        dict(name="loss-train-16000x32000x1024", kind="loss-train", type="bf16", N=16000,
             V=32000, H=1024),
    ]


def _log_int(rng, lo, hi):
    """An integer of [lo, hi], even over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng, lo, hi):
    """A layer's width: half of them multiples of 64, the others any number."""
    w = _log_int(rng, lo, hi)
    return max(64, w // 64 * 64) if rng.random() < 0.5 else w


def draw(rng):
    kind = rng.choice(["step", "scan", "scan-train", "scan-train", "emit", "emit-train",
                       "emit-train", "loss", "loss-train", "loss-train"])
    typ = rng.choice(["bf16", "bf16", "f16", "f32"])
    case = dict(kind=kind, type=typ)
    if kind == "step":
        return dict(case, n=_log_int(rng, 1, 4096), D=_width(rng, 100, 1024))
    if kind in ("scan", "scan-train"):
        D = _width(rng, 64, 1024)
        rows = 30000 if typ == "f32" else 60000
        T = _log_int(rng, 1, 40000 if kind == "scan" else 2000)
        n = _log_int(rng, 1, max(1, min(64, rows // T)))
        return dict(case, n=n, T=T, D=D, empty=n > 1 and rng.random() < 0.3,
                    reverse=rng.random() < 0.5)
    H = _width(rng, 100, 1024)
    if kind in ("emit", "emit-train"):
        N = _log_int(rng, 1, 16000)
        C = rng.randint(20, 100) if rng.random() < 0.7 else _log_int(rng, 100, 1000)
        return dict(case, N=N, C=C, H=H)
    small = typ == "f32"
    N = _log_int(rng, 1, 2000 if small else 16000)
    return dict(case, N=N, V=_log_int(rng, 500, 8000 if small else 32000), H=H)


def _lengths(case):
    """Frames of each sequence: unequal, from T down to half of it."""
    n, T = case["n"], case["T"]
    out = [max(1, T - (i * T) // (2 * n)) for i in range(n)]
    if case["empty"]:
        out[n // 2] = 0
    return out


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
    dt = TYPES[case["type"]]

    def normal(*shape, mean=0.0, std=1.0, dtype=dt):
        t = torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.float32)
        return (mean + std * t).to(dtype)

    f32 = torch.float32
    s = dict(case=case, comp=_context() if own else None)
    kind = case["kind"]
    if kind == "step":
        n, D = case["n"], case["D"]
        s.update(x=normal(n, D), gate=normal(n, D, mean=1.5, std=1.5),
                 state=normal(n, D, std=0.6, dtype=f32))
    elif kind in ("scan", "scan-train"):
        n, D = case["n"], case["D"]
        lens = _lengths(case)
        off = [0]
        for k in lens:
            off.append(off[-1] + k)
        N = off[-1]
        # gates lean to keeping: memories of tens of frames
        s.update(offset=torch.tensor(off, dtype=torch.int32, device=DEVICE), T=max(lens),
                 x=normal(N, D), gate=normal(N, D, mean=1.5, std=1.5),
                 state=normal(n, D, std=0.6, dtype=f32))
        if kind == "scan-train":
            s.update(grad_y=normal(N, D, std=0.1), grad_last=normal(n, D, std=0.1, dtype=f32))
    elif kind in ("emit", "emit-train"):
        N, C, H = case["N"], case["C"], case["H"]
        s.update(x=normal(N, H), w=normal(C, H, std=2.0 / math.sqrt(H)))
        if kind == "emit-train":
            # minus the arcs' posteriors: a few likely tokens a frame
            post = torch.softmax(normal(N, C, std=4.0, dtype=f32), 1)
            s.update(grad=(-post).contiguous())
    else:
        N, V, H = case["N"], case["V"], case["H"]
        # frequent words are more likely; a sixteenth of the rows have no word
        u = torch.rand(N, generator=gen, device=DEVICE)
        target = (V * u * u).to(torch.int32).clamp_(max=V - 1)
        none = torch.rand(N, generator=gen, device=DEVICE) < 0.0625
        target = torch.where(none, torch.full_like(target, -1), target)
        s.update(x=normal(N, H), w=normal(V, H, std=2.0 / math.sqrt(H)), target=target)
        if kind == "loss-train":
            # the mean over rows, rows weighted between 0.5 and 1.5
            scale = 0.5 + torch.rand(N, generator=gen, device=DEVICE)
            s.update(grad=scale / N)
    return s


# ---------------------------------------------------------------------------
# one pass: the framework's operators
# ---------------------------------------------------------------------------

def _run_own(s):
    comp, kind = s["comp"], s["case"]["kind"]
    if kind == "step":
        y, state = comp.recurrence_step(s["x"], s["gate"], s["state"])
        return dict(y=y, state=state)
    if kind in ("scan", "scan-train"):
        rev, train = s["case"]["reverse"], kind == "scan-train"
        r = comp.recurrence(s["x"], s["gate"], s["offset"], state=s["state"], reverse=rev,
                            save=train)
        out = dict(y=r["y"], last=r["last"])
        if train:
            g = comp.recurrence_grads(s["x"], s["gate"], s["offset"], s["grad_y"], r["saved"],
                                      state=s["state"], grad_last=s["grad_last"], reverse=rev)
            out.update(grad_x=g["x"], grad_gate=g["gate"], grad_state=g["state"])
        return out
    if kind in ("emit", "emit-train"):
        weight = comp.emission_weights(s["x"], s["w"])
        if kind == "emit":
            return dict(weight=weight)
        gx, gw = comp.emission_grads(s["x"], s["w"], weight, s["grad"])
        return dict(weight=weight, grad_x=gx, grad_w=gw)
    r = comp.cross_entropy(s["x"], s["w"], s["target"])
    if kind == "loss":
        return dict(loss=r["loss"], lse=r["lse"])
    gx, gw = comp.cross_entropy_grads(s["x"], s["w"], s["target"], r["lse"], s["grad"])
    return dict(loss=r["loss"], lse=r["lse"], grad_x=gx, grad_w=gw)


# ---------------------------------------------------------------------------
# one pass: the plain forms
# ---------------------------------------------------------------------------

def _scan(f, b):
    """h[:, t] = f[:, t] h[:, t - 1] + b[:, t] by doubling."""
    k, T = 1, f.shape[1]
    while k < T:
        b = torch.cat([b[:, :k], b[:, k:] + f[:, k:] * b[:, :-k]], 1)
        f = torch.cat([f[:, :k], f[:, k:] * f[:, :-k]], 1)
        k *= 2
    return b


def _plain_scan(s):
    case, off, T = s["case"], s["offset"].long(), s["T"]
    x, gate = s["x"].float(), s["gate"].float()
    dt = s["x"].dtype
    length = (off[1:] - off[:-1])[:, None]
    pos = torch.arange(T, device=DEVICE)[None, :]
    there = pos < length
    row = off[:-1, None] + (length - 1 - pos if case["reverse"] else pos)
    row = torch.where(there, row, torch.zeros_like(row))
    last = (length - 1).clamp(min=0)[:, :, None].expand(-1, 1, x.shape[1])
    some = length > 0
    m = there[:, :, None].float()
    f = torch.sigmoid(gate)[row] * m
    xs = x[row] * m
    b = (1 - f) * xs
    b[:, 0] += f[:, 0] * s["state"]
    h = _scan(f, b)
    # back to rows; what lies past a sequence's end goes to a row of its own
    to = torch.where(there, row, torch.full_like(row, x.shape[0])).reshape(-1)

    def rows(t):
        out = torch.empty(x.shape[0] + 1, x.shape[1], device=x.device)
        return out.index_copy_(0, to, t.reshape(-1, x.shape[1]))[:-1]

    out = dict(y=rows(h).to(dt), last=torch.where(some, h.gather(1, last)[:, 0], s["state"]))
    if case["kind"] == "scan":
        return out
    # the other way round: D[t] = gy[t] + f[t + 1] D[t + 1]
    gy = s["grad_y"].float()[row] * m
    gy.scatter_add_(1, last, (s["grad_last"] * some)[:, None])
    fn = torch.cat([f[:, 1:], torch.zeros_like(f[:, :1])], 1)
    d = _scan(fn.flip(1), gy.flip(1)).flip(1)
    hp = torch.cat([s["state"][:, None], h[:, :-1]], 1)
    gx, gu = rows((1 - f) * d), rows(d * (hp - xs) * f * (1 - f))
    gs = torch.where(some, f[:, 0] * d[:, 0], s["grad_last"])
    return dict(out, grad_x=gx.to(dt), grad_gate=gu.to(dt), grad_state=gs)


def _log_sum(z):
    m = z.max(1, keepdim=True).values
    return m + torch.log(torch.exp(z - m).sum(1, keepdim=True))


def _run_plain(s):
    kind, dt = s["case"]["kind"], s["x"].dtype
    if kind == "step":
        f = torch.sigmoid(s["gate"].float())
        h = f * s["state"] + (1 - f) * s["x"].float()
        return dict(y=h.to(dt), state=h)
    if kind in ("scan", "scan-train"):
        return _plain_scan(s)
    x, w = s["x"].float(), s["w"].float()
    z = x @ w.t()
    lse = _log_sum(z)
    if kind in ("emit", "emit-train"):
        weight = z - lse
        if kind == "emit":
            return dict(weight=weight)
        g = s["grad"]
        d = g - torch.exp(weight) * g.sum(1, keepdim=True)
        return dict(weight=weight, grad_x=(d @ w).to(dt), grad_w=(d.t() @ x).to(dt))
    word = s["target"].long()
    some = word >= 0
    at = word.clamp(min=0)[:, None]
    loss = torch.where(some, (lse - z.gather(1, at))[:, 0], torch.zeros_like(lse[:, 0]))
    out = dict(loss=loss, lse=lse[:, 0])
    if kind == "loss":
        return out
    p = torch.exp(z - lse)
    p.scatter_add_(1, at, torch.full_like(at, -1, dtype=torch.float32))
    p *= (s["grad"] * some)[:, None]
    return dict(out, grad_x=(p @ w).to(dt), grad_w=(p.t() @ x).to(dt))


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---------------------------------------------------------------------------
# the least work of one pass
# ---------------------------------------------------------------------------

def work(case):
    """Every input read once, every output written once.  A recurrence's
    element takes about 8 operations forward and 10 more for its gradients;
    a head takes one product forward and two for its gradients."""
    kind, e = case["kind"], 4 if case["type"] == "f32" else 2
    if kind == "step":
        m = case["n"] * case["D"]
        return dict(bytes=m * (3 * e + 8), flops=8 * m)
    if kind in ("scan", "scan-train"):
        m, nd = sum(_lengths(case)) * case["D"], case["n"] * case["D"]
        if kind == "scan":
            return dict(bytes=m * 3 * e + 8 * nd, flops=8 * m)
        return dict(bytes=m * 6 * e + 16 * nd, flops=18 * m)
    N, H = case["N"], case["H"]
    C = case["C"] if kind in ("emit", "emit-train") else case["V"]
    ends = (N + C) * H * e
    if kind == "emit":
        return dict(bytes=ends + 4 * N * C, flops=2 * N * C * H)
    if kind == "emit-train":
        return dict(bytes=2 * ends + 8 * N * C, flops=6 * N * C * H)
    if kind == "loss":
        return dict(bytes=ends + 12 * N, flops=2 * N * C * H)
    return dict(bytes=2 * ends + 16 * N, flops=6 * N * C * H)


# ---------------------------------------------------------------------------
# values in 64 bits
# ---------------------------------------------------------------------------

def _exact_scan(s):
    """Frame by frame, as the recurrence is defined."""
    case, f64 = s["case"], torch.float64
    lens = _lengths(case)
    T, n, D = max(lens), case["n"], case["D"]
    start = [0]
    for k in lens:
        start.append(start[-1] + k)
    # rows[t]: the row of each sequence that step t reads, -1 past its end
    rows = torch.full((T, n), -1, dtype=torch.int64)
    for i, k in enumerate(lens):
        order = torch.arange(start[i], start[i + 1])
        rows[:k, i] = order.flip(0) if case["reverse"] else order
    live = (rows >= 0).to(DEVICE)
    rows = rows.clamp(min=0).to(DEVICE)
    x, u = s["x"].to(f64), s["gate"].to(f64)
    keep, new = 1 / (1 + torch.exp(-u)), 1 / (1 + torch.exp(u))
    h = s["state"].to(f64)
    train = case["kind"] == "scan-train"
    y = torch.zeros_like(x)
    before = torch.zeros_like(x) if train else None
    ragged = min(lens) != T
    for t in range(T):
        r = rows[t]
        v = keep[r] * h + new[r] * x[r]
        if ragged:
            on = live[t]
            if train:
                before[r[on]] = h[on]
            h = torch.where(on[:, None], v, h)
            y[r[on]] = h[on]
        else:
            if train:
                before[r] = h
            h = v
            y[r] = h
    out = dict(y=y, last=h)
    if not train:
        return out
    gy = s["grad_y"].to(f64)
    total = torch.zeros_like(x)
    into = s["grad_last"].to(f64)
    for t in range(T - 1, -1, -1):
        r, on = rows[t], live[t]
        d = gy[r] + into
        total[r[on]] = d[on]
        into = torch.where(on[:, None], keep[r] * d, into)
    return dict(out, grad_x=new * total, grad_gate=total * (before - x) * keep * new,
                grad_state=into)


def exact(case, seed):
    """What run() returns, in 64 bits: sequences frame by frame, heads in
    blocks of rows."""
    s = prepare(case, seed)
    kind, f64 = case["kind"], torch.float64
    if kind == "step":
        u = s["gate"].to(f64)
        h = s["state"].to(f64) / (1 + torch.exp(-u)) + s["x"].to(f64) / (1 + torch.exp(u))
        return dict(y=h, state=h)
    if kind in ("scan", "scan-train"):
        return _exact_scan(s)
    x, w = s["x"].to(f64), s["w"].to(f64)
    train = kind.endswith("train")
    parts = []
    gw = torch.zeros_like(w)
    for i in range(0, x.shape[0], 2048):
        xb = x[i:i + 2048]
        z = torch.mm(xb, w.t().contiguous())
        lse = torch.logsumexp(z, 1)
        p = torch.exp(z - lse[:, None])
        if kind.startswith("emit"):
            one = [z - lse[:, None]]
            if train:
                g = s["grad"][i:i + 2048].to(f64)
                d = g - p * g.sum(1, keepdim=True)
        else:
            word = s["target"][i:i + 2048].long()
            hit = torch.nonzero(word >= 0).reshape(-1)
            loss = torch.zeros_like(lse)
            loss[hit] = lse[hit] - z[hit, word[hit]]
            one = [loss, lse]
            if train:
                d = torch.zeros_like(z)
                g = s["grad"][i:i + 2048].to(f64)
                d[hit] = p[hit] * g[hit, None]
                d[hit, word[hit]] -= g[hit]
        if train:
            one.append(torch.mm(d, w))
            gw += torch.mm(d.t().contiguous(), xb)
        parts.append(one)
    joined = [torch.cat(c) for c in zip(*parts)]
    names = ["weight"] if kind.startswith("emit") else ["loss", "lse"]
    out = dict(zip(names + ["grad_x"], joined))
    if train:
        out["grad_w"] = gw
    return out
