"""Plain implementations, in 64 bits on the CPU, of the attention layers over
frames, written as they are defined, and the bounds that their tests hold results
to.  U is half the spacing of float32, HALF_ULP a type's.

Bounds count roundings: a sum of n products in 32 bits, in any order, is off by at
most n U' times the sum of the terms' sizes, U' = 2 U (the matrix cores may cut
instead of round); what is rounded to a 16-bit type before it is multiplied adds
HALF_ULP of the type times the same."""
import torch

from layershelp import F64, HALF_ULP, TINY, TYPES  # noqa: F401

U = 2.0 ** -24
H16 = {torch.float32: 0.0, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
INF = float("inf")


def within(name, got, want, bound):
    """|got - want| <= bound + the rounding of got's type, element by element."""
    got = got.detach().cpu()
    dt = got.dtype
    got = got.to(F64)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    most = bound + 1.01 * HALF_ULP[dt] * want.abs() + TINY[dt]
    bad = ~((got - want).abs() <= most)
    # from half a spacing past its largest number on, a type rounds to infinity
    limit = torch.finfo(dt).max * (1 + HALF_ULP[dt] / 2)
    bad &= ~((want.abs() + most >= limit) & (got == torch.sign(want) * INF))
    if bad.any():
        i = tuple(torch.nonzero(bad)[0].tolist())
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {i}: "
                             f"{got[i].item()} for {want[i].item()}, bound {most[i].item()}, "
                             f"worst {((got - want).abs() / most).max().item():.3g} of it")


def offsets(lens):
    off = [0]
    for k in lens:
        off.append(off[-1] + k)
    return off


# ---- norms and rotation ----

def rotate(z, pos, freq, pairs, back=False):
    """z [N, heads, D], pos [N], freq [P]: pair by pair."""
    out = z.clone()
    P = 0 if freq is None else len(freq)
    for i in range(P):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, P + i)
        t = pos.to(F64) * freq[i].to(F64)
        c, s = torch.cos(t)[:, None], torch.sin(t)[:, None]
        if back:
            s = -s
        out[..., a] = z[..., a] * c - z[..., b] * s
        out[..., b] = z[..., b] * c + z[..., a] * s
    return out


def spread(z, freq, pairs):
    """Sizes of what a rotation adds up: |a| + |b| for each of a pair."""
    out = z.abs().clone()
    P = 0 if freq is None else len(freq)
    for i in range(P):
        a, b = (2 * i, 2 * i + 1) if pairs else (i, P + i)
        out[..., a] = out[..., b] = z[..., a].abs() + z[..., b].abs()
    return out


def head_norm(x, w, freq, pos, eps, pairs):
    """(result, bound) of x [N, heads * D] in 64 bits."""
    N, D = x.shape[0], len(w)
    z = x.view(N, x.shape[1] // D, D)
    r = 1 / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)
    y = z * r * w
    # the sum of D squares, its root and quotient, the weight, the turn (its
    # angle is a number below 1 rounded once, times 2 pi) and its two products
    return (rotate(y, pos, freq, pairs).flatten(1),
            (D + 40) * U * spread(y, freq, pairs).flatten(1))


def head_norm_grads(x, w, freq, pos, eps, pairs, g):
    """((grad_x, bound), (grad_w, bound))."""
    N, D = x.shape[0], len(w)
    z = x.view(N, x.shape[1] // D, D)
    r = 1 / torch.sqrt((z * z).mean(-1, keepdim=True) + eps)
    z = z * r
    turned = rotate(g.view(N, g.shape[1] // D, D), pos, freq, pairs, back=True)
    size = spread(g.view(N, g.shape[1] // D, D), freq, pairs)
    h = turned * w
    gx = r * (h - z * (h * z).mean(-1, keepdim=True))
    most = size * w.abs()
    bx = (3 * D + 80) * U * r * (most + z.abs() * (most * z.abs()).mean(-1, keepdim=True))
    gw = (turned * z).sum((0, 1))
    bw = (2 * N * z.shape[1] + D + 80) * U * (size * z.abs()).sum((0, 1))
    return (gx.flatten(1), bx.flatten(1)), (gw, bw)


# ---- linear attention ----

def linear(q, k, v, g, off, state, reverse, scale):
    """(y, last): q, k [N, H * K], v [N, H * V], g [H] in 64 bits."""
    H, n = len(g), len(off) - 1
    N = q.shape[0]
    q, k, v = (t.view(N, H, t.shape[1] // H) for t in (q, k, v))
    y = torch.zeros_like(v)
    last = torch.zeros(n, H, q.shape[2], v.shape[2], dtype=F64)
    keep = torch.exp(g)[:, None, None]
    for s in range(n):
        S = state[s].clone() if state is not None else torch.zeros_like(last[s])
        rows = range(off[s], off[s + 1])
        for t in reversed(rows) if reverse else rows:
            S = keep * S + k[t][:, :, None] * v[t][:, None, :]
            y[t] = scale * (q[t][:, :, None] * S).sum(1)
        last[s] = S
    return y.flatten(1), last


def linear_grads(q, k, v, g, off, state, reverse, scale, gy, glast):
    """(grad_q, grad_k, grad_v, grad_state)."""
    H, n, N = len(g), len(off) - 1, q.shape[0]
    q, k, v, gy = (t.view(N, H, t.shape[1] // H) for t in (q, k, v, gy))
    gq, gk, gv = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    K, V = q.shape[2], v.shape[2]
    gs = torch.zeros(n, H, K, V, dtype=F64)
    keep = torch.exp(g)[:, None, None]
    for s in range(n):
        rows = list(range(off[s], off[s + 1]))
        if reverse:
            rows.reverse()
        S = state[s].clone() if state is not None else torch.zeros_like(gs[s])
        for t in rows:
            S = keep * S + k[t][:, :, None] * v[t][:, None, :]
            gq[t] = scale * (S * gy[t][:, None, :]).sum(2)
        D = glast[s].clone() if glast is not None else torch.zeros_like(gs[s])
        for t in reversed(rows):
            D = D + scale * q[t][:, :, None] * gy[t][:, None, :]
            gk[t] = (D * v[t][:, None, :]).sum(2)
            gv[t] = (D * k[t][:, :, None]).sum(1)
            D = keep * D
        gs[s] = D
    return gq.flatten(1), gk.flatten(1), gv.flatten(1), gs


def linear_bounds(dt, sizes, states, longest):
    """Bounds of results that add terms of these sizes (the operator of the
    inputs' absolute values): a score or a number of the state is a sum of up to
    128 products, one of 64 scores or 128 numbers of the state follows, and the
    state is carried through longest / 64 chunks, of 64 products each, and a
    power of the decay times it (two numbers, off by U each chunk)."""
    C = 2 * (128 + 128) + 3 * 64 + 6 * (longest // 64 + 1)
    small = 2.0 ** -36 if dt == torch.float16 else 0.0  # scaled float16's spacing at 0
    # The matrix cores take bfloat16 numbers below 2^-126 as 0 (a head that keeps
    # e^-80 of its state has decayed k of that size): each of the three numbers that a
    # decayed k is loses up to 2^-126 times a v, here at most 6, in up to 64 rows of a
    # chunk, and earlier chunks' losses decay: 3 * 6 * 64 * 2^-126 * 2 < 2^-114.
    lost = 2.0 ** -114 if dt == torch.bfloat16 else 0.0
    out = [(C * U + H16[dt]) * a + small * (a.max() if a.numel() else 0) + lost for a in sizes]
    return out, [C * U * a + (2.0 ** -32 * a.max() if small and a.numel() else 0) + lost
                 for a in states]


# ---- attention to a window ----

def visible(T, window, sinks):
    t = torch.arange(T)
    ahead = t[:, None] - t[None, :]
    return (ahead >= 0) & ((ahead < window) | (t[None, :] < sinks))


def window(q, k, v, off, heads, kv_heads, win, sinks, scale, gy=None):
    """dict of (value, sizes for bounds) in 64 bits."""
    N = q.shape[0]
    D = q.shape[1] // heads
    E = heads // kv_heads
    out = {c: torch.zeros_like(t) for c, t in (("y", q), ("gq", q), ("gk", k), ("gv", v))}
    out["lse"] = torch.zeros(N, heads, dtype=F64)
    for c in ("y", "lse", "gq", "gk", "gv"):
        out["b" + c] = torch.zeros_like(out[c])
        out["r" + c] = torch.zeros_like(out[c])
    for s in range(len(off) - 1):
        a, b = off[s], off[s + 1]
        if a == b:
            continue
        see = visible(b - a, win, sinks)
        for h in range(heads):
            col, kc = slice(h * D, h * D + D), slice(h // E * D, h // E * D + D)
            Q, K, V = q[a:b, col], k[a:b, kc], v[a:b, kc]
            z = scale * Q @ K.t()
            size = abs(scale) * Q.abs() @ K.abs().t()
            z = torch.where(see, z, torch.full_like(z, -INF))
            lse = torch.logsumexp(z, 1)
            P = torch.exp(z - lse[:, None])
            P = torch.where(see, P, torch.zeros_like(P))
            # how far a score, its exponent and the log-sum are off, at most
            top = torch.where(see, size, torch.zeros_like(size)).max(1).values
            off_z = (2 * D + 24) * U * (top + 1) + 16 * U * (lse.abs() + top)
            rel = 2 * off_z + 2 * (b - a) * U
            out["y"][a:b, col] = P @ V
            out["by"][a:b, col] = (rel + 2 * (b - a) * U)[:, None] * (P @ V.abs())
            out["ry"][a:b, col] = P @ V.abs()
            out["lse"][a:b, h] = lse
            out["blse"][a:b, h] = 2 * off_z + 2 * (b - a) * U
            if gy is None:
                continue
            G = gy[a:b, col]
            Y = P @ V
            dP = G @ V.t()
            dS = P * (dP - (Y * G).sum(1, keepdim=True))
            mass = G.abs() @ V.abs().t()            # sizes of the terms of dP
            own = (G.abs() * (P @ V.abs())).sum(1, keepdim=True)  # and of delta
            n = 2 * (b - a) + 2 * D + 32
            e = rel[:, None] * dS.abs() + n * U * P * (mass + own)
            e = e + P * rel[:, None] * own
            ones = (P != 0).sum(1, keepdim=True) == 1
            e = torch.where(ones, torch.zeros_like(e), e)
            dS = torch.where(ones, torch.zeros_like(dS), dS)
            # with 16 bits: dS rounded once, and delta from y as it was rounded
            r = dS.abs() + torch.where(ones, torch.zeros_like(P), P) * own
            out["gq"][a:b, col] = scale * dS @ K
            out["bgq"][a:b, col] = abs(scale) * (e + n * U * dS.abs()) @ K.abs()
            out["rgq"][a:b, col] = abs(scale) * r @ K.abs()
            out["gk"][a:b, kc] += scale * dS.t() @ Q
            out["bgk"][a:b, kc] += abs(scale) * (e + n * E * U * dS.abs()).t() @ Q.abs()
            out["rgk"][a:b, kc] += abs(scale) * r.t() @ Q.abs()
            out["gv"][a:b, kc] += P.t() @ G
            out["bgv"][a:b, kc] += ((rel[:, None] + n * E * U) * P).t() @ G.abs()
            out["rgv"][a:b, kc] += P.t() @ G.abs()
    return out


def window_bound(out, c, dt):
    """The bound of result c: float32 steps, and with 16 bits half a spacing of
    what was rounded (float16: and of the spacing at 0 of numbers scaled to 2^15)."""
    b = out["b" + c] + H16[dt] * out["r" + c]
    if dt == torch.float16 and b.numel():
        b = b + 2.0 ** -24 * out["r" + c].max()
    return b
