"""The attention layers over frames on the GPU (norms with rotation, linear
attention, attention to a window, and a run of them together) against the plain
forms in 64 bits, with the bounds of attentionhelp."""
import pytest
import torch

import attentionhelp as ref
from attentionhelp import F64, TYPES

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


@pytest.fixture(scope="module")
def comp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2110_02848_amd import gpu
    c = gpu.Composer(0)
    yield c
    c.close()


def _mat(g, rows, cols, typ, pad=0, std=1.0):
    """A view of rows `pad` elements longer, that start `pad` elements in."""
    t = (std * torch.randn(rows, cols + 2 * pad, generator=g)).to(TYPES[typ])
    return t.cuda()[:, pad:pad + cols]


def _vec(g, *shape, std=1.0):
    return (std * torch.randn(*shape, generator=g)).cuda()


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _d(t):
    return None if t is None else t.detach().cpu().to(F64)


def _gen(*seed):
    return torch.Generator().manual_seed(hash(seed) % (1 << 31))


# ---------------------------------------------------------------------------
# norms and rotation
# ---------------------------------------------------------------------------

def _check_norms(comp, q, k, qw, kw, freq, pos, gq, gk, eps, pairs, stream=None):
    print(f"[norms] {tuple(q.shape)} {q.dtype} strides {q.stride()} D={qw.numel()} "
          f"P={0 if freq is None else freq.numel()} pairs={pairs}", flush=True)
    yq, yk = comp.head_norms(q, k, qw, kw, freq, pos, eps, pairs, stream=stream)
    r = comp.head_norms_grads(q, k, qw, kw, freq, pos, gq, gk, eps, pairs, stream=stream)
    torch.cuda.synchronize()
    P, F = (None, None) if pos is None else (pos.cpu(), freq.cpu())
    for c, x, w, y, g in (("q", q, qw, yq, gq), ("k", k, kw, yk, gk)):
        if x is None:
            assert y is None and r["k"] is None and r["k_weight"] is None
            continue
        ref.within("y_" + c, y, *ref.head_norm(_d(x), _d(w), F, P, eps, pairs))
        a, b = ref.head_norm_grads(_d(x), _d(w), F, P, eps, pairs, _d(g))
        ref.within("grad_" + c, r[c], *a)
        ref.within("grad_weight_" + c, r[c + "_weight"], *b)


def _norm_inputs(N, H, G, D, P, typ, pad=0, far=1000):
    g = _gen(N, H, G, D, P)
    q, k = _mat(g, N, H * D, typ, pad, 2.0), _mat(g, N, G * D, typ, pad, 0.5)
    gq, gk = _mat(g, N, H * D, typ, pad), _mat(g, N, G * D, typ, pad)
    qw, kw = _vec(g, D) + 1, _vec(g, D) + 1
    freq = (10000.0 ** (-torch.arange(P) / max(P, 1))).float().cuda() if P else None
    pos = torch.randint(0, far, (N,), generator=g).int().cuda() if P else None
    return q, k, qw, kw, freq, pos, gq, gk


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("N,H,G,D,P", [
    (1, 1, 1, 1, 0), (1, 1, 1, 2, 1), (3, 2, 1, 7, 3), (5, 4, 2, 64, 32), (2, 3, 3, 64, 20),
    (70, 8, 2, 128, 64), (9, 5, 1, 43, 13), (33, 1, 7, 96, 48), (4, 2, 2, 512, 256),
    (3, 1, 1, 300, 0), (2, 16, 4, 256, 128), (17, 2, 2, 80, 40), (13, 40, 8, 24, 12),
    (2100, 1, 1, 64, 32),
])
def test_norms(comp, N, H, G, D, P, typ, pairs):
    _check_norms(comp, *_norm_inputs(N, H, G, D, P, typ), 1e-6, pairs)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("pad", [1, 2, 4, 8])
def test_norms_of_strided_rows(comp, typ, pad):
    _check_norms(comp, *_norm_inputs(11, 3, 2, 64, 32, typ, pad), 1e-5, False)
    _check_norms(comp, *_norm_inputs(11, 3, 2, 40, 10, typ, pad), 1e-5, True)


def test_norms_of_parts_of_one_matrix(comp):
    g = _gen(4)
    qkv = _mat(g, 20, 6 * 64, "bf16")
    q, k = qkv[:, :3 * 64], qkv[:, 3 * 64:5 * 64]
    _, _, qw, kw, freq, pos, gq, gk = _norm_inputs(20, 3, 2, 64, 32, "bf16")
    _check_norms(comp, q, k, qw, kw, freq, pos, gq, gk, 1e-6, False)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_norms_at_far_positions(comp, typ):
    args = list(_norm_inputs(6, 2, 2, 64, 32, typ))
    args[5] = _i32([0, 1, 2 ** 20 + 1, 10 ** 8 + 3, 2 ** 31 - 1, -5])
    _check_norms(comp, *args, 1e-6, False)


def test_norms_of_queries_alone(comp):
    q, _, qw, _, freq, pos, gq, _ = _norm_inputs(7, 3, 1, 64, 32, "f16")
    _check_norms(comp, q, None, qw, None, freq, pos, gq, None, 1e-6, False)


def test_norms_of_no_rows_and_of_zeros(comp):
    args = _norm_inputs(0, 2, 2, 64, 32, "f32")
    y, _ = comp.head_norms(*args[:6])
    r = comp.head_norms_grads(*args)
    assert y.shape == (0, 128) and not r["q_weight"].any() and not r["k_weight"].any()
    args = list(_norm_inputs(3, 2, 2, 64, 32, "f32"))
    args[0] = torch.zeros_like(args[0])
    _check_norms(comp, *args, 1e-6, False)
    # a NaN stays in its own head's row
    args[0][1, 5] = NAN
    y, k = comp.head_norms(*args[:6])
    assert y[1, :64].isnan().all() and not y[1, 64:].isnan().any()
    assert not y[0].isnan().any() and not y[2].isnan().any() and not k.isnan().any()


# ---------------------------------------------------------------------------
# linear attention
# ---------------------------------------------------------------------------

def _linear_inputs(lens, H, K, V, typ, pad=0, seed=0):
    g = _gen(sum(lens), len(lens), H, K, V, seed)
    N, n = sum(lens), len(lens)
    q, k, v = (_mat(g, N, H * w, typ, pad) for w in (K, K, V))
    gy = _mat(g, N, H * V, typ, pad)
    state, glast = _vec(g, n, H, K, V), _vec(g, n, H, K, V)
    decay = -torch.logspace(-3, 0.5, H).cuda() if H > 1 else torch.tensor([-0.05]).cuda()
    return q, k, v, decay, state, gy, glast


def _check_linear(comp, q, k, v, decay, off, state, gy, glast, rev, scale=None, stream=None):
    H = decay.numel()
    print(f"[linear] {tuple(q.shape)} {tuple(v.shape)} {q.dtype} strides {q.stride()} H={H} "
          f"n={len(off) - 1} rev={rev}", flush=True)
    r = comp.linear_attention(q, k, v, decay, _i32(off), state=state, scale=scale, reverse=rev,
                              stream=stream)
    g = comp.linear_attention_grads(q, k, v, decay, _i32(off), gy, state=state, grad_last=glast,
                                    scale=scale, reverse=rev, stream=stream)
    torch.cuda.synchronize()
    s = (q.shape[1] // H) ** -0.5 if scale is None else scale
    args = [_d(t) for t in (q, k, v)]
    size = [t.abs() for t in args]
    d, st, gl, GY = _d(decay), _d(state), _d(glast), _d(gy)
    ab = [None if t is None else t.abs() for t in (st, gl)]
    dt = q.dtype
    longest = max([b - a for a, b in zip(off, off[1:])], default=0)
    y, last = ref.linear(*args, d, off, st, rev, s)
    (by,), (bl,) = ref.linear_bounds(dt, *[[t] for t in ref.linear(*size, d, off, ab[0], rev,
                                                                   abs(s))], longest)
    ref.within("y", r["y"], y, by)
    ref.within("last", r["last"], last, bl)
    want = ref.linear_grads(*args, d, off, st, rev, s, GY, gl)
    sizes = ref.linear_grads(*size, d, off, ab[0], rev, abs(s), GY.abs(), ab[1])
    bounds, (bs,) = ref.linear_bounds(dt, sizes[:3], sizes[3:], longest)
    for c, w, b in zip(("q", "k", "v", "state"), want, bounds + [bs]):
        ref.within("grad_" + c, g[c], w, b)
    return r, g


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("lens,H,K,V", [
    ([1], 1, 1, 1), ([1, 1, 1], 2, 3, 2), ([0], 1, 8, 8), ([3, 0, 2], 2, 64, 64),
    ([15, 16, 17], 1, 63, 65), ([63, 64, 65], 3, 41, 57), ([127, 128, 129], 2, 128, 128),
    ([200], 4, 64, 128), ([130, 0, 1, 5], 2, 128, 32), ([90], 1, 96, 80), ([70], 5, 16, 24),
])
def test_linear_lengths_and_widths(comp, lens, H, K, V, typ, rev):
    q, k, v, d, st, gy, gl = _linear_inputs(lens, H, K, V, typ)
    _check_linear(comp, q, k, v, d, ref.offsets(lens), st, gy, gl, rev)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,H,K,V", [(37, 3, 64, 128), (16, 8, 41, 33), (1, 9, 8, 100),
                                     (5, 1, 128, 60)])
def test_linear_of_many_sequences_and_heads(comp, n, H, K, V, typ):
    """Every job, head and slice of columns is some workgroup's, whatever is left of
    the division by the card's eight XCDs."""
    lens = [(7 * i) % 19 for i in range(n)] if n > 1 else [70]
    q, k, v, d, st, gy, gl = _linear_inputs(lens, H, K, V, typ)
    _check_linear(comp, q, k, v, d, ref.offsets(lens), st, gy, gl, False)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [[9000], [9000] + [1] * 11])
def test_linear_of_more_units_than_registers(comp, lens, typ):
    q, k, v, d, st, gy, gl = _linear_inputs(lens, 1, 16, 8, typ)
    _check_linear(comp, q, k, v, d, ref.offsets(lens), st, gy, gl, False)


@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens,H,K,V", [([1500], 2, 64, 64), ([700, 0, 403], 1, 33, 65),
                                        ([600, 600], 2, 128, 128)])
def test_linear_cut_into_units(comp, lens, H, K, V, typ, rev):
    q, k, v, d, st, gy, gl = _linear_inputs(lens, H, K, V, typ)
    _check_linear(comp, q, k, v, d, ref.offsets(lens), st, gy, gl, rev)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_linear_without_states_and_with_a_scale(comp, typ):
    lens = [70, 0, 9]
    q, k, v, d, _, gy, _ = _linear_inputs(lens, 2, 34, 20, typ)
    for scale in (0.0, -2.5, 1.0):
        r, g = _check_linear(comp, q, k, v, d, ref.offsets(lens), None, gy, None, False, scale)
        assert not r["last"][1].any() and not g["state"][1].any()


@pytest.mark.parametrize("pad", [1, 2, 4, 8])
@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_linear_of_strided_rows(comp, typ, pad):
    for lens, K, V in (([40, 70], 64, 64), ([1030], 24, 40)):
        q, k, v, d, st, gy, gl = _linear_inputs(lens, 2, K, V, typ, pad)
        _check_linear(comp, q, k, v, d, ref.offsets(lens), st, gy, gl, False)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens", [[150], [1100]])
def test_linear_decays_at_their_ends(comp, lens, typ):
    """Heads that keep everything, next to nothing, and nothing."""
    q, k, v, _, st, gy, gl = _linear_inputs(lens, 4, 20, 20, typ)
    d = torch.tensor([0.0, -80.0, -INF, -1e-7]).cuda()
    r, g = _check_linear(comp, q, k, v, d, ref.offsets(lens), st, gy, gl, False)
    # -inf: a row sees itself alone
    a, b = _d(k)[-1, 40:60], _d(v)[-1, 40:60]
    ref.within("last", r["last"][0, 2], a[:, None] * b, 2.0 ** -20 * (a[:, None] * b).abs())
    assert not g["state"][0, 2].any()


@pytest.mark.parametrize("size", [2.0 ** -12, 2.0 ** 10])
def test_linear_of_small_and_large_float16(comp, size):
    """Scores and states past float16's largest, and below its smallest."""
    for lens in ([130], [1100]):
        q, k, v, d, st, gy, gl = _linear_inputs(lens, 2, 64, 64, "f16")
        q, k = (q.float() * size).half(), (k.float() * size).half()
        scale = size ** -2 / 8
        _check_linear(comp, q, k, v, d, ref.offsets(lens), st * size, gy, gl / size, False, scale)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [NAN, INF])
@pytest.mark.parametrize("rev", [False, True])
def test_linear_rows_do_not_see_later_ones(comp, typ, bad, rev):
    # (sums that a product has made no number of are taken again in another
    # order: within the same bounds, not bit for bit)
    lens = [100, 40]
    off = ref.offsets(lens)
    q, k, v, d, st, gy, gl = _linear_inputs(lens, 2, 32, 32, typ)
    at = 37 if not rev else 62
    args = [_d(t) for t in (q, k, v)]
    size = [t.abs() for t in args]
    how = (_d(d), off), (rev, 32 ** -0.5)
    y, _ = ref.linear(*args, *how[0], _d(st), *how[1])
    ay, _ = ref.linear(*size, *how[0], _d(st).abs(), *how[1])
    want = ref.linear_grads(*args, *how[0], _d(st), *how[1], _d(gy), _d(gl))
    ag = ref.linear_grads(*size, *how[0], _d(st).abs(), *how[1], _d(gy).abs(), _d(gl).abs())
    (by, bq, bk, bv), _ = ref.linear_bounds(TYPES[typ], [ay, *ag[:3]], [], 100)
    later = range(at, 100) if not rev else range(0, at + 1)
    others = [t for t in range(140) if t not in later]
    for x in (q, k, v):
        z = x.clone()
        z[at, :32] = bad
        got = comp.linear_attention(*[z if t is x else t for t in (q, k, v)], d, _i32(off),
                                    state=st, reverse=rev)["y"].cpu()
        ref.within("y", got[others], y[others], by[others])
        ref.within("y, other head", got[:, 32:], y[:, 32:], by[:, 32:])
        assert not got[at, :32].float().isfinite().any()
    # gradients by k and v go the other way: rows past a bad dy are as they were
    z = gy.clone()
    z[at, :32] = bad
    got = comp.linear_attention_grads(q, k, v, d, _i32(off), z, state=st, grad_last=gl,
                                      reverse=rev)
    after = [t for t in later if t != at] + list(range(100, 140))
    for c, w, b in (("k", want[1], bk), ("v", want[2], bv)):
        ref.within(c, got[c][after], w[after], b[after])
        ref.within(c, got[c][:, 32:], w[:, 32:], b[:, 32:])
    rest = [t for t in range(140) if t != at]
    ref.within("q", got["q"][rest], want[0][rest], bq[rest])


def test_linear_leaves_rows_of_no_sequence(comp):
    q, k, v, d, st, gy, _ = _linear_inputs([10, 20], 2, 64, 64, "bf16")
    q[25:], k[25:], v[25:] = NAN, NAN, NAN
    off = [0, 10, 25]
    y = torch.full_like(v, 7.0)
    from paper_2110_02848_amd import gpu
    import ctypes
    A, n, _ = comp._linear(q, k, v, d, _i32(off), st, None, False)
    last = torch.empty_like(st)
    rc = comp._lib.fst_linear_attention_run(comp._h, ctypes.byref(A), comp._pass.made(0, y, 2),
                                            last.data_ptr(), comp._call_stream(None))
    assert rc == gpu.FST_OK
    assert (y[25:] == 7.0).all() and y[:25].isfinite().all() and last.isfinite().all()


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,H,K,V", [(1, 1, 1, 1), (3, 2, 64, 64), (5, 3, 41, 57),
                                     (2, 8, 128, 128), (4, 2, 128, 3), (2, 2, 5, 128),
                                     (300, 1, 16, 20)])
def test_linear_steps(comp, n, H, K, V, typ):
    g = _gen(n, H, K, V)
    q, k, v = (_mat(g, n, H * w, typ, 1) for w in (K, K, V))
    state, d = _vec(g, n + 2, H, K, V), -torch.rand(H, generator=g).cuda()
    y, new = comp.linear_attention_step(q, k, v, d, state)
    args = [_d(t) for t in (q, k, v)]
    off = list(range(n + 1))
    want, last = ref.linear(*args, _d(d), off, _d(state)[:n], False, K ** -0.5)
    ay, al = ref.linear(*[t.abs() for t in args], _d(d), off, _d(state)[:n].abs(), False,
                        K ** -0.5)
    ref.within("y", y, want, (K + 16) * ref.U * ay)
    ref.within("state", new[:n], last, 8 * ref.U * al)
    assert torch.equal(new[n:], state[n:])
    # by slots, in place, one row idle
    slot = torch.randperm(n + 2, generator=g)[:n].int().cuda()
    slot[0] = -1
    pool = state.clone()
    y2, same = comp.linear_attention_step(q, k, v, d, pool, slot=slot)
    assert same is pool and not y2[0].any()
    rows = slot[1:].long()
    y3, new3 = comp.linear_attention_step(q[1:], k[1:], v[1:], d, state[rows].contiguous())
    assert torch.equal(y2[1:], y3) and torch.equal(pool[rows], new3)
    rest = [i for i in range(n + 2) if i not in rows.tolist()]
    assert torch.equal(pool[rest], state[rest])
    out = torch.full_like(state, 3.0)
    comp.linear_attention_step(q[1:], k[1:], v[1:], d, state, slot=slot[1:].contiguous(), out=out)
    assert torch.equal(out[rows], new3) and (out[rest] == 3.0).all()


def test_linear_steps_are_the_sequence(comp):
    q, k, v, d, st, _, _ = _linear_inputs([150], 3, 40, 24, "f32")
    r = comp.linear_attention(q, k, v, d, _i32([0, 150]), state=st)
    state, rows = st.clone(), []
    for t in range(150):
        y, state = comp.linear_attention_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], d, state,
                                              out=state)
        rows.append(y)
    args = [t.cpu().to(F64) for t in (q, k, v)]
    ay, al = ref.linear(*[t.abs() for t in args], _d(d), [0, 150], _d(st).abs(), False,
                        40 ** -0.5)
    (by,), (bl,) = ref.linear_bounds(torch.float32, [ay], [al], 150 * 64)  # a chunk a step
    want, last = ref.linear(*args, _d(d), [0, 150], _d(st), False, 40 ** -0.5)
    ref.within("y", torch.cat(rows), want, by)
    ref.within("last", state, last, bl)
    assert r["y"].shape == (150, 72)


# ---------------------------------------------------------------------------
# attention to a window
# ---------------------------------------------------------------------------

def _window_inputs(lens, H, G, D, typ, pad=0, seed=0):
    g = _gen(sum(lens), len(lens), H, G, D, seed)
    N = sum(lens)
    q, gy = _mat(g, N, H * D, typ, pad), _mat(g, N, H * D, typ, pad)
    k, v = _mat(g, N, G * D, typ, pad), _mat(g, N, G * D, typ, pad)
    return q, k, v, gy


def _check_window(comp, q, k, v, gy, off, H, G, win, sinks, scale=None, stream=None):
    print(f"[window] {tuple(q.shape)} {q.dtype} strides {q.stride()} heads {H}/{G} "
          f"n={len(off) - 1} window={win} sinks={sinks}", flush=True)
    how = dict(heads=H, kv_heads=G, window=win, sinks=sinks, scale=scale, stream=stream)
    r = comp.window_attention(q, k, v, _i32(off), **how)
    g = comp.window_attention_grads(q, k, v, _i32(off), r["y"], r["lse"], gy, **how)
    torch.cuda.synchronize()
    s = (q.shape[1] // H) ** -0.5 if scale is None else scale
    o = ref.window(_d(q), _d(k), _d(v), off, H, G, win, sinks, s, _d(gy))
    got = dict(y=r["y"], lse=r["lse"], gq=g["q"], gk=g["k"], gv=g["v"])
    for c, t in got.items():
        ref.within(c, t, o[c], o["blse"] if c == "lse" else ref.window_bound(o, c, q.dtype))
    return r, g


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens,H,G,D,win,sinks", [
    ([1], 1, 1, 1, 1, 0), ([2], 1, 1, 8, 1, 1), ([1, 1, 1], 2, 1, 5, 9, 0), ([0], 1, 1, 8, 3, 0),
    ([3, 0, 2], 2, 2, 64, 2, 1), ([63, 64, 65], 2, 1, 64, 1000, 0), ([150], 4, 2, 64, 17, 4),
    ([130, 0, 1, 129], 3, 1, 43, 64, 3), ([200], 2, 2, 128, 65, 0), ([140, 70], 6, 3, 96, 63, 70),
    ([129], 1, 1, 33, 1, 0), ([300], 2, 1, 16, 5, 20), ([257], 2, 2, 80, 128, 1),
    ([100], 5, 5, 24, 2 ** 31 - 1, 0), ([260], 8, 1, 64, 2, 130),
])
def test_window_lengths_widths_and_masks(comp, lens, H, G, D, win, sinks, typ):
    q, k, v, gy = _window_inputs(lens, H, G, D, typ)
    _check_window(comp, q, k, v, gy, ref.offsets(lens), H, G, win, sinks)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens,H,G,D,win,sinks", [([1300], 2, 1, 64, 200, 4),
                                                  ([700, 600], 1, 1, 128, 30, 17)])
def test_window_of_long_sequences(comp, lens, H, G, D, win, sinks, typ):
    q, k, v, gy = _window_inputs(lens, H, G, D, typ)
    _check_window(comp, q, k, v, gy, ref.offsets(lens), H, G, win, sinks)


@pytest.mark.parametrize("pad", [1, 2, 4, 8])
@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_window_of_strided_rows(comp, typ, pad):
    for D in (64, 40, 128):
        q, k, v, gy = _window_inputs([70, 90], 4, 2, D, typ, pad)
        _check_window(comp, q, k, v, gy, [0, 70, 160], 4, 2, 33, 3)


@pytest.mark.parametrize("scale", [0.0, -0.5, 3.0])
def test_window_scales(comp, scale):
    q, k, v, gy = _window_inputs([90], 2, 2, 32, "f32")
    _check_window(comp, q, k, v, gy, [0, 90], 2, 2, 40, 2, scale)


@pytest.mark.parametrize("size", [2.0 ** -12, 2.0 ** 8])
def test_window_gradients_of_small_and_large_float16(comp, size):
    q, k, v, gy = _window_inputs([300], 2, 1, 64, "f16")
    gy = (gy.float() * size).half()
    _check_window(comp, q, k, v, gy, [0, 300], 2, 1, 90, 3)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_window_rows_see_no_others(comp, typ, bad):
    """A row that is no number reaches the rows that see it, and no other."""
    off, H, G, D, win, sinks = [0, 600, 640], 2, 1, 64, 20, 3
    q, k, v, gy = _window_inputs([600, 40], H, G, D, typ)
    how = dict(heads=H, kv_heads=G, window=win, sinks=sinks)

    o = ref.window(_d(q), _d(k), _d(v), off, H, G, win, sinks, D ** -0.5, _d(gy))

    def both(q, k, v, gy):
        r = comp.window_attention(q, k, v, _i32(off), **how)
        g = comp.window_attention_grads(q, k, v, _i32(off), r["y"], r["lse"], gy, **how)
        return dict(y=r["y"], gq=g["q"], gk=g["k"], gv=g["v"])

    def same(got, c, but):
        rest = [t for t in range(640) if t not in but]
        ref.within(c, got[c][rest], o[c][rest], ref.window_bound(o, c, TYPES[typ])[rest])

    at = 530
    for i in (1, 2):
        args = [q, k, v, gy]
        args[i] = args[i].clone()
        args[i][at] = bad
        got = both(*args)
        sees = range(at, at + win)
        same(got, "y", sees)
        same(got, "gq", sees)
        if i == 2 or bad != bad:
            assert not got["y"][list(sees)].float().isfinite().any()
        # keys that one of those queries sees
        keys = [*range(sinks), *range(at - win + 1, at + win)]
        same(got, "gk", keys)
        same(got, "gv", keys)
    for i in (0, 3):
        args = [q, k, v, gy]
        args[i] = args[i].clone()
        args[i][at] = bad
        got = both(*args)
        same(got, "y", [at])
        same(got, "gq", [at])
        keys = [*range(sinks), *range(at - win + 1, at + 1)]
        same(got, "gk", keys)
        same(got, "gv", keys)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_window_of_many_first_frames(comp, typ):
    """More of them than are cut into units, and more than there are frames."""
    q, k, v, gy = _window_inputs([700, 30], 2, 1, 32, typ)
    for sinks in (257, 300, 256, 2 ** 30):
        _check_window(comp, q, k, v, gy, [0, 700, 730], 2, 1, 10, sinks)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_all_of_it_no_number(comp, typ):
    """Every input NaN: every result is, in no time worth speaking of."""
    q, k, v, gy = (torch.full_like(t, NAN) for t in _window_inputs([3000], 4, 2, 64, typ))
    off = _i32([0, 3000])
    how = dict(heads=4, kv_heads=2, window=2000, sinks=4)
    r = comp.window_attention(q, k, v, off, **how)
    g = comp.window_attention_grads(q, k, v, off, r["y"], r["lse"], gy, **how)
    d = torch.full((4,), -0.1, device="cuda")
    lin = comp.linear_attention(q, q, gy, d, off)
    for t in (r["y"], g["q"][1:], g["k"], g["v"], lin["y"], lin["last"]):
        assert t.isnan().all()


def test_single_rows_of_any_stride(comp):
    """One row has no distance to a next one: any is taken for it."""
    q, k, v, d, st, gy, gl = _linear_inputs([1], 2, 16, 16, "f32")
    far = torch.empty_strided((1, 32), (1 << 40, 1), device="cuda")
    far.copy_(q)
    a = comp.linear_attention(q, k, v, d, _i32([0, 1]), state=st)["y"]
    assert torch.equal(comp.linear_attention(far, k, v, d, _i32([0, 1]), state=st)["y"], a)
    a = comp.window_attention(q, q, q, _i32([0, 1]), heads=2)
    b = comp.window_attention(far, far, far, _i32([0, 1]), heads=2)
    assert torch.equal(a["y"], b["y"]) and torch.equal(a["lse"], b["lse"])
    g = [comp.window_attention_grads(t, t, t, _i32([0, 1]), a["y"], a["lse"], t, heads=2)
         for t in (q, far)]
    assert all(torch.equal(g[0][c], g[1][c]) for c in "qkv") and not g[0]["q"].any()


def test_rows_too_far_apart_are_refused(comp):
    from paper_2110_02848_amd import gpu
    wide = torch.zeros(2, (1 << 22) + 1, dtype=torch.float16, device="cuda")
    x, d = wide[:, :16], torch.zeros(2, device="cuda")
    near = torch.zeros(2, 16, dtype=torch.float16, device="cuda")
    off = _i32([0, 2])
    calls = [lambda: comp.linear_attention(x, near, near, d, off),
             lambda: comp.linear_attention_grads(near, near, near, d, off, x),
             lambda: comp.window_attention(near, x, near, off, heads=2),
             lambda: comp.window_attention_grads(near, near, near, off, near,
                                                 torch.zeros(2, 2, device="cuda"), x, heads=2)]
    for call in calls:
        with pytest.raises(gpu.FstError) as e:
            call()
        assert e.value.code == gpu.FST_ERR_TOO_LARGE
    # as far as may be, and queries of the window attention any way
    x = torch.zeros(2, 1 << 22, dtype=torch.float16, device="cuda")[:, :16]
    x.normal_()
    want = comp.linear_attention(x.contiguous(), near, near + 1, d, off)["y"]
    assert torch.equal(comp.linear_attention(x, near, near + 1, d, off)["y"], want)
    q = wide[:, :16]
    q.normal_()
    want = comp.window_attention(q.contiguous(), near + 1, near + 2, off, heads=2)["y"]
    assert torch.equal(comp.window_attention(q, near + 1, near + 2, off, heads=2)["y"], want)


def test_window_leaves_rows_of_no_sequence(comp):
    from paper_2110_02848_amd import gpu
    import ctypes
    q, k, v, gy = _window_inputs([40], 2, 1, 64, "bf16")
    for t in (q, k, v, gy):
        t[30:] = NAN
    off = _i32([0, 10, 30])
    y, lse = torch.full_like(q, 7.0), torch.full((40, 2), 7.0, device="cuda")
    A, _ = comp._window(q, k, v, off, 2, 1, 5, 2, None)
    m = comp._pass
    rc = comp._lib.fst_window_attention_run(comp._h, ctypes.byref(A), m.made(0, y, 2),
                                            lse.data_ptr(), comp._call_stream(None))
    assert rc == gpu.FST_OK
    assert (y[30:] == 7.0).all() and (lse[30:] == 7.0).all()
    assert y[:30].isfinite().all() and lse[:30].isfinite().all()
    gq, gk, gv = (torch.full_like(t, 7.0) for t in (q, k, v))
    A, _ = comp._window(q, k, v, off, 2, 1, 5, 2, None)
    rc = comp._lib.fst_window_attention_grads(
        comp._h, ctypes.byref(A), m.made(0, y, 2), lse.data_ptr(), m.made(1, gy, 2),
        m.made(2, gq, 2), m.made(3, gk, 2), m.made(4, gv, 2), comp._call_stream(None))
    assert rc == gpu.FST_OK
    for t in (gq, gk, gv):
        assert (t[30:] == 7.0).all() and t[:30].isfinite().all()


def _ring(p, win, sinks):
    return p if p < sinks else sinks + (p - sinks) % win


def _step_reference(q, kf, vf, H, G, win, sinks, scale):
    """(y, bound) of the last of the frames kf, vf ([t, G * D], 64 bits)."""
    t, D = kf.shape[0], q.shape[0] // H
    E = H // G
    y, b, r = (torch.zeros(H * D, dtype=F64) for _ in range(3))
    see = ref.visible(t, win, sinks)[-1]
    for h in range(H):
        c, kc = slice(h * D, h * D + D), slice(h // E * D, h // E * D + D)
        K, V = kf[see, kc], vf[see, kc]
        z = scale * K @ q[c]
        w = torch.softmax(z, 0)
        size = (scale * K.abs() @ q[c].abs()).max()
        off = (2 * D + 24) * ref.U * (size + 1) + 16 * ref.U * (z.abs().max() + 1)
        y[c] = w @ V
        r[c] = w @ V.abs()
        b[c] = (4 * off + (2 * len(z) + 64) * ref.U) * r[c]
    return y, b, r


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("H,G,D,win,sinks,lens", [
    (1, 1, 8, 1, 0, [1, 2, 5]), (2, 1, 64, 4, 2, [1, 2, 3, 6, 7, 40]),
    (4, 2, 43, 33, 3, [1, 33, 36, 37, 100]), (8, 8, 128, 64, 0, [64, 65, 200]),
    (20, 1, 32, 10, 1, [4, 30]), (6, 3, 96, 500, 4, [1, 505, 700]), (3, 3, 64, 2, 64, [70, 200]),
])
def test_window_steps(comp, H, G, D, win, sinks, lens, typ):
    """The last frame of each of some sequences, after filling the caches with
    what comes before it; entries that no frame is in are NaN."""
    n, L = len(lens), win + sinks
    q, k, v, _ = _window_inputs(lens, H, G, D, typ, pad=1)
    off = ref.offsets(lens)
    before = [t for i in range(n) for t in range(off[i], off[i + 1] - 1)]
    kb, vb = k[before], v[before]
    g = _gen(H, G, D)
    slot = torch.randperm(n + 3, generator=g)[:n].int().cuda()
    shape = ((n + 3) * L, G * D)
    kc, vc = (torch.full(shape, NAN, dtype=TYPES[typ], device="cuda") for _ in range(2))
    boff = _i32([o - i for i, o in enumerate(off)])
    comp.window_attention_fill(kb, vb, boff, kc, vc, win, sinks, slot=slot)
    want_k, want_v = torch.full(shape, NAN, dtype=F64), torch.full(shape, NAN, dtype=F64)
    for i, T in enumerate(lens):
        for p in range(T - 1):
            row = int(slot[i]) * L + _ring(p, win, sinks)
            want_k[row], want_v[row] = _d(k)[off[i] + p], _d(v)[off[i] + p]
    assert torch.equal(_d(kc).nan_to_num(9.5), want_k.nan_to_num(9.5))
    assert torch.equal(_d(vc).nan_to_num(9.5), want_v.nan_to_num(9.5))
    lastrow = [o - 1 for o in off[1:]]
    pos = _i32([T - 1 for T in lens])
    print(f"[step] heads {H}/{G} D={D} window={win} sinks={sinks} {typ}", flush=True)
    how = dict(heads=H, kv_heads=G, window=win, sinks=sinks)
    y = comp.window_attention_step(q[lastrow], k[lastrow], v[lastrow], pos, kc, vc, slot=slot,
                                   **how)
    dt = TYPES[typ]
    for i in range(n):
        a, b = off[i], off[i + 1]
        w, bound, r = _step_reference(_d(q)[b - 1], _d(k)[a:b], _d(v)[a:b], H, G, win, sinks,
                                      D ** -0.5)
        small = 2.0 ** -24 if typ == "f16" else 0.0
        ref.within("y", y[i], w, bound + ref.H16[dt] * r + small * r.max())
        row = int(slot[i]) * L + _ring(lens[i] - 1, win, sinks)
        want_k[row], want_v[row] = _d(k)[b - 1], _d(v)[b - 1]
    assert torch.equal(_d(kc).nan_to_num(9.5), want_k.nan_to_num(9.5))
    assert torch.equal(_d(vc).nan_to_num(9.5), want_v.nan_to_num(9.5))
    # idle rows: no slot, or no position; nothing is touched
    kept = kc.clone(), vc.clone()
    idle = slot.clone()
    idle[0] = n + 3
    if n > 1:
        pos[1] = -1
    y2 = comp.window_attention_step(q[lastrow], k[lastrow], v[lastrow], pos, kc, vc, slot=idle,
                                    **how)
    assert not y2[:2].any() and torch.equal(y2[2:], y[2:])
    assert torch.equal(kept[0].nan_to_num(9.5), kc.nan_to_num(9.5))
    assert torch.equal(kept[1].nan_to_num(9.5), vc.nan_to_num(9.5))


def test_window_steps_from_the_first_frame(comp):
    """Streams that begin at different steps, through several turns of the ring,
    give what the whole sequences give."""
    H, G, D, win, sinks, T = 4, 2, 64, 7, 2, 40
    starts = [0, 3, 11]
    lens = [T - s for s in starts]
    off = ref.offsets(lens)
    q, k, v, _ = _window_inputs(lens, H, G, D, "f32")
    whole = comp.window_attention(q, k, v, _i32(off), heads=H, kv_heads=G, window=win,
                                  sinks=sinks)["y"]
    kc, vc = (torch.full((3 * (win + sinks), G * D), NAN, device="cuda") for _ in range(2))
    o = ref.window(_d(q), _d(k), _d(v), off, H, G, win, sinks, D ** -0.5)
    bound = 2 * ref.window_bound(o, "y", torch.float32)
    for t in range(T):
        rows = [off[i] + max(t - s, 0) for i, s in enumerate(starts)]
        y = comp.window_attention_step(q[rows], k[rows], v[rows], _i32([t - s for s in starts]),
                                       kc, vc, heads=H, kv_heads=G, window=win, sinks=sinks)
        for i, s in enumerate(starts):
            if t < s:
                assert not y[i].any()
            else:
                ref.within(f"y {t}", y[i], _d(whole)[rows[i]], bound[rows[i]])


def test_window_caches_of_strided_rows(comp):
    """Caches side by side in one tensor, as a layer's keys and values."""
    H, G, D, win, sinks, n = 4, 2, 64, 9, 1, 3
    both = torch.zeros(n * (win + sinks), 2 * G * D, dtype=torch.bfloat16, device="cuda")
    kc, vc = both[:, :G * D], both[:, G * D:]
    q, k, v, _ = _window_inputs([5] * n, H, G, D, "bf16")
    off = ref.offsets([5] * n)
    whole = comp.window_attention(q, k, v, _i32(off), heads=H, kv_heads=G, window=win,
                                  sinks=sinks)["y"]
    rows = [4, 9, 14]
    before = [t for t in range(15) if t not in rows]
    comp.window_attention_fill(k[before], v[before], _i32([0, 4, 8, 12]), kc, vc, win, sinks)
    y = comp.window_attention_step(q[rows], k[rows], v[rows], _i32([4, 4, 4]), kc, vc, heads=H,
                                   kv_heads=G, window=win, sinks=sinks)
    o = ref.window(_d(q), _d(k), _d(v), off, H, G, win, sinks, D ** -0.5)
    ref.within("y", y, o["y"][rows], ref.window_bound(o, "y", torch.bfloat16)[rows])
    ref.within("whole", whole, o["y"], ref.window_bound(o, "y", torch.bfloat16))


# ---------------------------------------------------------------------------
# all of them: streams, graphs, repeats, and a run of them together
# ---------------------------------------------------------------------------

def test_on_another_stream(comp):
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    args = _norm_inputs(50, 4, 2, 64, 32, "bf16")
    q, k, v, d, st, gy, gl = _linear_inputs([200, 30], 2, 64, 64, "bf16")
    wq, wk, wv, wg = _window_inputs([200, 30], 4, 2, 64, "bf16")
    torch.cuda.synchronize()
    _check_norms(comp, *args, 1e-6, False, stream=s)
    _check_linear(comp, q, k, v, d, [0, 200, 230], st, gy, gl, False, stream=s)
    _check_window(comp, wq, wk, wv, wg, [0, 200, 230], 4, 2, 50, 3, stream=s)
    y, state = comp.linear_attention_step(q[:2], k[:2], v[:2], d, st, stream=s)
    kc, vc = (torch.zeros(2 * 53, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    s.wait_stream(torch.cuda.current_stream())
    y2 = comp.window_attention_step(wq[:2], wk[:2], wv[:2], _i32([0, 0]), kc, vc, heads=4,
                                    kv_heads=2, window=50, sinks=3, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(y, comp.linear_attention_step(q[:2], k[:2], v[:2], d, st)[0])
    # alone in its sequence a frame gets its own value
    assert torch.equal(y2.view(2, 2, 2, 64)[:, :, 0], wv[:2].view(2, 2, 64))


class _Layer:
    """Norms with rotation, linear attention and window attention one after
    another, forward and back, as a network's layer uses them."""

    def __init__(self, comp, lens, H, G, D, win, sinks, typ):
        g = _gen(len(lens), H, G, D)
        self.comp, self.how = comp, dict(heads=H, kv_heads=G, window=win, sinks=sinks)
        self.N, self.H, self.G, self.D, self.typ = sum(lens), H, G, D, typ
        self.off = _i32(ref.offsets(lens))
        self.pos = torch.cat([torch.arange(n) for n in lens]).int().cuda()
        self.freq = (1000.0 ** (-torch.arange(D // 2) / (D // 2))).float().cuda()
        self.qw, self.kw = 1 + _vec(g, D, std=0.1), 1 + _vec(g, D, std=0.1)
        self.decay = -torch.logspace(-2, -0.5, G).cuda()
        self.qkv = _mat(g, self.N, (H + 2 * G) * D, typ)
        self.gy = _mat(g, self.N, H * D, typ)

    def parts(self, t):
        a, b = self.H * self.D, (self.H + self.G) * self.D
        return t[:, :a], t[:, a:b], t[:, b:]

    def run(self):
        c, o = self.comp, self.off
        q0, k0, v = self.parts(self.qkv)
        q, k = c.head_norms(q0, k0, self.qw, self.kw, self.freq, self.pos)
        lin = c.linear_attention(k, k, v, self.decay, o)
        w = c.window_attention(q, k, lin["y"], o, **self.how)
        gw = c.window_attention_grads(q, k, lin["y"], o, w["y"], w["lse"], self.gy, **self.how)
        gl = c.linear_attention_grads(k, k, v, self.decay, o, gw["v"])
        gk = gw["k"] + gl["q"] + gl["k"]
        gn = c.head_norms_grads(q0, k0, self.qw, self.kw, self.freq, self.pos, gw["q"], gk)
        return dict(y=w["y"], last=lin["last"], q=gn["q"], k=gn["k"], v=gl["v"],
                    qw=gn["q_weight"], kw=gn["k_weight"], q1=q, k1=k, v1=lin["y"])


def test_together_in_float32(comp):
    """The layer's results and gradients against the plain forms in 64 bits
    behind one another: each stage's bound, and what it makes of the bound of
    the one before, is under 2^-12 of the result's size here."""
    lens, H, G, D = [70, 0, 33], 4, 2, 16
    L = _Layer(comp, lens, H, G, D, 20, 2, "f32")
    got = L.run()
    off = ref.offsets(lens)
    q0, k0, v = [_d(t) for t in L.parts(L.qkv)]
    pos, freq, d, gy = L.pos.cpu(), L.freq.cpu(), _d(L.decay), _d(L.gy)
    q, _ = ref.head_norm(q0, _d(L.qw), freq, pos, 1e-6, False)
    k, _ = ref.head_norm(k0, _d(L.kw), freq, pos, 1e-6, False)
    s = D ** -0.5
    lv, last = ref.linear(k, k, v, d, off, None, False, s)
    o = ref.window(q, k, lv, off, H, G, 20, 2, s, gy)
    gq, gk, gv, _ = ref.linear_grads(k, k, v, d, off, None, False, s, o["gv"], None)
    (nq, _), (nqw, _) = ref.head_norm_grads(q0, _d(L.qw), freq, pos, 1e-6, False, o["gq"])
    (nk, _), (nkw, _) = ref.head_norm_grads(k0, _d(L.kw), freq, pos, 1e-6, False,
                                            o["gk"] + gq + gk)
    for c, w in dict(y=o["y"], last=last, q=nq, k=nk, v=gv, qw=nqw, kw=nkw).items():
        ref.within(c, got[c], w, 2.0 ** -12 * w.abs().max())


@pytest.mark.parametrize("D,typ", [(64, "bf16"), (128, "f16"), (128, "f32"), (40, "bf16")])
def test_together_the_same_again_and_as_a_graph(comp, D, typ):
    """Bit for bit: repeats, and replays of a graph between other calls."""
    L = _Layer(comp, [700, 0, 129, 1], 4, 2, D, 70, 3, typ)
    want = L.run()
    again = L.run()
    for c in want:
        assert torch.equal(want[c], again[c]), c
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        out = L.run()
    bigger = _Layer(comp, [1900, 400], 4, 2, D, 100, 3, typ)
    for _ in range(3):
        for t in out.values():
            t.fill_(5.0)
        graph.replay()
        torch.cuda.synchronize()
        for c in want:
            assert torch.equal(want[c], out[c]), c
        bigger.run()  # a larger workspace than the graph's
        torch.cuda.synchronize()


def test_steps_as_a_graph(comp):
    """A captured step of all three, replayed with new frames and positions."""
    H, G, D, win, sinks, n, T = 4, 2, 64, 9, 2, 3, 30
    g = _gen(77)
    frames = _mat(g, T * n, (H + 2 * G) * D, "f16").view(T, n, -1)
    qw, kw = 1 + _vec(g, D, std=0.1), 1 + _vec(g, D, std=0.1)
    freq = (1000.0 ** (-torch.arange(D // 2) / (D // 2))).float().cuda()
    decay = -torch.logspace(-2, -0.5, G).cuda()

    def step(x, pos, kc, vc, state):
        q, k, v = x[:, :H * D], x[:, H * D:(H + G) * D], x[:, (H + G) * D:]
        q, k = comp.head_norms(q, k, qw, kw, freq, pos)
        v, _ = comp.linear_attention_step(k, k, v, decay, state, out=state)
        return comp.window_attention_step(q, k, v, pos, kc, vc, heads=H, kv_heads=G, window=win,
                                          sinks=sinks)

    def fresh():
        return (torch.zeros(n * (win + sinks), G * D, dtype=torch.float16, device="cuda"),
                torch.zeros(n * (win + sinks), G * D, dtype=torch.float16, device="cuda"),
                torch.zeros(n, G, D, D, device="cuda"))

    a, want = fresh(), []
    for t in range(T):
        want.append(step(frames[t], _i32([t] * n), *a))
    b = fresh()
    x, pos = frames[0].clone(), _i32([0] * n)
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        y = step(x, pos, *b)
    for t in range(T):
        x.copy_(frames[t])
        pos.fill_(t)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[t]), t
    for p, r in zip(a, b):
        assert torch.equal(p, r)


def test_layer_streams_as_its_sequence(comp):
    """Frames one at a time through steps give the sequence's results: a float32
    layer within 2^-12 of the largest."""
    T, H, G, D, win, sinks = 60, 4, 2, 16, 20, 2
    L = _Layer(comp, [T], H, G, D, win, sinks, "f32")
    whole = L.run()
    kc, vc = (torch.zeros(win + sinks, G * D, device="cuda") for _ in range(2))
    state = torch.zeros(1, G, D, D, device="cuda")
    rows = []
    for t in range(T):
        q, k, v = L.parts(L.qkv[t:t + 1])
        q, k = comp.head_norms(q, k, L.qw, L.kw, L.freq, _i32([t]))
        v, state = comp.linear_attention_step(k, k, v, L.decay, state, out=state)
        rows.append(comp.window_attention_step(q, k, v, _i32([t]), kc, vc, heads=H, kv_heads=G,
                                               window=win, sinks=sinks))
    y = _d(whole["y"])
    ref.within("y", torch.cat(rows), y, 2.0 ** -12 * y.abs().max())


def test_arguments_that_the_binding_refuses(comp):
    q, k, v, d, st, gy, _ = _linear_inputs([6], 2, 8, 8, "f32")
    off = _i32([0, 6])
    with pytest.raises(ValueError):
        comp.linear_attention(q, k, v, d, off[:0])
    with pytest.raises(ValueError):
        comp.linear_attention(q, k, v, d.double(), off)
    with pytest.raises(ValueError):
        comp.linear_attention(q, k, v, d, off, state=st[:, :1])
    with pytest.raises(ValueError):
        comp.linear_attention(q[:, :15], k, v, d, off)
    with pytest.raises(ValueError):
        comp.window_attention(q, k, v, off, heads=3)
    with pytest.raises(ValueError):
        comp.window_attention(q, k, v, off, heads=2, window=1 << 31)
    with pytest.raises(ValueError):
        comp.window_attention(q.cpu(), k, v, off, heads=2)
    with pytest.raises(ValueError):
        comp.head_norms(q, k, torch.ones(8, device="cuda"), None)
    with pytest.raises(ValueError):
        comp.head_norms(q, k, torch.ones(8, device="cuda"), torch.ones(8, device="cuda"),
                        torch.ones(4, device="cuda"))
    from paper_2110_02848_amd import gpu
    with pytest.raises(gpu.FstError):
        comp.window_attention(q, k, v, off, heads=2, window=0)
    with pytest.raises(gpu.FstError):
        comp.linear_attention(q, k[:, :14], v, d, off)


# ---------------------------------------------------------------------------
# sizes, masks and magnitudes at their ends
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_window_of_heads_without_columns(comp, typ):
    """Every score is 0: lse is the logarithm of how many frames a query sees."""
    off, H, G, win, sinks = [0, 150, 150, 157], 4, 2, 70, 3
    q, k = (torch.empty(157, 0, dtype=TYPES[typ], device="cuda") for _ in range(2))
    how = dict(heads=H, kv_heads=G, window=win, sinks=sinks)
    print(f"[window] {tuple(q.shape)} strides {q.stride()} {typ}", flush=True)
    r = comp.window_attention(q, k, k, _i32(off), **how)
    torch.cuda.synchronize()
    count = torch.cat([ref.visible(b - a, win, sinks).sum(1) for a, b in zip(off, off[1:])])
    want = torch.log(count.to(F64))[:, None].expand(-1, H)
    # (a logarithm of at most 73 in powers of 2, 6.2, and its product with log 2)
    ref.within("lse", r["lse"], want, torch.full_like(want, 16 * ref.U))
    g = comp.window_attention_grads(q, k, k, _i32(off), r["y"], r["lse"], q, **how)
    assert r["y"].shape == (157, 0) and all(g[c].shape == (157, 0) for c in "qkv")


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("lens", [[10], [1000]])
@pytest.mark.parametrize("K,V", [(0, 5), (5, 0), (0, 0), (100, 0), (0, 100)])
def test_linear_of_heads_without_columns(comp, K, V, lens, typ):
    """Zeros, whether or not sequences are long enough to be cut into units."""
    q, k, v, d, st, gy, gl = _linear_inputs(lens, 2, K, V, typ)
    off = _i32(ref.offsets(lens))
    print(f"[linear] {tuple(q.shape)} {tuple(v.shape)} {typ} lengths {lens}", flush=True)
    r = comp.linear_attention(q, k, v, d, off, state=st)
    g = comp.linear_attention_grads(q, k, v, d, off, gy, state=st, grad_last=gl)
    torch.cuda.synchronize()
    for t, like in ((r["y"], v), (g["q"], q), (g["k"], k), (g["v"], v)):
        assert t.shape == like.shape and not t.any()
    assert r["last"].shape == g["state"].shape == (len(lens), 2, K, V)


def _near(out, c, rows):
    """window_bound of float16 with the spacing of scaled numbers at 0 taken from the
    row's own largest: dS is scaled to 2^11 or more, so that each of n terms, here at
    most 400, is off by at most 2^-25 / 2^11 of the largest dS of the row, and this
    times a number of the other operand, up to 5 where the row's largest has 1 or more
    in some column: 400 * 5 * 2^-36 < 2^-25 of the row's largest size."""
    r = out["r" + c]
    return (out["b" + c] + ref.H16[torch.float16] * r
            + 2.0 ** -25 * r.amax(1, keepdim=True).expand_as(r))[rows]


@pytest.mark.parametrize("where", ["other sequence", "no sequence", "later"])
@pytest.mark.parametrize("D", [64, 40, 128])
def test_window_float16_gradients_beside_large_rows(comp, where, D):
    """A large row takes no digits of the gradients of rows that do not see it."""
    off, H, G, win, sinks = [0, 200, 260], 2, 1, 90, 3
    q, k, v, gy = _window_inputs([200, 60, 20], H, G, D, "f16")
    gy = (gy.float() * 2.0 ** -10).half()
    how = dict(heads=H, kv_heads=G, window=win, sinks=sinks)
    o = ref.window(_d(q), _d(k), _d(v), off, H, G, win, sinks, D ** -0.5, _d(gy))
    at = {"other sequence": 230, "no sequence": 270, "later": 190}[where]
    queries = range(190 if where == "later" else 200)
    # (keys that row 190 sees: the first ones and its window)
    keys = range(sinks, 190 - win + 1) if where == "later" else range(200)
    print(f"[window] large row {at}, D={D}", flush=True)
    for big in ((gy,), (v,), (gy, v), (q, gy)):
        args = []
        for t in (q, k, v, gy):
            z = t.clone()
            if any(t is b for b in big):
                z[at] = 8000.0
            args.append(z)
        r = comp.window_attention(*args[:3], _i32(off), **how)
        g = comp.window_attention_grads(*args[:3], _i32(off), r["y"], r["lse"], args[3], **how)
        for c, rows in (("q", queries), ("k", keys), ("v", keys)):
            rows = list(rows)
            ref.within("g" + c, g[c][rows], o["g" + c][rows], _near(o, "g" + c, rows))


def test_window_float16_gradients_that_grow(comp):
    """dS that grow, and shrink, by thousands from tile to tile, each row within its
    own bound."""
    H, G, D, T, win, sinks = 2, 1, 64, 700, 150, 3
    q, k, v, gy = _window_inputs([T], H, G, D, "f16")
    t = torch.arange(T, device="cuda")
    for e in (10 * torch.sin(t / 40.0), (t - T // 2) / 30.0, (T // 2 - t) / 30.0):
        size = torch.exp2(e.round().clamp(-10, 10))[:, None]
        x = [(a.float() * b).half() for a, b in ((v, size), (gy, size.flip(0)))]
        how = dict(heads=H, kv_heads=G, window=win, sinks=sinks)
        r = comp.window_attention(q, k, x[0], _i32([0, T]), **how)
        g = comp.window_attention_grads(q, k, x[0], _i32([0, T]), r["y"], r["lse"], x[1], **how)
        o = ref.window(_d(q), _d(k), _d(x[0]), [0, T], H, G, win, sinks, D ** -0.5, _d(x[1]))
        rows = list(range(T))
        for c in "qk":
            ref.within("g" + c, g[c], o["g" + c], _near(o, "g" + c, rows))


@pytest.mark.parametrize("win,sinks", [(1000, 0), (40, 2)])
def test_window_float16_gradients_of_values_seen_faintly(comp, win, sinks):
    """A first frame that takes all but 2^-22 of every query's weight: what is left to
    the others has float16's digits all the same.  (P is scaled to 2^12, and each of at
    most 300 terms off by 2^-25 2^-12 of a dy, at most 5 * 2^11.)"""
    T, D = 300, 16
    q, k, v, gy = _window_inputs([T], 1, 1, D, "f16")
    q, k = (t.float() / 8 for t in (q, k))
    q[:, 0], k[:, 0] = 4.0, 0.0
    k[0, 0] = 15.25
    q, k, gy = q.half(), k.half(), (gy.float() * 2.0 ** 11).half()
    how = dict(heads=1, kv_heads=1, window=win, sinks=max(sinks, 1))
    r = comp.window_attention(q, k, v, _i32([0, T]), **how)
    g = comp.window_attention_grads(q, k, v, _i32([0, T]), r["y"], r["lse"], gy, **how)
    o = ref.window(_d(q), _d(k), _d(v), [0, T], 1, 1, win, max(sinks, 1), D ** -0.5, _d(gy))
    bound = (o["bgv"] + ref.H16[torch.float16] * o["rgv"]
             + 300 * 2.0 ** -37 * 5 * 2.0 ** 11)
    ref.within("gv", g["v"], o["gv"], bound)


@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("lens,at", [([150], 37), ([150], 149), ([70, 64], 20), ([1100], 700)])
@pytest.mark.parametrize("K,V", [(64, 64), (33, 20), (128, 128)])
def test_linear_float16_beside_large_rows(comp, K, V, lens, at, rev):
    """A large row takes no digits of rows that do not see it."""
    q, k, v, d, st, gy, gl = _linear_inputs(lens, 2, K, V, "f16")
    off, n = ref.offsets(lens), sum(lens)
    args = [_d(t) for t in (q, k, v)]
    size = [t.abs() for t in args]
    how = (_d(d), off), (rev, K ** -0.5)
    y, _ = ref.linear(*args, *how[0], _d(st), *how[1])
    ay, _ = ref.linear(*size, *how[0], _d(st).abs(), *how[1])
    want = ref.linear_grads(*args, *how[0], _d(st), *how[1], _d(gy), _d(gl))
    ag = ref.linear_grads(*size, *how[0], _d(st).abs(), *how[1], _d(gy).abs(), _d(gl).abs())
    (by, bq, bk, bv), _ = ref.linear_bounds(torch.float16, [ay, *ag[:3]], [], max(lens))
    print(f"[linear] large row {at} of {lens}, {K} x {V} rev={rev}", flush=True)
    for t, w in ((q, K), (k, K), (v, V), (gy, V)):
        t[at, :w] = 6e4
    r = comp.linear_attention(q, k, v, d, _i32(off), state=st, reverse=rev)
    g = comp.linear_attention_grads(q, k, v, d, _i32(off), gy, state=st, grad_last=gl,
                                    reverse=rev)
    s = max(i for i in range(len(lens)) if off[i] <= at)
    before, after = range(off[s], at), range(at + 1, off[s + 1])
    if rev:
        before, after = after, before
    others = [t for t in range(n) if not off[s] <= t < off[s + 1]]
    for c, got, w, b, rows, cols in (("y", r["y"], y, by, before, V),
                                     ("q", g["q"], want[0], bq, before, K),
                                     ("k", g["k"], want[1], bk, after, K),
                                     ("v", g["v"], want[2], bv, after, V)):
        rows = [*rows, *others]
        ref.within(c, got[rows], w[rows], b[rows])
        ref.within(c + ", other head", got[:, cols:], w[:, cols:], b[:, cols:])


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("bad", [NAN, INF, -INF])
def test_window_rows_that_see_only_themselves(comp, typ, bad):
    """dS = P (dy v^T - delta) is 0 there, and no number where one of its factors is
    none: the first rows of sequences, and all rows of a window of 1."""
    H, G, D = 2, 1, 16
    for lens, win in (([1, 40, 1, 1], 30), ([50, 3], 1)):
        off = ref.offsets(lens)
        q, k, v, gy = _window_inputs(lens, H, G, D, typ)
        how = dict(heads=H, kv_heads=G, window=win, sinks=0)
        alone = [t for t in range(off[-1]) if win == 1 or t + 1 in off and t in off]
        for i, at in ((i, at) for i in range(4) for at in alone[:1] + alone[-2:]):
            args = [t.clone() for t in (q, k, v, gy)]
            args[i][at, :D] = bad
            r = comp.window_attention(*args[:3], _i32(off), **how)
            g = comp.window_attention_grads(*args[:3], _i32(off), r["y"], r["lse"], args[3],
                                            **how)
            own = slice(0, 2 * D if i in (1, 2) else D)  # (k and v are both heads')
            print(f"[window] {typ} window={win} row {at} of input {i}", flush=True)
            assert g["q"][at, own].isnan().all() and g["k"][at].isnan().all()
            assert not i == 0 or not g["q"][at, D:].any()
            assert i == 2 or not g["v"][at].isfinite().any()
            rest = [t for t in alone if t != at]
            assert not g["q"][rest].any() and not g["k"][rest].any()
            assert g["q"].isfinite().sum() == g["q"].numel() - g["q"][at, own].numel()


def test_window_rows_that_see_only_themselves_and_no_score(comp):
    """A score of -infinity alone: its weight e^(z - lse) is no number."""
    q, k = (torch.full((2, 8), x, device="cuda") for x in (-INF, 1.0))
    q[1] = 1.0
    off = _i32([0, 1, 2])
    r = comp.window_attention(q, k, k, off, heads=1)
    g = comp.window_attention_grads(q, k, k, off, r["y"], r["lse"], k, heads=1)
    assert r["y"][0].isnan().all() and torch.equal(r["y"][1], k[1])
    assert all(g[c][0].isnan().all() for c in "qkv")
    assert not g["q"][1].any() and not g["k"][1].any() and torch.equal(g["v"][1], k[1])


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("H,G,D,win,sinks,lens", [
    (2, 1, 64, 900, 0, [1]), (2, 1, 64, 900, 0, [20, 900, 901]), (8, 2, 64, 2000, 4, [700, 2003]),
    (8, 2, 64, 2000, 4, [2004, 2005, 3000]), (20, 1, 32, 800, 64, [100, 864, 1900]),
    (4, 4, 128, 1600, 1, [1601, 1]), (6, 3, 43, 1500, 10, [1300, 2900]),
    (3, 1, 128, 30000, 0, [40]),
])
def test_window_steps_in_parts(comp, H, G, D, win, sinks, lens, typ):
    """Few streams with long rings: parts of a ring, and their join.  A new frame in the
    first part, a later one, and rings that leave later parts without frames."""
    rows = len(lens) * G * ((H // G + 15) // 16)
    assert min((512 + rows - 1) // rows, (win + sinks) // 384) > 1  # parts
    test_window_steps(comp, H, G, D, win, sinks, lens, typ)


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("T", [29000, 30500])
def test_window_step_of_a_long_ring(comp, T, typ):
    H, G, D, win, sinks = 2, 1, 64, 30000, 64
    q, k, v, _ = _window_inputs([T], H, G, D, typ)
    kc, vc = (torch.full((win + sinks, G * D), NAN, dtype=TYPES[typ], device="cuda")
              for _ in range(2))
    print(f"[step] ring {win + sinks}, frame {T} {typ}", flush=True)
    comp.window_attention_fill(k[:-1], v[:-1], _i32([0, T - 1]), kc, vc, win, sinks)
    y = comp.window_attention_step(q[-1:], k[-1:], v[-1:], _i32([T - 1]), kc, vc, heads=H,
                                   kv_heads=G, window=win, sinks=sinks)
    far = max(T - win, 0)  # the window's first frame
    sees = list(range(min(sinks, far))) + list(range(far, T))
    K, V, x = _d(k)[sees], _d(v)[sees], _d(q)[-1].view(H, D)
    z = D ** -0.5 * x @ K.t()
    w = torch.softmax(z, 1)
    size = D ** -0.5 * (x.abs() @ K.abs().t()).max(1, keepdim=True).values
    off = (2 * D + 24) * ref.U * (size + 1) + 16 * ref.U * (z.abs().max() + 1)
    r = w @ V.abs()
    # (as _step_reference has it, for every head)
    bound = (4 * off + (2 * len(sees) + 64) * ref.U + ref.H16[TYPES[typ]]) * r
    small = 2.0 ** -24 if typ == "f16" else 0.0
    ref.within("y", y[0], (w @ V).view(-1), (bound + small * r.max()).view(-1))


@pytest.mark.parametrize("typ", ["f32", "bf16"])
def test_window_steps_in_parts_as_a_graph(comp, typ):
    """Replays with new frames and positions, other calls of a larger workspace between
    them, against eager calls bit for bit."""
    H, G, D, win, sinks, n, T = 8, 2, 64, 1200, 4, 2, 6
    L = win + sinks
    g = _gen(5)
    frames = [[_mat(g, n, w * D, typ) for w in (H, G, G)] for _ in range(T)]
    begun = _mat(g, n * L, G * D, typ), _mat(g, n * L, G * D, typ)
    at = [[0, 1203], [400, 1204], [1202, 1205], [1203, 2407], [1204, 2408], [2500, -1]]
    how = dict(heads=H, kv_heads=G, window=win, sinks=sinks)
    a, b = ([t.clone() for t in begun] for _ in range(2))
    want = [comp.window_attention_step(*frames[t], _i32(at[t]), *a, **how) for t in range(T)]
    x, pos = [t.clone() for t in frames[0]], _i32(at[0])
    graph = torch.cuda.CUDAGraph()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=s):
        y = comp.window_attention_step(*x, pos, *b, **how)
    big = [_mat(g, 16, w * D, typ) for w in (H, G, G)]
    ring = [torch.zeros(16 * L, G * D, dtype=TYPES[typ], device="cuda") for _ in range(2)]
    for t in range(T):
        for p, f in zip(x, frames[t]):
            p.copy_(f)
        pos.copy_(_i32(at[t]))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[t]), t
        comp.window_attention_step(*big, _i32([1500] * 16), *ring, **how)
        torch.cuda.synchronize()
    assert all(torch.equal(p, r) for p, r in zip(a, b))


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_linear_sequences_are_their_steps(comp, typ):
    """The whole sequence's results and states within their bounds of the plain form,
    that of the steps within theirs of the same."""
    q, k, v, d, st, _, _ = _linear_inputs([150], 3, 40, 24, typ)
    r = comp.linear_attention(q, k, v, d, _i32([0, 150]), state=st)
    args = [_d(t) for t in (q, k, v)]
    how = _d(d), [0, 150]
    y, last = ref.linear(*args, *how, _d(st), False, 40 ** -0.5)
    ay, al = ref.linear(*[t.abs() for t in args], *how, _d(st).abs(), False, 40 ** -0.5)
    (by,), (bl,) = ref.linear_bounds(TYPES[typ], [ay], [al], 150)
    ref.within("y", r["y"], y, by)
    ref.within("last", r["last"], last, bl)
    state = st.clone()
    (by,), (bl,) = ref.linear_bounds(torch.float32, [ay], [al], 150 * 64)  # a chunk a step
    for t in range(150):
        x, state = comp.linear_attention_step(q[t:t + 1], k[t:t + 1], v[t:t + 1], d, state,
                                              out=state)
        ref.within(f"y {t}", x, y[t:t + 1], by[t:t + 1])
    ref.within("last", state, last, bl)


@pytest.mark.parametrize("win,sinks", [(1000, 0), (40, 1)])
@pytest.mark.parametrize("D", [16, 128])
def test_window_float16_values_seen_faintly(comp, D, win, sinks):
    """A first frame without a value that takes all but 2^-20 of every query's weight:
    what the others give has float16's digits all the same, in whole sequences and in
    a step.  (Weights are scaled to 2^12, and each of at most 300 off by 2^-25 2^-12 of a v,
    at most 5 * 2^10.)"""
    T = 300
    q, k, v, _ = _window_inputs([T], 1, 1, D, "f16")
    q, k = (t.float() / 8 for t in (q, k))
    q[:, 0], k[:, 0] = D ** 0.5, 0.0
    k[0, 0] = 13.875
    q, k, v = q.half(), k.half(), (v.float() * 2.0 ** 10).half()
    v[0] = 0.0
    how = dict(heads=1, kv_heads=1, window=win, sinks=sinks)
    r = comp.window_attention(q, k, v, _i32([0, T]), **how)
    o = ref.window(_d(q), _d(k), _d(v), [0, T], 1, 1, win, sinks, D ** -0.5)
    bound = (o["by"] + ref.H16[torch.float16] * o["ry"]
             + 300 * 2.0 ** -37 * 5 * 2.0 ** 10)
    ref.within("y", r["y"], o["y"], bound)
    ref.within("lse", r["lse"], o["lse"], o["blse"])
    L = win + sinks
    kc, vc = (torch.zeros(L, D, dtype=torch.float16, device="cuda") for _ in range(2))
    comp.window_attention_fill(k[:-1], v[:-1], _i32([0, T - 1]), kc, vc, win, sinks)
    y = comp.window_attention_step(q[-1:], k[-1:], v[-1:], _i32([T - 1]), kc, vc, **how)
    ref.within("step", y, o["y"][-1:], bound[-1:])


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("D,P,pairs", [(64, 32, False), (48, 16, True), (43, 13, False),
                                       (300, 20, True), (512, 256, False)])
def test_norms_of_numbers_whose_squares_leave_float32(comp, D, P, pairs, typ):
    """Results and gradients within the same bounds, beside rows of ordinary size."""
    for e, eps in ((70, 1e-6), (120, 1e-6), (60, 0.0), (-60, 1e-37), (-70, 0.0), (-110, 0.0)):
        args = list(_norm_inputs(6, 3, 2, D, P, typ))
        for i in (0, 1):
            args[i] = args[i].clone()
            args[i][1:] *= 2.0 ** e
        _check_norms(comp, *args, eps, pairs)


@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("T,V", [(64, 32), (150, 32), (1100, 100)])
def test_linear_float16_states_after_silence(comp, T, V, rev):
    """Rows without keys behind a few with them: what is left of those after a fast decay
    has float32's digits in the last state.  (A decayed k is two numbers of 11 bits, of
    the chunk's largest decayed k scaled to 2^11 or more: off by 2^-22 of itself and by
    2^-36 of the largest, a v at most 5 and one of 64 rows.)"""
    q, k, v, _, _, gy, gl = _linear_inputs([T], 2, 32, V, "f16")
    d = torch.tensor([-0.5, -0.9]).cuda()
    at = slice(T - 60, T - 50) if not rev else slice(50, 60)
    for t in (k, q):
        keep = t[at].clone()
        t.zero_()
        t[at] = keep
    print(f"[linear] silence, {T} x {V} rev={rev}", flush=True)
    last = comp.linear_attention(q, k, v, d, _i32([0, T]), reverse=rev)["last"]
    args = [_d(t) for t in (q, k, v)]
    _, want = ref.linear(*args, _d(d), [0, T], None, rev, 32 ** -0.5)
    _, size = ref.linear(*[t.abs() for t in args], _d(d), [0, T], None, rev, 32 ** -0.5)
    most = size.flatten(2).max(2).values[:, :, None, None]
    bound = (600 * ref.U + 2.0 ** -22) * size + 64 * 5 * 2.0 ** -36 * most
    ref.within("last", last, want, bound)


def test_linear_float16_with_a_large_state(comp):
    """Small keys beside a state of 2^100."""
    q, k, v, d, st, _, _ = _linear_inputs([100], 2, 32, 32, "f16")
    k = (k.float() * 2.0 ** -20).half()
    st = st * 2.0 ** 100
    last = comp.linear_attention(q, k, v, d, _i32([0, 100]), state=st)["last"]
    args = [_d(t) for t in (q, k, v)]
    _, want = ref.linear(*args, _d(d), [0, 100], _d(st), False, 32 ** -0.5)
    _, size = ref.linear(*[t.abs() for t in args], _d(d), [0, 100], _d(st).abs(), False,
                         32 ** -0.5)
    ref.within("last", last, want, 600 * ref.U * size)
