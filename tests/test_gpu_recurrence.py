"""The gated recurrence on the GPU (forward, gradients, single steps) against
the plain loops in 64 bits, with bounds from a running error analysis: where
A_t = f A_(t-1) + (1 - f) |x| is the sum of the terms' sizes, each step adds
at most C u A_t to the error that f carries over (u = 2^-24; C = 16: the two
gates are within 6 u, a step rounds twice, a chunk's map twice more)."""
import pytest
import torch

import layershelp as ref

pytestmark = pytest.mark.gpu

U, C = 2.0 ** -24, 16


@pytest.fixture(scope="module")
def comp():
    assert torch.cuda.is_available(), "GPU tests need a GPU"
    from paper_2110_02848_amd import gpu
    c = gpu.Composer(0)
    yield c
    c.close()


def _offsets(lens):
    off = [0]
    for k in lens:
        off.append(off[-1] + k)
    return off


def _inputs(seed, lens, D, typ, pad=0):
    """x, gate and grad_y as views of rows `pad` elements longer, that start
    `pad` elements in."""
    g = torch.Generator().manual_seed(seed)
    N, n = sum(lens), len(lens)

    def mat():
        t = torch.randn(N, D + 2 * pad, generator=g).to(ref.TYPES[typ])
        return t.cuda()[:, pad:pad + D]
    x, gate, gy = mat(), mat(), mat()
    gate.mul_(2).add_(1)
    state = torch.randn(n, D, generator=g).cuda()
    glast = torch.randn(n, D, generator=g).cuda()
    return x, gate, gy, state, glast


def _errors(x, gate, off, state, rev):
    """(A, E) of the states entering and leaving each row."""
    A, E = torch.zeros_like(x), torch.zeros_like(x)
    Ain, Ein = torch.zeros_like(x), torch.zeros_like(x)
    la, le = torch.zeros(len(off) - 1, x.shape[1]).to(x), torch.zeros(len(off) - 1, x.shape[1]).to(x)
    for s in range(len(off) - 1):
        a = state[s].abs() if state is not None else torch.zeros(x.shape[1]).to(x)
        e = torch.zeros_like(a)
        rows = range(off[s], off[s + 1])
        for r in reversed(rows) if rev else rows:
            Ain[r], Ein[r] = a, e
            f, g = torch.sigmoid(gate[r]), torch.sigmoid(-gate[r])
            a = f * a + g * x[r].abs()
            e = f * e + C * U * a
            A[r], E[r] = a, e
        la[s], le[s] = a, e
    return A, E, Ain, Ein, la, le


def _back_errors(gate, off, gy, glast, rev):
    A, E = torch.zeros_like(gate), torch.zeros_like(gate)
    ia = torch.zeros(len(off) - 1, gate.shape[1]).to(gate)
    ie = torch.zeros_like(ia)
    for s in range(len(off) - 1):
        a = glast[s].abs() if glast is not None else torch.zeros(gate.shape[1]).to(gate)
        e = torch.zeros_like(a)
        rows = list(range(off[s], off[s + 1]))
        for r in rows if rev else reversed(rows):
            f = torch.sigmoid(gate[r])
            a = gy[r].abs() + a
            e = e + C * U * a
            A[r], E[r] = a, e
            a, e = f * a, f * e
        ia[s], ie[s] = a, e + C * U * a
    return A, E, ia, ie


def _check(comp, x, gate, gy, off, state, glast, rev, stream=None):
    print(f"[recurrence] {tuple(x.shape)} {x.dtype} strides {x.stride()} n={len(off) - 1} "
          f"rev={rev}", flush=True)
    offset = torch.tensor(off, dtype=torch.int32, device="cuda")
    r = comp.recurrence(x, gate, offset, state=state, reverse=rev, save=True, stream=stream)
    g = comp.recurrence_grads(x, gate, offset, gy, r["saved"], state=state, grad_last=glast,
                              reverse=rev, stream=stream)
    torch.cuda.synchronize()
    X, G, GY = [t.cpu().double() for t in (x, gate, gy)]
    S = None if state is None else state.cpu().double()
    GL = None if glast is None else glast.cpu().double()
    y, last = ref.recurrence(X, G, off, S, rev)
    A, E, Ain, Ein, la, le = _errors(X, G, off, S, rev)
    ref.close("y", r["y"], y, 1.0, E)
    ref.close("last", r["last"], last, 1.0, le)
    gx, gu, gs = ref.recurrence_grads(X, G, off, S, GY, GL, rev)
    DA, DE, ia, ie = _back_errors(G, off, GY, GL, rev)
    f, h = torch.sigmoid(G), torch.sigmoid(-G)
    ref.close("grad_x", g["x"], gx, 1.0, h * (DE + C * U * DA))
    size = Ain + X.abs()
    ref.close("grad_gate", g["gate"], gu, 1.0,
              f * h * (DE * size + DA * (Ein + C * U * size)))
    ref.close("grad_state", g["state"], gs, 1.0, ie)
    return r, g


@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("lens,D", [
    ([1], 1), ([1, 1, 1], 2), ([0], 5), ([3, 0, 2], 64), ([15, 16, 17], 63), ([63, 64, 65], 65),
    ([127, 128, 129], 128), ([300], 130), ([257, 0, 1, 5], 257), ([511, 2], 40),
])
def test_lengths_and_widths(comp, lens, D, typ, rev):
    x, gate, gy, state, glast = _inputs(len(lens) * 1000 + D, lens, D, typ)
    _check(comp, x, gate, gy, _offsets(lens), state, glast, rev)


@pytest.mark.parametrize("typ", ["f32", "bf16"])
@pytest.mark.parametrize("lens,D", [([5000], 96), ([2100, 1], 33), ([1040] * 3, 128)])
def test_long_sequences(comp, lens, D, typ):
    x, gate, gy, state, glast = _inputs(7, lens, D, typ)
    _check(comp, x, gate, gy, _offsets(lens), state, glast, False)


@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_without_states(comp, typ, rev):
    lens = [70, 0, 9]
    x, gate, gy, _, _ = _inputs(3, lens, 34, typ)
    r, _ = _check(comp, x, gate, gy, _offsets(lens), None, None, rev)
    assert not r["last"][1].any()


@pytest.mark.parametrize("pad", [1, 2, 3, 4])
@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_strided_and_unaligned_rows(comp, typ, pad):
    lens = [33, 70]
    x, gate, gy, state, glast = _inputs(pad, lens, 66, typ, pad=pad)
    _check(comp, x, gate, gy, _offsets(lens), state, glast, False)


def test_no_rows_and_no_sequences(comp):
    e = torch.empty(0, 8, device="cuda")
    r = comp.recurrence(e, e, torch.zeros(1, dtype=torch.int32, device="cuda"))
    assert r["y"].shape == (0, 8) and r["last"].shape == (0, 8)
    state = torch.randn(3, 8, device="cuda")
    z = torch.zeros(4, dtype=torch.int32, device="cuda")
    r = comp.recurrence(e, e, z, state=state, save=True)
    assert torch.equal(r["last"], state)
    g = comp.recurrence_grads(e, e, z, e, r["saved"], state=state, grad_last=state * 2)
    assert torch.equal(g["state"], state * 2)


def test_gates_at_their_ends(comp):
    """Gates that keep everything, add everything, or are infinite: the state
    is held, or replaced by x, exactly."""
    big = torch.tensor([float("inf"), 200.0, -200.0, float("-inf")], device="cuda")
    x = torch.randn(40, 4, device="cuda")
    gate = big.expand(40, 4).contiguous()
    state = torch.randn(1, 4, device="cuda")
    off = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    r = comp.recurrence(x, gate, off, state=state, save=True)
    assert torch.equal(r["y"][:, :2], state[:, :2].expand(40, 2))
    assert torch.equal(r["y"][:, 2:], x[:, 2:])
    g = comp.recurrence_grads(x, gate, off, torch.ones_like(x), r["saved"], state=state)
    assert torch.isfinite(g["x"]).all() and torch.isfinite(g["gate"]).all()
    assert torch.equal(g["state"], torch.tensor([[40.0, 40.0, 0.0, 0.0]], device="cuda"))


def test_one_bad_channel_stays_alone(comp):
    x = torch.randn(150, 70, device="cuda")
    gate = torch.randn(150, 70, device="cuda")
    off = torch.tensor([0, 100, 150], dtype=torch.int32, device="cuda")
    good = comp.recurrence(x, gate, off)["y"].clone()
    x2 = x.clone()
    x2[20, 7] = float("nan")
    y = comp.recurrence(x2, gate, off)["y"]
    assert torch.isnan(y[20:100, 7]).all()
    hit = torch.zeros(150, 70, dtype=torch.bool, device="cuda")
    hit[20:100, 7] = True
    assert torch.equal(y[~hit], good[~hit])


def test_offsets_that_are_wrong_stay_inside(comp):
    """Offsets past the rows, negative or falling: whatever comes out, rows
    beside the matrices keep their values."""
    room = torch.full((64, 32), 7.0, device="cuda")
    x = torch.randn(48, 32, device="cuda")
    y = room[8:56]
    from paper_2110_02848_amd import gpu
    off = torch.tensor([-5, 30, 10, 1 << 30], dtype=torch.int32, device="cuda")
    R, n = comp._recurrence(x, x, off, None, False)
    rc = comp._lib.fst_recurrence_run(comp._h, R, gpu._matrix(y, "y"), None, None,
                                      gpu._stream_handle(None))
    assert rc == 0
    torch.cuda.synchronize()
    assert (room[:8] == 7).all() and (room[56:] == 7).all()


def test_gradients_against_differences(comp):
    """Along random directions, in float32: the loss sum(gy y) + sum(gl last)
    by plain loops in 64 bits at steps of 1e-4 (curvature: 1e-8 of it)."""
    lens, D = [20, 0, 75], 10
    x, gate, gy, state, glast = _inputs(11, lens, D, "f32")
    off = _offsets(lens)
    offset = torch.tensor(off, dtype=torch.int32, device="cuda")
    for rev in (False, True):
        r = comp.recurrence(x, gate, offset, state=state, reverse=rev, save=True)
        g = comp.recurrence_grads(x, gate, offset, gy, r["saved"], state=state, grad_last=glast,
                                  reverse=rev)
        at = [t.cpu().double() for t in (x, gate, state)]
        GY, GL = gy.cpu().double(), glast.cpu().double()

        def loss(v):
            y, last = ref.recurrence(v[0], v[1], off, v[2], rev)
            return float((GY * y).sum() + (GL * last).sum())

        gen = torch.Generator().manual_seed(5)
        for k, grad in enumerate((g["x"], g["gate"], g["state"])):
            d = torch.randn(at[k].shape, generator=gen, dtype=torch.float64)
            h = 1e-4
            up, dn = [list(at) for _ in range(2)]
            up[k], dn[k] = at[k] + h * d, at[k] - h * d
            want = (loss(up) - loss(dn)) / (2 * h)
            got = float((grad.cpu().double() * d).sum())
            size = float((grad.cpu().double() * d).abs().sum())
            assert abs(got - want) <= 1e-5 * size, (rev, k, got, want)


# ---- single steps ----

@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,D,pad", [(1, 1, 0), (3, 7, 0), (8, 256, 0), (65, 130, 3), (2, 64, 4)])
def test_step(comp, n, D, pad, typ):
    x, gate, _, _, _ = _inputs(n * D, [n], D, typ, pad=pad)
    state = torch.randn(n, D, device="cuda")
    before = state.clone()
    y, new = comp.recurrence_step(x, gate, state)
    assert torch.equal(state, before)
    f = torch.sigmoid(gate.cpu().double())
    g = torch.sigmoid(-gate.cpu().double())
    want = f * state.cpu().double() + g * x.cpu().double()
    size = f * state.cpu().double().abs() + g * x.cpu().double().abs()
    ref.close("state", new, want, C * U, size)
    ref.close("y", y, want, C * U, size)
    # in place
    y2, same = comp.recurrence_step(x, gate, state, out=state)
    assert same is state and torch.equal(state, new) and torch.equal(y, y2)


def test_steps_follow_the_scan(comp):
    x, gate, _, state, _ = _inputs(1, [12], 96, "bf16")
    off = torch.tensor([0, 12], dtype=torch.int32, device="cuda")
    r = comp.recurrence(x, gate, off, state=state)
    h = state
    for t in range(12):
        y, h = comp.recurrence_step(x[t:t + 1], gate[t:t + 1], h)
    # 12 steps' error of both sides, on sums of terms of at most this size
    size = float(max(x.float().abs().max(), state.abs().max()))
    assert float((h - r["last"]).abs().max()) <= 2 * 12 * C * U * size


def test_step_slots(comp):
    D = 40
    pool = torch.randn(9, D, device="cuda")
    before = pool.clone()
    x, gate, _, _, _ = _inputs(2, [5], D, "f16")
    slot = torch.tensor([7, -1, 0, 9, 3], dtype=torch.int32, device="cuda")
    y, out = comp.recurrence_step(x, gate, pool, slot=slot)
    assert out is pool
    live = [0, 2, 4]
    rows = [7, 0, 3]
    y1, new = comp.recurrence_step(x[live], gate[live], before[rows].contiguous())
    assert torch.equal(y[live], y1) and torch.equal(pool[rows], new)
    idle = [i for i in range(9) if i not in rows]
    assert torch.equal(pool[idle], before[idle])
    assert not y[[1, 3]].any()


# ---- streams, graphs, refusals ----

def test_other_stream(comp):
    lens = [200, 40]
    x, gate, gy, state, glast = _inputs(9, lens, 64, "bf16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    _check(comp, x, gate, gy, _offsets(lens), state, glast, False, stream=s)


def test_graph_replays(comp):
    lens = [150, 3]
    x, gate, gy, state, glast = _inputs(21, lens, 64, "bf16")
    off = torch.tensor(_offsets(lens), dtype=torch.int32, device="cuda")

    def step():
        r = comp.recurrence(x, gate, off, state=state, save=True)
        g = comp.recurrence_grads(x, gate, off, gy, r["saved"], state=state, grad_last=glast)
        return [r["y"], r["last"], g["x"], g["gate"], g["state"]]
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for k in range(3):
        x.copy_(torch.randn_like(x))
        want = [t.clone() for t in step()]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), k


def test_refusals(comp):
    from paper_2110_02848_amd import gpu
    x = torch.randn(6, 8, device="cuda")
    off = torch.tensor([0, 6], dtype=torch.int32, device="cuda")

    def refused(f):
        with pytest.raises(gpu.FstError) as e:
            f()
        assert e.value.code == gpu.FST_ERR_INVALID_ARG
    refused(lambda: comp.recurrence(x, x[:, :4], off))
    refused(lambda: comp.recurrence(x, x[:5], off))
    refused(lambda: comp.recurrence(x, x.half(), off))
    refused(lambda: comp.recurrence(x, x, off[:1]))  # rows of no sequence
    saved = torch.empty(1, 8, device="cuda")
    refused(lambda: comp.recurrence_grads(x, x, off, x[:5], saved))
    refused(lambda: comp.recurrence_step(x, x, x[:5].contiguous()))
    refused(lambda: comp.recurrence_step(x, x[:, :3], x))
    for bad in (x.double(), x.t(), x[0], x.cpu()):
        with pytest.raises(ValueError):
            comp.recurrence(bad, x, off)
    with pytest.raises(ValueError):
        comp.recurrence(x, x, off.long())
    with pytest.raises(ValueError):
        comp.recurrence(x, x, off, state=x)
    lib, M = comp._lib, gpu._matrix
    R, _ = comp._recurrence(x, x, off, None, False)
    s = gpu._stream_handle(None)
    assert lib.fst_recurrence_run(None, R, M(x, "y"), None, None, s) == gpu.FST_ERR_INVALID_ARG
    assert lib.fst_recurrence_run(comp._h, None, M(x, "y"), None, None, s) == \
        gpu.FST_ERR_INVALID_ARG
    assert lib.fst_recurrence_grads(comp._h, R, None, M(x, "g"), None, M(x, "a"), M(x, "b"), None,
                                    s) == gpu.FST_ERR_INVALID_ARG
    for field, value in (("rows", -1), ("stride", 7), ("type", 3), ("data", None),
                         ("data", x.data_ptr() + 2), ("cols", 1 << 40)):
        m = M(x, "x")
        setattr(m, field, value)
        assert lib.fst_recurrence_run(comp._h, R, m, None, None, s) == gpu.FST_ERR_INVALID_ARG
    R2 = gpu._Recurrence(gpu.FST_RECURRENCE_MAX_SEQS + 1, R.offset, 0, R.x, R.gate, None)
    assert lib.fst_recurrence_run(comp._h, R2, M(x, "y"), None, None, s) == \
        gpu.FST_ERR_INVALID_ARG


def _no_numbers(*tensors):
    return [torch.isnan(t.float()).cpu() for t in tensors]


@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("where", ["x", "gate", "state"])
@pytest.mark.parametrize("lens,D", [([70, 0, 133], 66), ([700], 64), ([9] * 255 + [100], 128)])
@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_what_is_no_number_goes_on(comp, typ, lens, D, where, rev):
    """A NaN in x, gate or state comes out wherever the formulas carry it, and
    nowhere else: whole sequences, one cut into units, two channels a lane."""
    x, gate, gy, state, glast = _inputs(13, lens, D, typ)
    off = _offsets(lens)
    offset = torch.tensor(off, dtype=torch.int32, device="cuda")

    def run():
        r = comp.recurrence(x, gate, offset, state=state, reverse=rev, save=True)
        g = comp.recurrence_grads(x, gate, offset, gy, r["saved"], state=state, grad_last=glast,
                                  reverse=rev)
        return [r["y"], r["last"], g["x"], g["gate"], g["state"]]
    good = run()
    t, r = dict(x=x, gate=gate, state=state)[where], 0 if where == "state" else 41
    t[r, 7] = t[r, 62] = float("nan")
    got = run()
    X, G, GY, S, GL = [v.cpu().double() for v in (x, gate, gy, state, glast)]
    want = _no_numbers(*ref.recurrence(X, G, off, S, rev),
                       *ref.recurrence_grads(X, G, off, S, GY, GL, rev))
    for a, b, m in zip(got, good, want):
        assert m.any() or where != "gate"
        assert torch.equal(_no_numbers(a)[0], m)
        assert torch.equal(a.cpu()[~m], b.cpu()[~m])


@pytest.mark.parametrize("D", [8, 7])
@pytest.mark.parametrize("where", ["x", "gate", "state"])
@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_step_of_what_is_no_number(comp, typ, where, D):
    x, gate, _, _, _ = _inputs(4, [5], D, typ)
    state = torch.randn(5, D, device="cuda")
    y0, s0 = comp.recurrence_step(x, gate, state)
    dict(x=x, gate=gate, state=state)[where][2, 3] = float("nan")
    y, s = comp.recurrence_step(x, gate, state)
    m = torch.zeros(5, D, dtype=torch.bool)
    m[2, 3] = True
    for a, b in ((y, y0), (s, s0)):
        assert torch.equal(_no_numbers(a)[0], m)
        assert torch.equal(a.cpu()[~m], b.cpu()[~m])


@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_gates_at_their_ends_in_16_bits(comp, typ):
    dt = ref.TYPES[typ]
    big = torch.tensor([float("inf"), 200.0, -200.0, float("-inf")], device="cuda").to(dt)
    x = torch.randn(40, 4, device="cuda").to(dt)
    gate = big.expand(40, 4).contiguous()
    state = torch.randn(1, 4, device="cuda")
    off = torch.tensor([0, 40], dtype=torch.int32, device="cuda")
    r = comp.recurrence(x, gate, off, state=state, save=True)
    assert torch.equal(r["last"][:, :2], state[:, :2])
    assert torch.equal(r["y"][:, :2], state[:, :2].to(dt).expand(40, 2))
    assert torch.equal(r["y"][:, 2:], x[:, 2:]) and torch.equal(r["last"][0, 2:], x[-1, 2:].float())
    g = comp.recurrence_grads(x, gate, off, torch.ones_like(x), r["saved"], state=state)
    assert torch.isfinite(g["x"]).all() and torch.isfinite(g["gate"]).all()
    assert torch.equal(g["state"][:, :2], torch.full((1, 2), 40.0, device="cuda"))
    # (what keeps nothing keeps 2^-126 at most)
    assert (g["state"][:, 2:].abs() <= 2.0 ** -126).all()
    y, new = comp.recurrence_step(x[:1], gate[:1], state)
    assert torch.equal(new[:, :2], state[:, :2]) and torch.equal(new[:, 2:], x[:1, 2:].float())
    assert torch.equal(y, new.to(dt))


@pytest.mark.parametrize("other", [False, True])
def test_step_with_states_to_spare(comp, other):
    """More states than rows: those that no row names keep their values in the
    new tensor, and `out` keeps its own."""
    D = 40
    x, gate, _, _, _ = _inputs(2, [5], D, "f16")
    pool = torch.randn(9, D, device="cuda")
    s = torch.cuda.Stream() if other else None
    torch.cuda.synchronize()
    y1, want = comp.recurrence_step(x, gate, pool[:5].contiguous())
    torch.full((9, D), 7.0, device="cuda")  # (what a new tensor may hold)
    torch.cuda.synchronize()
    before = pool.clone()
    y, new = comp.recurrence_step(x, gate, pool, stream=s)
    torch.cuda.synchronize()
    assert torch.equal(y, y1) and torch.equal(new[:5], want) and torch.equal(new[5:], pool[5:])
    assert new.shape == pool.shape and torch.equal(pool, before)
    none, same = comp.recurrence_step(x[:0], gate[:0], pool, stream=s)
    torch.cuda.synchronize()
    assert none.shape == (0, D) and torch.equal(same, pool)
    for slot in (None, torch.tensor([8, 0, -1, 9, 3], dtype=torch.int32, device="cuda")):
        out = torch.full((9, D), 7.0, device="cuda")
        torch.cuda.synchronize()
        _, got = comp.recurrence_step(x, gate, pool, slot=slot, out=out, stream=s)
        torch.cuda.synchronize()
        rows = [0, 1, 2, 3, 4] if slot is None else [8, 0, 3]
        assert got is out and torch.equal(pool, before)
        assert (out[[i for i in range(9) if i not in rows]] == 7).all()
        assert not (out[rows] == 7).any()


def test_widest_rows(comp):
    """As many columns as a launch takes, and one more."""
    from paper_2110_02848_amd import gpu
    D = 65535 * 64
    x, gate = torch.randn(2, D, device="cuda"), torch.randn(2, D, device="cuda")
    off = torch.tensor([0, 2], dtype=torch.int32, device="cuda")
    r = comp.recurrence(x, gate, off, save=True)
    f = torch.sigmoid(gate.double())
    want = f[1] * (1 - f[0]) * x[0].double() + (1 - f[1]) * x[1].double()
    assert float((r["last"][0].double() - want).abs().max()) <= 4 * C * U * float(x.abs().max())
    g = comp.recurrence_grads(x, gate, off, x, r["saved"])
    assert torch.isfinite(g["gate"]).all()
    x, gate = torch.zeros(2, D + 1, device="cuda"), torch.zeros(2, D + 1, device="cuda")
    saved = torch.zeros(1, D + 1, device="cuda")
    for call in (lambda: comp.recurrence(x, gate, off),
                 lambda: comp.recurrence_grads(x, gate, off, x, saved)):
        with pytest.raises(gpu.FstError) as e:
            call()
        assert e.value.code == gpu.FST_ERR_TOO_LARGE


@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("lens,D", [([130, 0, 65, 64] + [i % 13 for i in range(252)], 128),
                                    ([70] + [1 + i % 9 for i in range(130)], 258)])
@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_two_channels_a_lane(comp, typ, lens, D, rev):
    """Batches of many sequences in 16 bits: each one workgroup's for every 128
    channels."""
    x, gate, gy, state, glast = _inputs(D, lens, D, typ)
    _check(comp, x, gate, gy, _offsets(lens), state, glast, rev)


@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("typ", ["f32", "f16", "bf16"])
def test_long_units(comp, typ, rev):
    """10,100 steps of 1024 channels in units of 128 (two channels a lane) or
    256: several chunks of steps for each wavefront of a unit, an empty sequence
    between, ends inside a unit and inside a chunk."""
    lens = [6001, 0, 4099]
    x, gate, gy, state, glast = _inputs(17, lens, 1024, typ)
    _check(comp, x, gate, gy, _offsets(lens), state, glast, rev)


@pytest.mark.parametrize("rev", [False, True])
@pytest.mark.parametrize("typ", ["f16", "bf16"])
def test_units_of_one_channel(comp, typ, rev):
    """Rows that begin anywhere, long, in 16 bits: one channel a lane."""
    lens = [900, 0, 1500]
    x, gate, gy, state, glast = _inputs(19, lens, 67, typ, pad=1)
    _check(comp, x, gate, gy, _offsets(lens), state, glast, rev)
