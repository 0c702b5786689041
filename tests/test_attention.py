"""The attention layers over frames without a GPU: the plain forms' gradients
against differences, and what the entry points refuse (a refusal comes before
anything that needs a device, so that a context of zeros is enough)."""
import ctypes
import os

import pytest
import torch

import attentionhelp as ref
from attentionhelp import F64


def _rand(g, *shape):
    return torch.randn(*shape, generator=g, dtype=F64)


def _differences(f, args, grads, g, eps=1e-5):
    """<grad, d> against the central difference along a random d, for each."""
    for i, grad in enumerate(grads):
        d = _rand(g, *args[i].shape)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + eps * d, args[i] - eps * d
        slope = (f(*up) - f(*down)) / (2 * eps)
        # (a third derivative times eps^2 / 6, and the difference's own rounding:
        # 1e-16 |f| / eps)
        assert abs(slope - (grad * d).sum()) <= 1e-6 * (1 + abs(slope)), i


@pytest.mark.parametrize("pairs", [False, True])
def test_norm_gradients_are_slopes(pairs):
    g = torch.Generator().manual_seed(1)
    x, w, c = _rand(g, 5, 3 * 7), 1 + 0.2 * _rand(g, 7), _rand(g, 5, 21)
    freq, pos = torch.tensor([1.0, 0.3, 0.01]), torch.tensor([0, 3, 70, 1000, 2])

    def loss(x, w):
        return (ref.head_norm(x, w, freq, pos, 1e-6, pairs)[0] * c).sum()

    (gx, _), (gw, _) = ref.head_norm_grads(x, w, freq, pos, 1e-6, pairs, c)
    _differences(loss, [x, w], [gx, gw], g)


@pytest.mark.parametrize("reverse", [False, True])
def test_linear_gradients_are_slopes(reverse):
    g = torch.Generator().manual_seed(2)
    off, H, K, V = [0, 4, 4, 11], 2, 3, 5
    q, k, v = _rand(g, 11, H * K), _rand(g, 11, H * K), _rand(g, 11, H * V)
    state, decay = _rand(g, 3, H, K, V), torch.tensor([-0.1, -1.0], dtype=F64)
    c, c2 = _rand(g, 11, H * V), _rand(g, 3, H, K, V)

    def loss(q, k, v, state):
        y, last = ref.linear(q, k, v, decay, off, state, reverse, 0.7)
        return (y * c).sum() + (last * c2).sum()

    grads = ref.linear_grads(q, k, v, decay, off, state, reverse, 0.7, c, c2)
    _differences(loss, [q, k, v, state], grads, g)


@pytest.mark.parametrize("win,sinks", [(100, 0), (3, 2), (1, 0), (2, 1)])
def test_window_gradients_are_slopes(win, sinks):
    g = torch.Generator().manual_seed(3)
    off, H, G, D = [0, 6, 6, 7, 16], 4, 2, 3
    q, k, v = _rand(g, 16, H * D), _rand(g, 16, G * D), _rand(g, 16, G * D)
    c = _rand(g, 16, H * D)

    def loss(q, k, v):
        return (ref.window(q, k, v, off, H, G, win, sinks, 0.6)["y"] * c).sum()

    o = ref.window(q, k, v, off, H, G, win, sinks, 0.6, c)
    _differences(loss, [q, k, v], [o["gq"], o["gk"], o["gv"]], g)


# ---- refusals ----

@pytest.fixture(scope="module")
def lib():
    from paper_2110_02848_amd import gpu
    if not os.path.exists(gpu.LIB_PATH):
        pytest.skip("library not built")
    if torch.cuda.is_available():
        pytest.skip("calls with addresses of nothing: only where no device can follow them")
    return gpu.load()


CTX = ctypes.create_string_buffer(1 << 16)
SOME = 1 << 20  # an address that no refused call follows
INVALID, LARGE = 1, 3


def _m(rows, cols, typ=2, data=SOME, stride=None):
    from paper_2110_02848_amd import gpu
    return gpu._Matrix(data, rows, cols, cols if stride is None else stride, typ)


def _fields(s, kw, more):
    for k, v in {**kw, **more}.items():
        setattr(s, k, v)
    return s


def _norms(**more):
    from paper_2110_02848_amd import gpu
    return _fields(gpu._HeadNorms(), dict(q=_m(4, 24), k=_m(4, 8), width=8, q_weight=SOME,
                                          k_weight=SOME, freq=SOME, num_freq=4, pos=SOME,
                                          pairs=0, eps=1e-6), more)


def _linear(**more):
    from paper_2110_02848_amd import gpu
    return _fields(gpu._LinearAttention(), dict(num_seqs=2, offset=SOME, reverse=0, heads=2,
                                                log_decay=SOME, scale=1.0, q=_m(4, 16),
                                                k=_m(4, 16), v=_m(4, 12), state=None), more)


def _window(**more):
    from paper_2110_02848_amd import gpu
    return _fields(gpu._WindowAttention(), dict(num_seqs=2, offset=SOME, heads=4, kv_heads=2,
                                                window=3, sinks=1, scale=1.0, q=_m(4, 32),
                                                k=_m(4, 16), v=_m(4, 16)), more)


NAN = float("nan")


@pytest.mark.parametrize("more,code", [
    (dict(width=0), INVALID), (dict(width=7), INVALID), (dict(width=-8), INVALID),
    (dict(num_freq=5), INVALID), (dict(num_freq=-1), INVALID), (dict(freq=None), INVALID),
    (dict(pos=None), INVALID), (dict(q_weight=None), INVALID), (dict(k_weight=None), INVALID),
    (dict(eps=-1e-6), INVALID), (dict(eps=NAN), INVALID), (dict(eps=ref.INF), INVALID),
    (dict(k=_m(5, 8)), INVALID), (dict(k=_m(4, 8, typ=1)), INVALID),
    (dict(q=_m(4, 24, stride=23)), INVALID), (dict(q=_m(4, 24, data=SOME + 1)), INVALID),
    (dict(q=_m(4, 1026), k=_m(4, 513), width=513, num_freq=0), LARGE),
])
def test_norms_refuse(lib, more, code):
    a = _norms(**more)
    q, k = (_m(m.rows, m.cols) for m in (a.q, a.k))
    r = ctypes.byref
    assert lib.fst_head_norms_run(CTX, r(a), r(q), r(k), None) == code
    assert lib.fst_head_norms_grads(CTX, r(a), r(q), r(k), r(q), r(k), None, None, None) == code


def test_norms_refuse_other_outputs(lib):
    a, q, k, r = _norms(), _m(4, 24), _m(4, 8), ctypes.byref
    for bad in (_m(3, 24), _m(4, 16), _m(4, 24, typ=0), _m(4, 24, data=None)):
        assert lib.fst_head_norms_run(CTX, r(a), r(bad), r(k), None) == INVALID
        for i in range(4):
            m = [q, k, q, k]
            m[i] = bad
            assert lib.fst_head_norms_grads(CTX, r(a), *map(r, m), None, None, None) == INVALID
    assert lib.fst_head_norms_run(None, r(a), r(q), r(k), None) == INVALID
    assert lib.fst_head_norms_run(CTX, None, r(q), r(k), None) == INVALID


@pytest.mark.parametrize("more,code", [
    (dict(heads=0), INVALID), (dict(heads=3), INVALID), (dict(heads=-2), INVALID),
    (dict(heads=8), INVALID), (dict(log_decay=None), INVALID), (dict(scale=NAN), INVALID),
    (dict(scale=ref.INF), INVALID), (dict(offset=None), INVALID), (dict(num_seqs=-1), INVALID),
    (dict(num_seqs=0), INVALID), (dict(num_seqs=(1 << 22) + 1), INVALID),
    (dict(k=_m(4, 14)), INVALID), (dict(k=_m(3, 16)), INVALID), (dict(v=_m(3, 12)), INVALID),
    (dict(v=_m(4, 12, typ=0)), INVALID), (dict(q=_m(4, 258), k=_m(4, 258)), LARGE),
    (dict(v=_m(4, 258)), LARGE),
])
def test_linear_refuses(lib, more, code):
    a = _linear(**more)
    y, q, r = _m(4, a.v.cols), _m(4, a.q.cols), ctypes.byref
    assert lib.fst_linear_attention_run(CTX, r(a), r(y), None, None) == code
    assert lib.fst_linear_attention_grads(CTX, r(a), r(y), None, r(q), r(q), r(y), None,
                                          None) == code
    if not {"offset", "num_seqs"} & set(more):
        assert lib.fst_linear_attention_step(CTX, r(a.q), r(a.k), r(a.v), a.heads, a.log_decay,
                                             a.scale, SOME, SOME, None, 4, r(y), None) == code


def test_linear_refuses_other_outputs(lib):
    a, y, q, r = _linear(), _m(4, 12), _m(4, 16), ctypes.byref
    for bad in (_m(3, 12), _m(4, 10), _m(4, 12, typ=1), _m(4, 12, data=None)):
        assert lib.fst_linear_attention_run(CTX, r(a), r(bad), None, None) == INVALID
        for m in ([bad, q, q, y], [y, bad, q, y], [y, q, bad, y], [y, q, q, bad]):
            assert lib.fst_linear_attention_grads(CTX, r(a), r(m[0]), None, r(m[1]), r(m[2]),
                                                  r(m[3]), None, None) == INVALID
    step = [CTX, r(a.q), r(a.k), r(a.v), 2, SOME, 1.0, SOME, SOME, None, 4, r(y), None]
    for i, bad in ((5, None), (7, None), (8, None), (10, 3), (10, -1), (1, None), (11, None)):
        call = list(step)
        call[i] = bad
        assert lib.fst_linear_attention_step(*call) == INVALID, i


@pytest.mark.parametrize("more,code", [
    (dict(window=0), INVALID), (dict(window=-1), INVALID), (dict(sinks=-1), INVALID),
    (dict(window=2 ** 31 - 1, sinks=1), INVALID), (dict(heads=3), INVALID),
    (dict(heads=0), INVALID), (dict(kv_heads=0), INVALID), (dict(kv_heads=3), INVALID),
    (dict(kv_heads=4), INVALID), (dict(kv_heads=-2), INVALID), (dict(scale=NAN), INVALID),
    (dict(k=_m(4, 32)), INVALID), (dict(v=_m(4, 8)), INVALID), (dict(v=_m(5, 16)), INVALID),
    (dict(k=_m(4, 16, typ=0)), INVALID), (dict(offset=None), INVALID),
    (dict(num_seqs=0), INVALID),
    (dict(q=_m(4, 516), k=_m(4, 258), v=_m(4, 258)), LARGE),
])
def test_window_refuses(lib, more, code):
    a = _window(**more)
    y, kk, r = _m(4, a.q.cols), _m(4, a.k.cols), ctypes.byref
    L = max(1, a.window) + max(0, a.sinks)
    cache = _m(4 * L if L < 1 << 28 else 4, a.k.cols)
    assert lib.fst_window_attention_run(CTX, r(a), r(y), SOME, None) == code
    vv = _m(4, a.v.cols)
    assert lib.fst_window_attention_grads(CTX, r(a), r(y), SOME, r(y), r(y), r(kk), r(vv),
                                          None) == code
    if not {"offset", "num_seqs"} & set(more):
        assert lib.fst_window_attention_step(CTX, r(a.q), r(a.k), r(a.v), a.heads, a.kv_heads,
                                             a.window, a.sinks, a.scale, SOME, None, 4,
                                             r(cache), r(cache), r(y), None) == code


def test_window_refuses_other_arrays(lib):
    a, y, k, r = _window(), _m(4, 32), _m(4, 16), ctypes.byref
    assert lib.fst_window_attention_run(CTX, r(a), r(y), None, None) == INVALID
    for bad in (_m(3, 32), _m(4, 16), _m(4, 32, typ=1), _m(4, 32, data=None)):
        assert lib.fst_window_attention_run(CTX, r(a), r(bad), SOME, None) == INVALID
        for i in range(3):
            m = [y, y, y]
            m[i] = bad
            assert lib.fst_window_attention_grads(CTX, r(a), r(m[0]), SOME, r(m[1]), r(m[2]),
                                                  r(k), r(k), None) == INVALID
    for bad in (_m(3, 16), _m(4, 32), _m(4, 16, typ=1), _m(4, 16, data=None)):
        assert lib.fst_window_attention_grads(CTX, r(a), r(y), SOME, r(y), r(y), r(bad), r(k),
                                              None) == INVALID
        assert lib.fst_window_attention_grads(CTX, r(a), r(y), SOME, r(y), r(y), r(k), r(bad),
                                              None) == INVALID
    assert lib.fst_window_attention_grads(CTX, r(a), r(y), None, r(y), r(y), r(k), r(k),
                                          None) == INVALID


def test_window_caches_are_checked(lib):
    """window 3 and sinks 1: four rows a stream."""
    q, k, y, r = _m(4, 32), _m(4, 16), _m(4, 32), ctypes.byref
    cache = _m(20, 16)

    def step(kc=cache, vc=cache, pos=SOME, slot=SOME, slots=5, window=3, sinks=1):
        return lib.fst_window_attention_step(CTX, r(q), r(k), r(k), 4, 2, window, sinks, 1.0, pos,
                                             slot, slots, r(kc), r(vc), r(y), None)

    def fill(kc=cache, vc=cache, slot=SOME, slots=5, seqs=2, off=SOME, window=3, sinks=1):
        return lib.fst_window_attention_fill(CTX, seqs, off, r(k), r(k), window, sinks, slot,
                                             slots, r(kc), r(vc), None)

    assert step() not in (INVALID, LARGE) and fill() not in (INVALID, LARGE)
    for f in (step, fill):
        for bad in (_m(19, 16), _m(21, 16), _m(20, 15), _m(20, 16, typ=0), _m(20, 16, data=None),
                    _m(20, 16, stride=8)):
            assert f(kc=bad) == INVALID and f(vc=bad) == INVALID
        assert f(slots=4) == INVALID and f(slots=-1) == INVALID
        assert f(window=0) == INVALID and f(sinks=-1) == INVALID and f(window=4) == INVALID
    small = _m(12, 16)
    assert step(kc=small, vc=small, slots=3, slot=None) == INVALID
    one = _m(4, 16)
    assert fill(kc=one, vc=one, slots=1, slot=None) == INVALID
    assert step(pos=None) == INVALID
    assert fill(off=None) == INVALID and fill(seqs=-1) == INVALID and fill(seqs=0) == INVALID


def test_window_step_refuses_rings_past_its_row_numbers(lib):
    """Rows of a ring are counted in 32 bits, a few tiles past its end among them."""
    q, k, y, r = _m(1, 32), _m(1, 16), _m(1, 32), ctypes.byref

    def step(window, sinks):
        cache = _m(window + sinks, 16)
        return lib.fst_window_attention_step(CTX, r(q), r(k), r(k), 4, 2, window, sinks, 1.0,
                                             SOME, None, 1, r(cache), r(cache), r(y), None)

    most = 2 ** 31 - 257
    assert step(2 ** 31 - 1, 0) == step(most, 1) == step(1, most) == LARGE
    assert step(most, 0) not in (INVALID, LARGE)


def test_norms_refuse_more_heads_than_are_counted(lib):
    """Heads of queries and keys are counted together, in 32 bits."""
    def calls(nq, nk):
        q, k, r = _m(1, nq), _m(1, nk), ctypes.byref
        a = _norms(q=q, k=k, width=1, num_freq=0)
        return {lib.fst_head_norms_run(CTX, r(a), r(q), r(k), None),
                lib.fst_head_norms_grads(CTX, r(a), r(q), r(k), r(q), r(k), None, None, None)}

    most = 2 ** 31 - 1
    assert calls(most, most) == calls(most, 0) == calls(most - 64, 1) == {LARGE}
    assert not calls(most - 64, 0) & {INVALID, LARGE}
