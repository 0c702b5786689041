"""Plain implementations, in 64 bits on the CPU, of the operators between a
network and its graphs, and the bounds that their tests hold results to."""
import torch

F64 = torch.float64
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# half the spacing of numbers above 1
HALF_ULP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
# the spacing at 0
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -133}


def recurrence(x, gate, offset, state, reverse):
    """(y, last) row by row, in the type of x."""
    n, D = len(offset) - 1, x.shape[1]
    y = torch.zeros_like(x)
    last = torch.zeros(n, D, dtype=x.dtype)
    for s in range(n):
        h = state[s] if state is not None else torch.zeros(D, dtype=x.dtype)
        rows = range(offset[s], offset[s + 1])
        for r in reversed(rows) if reverse else rows:
            f = torch.sigmoid(gate[r])
            h = f * h + torch.sigmoid(-gate[r]) * x[r]
            y[r] = h
        last[s] = h
    return y, last


def recurrence_grads(x, gate, offset, state, grad_y, grad_last, reverse):
    """(grad_x, grad_gate, grad_state) by the formulas."""
    n, D = len(offset) - 1, x.shape[1]
    zero = torch.zeros(D, dtype=x.dtype)
    gx, gu = torch.zeros_like(x), torch.zeros_like(x)
    gs = torch.zeros(n, D, dtype=x.dtype)
    for s in range(n):
        rows = list(range(offset[s], offset[s + 1]))
        if reverse:
            rows.reverse()
        h = state[s] if state is not None else zero
        before = []
        for r in rows:
            before.append(h)
            h = torch.sigmoid(gate[r]) * h + torch.sigmoid(-gate[r]) * x[r]
        into = grad_last[s] if grad_last is not None else zero
        for r, hp in zip(reversed(rows), reversed(before)):
            f, g = torch.sigmoid(gate[r]), torch.sigmoid(-gate[r])
            d = grad_y[r] + into
            gx[r] = g * d
            gu[r] = d * (hp - x[r]) * f * g
            into = f * d
        gs[s] = into
    return gx, gu, gs


def scores(x, w):
    return torch.mm(x, w.t().contiguous())


def close(name, got, want, rel, floor=None):
    """Elementwise |got - want| <= rel * scale + the rounding of got's type,
    where scale is what the error is relative to: |want| unless given."""
    got = got.detach().cpu()
    dt = got.dtype
    got = got.to(F64)
    assert got.shape == want.shape, (name, got.shape, want.shape)
    size = want.abs() if floor is None else floor
    bound = rel * size + 1.01 * HALF_ULP[dt] * want.abs() + TINY[dt]
    bad = ~((got - want).abs() <= bound)
    if bad.any():
        i = torch.nonzero(bad)[0].tolist()
        raise AssertionError(f"{name}: {int(bad.sum())} of {bad.numel()} off, first at {i}: "
                             f"{got[tuple(i)].item()} for {want[tuple(i)].item()}, "
                             f"bound {bound[tuple(i)].item()}")
