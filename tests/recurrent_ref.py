"""The recurrent core's definitions in 64 bits, one step after the other; gradients by differentiating them."""
import torch

ACT = {"none": lambda v: v * 1, "relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}
HALF_STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}      # a rounding, relative to the value


def f64(v):
    return None if v is None else v.double()


def _live(lengths, t, N, device):
    return torch.ones(N, dtype=torch.bool, device=device) if lengths is None else t < lengths.clamp(min=0)


def conv(x, w, bias, starts, lengths, window_in, act):
    """-> y [T, N, D] (zero behind a sequence's end), window_out"""
    T, N, D = x.shape
    W = w.shape[1]
    win = [torch.zeros(N, D, dtype=x.dtype, device=x.device)] * (W - 1) if window_in is None else list(window_in.unbind(1))
    ys = []
    for t in range(T):
        on = _live(lengths, t, N, x.device)[:, None]
        fresh = on & (starts[t] != 0)[:, None] if starts is not None else on & False
        seen = [torch.where(fresh, torch.zeros_like(v), v) for v in win] + [x[t]]
        pre = sum(w[:, k] * seen[k] for k in range(W))
        y = ACT[act](pre if bias is None else pre + bias)
        ys.append(torch.where(on, y, torch.zeros_like(y)))
        win = [torch.where(on, v, u) for v, u in zip(seen[1:], win)]
    return torch.stack(ys), torch.stack(win, 1)


def scan(x, dt, a, b, c, d, dt_bias, z, starts, lengths, state_in, softplus):
    """-> y [T, N, D] (zero behind a sequence's end), state_out"""
    T, N, D = x.shape
    h = torch.zeros(N, D, a.shape[1], dtype=x.dtype, device=x.device) if state_in is None else state_in
    raw = dt if dt_bias is None else dt + dt_bias
    delta = torch.nn.functional.softplus(raw, threshold=700.0) if softplus else raw
    ys = []
    for t in range(T):
        on = _live(lengths, t, N, x.device)
        old = h
        if starts is not None:
            old = torch.where((starts[t] != 0)[:, None, None], torch.zeros_like(h), h)
        new = old * torch.exp(delta[t][:, :, None] * a) + (delta[t] * x[t])[:, :, None] * b[t][:, None, :]
        y = (new * c[t][:, None, :]).sum(-1)
        if d is not None:
            y = y + d * x[t]
        if z is not None:
            y = y * torch.nn.functional.silu(z[t])
        ys.append(torch.where(on[:, None], y, torch.zeros_like(y)))
        h = torch.where(on[:, None, None], new, h)
    return torch.stack(ys), h


def grads(outputs, seeds, inputs):
    """{name: gradient} of the sum over outputs x seeds; inputs: {name: leaf or None}"""
    names = [k for k, v in inputs.items() if v is not None]
    got = torch.autograd.grad(outputs, [inputs[k] for k in names], seeds, allow_unused=True)
    return {k: torch.zeros_like(inputs[k]) if g is None else g for k, g in zip(names, got)}


def rel2(got, ref):
    """2-norm of the difference over 2-norm of the reference"""
    return float((got.double() - ref).norm() / ref.norm().clamp(min=1e-30))


def within(got, ref, slack, what=""):
    """Every element is within a rounding of its type, and `slack` (a tensor or number) more."""
    err = (got.double() - ref).abs()
    room = HALF_STEP[got.dtype] * ref.abs() + slack
    worst = (err - room).max()
    assert bool(torch.isfinite(got.float()).all()) and float(worst) <= 0, f"{what}: beyond its bound by {float(worst):.3g}, largest error {float(err.max()):.3g}"


def lend(stream, *tensors):
    """Tensors of the current stream for a call on another: what fills them comes first, and their memory goes to nobody else before the call is done."""
    if stream is not None:
        s = torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream
        s.wait_stream(torch.cuda.current_stream())
        for t in tensors:
            if t is not None:
                t.record_stream(s)
