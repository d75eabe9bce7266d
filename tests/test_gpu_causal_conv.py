"""hts_causal_conv, its step and its gradient against the definition in 64 bits."""
import pytest
import torch

import paper_2012_09849_b200 as hts
import recurrent_ref as ref

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
# Of the magnitude |bias| + sum |w v|: W + 1 roundings of 2^-24, and for SiLU the exponent (up to 16 x 2^-24 at |pre| <= 16, and the
# exponential is steeper than SiLU nowhere), exponential and reciprocal (2^-22 each): below 2^-19.
SLACK = 2.0 ** -19


def case(T, N, D, W, type="fp32", seed=0, ragged=False, p=0.15, window=True, offset=0, pad=0, bias=True):
    """offset: elements in front of x's rows; pad: more behind them"""
    g = torch.Generator(device="cuda").manual_seed(seed + T * 131 + N * 17 + D)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    t = TYPES[type]
    c = dict(x=r(T, N, offset + D + pad).to(t)[..., offset:offset + D], w=r(D, W) / W ** 0.5, bias=0.1 * r(D) if bias else None,
             starts=(torch.rand(T, N, generator=g, device="cuda") < p).to(torch.uint8), window_in=r(N, W - 1, D).to(t) if window else None, lengths=None)
    if ragged:
        c["lengths"] = torch.randint(-1, T + 2, (N,), generator=g, device="cuda").to(torch.int32)
        c["lengths"][0] = 0
    return c


def outputs(c, sentinel=7.0):
    T, N, D = c["x"].shape
    y = torch.full((T, N, D), sentinel, dtype=c["x"].dtype, device="cuda")
    return y, torch.full((N, c["w"].shape[1] - 1, D), sentinel, dtype=c["x"].dtype, device="cuda")


def run(c, act, stream=None):
    y, out = outputs(c)
    ref.lend(stream, y, out)
    hts.hts_causal_conv(c["x"], c["w"], c["bias"], c["starts"], c["lengths"], c["window_in"], act, y, out, stream)
    return y, out


def live(c):
    T, N, _ = c["x"].shape
    n = torch.full((N,), T, device="cuda") if c["lengths"] is None else c["lengths"].clamp(0, T)
    return torch.arange(T, device="cuda")[:, None] < n[None]


def wide(c):
    return {k: ref.f64(v) if k in ("x", "w", "bias", "window_in") else v for k, v in c.items()}


def magnitude(c):
    m = {k: v.abs() if k in ("x", "w", "bias", "window_in") and v is not None else v for k, v in wide(c).items()}
    return ref.conv(**m, act="none")[0]


SHAPES = [(1, 1, 1, 4), (1, 3, 4, 2), (2, 2, 5, 4), (3, 1, 8, 4), (7, 5, 12, 3), (8, 3, 130, 4), (33, 4, 64, 4), (70, 2, 260, 2), (129, 1, 36, 4), (20, 300, 8, 3)]


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("shape", SHAPES)
def test_steps_and_window(shape, act, type):
    for ragged in (False, True):
        c = case(*shape, type=type, ragged=ragged, window=shape[0] % 2 == 1, bias=shape[2] != 12)
        y, out = run(c, act)
        ry, rout = ref.conv(**wide(c), act=act)
        on = live(c)
        ref.within(torch.where(on[..., None], y, torch.zeros_like(y)), ry, SLACK * magnitude(c))
        assert bool((y[~on] == 7).all())                       # rows behind a sequence's end are left as they were
        assert torch.equal(out.double(), rout)                 # copies of inputs


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("offset,pad", [(0, 0), (0, 4), (1, 0), (3, 2), (8, 8)])
def test_rows_of_wider_tensors(offset, pad, type):
    c = case(19, 3, 24, 4, type=type, offset=offset, pad=pad)
    y, _ = run(c, "silu")
    ref.within(y, ref.conv(**wide(c), act="silu")[0], SLACK * magnitude(c))
    dense = dict(c, x=c["x"].contiguous())
    assert torch.equal(y, run(dense, "silu")[0])


def test_nothing_is_seen_of_what_lies_before_a_start_or_behind_an_end():
    c = case(12, 2, 8, 4, p=0.0, ragged=False)
    c["starts"][5] = 1
    c["x"] = c["x"].clone()
    c["x"][4] = float("nan")
    c["x"][3] = float("inf")
    c["window_in"].fill_(float("nan"))
    c["starts"][0] = 1
    c["lengths"] = torch.tensor([9, 12], dtype=torch.int32, device="cuda")
    c["x"][9:, 0] = float("nan")
    y, out = run(c, "silu")
    assert bool(torch.isfinite(y[:3]).all()) and bool(torch.isfinite(y[5:]).all()) and bool(torch.isfinite(out).all())
    assert bool(torch.isnan(y[4]).all())


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("D,W", [(1, 2), (12, 3), (130, 4), (256, 4)])
def test_single_steps_have_the_same_bits(D, W, type):
    T, N, pool = 9, 5, 11
    c = case(T, N, D, W, type=type)
    y, out = run(c, "silu")
    slots = torch.randperm(pool, device="cuda")[:N].to(torch.int32)
    states = torch.full((pool, W - 1, D), 3.0, dtype=c["x"].dtype, device="cuda")
    states[slots.long()] = c["window_in"]
    for t in range(T):
        row = torch.empty(N, D, dtype=c["x"].dtype, device="cuda")
        hts.hts_causal_conv_step(c["x"][t], c["w"], c["bias"], c["starts"][t], slots, states, "silu", row, states)
        assert torch.equal(row, y[t])
    assert torch.equal(states[slots.long()], out)
    rest = torch.ones(pool, dtype=torch.bool, device="cuda")
    rest[slots.long()] = False
    assert bool((states[rest] == 3).all())


def test_rows_without_a_slot_are_skipped():
    c = case(1, 4, 20, 4)
    states = c["window_in"].clone()
    slots = torch.tensor([2, -1, 4, 0], dtype=torch.int32, device="cuda")          # two rows that only fill the batch up
    y = torch.full((4, 20), 7.0, device="cuda")
    hts.hts_causal_conv_step(c["x"][0], c["w"], c["bias"], None, slots, states, "none", y, states)
    assert bool((y[1] == 7).all()) and bool((y[2] == 7).all()) and bool((y[0] != 7).all())
    assert torch.equal(states[1], c["window_in"][1]) and torch.equal(states[3], c["window_in"][3])


def gradient(c, act, dy, dout, want=("dx", "dw", "dbias", "dwindow_in"), stream=None):
    T, N, D = c["x"].shape
    W = c["w"].shape[1]
    o = {"dx": torch.full((T, N, D), 7.0, dtype=c["x"].dtype, device="cuda"), "dw": torch.empty(D, W, device="cuda"), "dbias": torch.empty(D, device="cuda"),
         "dwindow_in": torch.empty(N, W - 1, D, device="cuda")}
    o = {k: v if k in want else None for k, v in o.items()}
    work = torch.empty(hts.hts_causal_conv_workspace(T, N, D, W), dtype=torch.uint8, device="cuda")
    ref.lend(stream, work, *o.values())
    hts.hts_causal_conv_gradient(c["x"], c["w"], c["bias"], c["starts"], c["lengths"], c["window_in"], act, dy, dout, o["dx"], o["dw"], o["dbias"], o["dwindow_in"], work,
                                 stream)
    return o


def reference_gradient(c, act, dy, dout):
    m = wide(c)
    if m["window_in"] is None:
        m["window_in"] = torch.zeros(c["x"].shape[1], c["w"].shape[1] - 1, c["x"].shape[2], dtype=torch.float64, device="cuda")
    if m["bias"] is None:
        m["bias"] = torch.zeros(c["x"].shape[2], dtype=torch.float64, device="cuda")
    leaves = {k: m[k].requires_grad_() for k in ("x", "w", "bias", "window_in")}
    outs = ref.conv(**m, act=act)
    g = ref.grads(list(outs), [dy.double(), torch.zeros_like(outs[1]) if dout is None else dout.double()], leaves)
    return {"dx": g["x"], "dw": g["w"], "dbias": g["bias"], "dwindow_in": g["window_in"]}


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("shape", SHAPES)
def test_gradient(shape, act, type):
    """dx and dwindow_in: sums of W terms of |w g|, |g| <= 1.1 |dy|; dw, dbias: sums of n = T N terms in a tree of depth below 64."""
    for ragged in (False, True):
        c = case(*shape, type=type, ragged=ragged, window=shape[0] % 2 == 0, bias=shape[2] != 12)
        T, N, D = c["x"].shape
        dy = torch.randn(T, N, D, device="cuda").to(c["x"].dtype)
        dout = torch.randn(N, shape[3] - 1, D, device="cuda") if shape[1] % 2 else None
        got, want = gradient(c, act, dy, dout), reference_gradient(c, act, dy, dout)
        on = live(c)
        most = float(dy.abs().max()) * 1.1
        slope = 1 + float(magnitude(c).max())                 # the slope of SiLU moves by at most half of what pre does
        room = SLACK * most * slope * c["w"].abs().sum(1).double() + (0 if dout is None else 2.0 ** -23 * dout.abs().max())
        ref.within(torch.where(on[..., None], got["dx"], torch.zeros_like(got["dx"])), want["dx"], room)
        assert bool((got["dx"][~on] == 7).all())
        ref.within(got["dwindow_in"], want["dwindow_in"], room)
        n = max(1, int(on.sum()))
        room = (SLACK * slope + 64 * 2.0 ** -24) * n * most
        ref.within(got["dw"], want["dw"], room * float(c["x"].abs().max().clamp(min=1)))
        ref.within(got["dbias"], want["dbias"], room)


def test_gradient_is_that_of_differences():
    c = case(11, 2, 3, 4)
    dy, dout = torch.randn(11, 2, 3, device="cuda"), torch.randn(2, 3, 3, device="cuda")
    got = gradient(c, "silu", dy, dout)
    m = wide(c)

    def value(**change):
        y, out = ref.conv(**{**m, **change}, act="silu")
        return float((y * dy.double()).sum() + (out * dout.double()).sum())
    h = 1e-5
    for key, out in (("x", "dx"), ("w", "dw"), ("bias", "dbias"), ("window_in", "dwindow_in")):
        e = torch.randn_like(m[key])
        slope = (value(**{key: m[key] + h * e}) - value(**{key: m[key] - h * e})) / (2 * h)
        assert abs(float((got[out].double() * e).sum()) - slope) <= 1e-4 * max(1.0, float((got[out].double() * e).abs().sum()))


def test_gradients_that_are_not_asked_for_and_repetition():
    c = case(40, 6, 32, 4, type="bf16", ragged=True)
    dy = torch.randn(40, 6, 32, device="cuda").bfloat16()
    full = gradient(c, "silu", dy, None)
    for want in (("dx",), ("dw",), ("dbias", "dwindow_in")):
        part = gradient(c, "silu", dy, None, want)
        for k in want:
            assert torch.equal(part[k], full[k]), k


def test_captured_calls_replay_and_other_streams():
    c = case(30, 4, 64, 4, type="bf16")
    dy = torch.randn(30, 4, 64, device="cuda").bfloat16()
    want_y, want_out = run(c, "silu")
    want = gradient(c, "silu", dy, None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    y, out = run(c, "silu", s)
    g = gradient(c, "silu", dy, None, stream=s.cuda_stream)
    s.synchronize()
    assert torch.equal(y, want_y) and torch.equal(out, want_out) and all(torch.equal(g[k], want[k]) for k in g)
    y, out = outputs(c)
    o = {k: torch.zeros_like(v) for k, v in want.items()}
    work = torch.empty(hts.hts_causal_conv_workspace(30, 4, 64, 4), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        hts.hts_causal_conv(c["x"], c["w"], c["bias"], c["starts"], None, c["window_in"], "silu", y, out)
        hts.hts_causal_conv_gradient(c["x"], c["w"], c["bias"], c["starts"], None, c["window_in"], "silu", dy, None, o["dx"], o["dw"], o["dbias"], o["dwindow_in"], work)
    for _ in range(2):
        for v in (y, out, *o.values()):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want_y) and torch.equal(out, want_out) and all(torch.equal(o[k], want[k]) for k in o)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("W", [2, 3, 4])
def test_weights_that_start_anywhere(W, type):
    c = case(40, 3, 24, W, type=type)
    dy = torch.randn_like(c["x"])
    want, want_g = run(c, "silu"), gradient(c, "silu", dy, None)
    for off in (1, 2):
        moved = dict(c)
        for k in ("w", "bias"):
            room = torch.zeros(c[k].numel() + off, device="cuda")
            moved[k] = room[off:].view(c[k].shape).copy_(c[k])
        got, got_g = run(moved, "silu"), gradient(moved, "silu", dy, None)
        assert all(torch.equal(u, v) for u, v in zip(got, want))
        assert torch.equal(got_g["dx"], want_g["dx"]) and all(ref.rel2(got_g[k], want_g[k].double()) <= 120 * 2.0 ** -24 for k in ("dw", "dbias"))      # 120 steps, in another order
        row, rows = torch.empty_like(c["x"][0]), torch.empty_like(want[1])
        other, others = torch.empty_like(row), torch.empty_like(rows)
        window = torch.zeros_like(want[1]) if c["window_in"] is None else c["window_in"]
        hts.hts_causal_conv_step(c["x"][0], c["w"], c["bias"], None, None, window, "silu", row, rows)
        hts.hts_causal_conv_step(c["x"][0], moved["w"], moved["bias"], None, None, window, "silu", other, others)
        assert torch.equal(row, other) and torch.equal(rows, others)
