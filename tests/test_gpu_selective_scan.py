"""hts_selective_scan, its step and its gradient against the definition in 64 bits."""
import pytest
import torch

import paper_2012_09849_b200 as hts
import recurrent_ref as ref

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
WIDE = ("x", "dt", "a", "b", "c", "d", "dt_bias", "z", "state_in")


def case(T, N, D, S, type="fp32", seed=0, ragged=False, p=0.1, softplus=True, gate=True, skip=True, state=True, offset=0):
    g = torch.Generator(device="cuda").manual_seed(seed + T * 131 + N * 17 + D * 7 + S)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    t = TYPES[type]
    size = torch.exp(-7 + 5 * torch.rand(D, generator=g, device="cuda"))
    bc = r(T, N, offset + 2 * S).to(t)[..., offset:]
    c = dict(x=r(T, N, D).to(t), dt=(0.5 * r(T, N, D)).to(t) if softplus else (size * torch.exp(0.5 * r(T, N, D))).to(t), a=-torch.exp(r(D, S)), b=bc[..., :S],
             c=bc[..., S:], d=r(D) if skip else None, dt_bias=torch.log(torch.expm1(size)) if softplus else None, z=r(T, N, offset + D).to(t)[..., offset:] if gate else None,
             starts=(torch.rand(T, N, generator=g, device="cuda") < p).to(torch.uint8), lengths=None, state_in=r(N, D, S) if state else None, softplus=softplus)
    if ragged:
        c["lengths"] = torch.randint(-1, T + 2, (N,), generator=g, device="cuda").to(torch.int32)
        c["lengths"][0] = 0
    return c


def run(c, stream=None):
    T, N, D = c["x"].shape
    S = c["a"].shape[1]
    y = torch.full((T, N, D), 7.0, dtype=c["x"].dtype, device="cuda")
    out = torch.full((N, D, S), 7.0, device="cuda")
    work = torch.empty(hts.hts_selective_scan_workspace(T, N, D, S), dtype=torch.uint8, device="cuda")
    ref.lend(stream, y, out, work)
    hts.hts_selective_scan(**c, y=y, state_out=out, workspace=work, stream=stream)
    return y, out


def live(c):
    T, N, _ = c["x"].shape
    n = torch.full((N,), T, device="cuda") if c["lengths"] is None else c["lengths"].clamp(0, T)
    return torch.arange(T, device="cuda")[:, None] < n[None]


def wide(c):
    return {k: ref.f64(v) if k in WIDE else v for k, v in c.items()}


def magnitudes(c):
    """What y and the states could at most be made of: the same sums with every term positive."""
    m = {k: v.abs() if k in ("x", "b", "c", "d", "state_in") and v is not None else v for k, v in wide(c).items()}
    z, m["z"] = m["z"], None
    y, h = ref.scan(**m)
    return (y if z is None else y * torch.nn.functional.silu(z).abs()), h


def slack(T):
    """A step adds to a state's error, relative to its magnitude: the decay's (exponent 2^-23 of v with v exp(-v) <= 0.37, ex2 2^-22, its
    correction 2^-25), delta's (2^-20: exponential, reciprocal, eight multiply-adds), two roundings.  Below 2^-19; T of them."""
    return (T + 4) * 2.0 ** -19


SHAPES = [(1, 1, 1, 1), (1, 3, 5, 16), (2, 2, 64, 4), (7, 3, 9, 3), (8, 1, 130, 16), (9, 2, 33, 13), (17, 3, 40, 8), (33, 2, 24, 17), (40, 3, 10, 32), (24, 2, 20, 33),
          (19, 1, 16, 64), (70, 2, 128, 16), (12, 130, 8, 5)]
LONG = [(500, 1, 64, 16), (257, 2, 24, 6), (300, 3, 40, 40)]              # cut into runs of steps


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("shape", SHAPES + LONG)
def test_outputs_and_states(shape, type):
    for ragged in (False, True):
        odd = sum(shape) % 2 == 1
        c = case(*shape, type=type, ragged=ragged, softplus=not odd, gate=shape[1] != 2, skip=shape[1] != 3, state=shape[3] != 16 or ragged, p=0.1 if shape[0] < 100 else 0.01)
        y, out = run(c)
        (ry, rh), (my, mh), on = ref.scan(**wide(c)), magnitudes(c), live(c)
        ref.within(torch.where(on[..., None], y, torch.zeros_like(y)), ry, slack(shape[0]) * my, "y")
        assert bool((y[~on] == 7).all())
        ref.within(out, rh, slack(shape[0]) * mh, "state")


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("offset", [1, 3, 8])
def test_rows_of_wider_tensors(offset, type):
    c = case(21, 3, 48, 16, type=type, offset=offset)
    dense = {k: v.contiguous() if isinstance(v, torch.Tensor) else v for k, v in c.items()}
    assert not c["z"].is_contiguous() and all(torch.equal(u, v) for u, v in zip(run(c), run(dense)))


def test_nothing_is_seen_of_what_lies_before_a_start_or_behind_an_end():
    c = case(300, 2, 40, 16, p=0.0)                             # in runs: the start lies in the middle of one
    for k in ("x", "dt", "z", "b", "c"):
        c[k] = c[k].clone()
    c["x"][100] = float("nan")
    c["dt"][101] = float("inf")
    c["starts"][102] = 1
    c["lengths"] = torch.tensor([250, 300], dtype=torch.int32, device="cuda")
    for k in ("x", "dt", "z", "b", "c"):
        c[k][250:, 0] = float("nan")
    y, out = run(c)
    assert bool(torch.isfinite(y[:100]).all()) and bool(torch.isfinite(y[102:]).all()) and bool(torch.isfinite(out).all())
    assert bool(torch.isnan(y[100]).all())
    clean = dict(c, x=torch.nan_to_num(c["x"]), dt=torch.nan_to_num(c["dt"], posinf=0.0))
    dy = torch.randn_like(y)
    dy[250:, 0] = float("nan")
    g, want = gradient(c, dy, None), gradient(clean, dy, None)
    for k in ("x", "dt", "b", "c", "z"):
        assert torch.equal(g[k][102:250], want[k][102:250]), k


@pytest.mark.parametrize("delta,decay", [(0.0, -3.0), (60.0, -50.0), (1e-6, -1.0), (0.5, 0.0), (0.1, 0.5), (300.0, -1.0)])
def test_decays_from_none_to_all(delta, decay):
    c = case(13, 2, 8, 16, softplus=False, p=0.0)
    c["dt"] = torch.full_like(c["dt"], delta)
    c["a"] = torch.full_like(c["a"], decay)
    y, out = run(c)
    (ry, rh), (my, mh) = ref.scan(**wide(c)), magnitudes(c)
    ref.within(y, ry, slack(13) * my)
    ref.within(out, rh, slack(13) * mh)


def test_large_and_small_inputs_of_softplus():
    c = case(4, 1, 8, 4, p=0.0)
    c["dt"] = torch.tensor([-100.0, -20.0, -5.0, -1.0, 0.0, 1.0, 20.0, 90.0], device="cuda").expand(4, 1, 8).contiguous()
    c["dt_bias"] = torch.zeros(8, device="cuda")
    y, out = run(c)
    (ry, rh), (my, mh) = ref.scan(**wide(c)), magnitudes(c)
    ref.within(y, ry, slack(4) * my)
    ref.within(out, rh, slack(4) * mh)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("D,S", [(1, 1), (40, 16), (17, 13), (24, 64), (520, 16)])
def test_single_steps_are_the_scan(D, S, type):
    T, N, pool = 8, 5, 9
    c = case(T, N, D, S, type=type)
    y, out = run(c)
    slots = torch.randperm(pool, device="cuda")[:N].to(torch.int32)
    states = torch.full((pool, D, S), 3.0, device="cuda")
    states[slots.long()] = c["state_in"]
    my, mh = magnitudes(c)
    for t in range(T):
        row = torch.empty(N, D, dtype=c["x"].dtype, device="cuda")
        hts.hts_selective_scan_step(c["x"][t], c["dt"][t], c["a"], c["b"][t], c["c"][t], c["d"], c["dt_bias"], c["z"][t], c["starts"][t], slots, states, True, row, states)
        ref.within(row, y[t].double(), 2 * slack(T) * my[t] + ref.HALF_STEP[row.dtype] * y[t].double().abs() * 2)
    ref.within(states[slots.long()], out.double(), 2 * slack(T) * mh)
    rest = torch.ones(pool, dtype=torch.bool, device="cuda")
    rest[slots.long()] = False
    assert bool((states[rest] == 3).all())


def test_steps_of_many_rows():
    c = case(1, 2600, 64, 16, type="bf16")
    y, out = run(c)
    row, states = torch.empty(2600, 64, dtype=torch.bfloat16, device="cuda"), torch.empty_like(out)
    hts.hts_selective_scan_step(c["x"][0], c["dt"][0], c["a"], c["b"][0], c["c"][0], c["d"], c["dt_bias"], c["z"][0], c["starts"][0], None, c["state_in"], True, row, states)
    my, mh = magnitudes(c)
    ref.within(row, y[0].double(), 2 * slack(1) * my[0] + 2.0 ** -7 * y[0].double().abs())
    ref.within(states, out.double(), 2 * slack(1) * mh)


def test_rows_without_a_slot_are_skipped():
    c = case(1, 4, 20, 16)
    states = c["state_in"].clone()
    slots = torch.tensor([2, -1, 4, 0], dtype=torch.int32, device="cuda")
    y = torch.full((4, 20), 7.0, device="cuda")
    hts.hts_selective_scan_step(c["x"][0], c["dt"][0], c["a"], c["b"][0], c["c"][0], None, None, None, None, slots, states, False, y, states)
    assert bool((y[1] == 7).all()) and bool((y[2] == 7).all()) and bool((y[0] != 7).all()) and bool((y[3] != 7).all())
    assert torch.equal(states[1], c["state_in"][1]) and torch.equal(states[3], c["state_in"][3])


# ---- gradient ----------------------------------------------------------------------------------------------------------
def grad_buffers(c):
    o = {k: torch.full(c[k].shape, 7.0, dtype=c[k].dtype, device="cuda") for k in ("x", "dt", "b", "c", "z", "a", "d", "dt_bias") if c[k] is not None}
    T, N, D = c["x"].shape
    o["state_in"] = torch.full((N, D, c["a"].shape[1]), 7.0, device="cuda")
    return o


def gradient(c, dy, dout, want=None, stream=None):
    T, N, D = c["x"].shape
    o = grad_buffers(c)
    if want:
        o = {k: o[k] for k in want}
    work = torch.empty(hts.hts_selective_scan_workspace(T, N, D, c["a"].shape[1], True), dtype=torch.uint8, device="cuda")
    ref.lend(stream, work, *o.values())
    hts.hts_selective_scan_gradient(**c, dy=dy, dstate_out=dout, grads=o, workspace=work, stream=stream)
    return o


def reference_gradient(c, dy, dout):
    m = wide(c)
    if m["state_in"] is None:
        m["state_in"] = torch.zeros(c["x"].shape[1], c["x"].shape[2], c["a"].shape[1], dtype=torch.float64, device="cuda")
    leaves = {k: m[k].clone().requires_grad_() for k in WIDE if m[k] is not None}
    outs = ref.scan(**{**m, **leaves})
    return ref.grads(list(outs), [dy.double(), torch.zeros_like(outs[1]) if dout is None else dout.double()], leaves)


@pytest.mark.parametrize("type", TYPES)
@pytest.mark.parametrize("shape", SHAPES + LONG)
def test_gradient(shape, type):
    """Norms: a gradient's terms have the relative errors of the states and of the gradients behind them, 2 T steps of 2^-19 at most; sums
    over channels, steps and sequences add 2^-24 a level.  Outputs in bf16 are rounded once more."""
    T, N, D, S = shape
    for ragged in (False, True):
        odd = sum(shape) % 2 == 1
        c = case(*shape, type=type, ragged=ragged, softplus=not odd, gate=N != 2, skip=N != 3, state=S != 16 or ragged, p=0.1 if T < 100 else 0.01)
        dy = torch.randn(T, N, D, device="cuda").to(c["x"].dtype)
        dout = torch.randn(N, D, S, device="cuda") if S % 2 else None
        got, want, on = gradient(c, dy, dout), reference_gradient(c, dy, dout), live(c)
        for k, v in got.items():
            if k in ("x", "dt", "b", "c", "z"):
                assert bool((v[~on] == 7).all()), k
                v = torch.where(on[..., None], v, torch.zeros_like(v))
            room = 2 * slack(T) + 64 * 2.0 ** -24 + (2.0 ** -8 if v.dtype == torch.bfloat16 else 0)
            if float(want[k].norm()) == 0:
                assert float(v.double().norm()) == 0, k
            else:
                assert ref.rel2(v, want[k]) <= room, (k, ref.rel2(v, want[k]), room)


def test_gradient_is_that_of_differences():
    c = case(10, 2, 3, 5)
    dy, dout = torch.randn(10, 2, 3, device="cuda"), torch.randn(2, 3, 5, device="cuda")
    got, m = gradient(c, dy, dout), wide(c)

    def value(**change):
        y, h = ref.scan(**{**m, **change})
        return float((y * dy.double()).sum() + (h * dout.double()).sum())
    for key in got:
        e = torch.randn_like(m[key])
        slope = (value(**{key: m[key] + 1e-5 * e}) - value(**{key: m[key] - 1e-5 * e})) / 2e-5
        assert abs(float((got[key].double() * e).sum()) - slope) <= 1e-4 * max(1.0, float((got[key].double() * e).abs().sum())), key


def test_gradients_that_are_not_asked_for_and_repetition():
    c = case(40, 3, 72, 16, type="bf16", ragged=True)
    dy = torch.randn(40, 3, 72, device="cuda").bfloat16()
    full = gradient(c, dy, None)
    for want in (("x",), ("b",), ("c", "a"), ("state_in",), ("dt_bias", "d"), ("z", "dt")):
        part = gradient(c, dy, None, want)
        for k in want:
            assert torch.equal(part[k], full[k]), k


@pytest.mark.parametrize("T,N", [(40, 3), (400, 1)])
def test_captured_calls_replay_and_other_streams(T, N):
    c = case(T, N, 64, 16, type="bf16")
    dy = torch.randn(T, N, 64, device="cuda").bfloat16()
    want, want_g = run(c), gradient(c, dy, None)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, got_g = run(c, s), gradient(c, dy, None, stream=s.cuda_stream)
    s.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(got, want)) and all(torch.equal(got_g[k], want_g[k]) for k in want_g)
    y, out, o = torch.zeros_like(want[0]), torch.zeros_like(want[1]), grad_buffers(c)
    work = [torch.empty(hts.hts_selective_scan_workspace(T, N, 64, 16, g), dtype=torch.uint8, device="cuda") for g in (False, True)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        hts.hts_selective_scan(**c, y=y, state_out=out, workspace=work[0])
        hts.hts_selective_scan_gradient(**c, dy=dy, dstate_out=None, grads=o, workspace=work[1])
    for _ in range(2):
        for v in (y, out, *o.values()):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(out, want[1]) and all(torch.equal(o[k], want_g[k]) for k in o)


def test_two_calls_at_once():
    cases = [case(300, 2, 64, 16, seed=s) for s in (1, 2)]
    want = [run(c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [run(c, s) for c, s in zip(cases, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for g, w in zip(got, want) for u, v in zip(g, w))


def test_advantages_are_a_scan():
    """hts_gae's recurrence, run backwards in time, is this one with one state: A_t = delta_t + gamma lambda (1 - d_t) A_{t+1}."""
    T, N, gamma, lam = 60, 7, 0.99, 0.95
    g = torch.Generator(device="cuda").manual_seed(3)
    r, v = (torch.randn(T, N, generator=g, device="cuda") for _ in range(2))
    done = (torch.rand(T, N, generator=g, device="cuda") < 0.1).to(torch.uint8)
    boot = torch.randn(N, generator=g, device="cuda")
    adv, ret = torch.empty(T, N, device="cuda"), torch.empty(T, N, device="cuda")
    hts.hts_gae(r, v, done, boot, gamma, lam, T, N, adv, ret)
    delta = r + gamma * (1 - done.float()) * torch.cat([v[1:], boot[None]]) - v
    flip = lambda u: u.flip(0)[..., None].contiguous()
    one = torch.ones(T, N, 1, device="cuda")
    # a start where the transition ended the episode: what lies behind it in time is not added
    y = torch.empty(T, N, 1, device="cuda")
    hts.hts_selective_scan(flip(delta), one, torch.full((1, 1), float(torch.log(torch.tensor(gamma * lam))), device="cuda"), one, one, None, None, None,
                           done.flip(0).contiguous(), None, None, False, y, None, torch.empty(hts.hts_selective_scan_workspace(T, N, 1, 1), dtype=torch.uint8, device="cuda"))
    assert float((y[..., 0].flip(0) - adv).abs().max()) <= slack(T) * float(adv.abs().max()) * 20      # 1 / (1 - gamma lambda) steps matter


def test_growth_of_nothing_is_nothing():
    """Decays above 1 whose product over a run of steps is beyond fp32, where there is nothing to multiply: before the first input, behind the last output."""
    T, D, S = 100, 8, 13
    c = case(T, 1, D, S, softplus=False, p=0.0, state=False)
    c["dt"] = torch.full_like(c["dt"], 8.0)
    c["a"] = torch.full_like(c["a"], 0.5)                       # e^4 a step
    c["x"] = c["x"].clone()
    c["x"][:-8] = 0
    y, out = run(c)
    (ry, rh), (my, mh) = ref.scan(**wide(c)), magnitudes(c)
    ref.within(y, ry, slack(T) * my)
    ref.within(out, rh, slack(T) * mh)
    dy = torch.randn_like(y)
    dy[8:] = 0
    got, want = gradient(c, dy, None), reference_gradient(c, dy, None)
    for k in got:                                               # an exponent of 4 log2(e) is rounded by less than 2^-21 a step
        if k != "state_in":
            assert bool(torch.isfinite(got[k]).all()) and ref.rel2(got[k], want[k]) <= 2 * slack(T), k


def test_steps_of_no_length_keep_the_state():
    c = case(40, 3, 24, 13, p=0.0, softplus=False)
    c["dt"] = torch.zeros_like(c["dt"])
    y, out = run(c)
    assert torch.equal(out, c["state_in"])
    for S in (13, 16):
        c = case(1, 3, 24, S, p=0.0, softplus=False)
        states = torch.empty_like(c["state_in"])
        hts.hts_selective_scan_step(c["x"][0], torch.zeros_like(c["dt"][0]), c["a"], c["b"][0], c["c"][0], None, None, None, None, None, c["state_in"], False, torch.empty_like(c["x"][0]),
                                    states)
        assert torch.equal(states, c["state_in"])


def test_many_single_steps_do_not_drift():
    """Decays near one over 2000 steps: what a decay is off by on average adds up over the steps that a state lives, 1 / (1 - decay) of them."""
    T, D, S = 2000, 16, 16
    c = case(T, 1, D, S, p=0.0, softplus=False, gate=False, skip=False)
    c["a"] = -(0.5 + torch.rand_like(c["a"]))
    c["dt"] = torch.full_like(c["dt"], 1e-3)
    c["x"], c["b"] = c["x"].abs() + 1, c["b"].abs() + 1         # nothing cancels
    state, y = c["state_in"].abs(), torch.empty(1, D, device="cuda")
    c["state_in"] = state.clone()
    for t in range(T):
        hts.hts_selective_scan_step(c["x"][t], c["dt"][t], c["a"], c["b"][t], c["c"][t], None, None, None, None, None, state, False, y, state)
    _, want = ref.scan(**wide(c))
    assert ref.rel2(state, want) <= 700 * 2.0 ** -24            # a life of 2000 steps at most, each off by 1e-8 on average and at random by a rounding
