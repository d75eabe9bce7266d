"""The recurrent core as a policy uses it: linear, causal convolution, linear, selective scan with its gate, linear with the residual.

The learner's pass over the storage, the actor's single steps over a pool of states, and the gradients of the whole chain."""
import pytest
import torch

import paper_2012_09849_b200 as hts
import recurrent_ref as ref

pytestmark = pytest.mark.gpu
WIDTH, INNER, STATE, TAPS = 64, 128, 16, 4


def weights(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")
    m = lambda n, k: (r(n, k) / k ** 0.5).bfloat16()
    return dict(w_in=m(2 * INNER, WIDTH), b_in=0.1 * r(2 * INNER), taps=r(INNER, TAPS) / 2, b_taps=0.1 * r(INNER), w_x=m(INNER + 2 * STATE, INNER),
                dt_bias=-3 + r(INNER), a=-torch.exp(r(INNER, STATE)), d=torch.ones(INNER, device="cuda"), w_out=m(WIDTH, INNER), b_out=0.1 * r(WIDTH))


def bf(*shape):
    return torch.empty(*shape, dtype=torch.bfloat16, device="cuda")


def linear(x, w, bias, residual=None):
    y = bf(x.shape[0], w.shape[0])
    hts.hts_linear(x, w, bias, residual, "none", y, None, torch.empty(hts.hts_linear_workspace(x.shape[0], x.shape[1], w.shape[0]), dtype=torch.uint8, device="cuda"))
    return y


def split(p, lead):
    p = p.view(*lead, -1)
    return p[..., :INNER], p[..., INNER:INNER + STATE], p[..., INNER + STATE:]


def forward(w, x, starts, window, state):
    """-> y, what the gradient needs, window and state behind the last step"""
    T, N, _ = x.shape
    flat = x.reshape(T * N, WIDTH)
    both = linear(flat, w["w_in"], w["b_in"]).view(T, N, 2 * INNER)
    u, window_out = bf(T, N, INNER), torch.empty_like(window)
    hts.hts_causal_conv(both[..., :INNER], w["taps"], w["b_taps"], starts, None, window, "silu", u, window_out)
    dt, b, c = split(linear(u.view(T * N, INNER), w["w_x"], None), (T, N))
    s, state_out = bf(T, N, INNER), torch.empty_like(state)
    hts.hts_selective_scan(u, dt, w["a"], b, c, w["d"], w["dt_bias"], both[..., INNER:], starts, None, state, True, s, state_out,
                           torch.empty(hts.hts_selective_scan_workspace(T, N, INNER, STATE), dtype=torch.uint8, device="cuda"))
    y = linear(s.view(T * N, INNER), w["w_out"], w["b_out"], flat).view(T, N, WIDTH)
    return y, (flat, both, u, dt, b, c, s), window_out, state_out


def reference(w, x, starts, window, state):
    both = x @ w["w_in"].t() + w["b_in"]
    u, _ = ref.conv(both[..., :INNER], w["taps"], w["b_taps"], starts, None, window, "silu")
    p = u @ w["w_x"].t()
    s, _ = ref.scan(u, p[..., :INNER], w["a"], p[..., INNER:INNER + STATE], p[..., INNER + STATE:], w["d"], w["dt_bias"], both[..., INNER:], starts, None, state, True)
    return s @ w["w_out"].t() + w["b_out"] + x


def inputs(T, N, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(T, N, WIDTH, generator=g, device="cuda").bfloat16(), (torch.rand(T, N, generator=g, device="cuda") < 0.1).to(torch.uint8),
            torch.randn(N, TAPS - 1, INNER, generator=g, device="cuda").bfloat16(), torch.randn(N, INNER, STATE, generator=g, device="cuda"))


@pytest.mark.parametrize("T,N", [(1, 1), (5, 16), (40, 3), (300, 1)])
def test_storage(T, N):
    """Five tensors on the way are rounded to bf16, each 2^-8 at most, and none of the layers enlarges a relative error twofold."""
    w, x = weights(), inputs(T, N)
    y, _, _, _ = forward(w, *x)
    want = reference({k: v.double() for k, v in w.items()}, x[0].double(), x[1], x[2].double(), x[3].double())
    assert ref.rel2(y, want) <= 2 * 5 * 2.0 ** -8


def test_single_steps_over_a_pool_are_the_pass_over_the_storage():
    T, N, pool = 20, 6, 10
    w, (x, starts, window, state) = weights(), inputs(T, N)
    y, _, window_out, state_out = forward(w, x, starts, window, state)
    slots = torch.randperm(pool, device="cuda")[:N].to(torch.int32)
    windows, states = torch.zeros(pool, TAPS - 1, INNER, dtype=torch.bfloat16, device="cuda"), torch.zeros(pool, INNER, STATE, device="cuda")
    windows[slots.long()], states[slots.long()] = window, state
    for t in range(T):
        both = linear(x[t], w["w_in"], w["b_in"])
        u, s = bf(N, INNER), bf(N, INNER)
        hts.hts_causal_conv_step(both[:, :INNER], w["taps"], w["b_taps"], starts[t], slots, windows, "silu", u, windows)
        dt, b, c = split(linear(u, w["w_x"], None), (N,))
        hts.hts_selective_scan_step(u, dt, w["a"], b, c, w["d"], w["dt_bias"], both[:, INNER:], starts[t], slots, states, True, s, states)
        row = linear(s, w["w_out"], w["b_out"], x[t])
        assert ref.rel2(row, y[t].double()) <= 2 * 5 * 2.0 ** -8
    assert ref.rel2(windows[slots.long()], window_out.double()) <= 2.0 ** -7 and ref.rel2(states[slots.long()], state_out.double()) <= 4 * 2.0 ** -8


def backward(w, x, starts, window, state, saved, dy):
    flat, both, u, dt, b, c, s = saved
    T, N, _ = x.shape
    R = T * N
    work = lambda k, n: torch.empty(hts.hts_linear_workspace(R, k, n, True), dtype=torch.uint8, device="cuda")
    g = {k: torch.empty(v.shape, device="cuda") for k, v in w.items()}
    d_s, d_u, d_p, d_both, d_x = bf(R, INNER), bf(T, N, INNER), bf(T, N, INNER + 2 * STATE), bf(T, N, 2 * INNER), bf(R, WIDTH)
    dyf = dy.view(R, WIDTH)
    hts.hts_linear_gradient(s.view(R, INNER), w["w_out"], None, dyf, "none", d_s, g["w_out"], g["b_out"], work(INNER, WIDTH))
    out = {"x": d_u, "dt": d_p[..., :INNER], "b": d_p[..., INNER:INNER + STATE], "c": d_p[..., INNER + STATE:], "z": d_both[..., INNER:], "a": g["a"], "d": g["d"],
           "dt_bias": g["dt_bias"]}
    hts.hts_selective_scan_gradient(u, dt, w["a"], b, c, w["d"], w["dt_bias"], both[..., INNER:], starts, None, state, True, d_s.view(T, N, INNER), None, out,
                                    torch.empty(hts.hts_selective_scan_workspace(T, N, INNER, STATE, True), dtype=torch.uint8, device="cuda"))
    more = bf(R, INNER)
    hts.hts_linear_gradient(u.view(R, INNER), w["w_x"], None, d_p.view(R, -1), "none", more, g["w_x"], None, work(INNER, INNER + 2 * STATE))
    d_u += more.view_as(d_u)
    hts.hts_causal_conv_gradient(both[..., :INNER], w["taps"], w["b_taps"], starts, None, window, "silu", d_u, None, d_both[..., :INNER], g["taps"], g["b_taps"], None,
                                 torch.empty(hts.hts_causal_conv_workspace(T, N, INNER, TAPS), dtype=torch.uint8, device="cuda"))
    hts.hts_linear_gradient(flat, w["w_in"], None, d_both.view(R, -1), "none", d_x, g["w_in"], g["b_in"], work(WIDTH, 2 * INNER))
    return g, d_x.view_as(dy) + dy


@pytest.mark.parametrize("T,N", [(5, 16), (40, 3)])
def test_gradients_of_the_chain(T, N):
    """Against differentiating the chain in 64 bits: nine tensors on the way there and back are rounded to bf16, and a product's
    factors carry two of those errors."""
    w, x = weights(), inputs(T, N)
    y, saved, _, _ = forward(w, *x)
    dy = torch.randn_like(y)
    got, dx = backward(w, *x, saved, dy)
    leaves = {k: v.double().requires_grad_() for k, v in w.items()}
    xin = x[0].double().requires_grad_()
    want = ref.grads([reference(leaves, xin, x[1], x[2].double(), x[3].double())], [dy.double()], {**leaves, "x": xin})
    for k in got:
        assert ref.rel2(got[k], want[k]) <= 2 * 9 * 2.0 ** -8, (k, ref.rel2(got[k], want[k]))
    assert ref.rel2(dx, want["x"]) <= 2 * 9 * 2.0 ** -8


def test_weights_learn_through_the_delayed_update():
    """The gradients are in the form that hts_delayed_update takes: one step of it changes the weights by lr times the gradient."""
    w, x = weights(), inputs(5, 16)
    y, saved, _, _ = forward(w, *x)
    g, _ = backward(w, *x, saved, torch.randn_like(y))
    theta = w["w_out"].float().clone()
    half = torch.empty_like(w["w_out"])
    hts.hts_delayed_update(theta, g["w_out"], None, theta.numel(), 0.5, 0.0, 1.0, half)
    want = w["w_out"].float() + 0.5 * g["w_out"]
    assert torch.allclose(theta, want, rtol=2.0 ** -22, atol=1e-7) and torch.equal(half, theta.bfloat16())
