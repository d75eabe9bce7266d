"""The recurrent core of a policy with memory, as cases: short causal convolution, selective scan, dense layer with its epilogue.

A policy that remembers runs, per token (one environment step or one token of a prompt):
linear -> causal convolution -> linear (dt, B, C) -> selective scan, gated -> linear + residual.  Its actor calls the single-token forms
once per environment step over a pool of states, its learner the forms over the whole [T, N] storage and their gradients.

Kinds of pass, and the call each makes
  conv, conv-step, conv-gradient        hts_causal_conv, hts_causal_conv_step, hts_causal_conv_gradient
  scan, scan-step, scan-gradient        hts_selective_scan, hts_selective_scan_step, hts_selective_scan_gradient
  linear, linear-gradient               hts_linear, hts_linear_gradient

Shapes: the environments (16, 256, 1024), unroll lengths (5, 128, 512) and the hidden width (512) of hts_workloads.py, an inner width of
twice the hidden one, states of 16 per channel; prompts of thousands of tokens for few sequences; odd and ragged sizes.
Inputs lie in memory as the layers before leave them: x and z are halves of one projection, B and C of another.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
WIDTH_LIMIT = 4096
LIMIT = {"conv": 128 * 256 * 1024, "conv-step": 1024 * 4096, "scan": 128 * 256 * 1024 * 16, "scan-step": 1024 * 1024 * 16,
         "linear": 32768 * 512 * 2048}


def listed():
    return [
        # the actor's step of 256 environments, states gathered from a pool of 1024 by slot: launch latency
        {"name": "conv-step-256", "kind": "conv-step", "type": "bf16", "N": 256, "pool": 1024, "D": 1024, "W": 4, "act": "silu"},
        # the learner's pass over a 128-step rollout of 256 environments with episode ends
        {"name": "conv-rollout-128x256", "kind": "conv", "type": "bf16", "T": 128, "N": 256, "D": 1024, "W": 4, "act": "silu", "ragged": False},
        # its gradient
        {"name": "conv-gradient-128x256", "kind": "conv-gradient", "type": "bf16", "T": 128, "N": 256, "D": 1024, "W": 4, "act": "silu", "ragged": False},
        # the actor's step of the tiny configuration: 16 environments, fp32
        {"name": "scan-step-fp32-16", "kind": "scan-step", "type": "fp32", "N": 16, "pool": 16, "D": 512, "S": 16, "softplus": True, "gate": True},
        # the actor's step of 1024 environments: reads and writes 64 MB of states
        {"name": "scan-step-1024", "kind": "scan-step", "type": "bf16", "N": 1024, "pool": 1024, "D": 1024, "S": 16, "softplus": True, "gate": True},
        # the learner's pass over the rollout
        {"name": "scan-rollout-128x256", "kind": "scan", "type": "bf16", "T": 128, "N": 256, "D": 1024, "S": 16, "softplus": True, "gate": True, "ragged": False},
        # prompts of up to 4095 tokens for three sequences, one of them of a single token: little to do at once besides the long axis
        {"name": "scan-prompts-4095x3", "kind": "scan", "type": "bf16", "T": 4095, "N": 3, "D": 1024, "S": 16, "softplus": True, "gate": True, "ragged": True},
        # the learner's gradient over the rollout
        {"name": "scan-gradient-128x256", "kind": "scan-gradient", "type": "bf16", "T": 128, "N": 256, "D": 1024, "S": 16, "softplus": True, "gate": True, "ragged": False},
        # gradient of two fp32 sequences of odd length, odd number of channels and of states
        {"name": "scan-gradient-fp32-2047x2", "kind": "scan-gradient", "type": "fp32", "T": 2047, "N": 2, "D": 509, "S": 13, "softplus": True, "gate": True, "ragged": False},
        # the output projection of an actor step of 16 environments, residual added: reads the weights
        {"name": "linear-step-16", "kind": "linear", "M": 16, "K": 1024, "N": 512, "act": "none", "bias": True, "residual": True, "keep": False},
        # the input projection over the rollout, pre-activations kept for the gradient
        {"name": "linear-rollout-32768", "kind": "linear", "M": 32768, "K": 512, "N": 2048, "act": "silu", "bias": True, "residual": False, "keep": True},
        # its gradient
        {"name": "linear-gradient-32768", "kind": "linear-gradient", "M": 32768, "K": 512, "N": 2048, "act": "silu"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _width(rng):
    """Channels: any number, half of the time a multiple of eight as layers have it."""
    d = _log(rng, 1, WIDTH_LIMIT)
    return d if rng.random() < 0.5 else max(8, d // 8 * 8)


def draw(rng):
    kind = rng.choice(("conv", "conv-step", "conv-gradient", "scan", "scan-step", "scan-gradient", "linear", "linear-gradient"))
    if kind.startswith("linear"):
        M = _log(rng, 1, 32768)
        K, N = _width(rng), _width(rng)
        M = max(1, min(M, LIMIT["linear"] // (K * N)))
        act = rng.choice(("none", "relu", "silu", "gelu"))
        c = {"kind": kind, "M": M, "K": K, "N": N, "act": act}
        if kind == "linear":
            c |= {"bias": rng.random() < 0.7, "residual": rng.random() < 0.5, "keep": rng.random() < 0.5}
        return c
    c = {"kind": kind, "type": rng.choice(("fp32", "bf16"))}
    D = _width(rng)
    if kind.startswith("conv"):
        c |= {"D": D, "W": rng.choice((2, 3, 4, 4)), "act": rng.choice(("none", "silu"))}
        each, most = D, LIMIT["conv-step" if kind == "conv-step" else "conv"]
    else:
        S = rng.choice((16, 16, _log(rng, 1, 64), _log(rng, 1, 64)))
        c |= {"D": D, "S": S, "softplus": rng.random() < 0.8, "gate": rng.random() < 0.7}
        each, most = D * S, LIMIT["scan-step" if kind == "scan-step" else "scan"]
    if kind.endswith("step"):
        N = max(1, min(_log(rng, 1, 4096), most // each))
        return c | {"N": N, "pool": N + rng.choice((0, 1, N))}
    T = max(1, min(_log(rng, 1, 4096), most // each))
    N = max(1, min(_log(rng, 1, 1024), most // (each * T)))
    return c | {"T": T, "N": N, "ragged": rng.random() < 0.4}


# ---- inputs ------------------------------------------------------------------------------------------------------------
def _lengths(case):
    """Steps of each sequence: evenly spread over 1..T, and with four sequences or more one that is empty; None if all have T."""
    if not case.get("ragged"):
        return None
    T, N = case["T"], case["N"]
    v = [max(1, T * (i + 1) // N) for i in range(N)]
    v[0] = 1
    if N >= 4:
        v[1] = 0
    if N == 1:
        v[0] = max(1, T - 1)
    return v


def _steps(case):
    v = _lengths(case)
    return sum(v) if v else case["T"] * case["N"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dev = "cuda"

    def normal(*shape, t=torch.float32):
        return torch.randn(*shape, generator=g, device=dev).to(t)

    def uniform(lo, hi, *shape):
        return torch.rand(*shape, generator=g, device=dev) * (hi - lo) + lo

    s = {"case": case}
    kind = case["kind"]
    if kind.startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        s["x"] = normal(M, K, t=torch.bfloat16)
        s["w"] = (normal(N, K) / math.sqrt(K)).to(torch.bfloat16)
        if kind == "linear":
            s["bias"] = uniform(-0.1, 0.1, N) if case["bias"] else None
            s["residual"] = normal(M, N, t=torch.bfloat16) if case["residual"] else None
            s["y"] = torch.zeros(M, N, dtype=torch.bfloat16, device=dev)
            s["pre"] = torch.zeros(M, N, dtype=torch.bfloat16, device=dev) if case["keep"] else None
        else:
            s["pre"] = normal(M, N, t=torch.bfloat16) if case["act"] != "none" else None
            s["dy"] = normal(M, N, t=torch.bfloat16)
            s["dx"] = torch.zeros(M, K, dtype=torch.bfloat16, device=dev)
            s["dw"] = torch.zeros(N, K, dtype=torch.bfloat16, device=dev)
            s["dbias"] = torch.zeros(N, device=dev)
        if own:
            import paper_2012_09849_b200 as hts
            s["work"] = torch.empty(hts.hts_linear_workspace(M, K, N, kind != "linear"), dtype=torch.uint8, device=dev)
        return s

    t, N, D = TYPES[case["type"]], case["N"], case["D"]
    step = kind.endswith("step")
    lead = (N,) if step else (case["T"], N)
    # an episode ends every hundred steps or so
    s["starts"] = (torch.rand(*lead, generator=g, device=dev) < 0.01).to(torch.uint8)
    if step:
        s["slots"] = torch.randperm(case["pool"], generator=g, device=dev)[:N].to(torch.int32)
        states = case["pool"]
    else:
        v = _lengths(case)
        s["lengths"] = None if v is None else torch.tensor(v, device=dev)[torch.randperm(N, generator=g, device=dev)].to(torch.int32)
        states = N
    both = normal(*lead, 2 * D, t=t)                       # the input projection: x and the gate
    if kind.startswith("conv"):
        W = case["W"]
        s["x"] = both[..., :D]
        s["w"] = uniform(-1, 1, D, W) / math.sqrt(W)
        s["bias"] = uniform(-0.1, 0.1, D)
        s["window_in"] = normal(states, W - 1, D, t=t)
        s["y"] = torch.zeros(*lead, D, dtype=t, device=dev)
        s["window_out"] = torch.zeros(states, W - 1, D, dtype=t, device=dev)
        if kind == "conv-gradient":
            s["dy"] = normal(*lead, D, t=t)
            s["dwindow_out"] = normal(states, W - 1, D)
            s["dx"] = torch.zeros(*lead, D, dtype=t, device=dev)
            s["dw"], s["dbias"] = torch.zeros(D, W, device=dev), torch.zeros(D, device=dev)
            s["dwindow_in"] = torch.zeros(states, W - 1, D, device=dev)
            if own:
                import paper_2012_09849_b200 as hts
                s["work"] = torch.empty(hts.hts_causal_conv_workspace(case["T"], N, D, W), dtype=torch.uint8, device=dev)
        return s

    S = case["S"]
    x = normal(*lead, D)
    s["x"] = (x * torch.sigmoid(x)).to(t)                  # what the convolution and its activation leave
    s["z"] = both[..., D:] if case["gate"] else None
    # decays of exp(-0.001) to exp(-0.1 S) per step
    size = torch.exp(uniform(math.log(1e-3), math.log(1e-1), D))
    if case["softplus"]:
        s["dt"], s["dt_bias"] = normal(*lead, D).mul_(0.5).to(t), torch.log(torch.expm1(size))
    else:
        s["dt"], s["dt_bias"] = (size * torch.exp(0.5 * normal(*lead, D))).to(t), None
    s["a"] = -torch.arange(1, S + 1, device=dev, dtype=torch.float32) * torch.exp(0.1 * normal(D, S))
    s["d"] = torch.ones(D, device=dev)
    bc = normal(*lead, 2 * S, t=t)
    s["b"], s["c"] = bc[..., :S], bc[..., S:]
    s["state_in"] = normal(states, D, S)
    s["y"] = torch.zeros(*lead, D, dtype=t, device=dev)
    s["state_out"] = torch.zeros(states, D, S, device=dev)
    if kind == "scan-gradient":
        s["dy"], s["dstate_out"] = normal(*lead, D, t=t), normal(states, D, S)
        out = {k: torch.zeros(*lead, n, dtype=t, device=dev) for k, n in (("x", D), ("dt", D), ("b", S), ("c", S))}
        if case["gate"]:
            out["z"] = torch.zeros(*lead, D, dtype=t, device=dev)
        out["a"], out["d"] = torch.zeros(D, S, device=dev), torch.zeros(D, device=dev)
        if s["dt_bias"] is not None:
            out["dt_bias"] = torch.zeros(D, device=dev)
        out["state_in"] = torch.zeros(states, D, S, device=dev)
        s["grads"] = out
    if own and not step:
        import paper_2012_09849_b200 as hts
        s["work"] = torch.empty(hts.hts_selective_scan_workspace(case["T"], N, D, S, kind != "scan"), dtype=torch.uint8, device=dev)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(s):
    return (_own if own else _plain)[s["case"]["kind"]](s)


def _own_conv(s):
    import paper_2012_09849_b200 as hts
    hts.hts_causal_conv(s["x"], s["w"], s["bias"], s["starts"], s["lengths"], s["window_in"], s["case"]["act"], s["y"], s["window_out"])
    return {"y": s["y"], "window_out": s["window_out"]}


def _own_conv_step(s):
    import paper_2012_09849_b200 as hts
    hts.hts_causal_conv_step(s["x"], s["w"], s["bias"], s["starts"], s["slots"], s["window_in"], s["case"]["act"], s["y"], s["window_out"])
    return {"y": s["y"], "window_out": s["window_out"]}


def _own_conv_gradient(s):
    import paper_2012_09849_b200 as hts
    hts.hts_causal_conv_gradient(s["x"], s["w"], s["bias"], s["starts"], s["lengths"], s["window_in"], s["case"]["act"], s["dy"], s["dwindow_out"],
                                 s["dx"], s["dw"], s["dbias"], s["dwindow_in"], s["work"])
    return {k: s[k] for k in ("dx", "dw", "dbias", "dwindow_in")}


def _own_scan(s):
    import paper_2012_09849_b200 as hts
    hts.hts_selective_scan(s["x"], s["dt"], s["a"], s["b"], s["c"], s["d"], s["dt_bias"], s["z"], s["starts"], s["lengths"], s["state_in"],
                           s["case"]["softplus"], s["y"], s["state_out"], s["work"])
    return {"y": s["y"], "state_out": s["state_out"]}


def _own_scan_step(s):
    import paper_2012_09849_b200 as hts
    hts.hts_selective_scan_step(s["x"], s["dt"], s["a"], s["b"], s["c"], s["d"], s["dt_bias"], s["z"], s["starts"], s["slots"], s["state_in"],
                                s["case"]["softplus"], s["y"], s["state_out"])
    return {"y": s["y"], "state_out": s["state_out"]}


def _own_scan_gradient(s):
    import paper_2012_09849_b200 as hts
    hts.hts_selective_scan_gradient(s["x"], s["dt"], s["a"], s["b"], s["c"], s["d"], s["dt_bias"], s["z"], s["starts"], s["lengths"], s["state_in"],
                                    s["case"]["softplus"], s["dy"], s["dstate_out"], s["grads"], s["work"])
    return s["grads"]


def _own_linear(s):
    import paper_2012_09849_b200 as hts
    hts.hts_linear(s["x"], s["w"], s["bias"], s["residual"], s["case"]["act"], s["y"], s["pre"], s["work"])
    return {"y": s["y"]} | ({} if s["pre"] is None else {"pre": s["pre"]})


def _own_linear_gradient(s):
    import paper_2012_09849_b200 as hts
    hts.hts_linear_gradient(s["x"], s["w"], s["pre"], s["dy"], s["case"]["act"], s["dx"], s["dw"], s["dbias"], s["work"])
    return {k: s[k] for k in ("dx", "dw", "dbias")}


def _act(v, act):
    if act == "relu":
        return torch.clamp(v, min=0)
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    return v


def _slope(v, act):
    if act == "relu":
        return (v > 0).to(v.dtype)
    if act == "silu":
        q = torch.sigmoid(v)
        return q * (1 + v * (1 - q))
    if act == "gelu":
        return 0.5 * (1 + torch.erf(v * math.sqrt(0.5))) + v * torch.exp(-0.5 * v * v) * (1 / math.sqrt(2 * math.pi))
    return torch.ones_like(v)


def _softplus(v):
    return torch.clamp(v, min=0) + torch.log1p(torch.exp(-torch.abs(v)))


def _live(s, T, N):
    """[T, N]: the step is one of its sequence's."""
    if s["lengths"] is None:
        return torch.ones(T, N, dtype=torch.bool, device="cuda")
    return torch.arange(T, device="cuda")[:, None] < s["lengths"][None, :]


def _conv_taps(s):
    """For every step the W inputs that it sees, [W][T, N, D], and whether a tap lies in the step's own episode, [W][T, N]."""
    c = s["case"]
    T, N, D, W = c["T"], c["N"], c["D"], c["W"]
    seen = torch.cat([s["window_in"].float().transpose(0, 1), s["x"].float()])
    episode = torch.cumsum(torch.cat([torch.zeros(W - 1, N, device="cuda"), s["starts"].float()]), 0)
    same = [episode[k:k + T] == episode[W - 1:] for k in range(W)]
    return [torch.where(same[k][..., None], seen[k:k + T], 0.0) for k in range(W)], same


def _plain_conv(s):
    c = s["case"]
    T, N, D, W = c["T"], c["N"], c["D"], c["W"]
    taps, _ = _conv_taps(s)
    pre = s["bias"] + sum(s["w"][:, k] * taps[k] for k in range(W))
    live = _live(s, T, N)
    y = torch.where(live[..., None], _act(pre, c["act"]), 0.0).to(s["x"].dtype)
    # the window after the last step: what a step at the sequence's end would see
    end = s["lengths"].long() if s["lengths"] is not None else torch.full((N,), T, device="cuda")
    seen = torch.cat([s["window_in"].transpose(0, 1), s["x"]])
    episode = torch.cumsum(torch.cat([torch.zeros(W - 1, N, device="cuda"), s["starts"].float()]), 0)
    n = torch.arange(N, device="cuda")
    last = episode[end + W - 2, n]
    out = [torch.where((episode[end + j, n] == last)[:, None], seen[end + j, n], 0.0).to(s["x"].dtype) for j in range(W - 1)]
    return {"y": y, "window_out": torch.stack(out, 1)}


def _plain_conv_step(s):
    c = s["case"]
    slots = s["slots"].long()
    win = torch.where((s["starts"] != 0)[:, None, None], 0.0, s["window_in"][slots].float())
    rows = torch.cat([win, s["x"].float()[:, None]], 1)
    y = _act(s["bias"] + sum(s["w"][:, k] * rows[:, k] for k in range(c["W"])), c["act"]).to(s["x"].dtype)
    out = s["window_out"].clone()
    out[slots] = rows[:, 1:].to(out.dtype)
    return {"y": y, "window_out": out}


def _plain_conv_gradient(s):
    c = s["case"]
    T, N, D, W = c["T"], c["N"], c["D"], c["W"]
    taps, same = _conv_taps(s)
    pre = s["bias"] + sum(s["w"][:, k] * taps[k] for k in range(W))
    live = _live(s, T, N)
    dpre = torch.where(live[..., None], s["dy"].float() * _slope(pre, c["act"]), 0.0)
    dw = torch.stack([(dpre * taps[k]).sum((0, 1)) for k in range(W)], 1)
    ext = torch.zeros(T + W - 1, N, D, device="cuda")          # gradients of the window, then of x
    for k in range(W):
        ext[k:k + T] += torch.where(same[k][..., None], s["w"][:, k] * dpre, 0.0)
    end = s["lengths"].long() if s["lengths"] is not None else torch.full((N,), T, device="cuda")
    episode = torch.cumsum(torch.cat([torch.zeros(W - 1, N, device="cuda"), s["starts"].float()]), 0)
    n = torch.arange(N, device="cuda")
    last = episode[end + W - 2, n]
    for j in range(W - 1):
        ext[end + j, n] += torch.where((episode[end + j, n] == last)[:, None], s["dwindow_out"][:, j], 0.0)
    return {"dx": torch.where(live[..., None], ext[W - 1:], 0.0).to(s["x"].dtype), "dw": dw, "dbias": dpre.sum((0, 1)), "dwindow_in": ext[:W - 1].transpose(0, 1).contiguous()}


def _delta(s):
    v = s["dt"].float()
    if s["dt_bias"] is not None:
        v = v + s["dt_bias"]
    return _softplus(v) if s["case"]["softplus"] else v


def _recurrence(a, b):
    """h[t] = a[t] h[t-1] + b[t] from h[-1] = 0, for all t at once: maps of 1, 2, 4, ... steps are composed.  a and b are used up."""
    T, k = a.shape[0], 1
    a2, b2 = torch.empty_like(a), torch.empty_like(b)
    while k < T:
        torch.addcmul(b[k:], a[k:], b[:-k], out=b2[k:])
        torch.mul(a[k:], a[:-k], out=a2[k:])
        b2[:k], a2[:k] = b[:k], a[:k]
        a, a2, b, b2, k = a2, a, b2, b, 2 * k
    return b


def _decays_and_inputs(s, delta, x, b):
    """[T, N, D, S]: what a step keeps of the state, and what it adds; a step behind its sequence's end keeps all and adds nothing."""
    a = torch.exp(delta[..., None] * s["a"])
    a.masked_fill_((s["starts"] != 0)[..., None, None], 0.0)
    u = (delta * x)[..., None] * b[..., None, :]
    if s["lengths"] is not None:
        over = ~_live(s, *x.shape[:2])[..., None, None]
        a.masked_fill_(over, 1.0)
        u.masked_fill_(over, 0.0)
    return a, u


def _plain_scan(s):
    c = s["case"]
    delta, x, b, cc = _delta(s), s["x"].float(), s["b"].float(), s["c"].float()
    a, u = _decays_and_inputs(s, delta, x, b)
    u[0] += a[0] * s["state_in"]
    h = _recurrence(a, u)
    y = (h * cc[..., None, :]).sum(-1) + s["d"] * x
    if s["z"] is not None:
        y = y * _act(s["z"].float(), "silu")
    return {"y": torch.where(_live(s, c["T"], c["N"])[..., None], y, 0.0).to(s["x"].dtype), "state_out": h[-1].clone()}


def _plain_scan_step(s):
    slots = s["slots"].long()
    delta, x = _delta(s), s["x"].float()
    h = torch.where((s["starts"] != 0)[:, None, None], 0.0, s["state_in"][slots])
    h = h * torch.exp(delta[..., None] * s["a"]) + (delta * x)[..., None] * s["b"].float()[:, None, :]
    y = (h * s["c"].float()[:, None, :]).sum(-1) + s["d"] * x
    if s["z"] is not None:
        y = y * _act(s["z"].float(), "silu")
    out = s["state_out"].clone()
    out[slots] = h
    return {"y": y.to(s["x"].dtype), "state_out": out}


def _plain_scan_gradient(s):
    c = s["case"]
    delta, x, b, cc, dy = _delta(s), s["x"].float(), s["b"].float(), s["c"].float(), s["dy"].float()
    live = _live(s, c["T"], c["N"])
    z = None if s["z"] is None else s["z"].float()
    g = torch.where(live[..., None], dy if z is None else dy * _act(z, "silu"), 0.0)
    a, u = _decays_and_inputs(s, delta, x, b)
    u[0] += a[0] * s["state_in"]
    h = _recurrence(a.clone(), u)
    kept = a * torch.cat([s["state_in"][None], h[:-1]])         # what a step kept of the state before it
    y = (h * cc[..., None, :]).sum(-1)
    dc = (h * g[..., None]).sum(2)
    del h, u
    # the gradient of the states runs back: what reaches step t from step t + 1 has that step's decay
    u = g[..., None] * cc[..., None, :]
    u[-1] += s["dstate_out"]
    grad = _recurrence(torch.cat([a[1:], torch.zeros_like(a[:1])]).flip(0), u.flip(0)).flip(0)
    state_in = a[0] * grad[0]
    grad.masked_fill_(~live[..., None, None], 0.0)
    db = (grad * (delta * x)[..., None]).sum(2)
    gb = (grad * b[..., None, :]).sum(-1)
    grad *= kept
    ddt = x * gb + (grad * s["a"]).sum(-1)
    da = (grad * delta[..., None]).sum((0, 1))
    dx = delta * gb + s["d"] * g
    if c["softplus"]:
        ddt = ddt * torch.sigmoid(s["dt"].float() if s["dt_bias"] is None else s["dt"].float() + s["dt_bias"])
    t = s["x"].dtype
    out = {"x": dx.to(t), "dt": ddt.to(t), "b": db.to(t), "c": dc.to(t)}
    if z is not None:
        out["z"] = torch.where(live[..., None], dy * (y + s["d"] * x) * _slope(z, "silu"), 0.0).to(t)
    out["a"], out["d"] = da, (g * x).sum((0, 1))
    if s["dt_bias"] is not None:
        out["dt_bias"] = ddt.sum((0, 1))
    out["state_in"] = state_in
    return out


def _plain_linear(s):
    pre = s["x"].float() @ s["w"].float().t()
    if s["bias"] is not None:
        pre = pre + s["bias"]
    y = _act(pre, s["case"]["act"])
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(torch.bfloat16)} | ({} if s["pre"] is None else {"pre": pre.to(torch.bfloat16)})


def _plain_linear_gradient(s):
    dz = s["dy"].float()
    if s["pre"] is not None:
        dz = dz * _slope(s["pre"].float(), s["case"]["act"])
    return {"dx": (dz @ s["w"].float()).to(torch.bfloat16), "dw": (dz.t() @ s["x"].float()).to(torch.bfloat16), "dbias": dz.sum(0)}


_own = {"conv": _own_conv, "conv-step": _own_conv_step, "conv-gradient": _own_conv_gradient, "scan": _own_scan, "scan-step": _own_scan_step,
        "scan-gradient": _own_scan_gradient, "linear": _own_linear, "linear-gradient": _own_linear_gradient}
_plain = {"conv": _plain_conv, "conv-step": _plain_conv_step, "conv-gradient": _plain_conv_gradient, "scan": _plain_scan, "scan-step": _plain_scan_step,
          "scan-gradient": _plain_scan_gradient, "linear": _plain_linear, "linear-gradient": _plain_linear_gradient}


# ---- what one pass cannot do without ---------------------------------------------------------------------------------------
def work(case):
    kind = case["kind"]
    if kind.startswith("linear"):
        M, K, N = case["M"], case["K"], case["N"]
        if kind == "linear":
            kept = case["keep"] + case["residual"]
            return {"bytes": 2 * (M * K + N * K + M * N * (1 + kept)) + 4 * N * case["bias"], "flops": 2 * M * N * K}
        return {"bytes": 2 * (2 * M * K + 2 * N * K + M * N * (1 + (case["act"] != "none"))) + 4 * N, "flops": 4 * M * N * K}
    e = 4 if case["type"] == "fp32" else 2
    D, step = case["D"], kind.endswith("step")
    R = case["N"] if step else _steps(case)
    if kind.startswith("conv"):
        W = case["W"]
        windows = case["N"] * (W - 1) * D
        fixed = 4 * D * (W + 1) + R
        if kind == "conv-gradient":
            return {"bytes": 3 * R * D * e + windows * (e + 8) + 2 * fixed, "flops": R * D * (6 * W + 12)}
        return {"bytes": 2 * R * D * e + 2 * windows * e + fixed, "flops": R * D * (2 * W + 4)}
    S = case["S"]
    states = case["N"] * D * S * 4
    fixed = 4 * D * (S + 2) + R
    tensors = 3 + case["gate"]
    if kind == "scan-gradient":
        return {"bytes": R * ((2 * tensors - 1) * D + 4 * S) * e + 3 * states + 2 * fixed, "flops": R * D * (20 * S + 30)}
    return {"bytes": R * (tensors * D + 2 * S) * e + 2 * states + fixed, "flops": R * D * (7 * S + 15)}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    """Every sequence by itself, episode by episode; gradients by differentiating the definition."""
    s = prepare(case, seed)
    kind = case["kind"]
    f = lambda v: None if v is None else v.double()
    with torch.enable_grad():
        if kind.startswith("linear"):
            if kind == "linear":
                pre = torch.einsum("mk,nk->mn", f(s["x"]), f(s["w"])) + (0 if s["bias"] is None else f(s["bias"]))
                y = _by_name(pre, case["act"]) + (0 if s["residual"] is None else f(s["residual"]))
                return {"y": y} | ({} if s["pre"] is None else {"pre": pre})
            dz = f(s["dy"])
            if s["pre"] is not None:
                p = f(s["pre"]).requires_grad_()
                dz, = torch.autograd.grad(_by_name(p, case["act"]), p, dz)
            return {"dx": torch.einsum("mn,nk->mk", dz, f(s["w"])), "dw": torch.einsum("mn,mk->nk", dz, f(s["x"])), "dbias": torch.einsum("mn->n", dz)}
        return _exact_conv(s, f) if kind.startswith("conv") else _exact_scan(s, f)


def _by_name(v, act):
    f = torch.nn.functional
    return {"none": lambda u: u * 1, "relu": f.relu, "silu": f.silu, "gelu": f.gelu}[act](v)


def _exact_conv(s, f):
    c = s["case"]
    W, step, grad = c["W"], c["kind"] == "conv-step", c["kind"] == "conv-gradient"
    x, w, bias, win = f(s["x"]), f(s["w"]), f(s["bias"]), f(s["window_in"])
    starts = s["starts"] != 0
    if step:
        slots = s["slots"].long()
        x, starts, win_all, win = x[None], starts[None], f(s["window_out"]), win[slots]
    if grad:
        for v in (x, w, bias, win):
            v.requires_grad_()
    T, N = x.shape[:2]
    lengths = s.get("lengths")
    window, ys = list(win.unbind(1)), []
    for t in range(T):
        on = torch.ones_like(starts[t]) if lengths is None else t < lengths
        fresh = (starts[t] & on)[:, None]
        seen = [torch.where(fresh, torch.zeros_like(v), v) for v in window] + [x[t]]
        y = _by_name(bias + sum(w[:, k] * seen[k] for k in range(W)), c["act"])
        ys.append(torch.where(on[:, None], y, torch.zeros_like(y)))
        window = [torch.where(on[:, None], v, u) for v, u in zip(seen[1:], window)]      # past its end a sequence keeps its window
    y, out = torch.stack(ys), torch.stack(window, 1)
    if step:
        win_all[slots] = out
        return {"y": y[0], "window_out": win_all}
    if not grad:
        return {"y": y, "window_out": out}
    dx, dw, db, dwin = torch.autograd.grad([y, out], [x, w, bias, win], [f(s["dy"]), f(s["dwindow_out"])])
    return {"dx": dx, "dw": dw, "dbias": db, "dwindow_in": dwin}


def _exact_scan(s, f):
    c = s["case"]
    step, grad = c["kind"] == "scan-step", c["kind"] == "scan-gradient"
    v = {k: f(s[k]) for k in ("x", "dt", "a", "b", "c", "d", "dt_bias", "z")}
    h = f(s["state_in"])
    starts = s["starts"] != 0
    if step:
        slots = s["slots"].long()
        h = h[slots]
        for k in ("x", "dt", "b", "c", "z"):
            v[k] = None if v[k] is None else v[k][None]
        starts = starts[None]
    v["state_in"] = h
    wanted = [k for k in v if v[k] is not None]
    if grad:
        for k in wanted:
            v[k].requires_grad_()
    raw = v["dt"] if v["dt_bias"] is None else v["dt"] + v["dt_bias"]
    delta = torch.nn.functional.softplus(raw, threshold=700.0) if c["softplus"] else raw
    lengths = s.get("lengths")
    h, ys = v["state_in"], []
    for t in range(v["x"].shape[0]):
        decay = torch.exp(torch.einsum("nd,ds->nds", delta[t], v["a"]))
        decay = torch.where(starts[t][:, None, None], torch.zeros_like(decay), decay)
        new = decay * h + torch.einsum("nd,ns->nds", delta[t] * v["x"][t], v["b"][t])
        y = torch.einsum("nds,ns->nd", new, v["c"][t])
        if lengths is None:
            h = new
        else:
            on = t < lengths
            h, y = torch.where(on[:, None, None], new, h), torch.where(on[:, None], y, torch.zeros_like(y))
        ys.append(y)
    y = torch.stack(ys) + v["d"] * v["x"]
    if v["z"] is not None:
        y = y * torch.nn.functional.silu(v["z"])
    if lengths is not None:
        y = torch.where((torch.arange(len(ys), device="cuda")[:, None] < lengths)[..., None], y, torch.zeros_like(y))
    if step:
        states = f(s["state_out"])
        states[slots] = h
        return {"y": y[0], "state_out": states}
    if not grad:
        return {"y": y, "state_out": h}
    got = dict(zip(wanted, torch.autograd.grad([y, h], [v[k] for k in wanted], [f(s["dy"]), f(s["dstate_out"])])))
    return {k: got[k] for k in s["grads"]}
