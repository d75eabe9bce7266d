"""hts_linear and its gradient against the definition in 64 bits."""
import pytest
import torch

import paper_2012_09849_b200 as hts
import recurrent_ref as ref

pytestmark = pytest.mark.gpu
# rows, in, out: single rows, odd sizes (rows off 16-byte boundaries), sizes around the tiles (128, 64, 256), products cut along k, and
# those that run on pairs of SMs
SHAPES = [(1, 1, 1), (1, 1024, 512), (3, 5, 7), (16, 1024, 512), (16, 512, 2048), (65, 4096, 200), (127, 64, 65), (128, 200, 128), (129, 136, 63), (300, 72, 520), (257, 2000, 257),
          (1000, 96, 1024), (2600, 64, 512), (2561, 1000, 264), (5000, 24, 72)]


def rows(M, N, offset=0, seed=0, pad=0):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + M * 31 + N)
    return torch.randn(M, offset + N + pad, generator=g, device="cuda").bfloat16()[:, offset:offset + N]


def case(M, K, N, offset=0, pad=0, bias=True, residual=True):
    return dict(x=rows(M, K, offset, 1, pad), w=(rows(N, K, 0, 2).float() / K ** 0.5).bfloat16().contiguous(), bias=rows(1, N, 0, 3)[0].float().contiguous() if bias else None,
                residual=rows(M, N, offset, 4, pad) if residual else None)


def run(c, act, keep=False, y=None, stream=None):
    M, N, K = c["x"].shape[0], c["w"].shape[0], c["x"].shape[1]
    y = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda") if y is None else y
    pre = torch.full((M, N), 7.0, dtype=torch.bfloat16, device="cuda") if keep else None
    work = torch.empty(hts.hts_linear_workspace(M, K, N), dtype=torch.uint8, device="cuda")
    ref.lend(stream, y, pre, work)
    hts.hts_linear(c["x"], c["w"], c["bias"], c["residual"], act, y, pre, work, stream)
    return y, pre


def check(c, act, y, pre):
    """The sums: at most 2^-23 of the magnitude for every 16 products (the tensor core cuts off), 2^-24 for every other addition;
    an activation's slope is below 1.13, and its own error 2^-19 of its argument."""
    x, w, K = c["x"].double(), c["w"].double(), c["x"].shape[1]
    s = x @ w.t() + (0 if c["bias"] is None else c["bias"].double())
    mag = x.abs() @ w.abs().t() + (0 if c["bias"] is None else c["bias"].double().abs())
    room = 1.13 * ((K / 16 + 12) * 2.0 ** -23 + 2.0 ** -19) * mag
    want = ref.ACT[act](s) + (0 if c["residual"] is None else c["residual"].double())
    ref.within(y, want, room + 2.0 ** -23 * want.abs(), "y")
    if pre is not None:
        ref.within(pre, s, room, "pre")


@pytest.mark.parametrize("shape", SHAPES)
def test_products_and_epilogues(shape):
    for i, act in enumerate(("none", "relu", "silu", "gelu")):
        c = case(*shape, bias=i != 1, residual=i != 2)
        check(c, act, *run(c, act, keep=i % 2 == 0))


@pytest.mark.parametrize("shape", [(17, 64, 40), (300, 128, 256), (2600, 64, 512)])
@pytest.mark.parametrize("offset,pad", [(8, 0), (0, 8), (1, 0), (4, 3)])
def test_rows_of_wider_tensors(shape, offset, pad):
    c = case(*shape, offset=offset, pad=pad)
    M, N = shape[0], shape[2]
    wide = torch.full((M, N + offset + pad), 7.0, dtype=torch.bfloat16, device="cuda")
    y, _ = run(c, "silu", y=wide[:, offset:offset + N])
    check(c, "silu", y, None)
    assert bool((wide[:, :offset] == 7).all()) and bool((wide[:, offset + N:] == 7).all())


@pytest.mark.parametrize("shape", [(40, 64, 72), (2600, 64, 512)])
def test_the_residual_may_be_written_over(shape):
    c = case(*shape)
    want, _ = run(c, "none")
    y = c["residual"].clone()
    got, _ = run(dict(c, residual=y), "none", y=y)
    assert torch.equal(got, want)


@pytest.mark.parametrize("shape", [(40, 100, 72), (2600, 64, 512)])
def test_a_row_is_not_touched_by_another(shape):
    c = case(*shape, residual=False)
    want, _ = run(c, "gelu")
    x = c["x"].clone()
    x[5] = float("nan")
    x[7, 3] = float("inf")
    got, _ = run(dict(c, x=x), "gelu")
    rest = torch.ones(shape[0], dtype=torch.bool, device="cuda")
    rest[5] = rest[7] = False
    assert torch.equal(got[rest], want[rest]) and bool(torch.isnan(got[5]).all()) and not bool(torch.isfinite(got[7]).all())


def gradient(c, act, pre, dy, dw_type=torch.float32, want=("dx", "dw", "dbias"), stream=None):
    M, N, K = c["x"].shape[0], c["w"].shape[0], c["x"].shape[1]
    o = {"dx": torch.full((M, K), 7.0, dtype=torch.bfloat16, device="cuda"), "dw": torch.full((N, K), 7.0, dtype=dw_type, device="cuda"), "dbias": torch.full((N,), 7.0, device="cuda")}
    o = {k: v if k in want else None for k, v in o.items()}
    work = torch.empty(hts.hts_linear_workspace(M, K, N, True), dtype=torch.uint8, device="cuda")
    ref.lend(stream, work, *o.values())
    hts.hts_linear_gradient(c["x"], c["w"], pre, dy, act, o["dx"], o["dw"], o["dbias"], work, stream)
    return o


@pytest.mark.parametrize("shape", SHAPES + [(9000, 72, 136)])
def test_gradient(shape):
    """dz is rounded to bf16 (2^-8 of each) where there is an activation; the sums as above, those of rows K = M."""
    M, K, N = shape
    for i, act in enumerate(("none", "relu", "silu", "gelu")):
        c = case(*shape, residual=False)
        pre, dy = rows(M, N, 0, 5), rows(M, N, 0, 6)
        got = gradient(c, act, None if act == "none" else pre, dy, torch.float32 if i % 2 else torch.bfloat16)
        p = pre.double().requires_grad_()
        dz = dy.double() if act == "none" else torch.autograd.grad(ref.ACT[act](p), p, dy.double())[0]
        exact = act == "none"
        each = 0 if exact else 2.0 ** -8 + 2.0 ** -18                       # of dz: its rounding and the slope's error
        small = 0 if exact else 2.0 ** -17 * dy.double().abs()              # the slope's error where it is near zero
        x, w, mag = c["x"].double(), c["w"].double(), dz.abs()
        for k, want, m, n in (("dx", dz @ w, (mag * each + small) @ w.abs() + (N / 16 + 12) * 2.0 ** -23 * (mag @ w.abs()), N),
                              ("dw", dz.t() @ x, (mag * each + small).t() @ x.abs() + (M / 16 + 60) * 2.0 ** -23 * (mag.t() @ x.abs()), M)):
            ref.within(got[k], want, m, k)
        room = 0 if exact else 2.0 ** -18 * mag.sum(0) + small.sum(0)
        ref.within(got["dbias"], dz.sum(0), room + 80 * 2.0 ** -24 * mag.sum(0), "dbias")


def test_gradient_is_that_of_differences():
    M, K, N = 6, 10, 5
    c = case(M, K, N, residual=False)
    x, w, dy = c["x"].double(), c["w"].double(), rows(M, N, 0, 6).double()
    pre = (x @ w.t() + c["bias"].double())
    got = gradient(c, "silu", pre.bfloat16(), dy.bfloat16())

    def value(x, w, b):
        return float((ref.ACT["silu"](x @ w.t() + b) * dy).sum())
    b = c["bias"].double()
    for key, at in (("dx", 0), ("dw", 1), ("dbias", 2)):
        args = [x, w, b]
        e = torch.randn_like(args[at])
        up, down = list(args), list(args)
        up[at], down[at] = args[at] + 1e-5 * e, args[at] - 1e-5 * e
        slope = (value(*up) - value(*down)) / 2e-5
        # the pre-activations are rounded to bf16 (2^-8 of them, SiLU's second derivative is at most 1/2), dz and dx are too
        room = float((got[key].double() * e).abs().sum()) * 3 * 2.0 ** -8 + float(pre.abs().max()) * 2.0 ** -8 * float(dy.abs().sum()) * float(args[1 - at].abs().max() if at < 2 else 1) * float(e.abs().max()) / 2
        assert abs(float((got[key].double() * e).sum()) - slope) <= room


def test_gradients_that_are_not_asked_for_and_repetition():
    c = case(700, 136, 72, residual=False)
    pre, dy = rows(700, 72, 0, 5), rows(700, 72, 1, 6)          # dy starts off a 16-byte boundary
    full = gradient(c, "silu", pre, dy)
    for want in (("dx",), ("dw",), ("dbias",), ("dx", "dbias")):
        part = gradient(c, "silu", pre, dy, want=want)
        for k in want:
            assert torch.equal(part[k], full[k]), k
    plain = gradient(c, "none", None, dy)
    assert all(torch.equal(plain[k], gradient(c, "none", None, dy.contiguous())[k]) for k in plain)


@pytest.mark.parametrize("shape", [(16, 1024, 512), (2600, 64, 512)])
def test_captured_calls_replay_and_other_streams(shape):
    M, K, N = shape
    c = case(*shape)
    pre, dy = rows(M, N, 0, 5), rows(M, N, 0, 6)
    want, want_g = run(c, "silu", keep=True), gradient(c, "silu", pre, dy)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, got_g = run(c, "silu", keep=True, stream=s), gradient(c, "silu", pre, dy, stream=s)
    s.synchronize()
    assert all(torch.equal(u, v) for u, v in zip(got, want)) and all(torch.equal(got_g[k], want_g[k]) for k in want_g)
    y, kept = torch.zeros_like(want[0]), torch.zeros_like(want[0])
    o = {k: torch.zeros_like(v) for k, v in want_g.items()}
    work = [torch.empty(hts.hts_linear_workspace(M, K, N, g), dtype=torch.uint8, device="cuda") for g in (False, True)]
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        hts.hts_linear(c["x"], c["w"], c["bias"], c["residual"], "silu", y, kept, work[0])
        hts.hts_linear_gradient(c["x"], c["w"], pre, dy, "silu", o["dx"], o["dw"], o["dbias"], work[1])
    for _ in range(2):
        for v in (y, kept, *o.values()):
            v.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[0]) and torch.equal(kept, want[1]) and all(torch.equal(o[k], want_g[k]) for k in o)


def test_two_calls_at_once():
    cases = [case(2600, 512, 512), case(3000, 256, 768)]
    want = [run(c, "silu")[0] for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        got = [run(c, "silu", stream=s)[0] for c, s in zip(cases, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(u, v) for u, v in zip(got, want))


@pytest.mark.parametrize("M,N", [(40, 72), (41, 71), (4100, 72)])
def test_nothing_passes_where_relu_is_shut(M, N):
    """An infinite or undefined dy in front of a pre-activation of zero or less."""
    c = case(M, 64, N, residual=False)
    _, pre = run(c, "relu", keep=True)
    pre[3, 5], pre[M - 1, 0] = -1.0, 0.0
    dy = rows(M, N, 0, 9).clone()
    clean = torch.where(pre > 0, dy, torch.zeros_like(dy))
    dy[3, 5], dy[M - 1, 0] = float("inf"), float("nan")
    results = []
    for d in (dy, clean):
        dx, dw, db = torch.empty(M, 64, dtype=torch.bfloat16, device="cuda"), torch.empty(N, 64, device="cuda"), torch.empty(N, device="cuda")
        hts.hts_linear_gradient(c["x"], c["w"], pre, d, "relu", dx, dw, db, torch.empty(hts.hts_linear_workspace(M, 64, N, True), dtype=torch.uint8, device="cuda"))
        results.append((dx, dw, db))
    assert all(bool(torch.isfinite(u).all()) and torch.equal(u, v) for u, v in zip(*results))
