"""Rows whose offsets pass 32 bits: the recurrent core on column ranges of a tensor of 2^31 elements and more."""
import pytest
import torch

import paper_2012_09849_b200 as hts

pytestmark = pytest.mark.gpu
T, D, S, LD = 40, 64, 16, 1 << 26                       # 40 rows, 2^26 elements apart: the last starts at 2.6e9


@pytest.fixture(scope="module")
def far():
    need = 3 * T * LD * 2
    if torch.cuda.mem_get_info()[0] < need + (4 << 30):
        pytest.skip("not enough memory")
    tensors = [torch.empty(T, 1, LD, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
    yield lambda i, at, cols: tensors[i][:, :, at:at + cols]
    tensors.clear()
    torch.cuda.empty_cache()


def near(*shape, seed):
    return torch.randn(*shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").bfloat16()


def put(view, value):
    view.copy_(value)
    return view


def test_convolution_and_gradient(far):
    x, dy, w = near(T, 1, D, seed=1), near(T, 1, D, seed=2), torch.rand(D, 4, device="cuda")
    got = []
    for fx, fdy, fy in ((x, dy, torch.empty_like(x)), (put(far(0, 8, D), x), put(far(1, 0, D), dy), far(2, 16, D))):
        work = torch.empty(hts.hts_causal_conv_workspace(T, 1, D, 4), dtype=torch.uint8, device="cuda")
        dw = torch.empty(D, 4, device="cuda")
        hts.hts_causal_conv(fx, w, None, None, None, None, "silu", fy, None)
        y = fy.clone()
        hts.hts_causal_conv_gradient(fx, w, None, None, None, None, "silu", fdy, None, fy, dw, None, None, work)
        got.append((y, fy.clone(), dw))
    assert all(torch.equal(u, v) for u, v in zip(*got))


def test_scan_and_gradient(far):
    x, dt, z, dy, b, c = (near(T, 1, n, seed=i) for i, n in enumerate((D, D, D, D, S, S)))
    a = -torch.exp(torch.randn(D, S, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda"))
    got = []
    for i in range(2):
        place = (lambda t, k, at: put(far(k, at, t.shape[2]), t)) if i else (lambda t, k, at: t)
        ins = (place(x, 0, 0), place(dt, 0, 128), a, place(b, 0, 256), place(c, 0, 512), None, None, place(z, 1, 8), None, None, None, True)
        y = far(2, 0, D) if i else torch.empty_like(x)
        state = torch.empty(1, D, S, device="cuda")
        hts.hts_selective_scan(*ins, y, state, torch.empty(hts.hts_selective_scan_workspace(T, 1, D, S), dtype=torch.uint8, device="cuda"))
        g = {k: far(2, 1024 + 128 * j, t.shape[2]) if i else torch.empty_like(t) for j, (k, t) in enumerate((("x", x), ("dt", dt), ("b", b), ("c", c), ("z", z)))}
        g["a"] = torch.empty_like(a)
        out = y.clone()
        hts.hts_selective_scan_gradient(*ins, place(dy, 1, 256), None, g, torch.empty(hts.hts_selective_scan_workspace(T, 1, D, S, True), dtype=torch.uint8, device="cuda"))
        got.append([out, state] + [v.clone() for v in g.values()])
    assert all(torch.equal(u, v) for u, v in zip(*got))


def test_linear_and_gradient(far):
    x, r, dy = near(T, 1, D, seed=1), near(T, 1, 72, seed=2), near(T, 1, 72, seed=3)
    w = near(72, D, seed=4)
    got = []
    for i in range(2):
        place = (lambda t, k, at: put(far(k, at, t.shape[2]), t)[:, 0]) if i else (lambda t, k, at: t[:, 0])
        y = far(2, 0, 72)[:, 0] if i else torch.empty(T, 72, dtype=torch.bfloat16, device="cuda")
        dx = far(2, 128, D)[:, 0] if i else torch.empty(T, D, dtype=torch.bfloat16, device="cuda")
        dw = torch.empty(72, D, device="cuda")
        hts.hts_linear(place(x, 0, 0), w, None, place(r, 1, 8), "none", y, None, torch.empty(hts.hts_linear_workspace(T, D, 72), dtype=torch.uint8, device="cuda"))
        hts.hts_linear_gradient(place(x, 0, 0), w, None, place(dy, 1, 256), "none", dx, dw, None, torch.empty(hts.hts_linear_workspace(T, D, 72, True), dtype=torch.uint8, device="cuda"))
        got.append((y.clone(), dx.clone(), dw))
    assert all(torch.equal(u, v) for u, v in zip(*got))
