"""What the recurrent core refuses (no GPU: every call below is refused before any CUDA call)."""
import ctypes

import pytest
import torch

import paper_2012_09849_b200 as hts

INVALID = 1
P = 1 << 20                                             # stands for an address; never used


def conv_desc(**kw):
    return hts.hts_conv_desc(**{**dict(T=4, N=2, channels=8, width=4, dtype=0, activation=2, ld_x=8, ld_y=8, ld_dy=8, ld_dx=8), **kw})


def conv(x=P, w=P + 1, y=P + 2, window_in=None, window_out=None, **kw):
    return hts.lib().hts_causal_conv(ctypes.byref(conv_desc(**kw)), x, w, None, None, None, window_in, y, window_out, None)


@pytest.mark.parametrize("kw", [dict(T=0), dict(N=0), dict(channels=0), dict(width=1), dict(width=5), dict(dtype=2), dict(activation=1), dict(activation=3), dict(ld_x=7), dict(ld_y=7),
                                dict(x=None), dict(w=None), dict(y=None), dict(y=P), dict(window_in=P + 9, window_out=P + 9)])
def test_convolution(kw):
    assert conv(**kw) == INVALID


@pytest.mark.parametrize("kw", [dict(window_in=None), dict(window_out=None), dict(pool=0), dict(pool=1), dict(y=P), dict(N=-1)])
def test_convolution_step(kw):
    a = {**dict(x=P, w=P + 1, slots=None, pool=2, window_in=P + 3, y=P + 2, window_out=P + 3, N=2), **kw}
    assert hts.lib().hts_causal_conv_step(ctypes.byref(conv_desc(N=a["N"])), a["x"], a["w"], None, None, a["slots"], a["pool"], a["window_in"], a["y"], a["window_out"], None) == INVALID


@pytest.mark.parametrize("kw", [dict(dx=None, dw=None, dbias=None, dwin=None), dict(dy=None), dict(dx=P), dict(dx=P + 4), dict(ld_dy=7), dict(ld_dx=7), dict(work=None), dict(work=P + 8),
                                dict(less=1)])
def test_convolution_gradient(kw):
    a = {**dict(dy=P + 4, dx=P + 5, dw=P + 6, dbias=None, dwin=None, work=P, less=0), **kw}
    need = hts.hts_causal_conv_workspace(4, 2, 8, 4)
    desc = conv_desc(**{k: v for k, v in kw.items() if k.startswith("ld")})
    assert need > 0 and hts.lib().hts_causal_conv_gradient(ctypes.byref(desc), P, P + 1, None, None, None, None, a["dy"], None, a["dx"], a["dw"], a["dbias"], a["dwin"], a["work"],
                                                           need - a["less"], None) == INVALID


def scan_call(form="", **kw):
    d = {**dict(T=4, N=2, channels=8, state=16, dtype=0, softplus=1, ld_x=8, ld_dt=8, ld_b=16, ld_c=16, ld_z=8, ld_y=8), **{k: v for k, v in kw.items() if k in dict(hts.hts_scan_desc._fields_)}}
    i = {**dict(x=P, dt=P + 1, b=P + 2, c=P + 3, z=P + 4, a=P + 5, state_in=P + 6), **{k: v for k, v in kw.items() if k in dict(hts.hts_scan_inputs._fields_)}}
    a = {**dict(y=P + 7, state_out=P + 8, work=P, bytes=1 << 40, slots=None, pool=2, dy=P + 9, ld_dy=8), **kw}
    desc, ins = hts.hts_scan_desc(**d), hts.hts_scan_inputs(**i)
    L = hts.lib()
    if form == "step":
        return L.hts_selective_scan_step(ctypes.byref(desc), ctypes.byref(ins), a["slots"], a["pool"], a["y"], a["state_out"], None)
    if form == "gradient":
        g = hts.hts_scan_grads(**{**dict(x=P + 10, ld_x=8), **kw.get("grads", {})})
        return L.hts_selective_scan_gradient(ctypes.byref(desc), ctypes.byref(ins), a["dy"], a["ld_dy"], None, ctypes.byref(g), a["work"], a["bytes"], None)
    return L.hts_selective_scan(ctypes.byref(desc), ctypes.byref(ins), a["y"], a["state_out"], a["work"], a["bytes"], None)


@pytest.mark.parametrize("kw", [dict(T=0), dict(N=0), dict(channels=0), dict(state=0), dict(state=65), dict(dtype=-1), dict(ld_x=7), dict(ld_dt=7), dict(ld_b=15), dict(ld_c=15), dict(ld_z=7),
                                dict(ld_y=7), dict(x=None), dict(dt=None), dict(a=None), dict(b=None), dict(c=None), dict(y=None), dict(y=P), dict(y=P + 4), dict(state_out=P + 6),
                                dict(ld_x=1 << 28), dict(T=1 << 30, N=1 << 10), dict(T=4096, work=None), dict(T=4096, bytes=16), dict(T=4096, work=P + 8)])
def test_scan(kw):
    assert scan_call(**kw) == INVALID


@pytest.mark.parametrize("kw", [dict(state_in=None), dict(state_out=None), dict(lengths=P), dict(pool=0), dict(pool=1), dict(y=P), dict(state=65), dict(ld_y=7)])
def test_scan_step(kw):
    assert scan_call("step", **kw) == INVALID


@pytest.mark.parametrize("kw", [dict(dy=None), dict(ld_dy=7), dict(grads=dict(x=None)), dict(grads=dict(x=P)), dict(grads=dict(x=P + 9)), dict(grads=dict(ld_x=7)),
                                dict(grads=dict(b=P + 11, ld_b=15)), dict(z=None, grads=dict(z=P + 11, ld_z=8)), dict(work=None), dict(work=P + 8), dict(bytes=64)])
def test_scan_gradient(kw):
    assert scan_call("gradient", **kw) == INVALID


def linear_call(gradient=False, **kw):
    d = {**dict(rows=4, in_features=8, out_features=16, activation=2, ld_x=8, ld_residual=16, ld_y=16, ld_pre=16, ld_dy=16, ld_dx=8, dw_dtype=0),
         **{k: v for k, v in kw.items() if k in dict(hts.hts_linear_desc._fields_)}}
    need = hts.hts_linear_workspace(4, 8, 16, gradient)
    a = {**dict(x=P, w=P + 1, residual=P + 2, y=P + 3, pre=P + 4, dy=P + 5, dx=P + 6, dw=P + 7, dbias=None, work=P, bytes=need), **kw}
    desc = hts.hts_linear_desc(**d)
    if gradient:
        return hts.lib().hts_linear_gradient(ctypes.byref(desc), a["x"], a["w"], a["pre"], a["dy"], a["dx"], a["dw"], a["dbias"], a["work"], a["bytes"], None)
    return hts.lib().hts_linear(ctypes.byref(desc), a["x"], a["w"], None, a["residual"], a["y"], a["pre"], a["work"], a["bytes"], None)


@pytest.mark.parametrize("kw", [dict(rows=0), dict(in_features=0), dict(out_features=-1), dict(activation=4), dict(activation=-1), dict(ld_x=7), dict(ld_residual=15), dict(ld_y=15), dict(ld_pre=15),
                                dict(x=None), dict(w=None), dict(y=None), dict(y=P), dict(pre=P + 3), dict(pre=P + 2), dict(work=None), dict(work=P + 8), dict(bytes=100)])
def test_linear(kw):
    assert linear_call(**kw) == INVALID


@pytest.mark.parametrize("kw", [dict(dy=None), dict(ld_dy=15), dict(ld_dx=7), dict(pre=None), dict(ld_pre=15), dict(dw_dtype=2), dict(dx=None, dw=None), dict(dx=P), dict(dx=P + 5), dict(dw=P + 1),
                                dict(work=None), dict(bytes=1000)])
def test_linear_gradient(kw):
    assert linear_call(True, **kw) == INVALID


def test_workspaces():
    assert hts.hts_causal_conv_workspace(0, 1, 1, 2) == hts.hts_causal_conv_workspace(1, 1, 1, 5) == 0
    assert hts.hts_selective_scan_workspace(1, 1, 1, 65) == hts.hts_linear_workspace(1, 0, 1) == 0
    assert hts.hts_selective_scan_workspace(128, 256, 1024, 16) == 0                # enough sequences: no runs
    assert hts.hts_selective_scan_workspace(4096, 1, 1024, 16) > 0
    assert hts.hts_linear_workspace(16, 8, 8, True) > hts.hts_linear_workspace(16, 8, 8) > 0


# ---- tensors ------------------------------------------------------------------------------------------------------------
def conv_tensors(**kw):
    t = dict(x=torch.zeros(4, 2, 8), w=torch.zeros(8, 4), bias=torch.zeros(8), starts=torch.zeros(4, 2, dtype=torch.uint8), lengths=None, window_in=torch.zeros(2, 3, 8), activation="silu",
             y=torch.zeros(4, 2, 8), window_out=None, stream=0)
    return {**t, **kw}


@pytest.mark.parametrize("kw,error", [
    (dict(x=None), TypeError), (dict(x=5), TypeError), (dict(x=torch.zeros(4, 2, 8, dtype=torch.float16)), TypeError), (dict(x=torch.zeros(8, 8)), ValueError),
    (dict(w=torch.zeros(8, 5)), ValueError), (dict(w=torch.zeros(8, 1)), ValueError), (dict(bias=torch.zeros(9)), ValueError), (dict(bias=torch.zeros(8, dtype=torch.bfloat16)), TypeError),
    (dict(starts=torch.zeros(4, 2)), TypeError), (dict(starts=torch.zeros(4, 3, dtype=torch.uint8)), ValueError), (dict(lengths=torch.zeros(2, dtype=torch.int64)), TypeError),
    (dict(window_in=torch.zeros(2, 4, 8)), ValueError), (dict(activation="tanh"), KeyError), (dict(y=torch.zeros(4, 2, 8, dtype=torch.bfloat16)), TypeError),
    (dict(x=torch.zeros(4, 2, 16)[..., ::2]), ValueError), (dict(x=torch.zeros(2, 4, 8).transpose(0, 1)), ValueError), (dict(x=torch.zeros(1, 1, 8).expand(4, 2, 8)), ValueError),
    (dict(x=torch.zeros(0, 2, 8)), ValueError), (dict(), ValueError)])                # the last: nothing wrong but that they are not on a GPU
def test_tensors_of_the_convolution(kw, error):
    with pytest.raises(error):
        hts.hts_causal_conv(**conv_tensors(**kw))


def test_tensors_of_the_others():
    z = torch.zeros
    x = z(4, 2, 8)
    good = dict(x=x, dt=x, a=z(8, 16), b=z(4, 2, 16), c=z(4, 2, 16), d=None, dt_bias=None, z=None, starts=None, lengths=None, state_in=None, softplus=True, y=z(4, 2, 8), state_out=None,
                workspace=None, stream=0)
    for kw, error in ((dict(dt=z(4, 2, 9)), ValueError), (dict(b=z(4, 2, 15)), ValueError), (dict(a=z(9, 16)), ValueError), (dict(a=z(8)), ValueError), (dict(state_in=z(2, 8, 15)), ValueError),
                      (dict(b=z(4, 2, 16).bfloat16()), TypeError), (dict(workspace=5), TypeError), (dict(), ValueError)):
        with pytest.raises(error):
            hts.hts_selective_scan(**{**good, **kw})
    step = dict(x=z(2, 8), dt=z(2, 8), a=z(8, 16), b=z(2, 16), c=z(2, 16), d=None, dt_bias=None, z=None, starts=None, slots=None, state_in=z(3, 8, 16), softplus=True, y=z(2, 8),
                state_out=z(3, 8, 16), stream=0)
    for kw, error in ((dict(state_in=None), TypeError), (dict(state_out=z(2, 8, 16)), ValueError), (dict(slots=z(2)), TypeError), (dict(), ValueError)):
        with pytest.raises(error):
            hts.hts_selective_scan_step(**{**step, **kw})
    h = lambda *s: z(*s, dtype=torch.bfloat16)
    lin = dict(x=h(4, 8), w=h(16, 8), bias=None, residual=None, activation="none", y=h(4, 16), pre=None, workspace=None, stream=0)
    for kw, error in ((dict(x=z(4, 8)), TypeError), (dict(w=h(16, 9)), ValueError), (dict(w=h(8, 16).t()), ValueError), (dict(y=h(4, 15)), ValueError), (dict(residual=h(3, 16)), ValueError),
                      (dict(), ValueError)):
        with pytest.raises(error):
            hts.hts_linear(**{**lin, **kw})
    grad = dict(x=h(4, 8), w=h(16, 8), pre=None, dy=h(4, 16), activation="none", dx=None, dw=z(16, 8, dtype=torch.int32), dbias=None, workspace=None, stream=0)
    with pytest.raises(TypeError):
        hts.hts_linear_gradient(**grad)
    with pytest.raises(TypeError):                       # not a dict
        hts.hts_selective_scan_gradient(**{k: None if k in ("y", "state_out") else v for k, v in good.items() if k not in ("y", "state_out")}, dy=x, dstate_out=None, grads=[])


def test_a_size_that_a_call_refuses_has_no_workspace():
    big = 1 << 30
    assert hts.hts_causal_conv_workspace(big + 1, 1, 8, 4) == hts.hts_causal_conv_workspace(4, big, 512, 4) == hts.hts_causal_conv_workspace(4, big + 1, 8, 4) == 0
    assert hts.hts_linear_workspace(big, 512, 8) == hts.hts_linear_workspace(8, big, 512, True) == hts.hts_linear_workspace(512, 8, big) == 0
    assert hts.hts_selective_scan_workspace(big, 2, 8, 16) == hts.hts_selective_scan_workspace(4, 1 << 21, 8, 16) == hts.hts_selective_scan_workspace(1 << 20, 16, 1 << 20, 16, True) == 0
    for sizes in (dict(T=4, N=big, channels=512, ld_x=512, ld_y=512), dict(T=4, N=big + 1), dict(T=big + 1)):
        assert conv(**sizes) == INVALID
    for sizes in (dict(rows=big, in_features=512, ld_x=512), dict(rows=512, out_features=big, ld_y=big, ld_pre=big, ld_residual=big)):
        assert linear_call(**sizes, bytes=1 << 60) == INVALID
    for sizes in (dict(T=big, N=2), dict(N=1 << 21)):
        assert scan_call(**sizes, bytes=1 << 60) == INVALID


def scan_tensors(**kw):
    z = torch.zeros
    return {**dict(x=z(4, 2, 8), dt=z(4, 2, 8), a=z(8, 16), b=z(4, 2, 16), c=z(4, 2, 16), d=None, dt_bias=None, z=None, starts=None, lengths=None, state_in=None, softplus=True, y=z(4, 2, 8),
                   state_out=None, workspace=None, stream=0), **kw}


def test_threads_do_not_see_each_others_tensors():
    """An argument that runs Python lets another thread's call in between the checks of this one, which reports its own first fault all the same."""
    import threading
    calls = []

    class Slow:
        def __bool__(self):
            def other():
                with pytest.raises(TypeError):
                    hts.hts_causal_conv(**conv_tensors(x=5))
                calls.append(1)
            t = threading.Thread(target=other)
            t.start()
            t.join()
            return True

    with pytest.raises(ValueError, match="x is not on a CUDA device"):
        hts.hts_selective_scan(**scan_tensors(softplus=Slow()))
    assert calls


@pytest.mark.parametrize("x,error", [(torch.zeros(4, 2, 8, device="meta"), "x is not"), (torch.zeros(4, 2, 8).to_sparse(), "x is not a tensor with memory"),
                                     (torch.zeros(4, 2, 8, dtype=torch.complex64), "element type"), (torch.zeros(4, 2, 8, dtype=torch.bool), "element type"),
                                     (torch.zeros(4, 2, 8, dtype=torch.int32), "element type"), (torch.zeros(4, 2, 8, dtype=torch.float64), "element type"),
                                     (torch.zeros(1, 1, 4, 2, 8), "shape"), (torch.zeros(()), "shape"), (torch.nn.Parameter(torch.zeros(4, 2, 8)), "x is not on a CUDA device"),
                                     (torch.zeros(4, 2, 16)[..., 3:11], "x is not on a CUDA device")])
def test_tensors_of_other_kinds(x, error):
    with pytest.raises((TypeError, ValueError), match=error):
        hts.hts_selective_scan(**scan_tensors(x=x))
    with pytest.raises((TypeError, ValueError), match="workspace is not|must be|x is not"):
        hts.hts_selective_scan(**scan_tensors(workspace="0"))


def test_workspaces_are_contiguous():
    with pytest.raises(AssertionError):
        hts.hts_selective_scan(**scan_tensors(workspace=torch.zeros(64, 2)[:, 0]))


def test_references_are_kept():
    """A refused call and its checks leave no reference behind and take none away."""
    import sys
    t = scan_tensors()
    before = {k: sys.getrefcount(v) for k, v in t.items() if isinstance(v, torch.Tensor)}
    for _ in range(100):
        with pytest.raises(ValueError):
            hts.hts_selective_scan(**t)
    assert before == {k: sys.getrefcount(v) for k, v in t.items() if isinstance(v, torch.Tensor)}
