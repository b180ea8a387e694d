"""The calls around the planner refuse what they cannot answer: inputs whose
gradient they would lose, shapes without the dimensions they need, tensors of
several devices."""
import contextlib
import types

import pytest
import torch

import paper_2608_03676_amd as taot

gpu_test = pytest.mark.gpu


def _calls(gpu):
    """name -> (call, its floating inputs)"""
    T, H, E, k = 4, 16, 8, 2
    f = {n: torch.ones(s, device=gpu) for n, s in dict(
        x=(T, H), residual=(T, H), weight=(H,), dy=(T, H), dh=(T, H), h=(T, H), rstd=(T,), logits=(T, E), bias=(E,),
        dweights=(T, k), rows=(T, H), scale=(T, 1), y=(T * k, H), weights=(T * k,), dout=(T, H)).items()}
    ids = torch.arange(T * k, dtype=torch.int32, device=gpu).view(T, k) % E
    pos = torch.arange(T * k, dtype=torch.int32, device=gpu)
    return f, {
        "add_rms_norm": (lambda a: taot.add_rms_norm(a["x"], a["weight"], 1e-6, residual=a["residual"]),
                         ("x", "weight", "residual")),
        "add_rms_norm_backward": (lambda a: taot.add_rms_norm_backward(a["dy"], a["h"], a["rstd"], a["weight"], dh=a["dh"]),
                                  ("dy", "h", "rstd", "weight", "dh")),
        "route": (lambda a: taot.route(a["logits"], k, bias=a["bias"]), ("logits", "bias")),
        "route_backward": (lambda a: taot.route_backward(a["dweights"], a["logits"], ids), ("dweights", "logits")),
        "dispatch_rows": (lambda a: taot.dispatch_rows(a["rows"], pos, scale=a["scale"]), ("rows", "scale")),
        "combine_rows": (lambda a: taot.combine_rows(a["y"], pos, weights=a["weights"], top_k=k), ("y", "weights")),
        "combine_rows_backward": (lambda a: taot.combine_rows_backward(a["dout"], a["y"], pos, a["weights"]),
                                  ("dout", "y", "weights"))}


@gpu_test
def test_inputs_that_want_a_gradient(gpu):
    """The results carry no gradient: refused while gradients are recorded, taken under no_grad and when detached."""
    f, calls = _calls(gpu)
    for name, (call, inputs) in calls.items():
        call(f)
        for i in inputs:
            a = dict(f, **{i: f[i].clone().requires_grad_()})
            with pytest.raises(RuntimeError, match=i if i != "rows" else "x"):
                call(a)
            with torch.no_grad():
                call(a)
            call(dict(f, **{i: a[i].detach()}))


@gpu_test
def test_what_lacks_a_dimension_or_is_no_tensor(gpu):
    f, _ = _calls(gpu)
    x, w, logits, y = f["x"], f["weight"], f["logits"], f["y"]
    pos = torch.arange(8, dtype=torch.int32, device=gpu)
    ids = torch.zeros((4, 2), dtype=torch.int32, device=gpu)
    one, zero_dim = torch.ones(8, device=gpu), torch.zeros((), dtype=torch.int32, device=gpu)
    for call in (lambda: taot.dispatch_rows(x[0], pos), lambda: taot.dispatch_rows(x, zero_dim),
                 lambda: taot.dispatch_rows(x, pos, scale=one[0]), lambda: taot.dispatch_rows(one[0], pos),
                 lambda: taot.combine_rows(one, pos), lambda: taot.combine_rows(one, zero_dim),
                 lambda: taot.combine_rows(one[0], zero_dim), lambda: taot.combine_rows_backward(one, y, pos, f["weights"]),
                 lambda: taot.combine_rows_backward(x, one, pos, f["weights"]),
                 lambda: taot.combine_rows_backward(x, one, zero_dim, f["weights"]),
                 lambda: taot.combine_rows_backward(one[0], one[0], zero_dim, one[0]),
                 lambda: taot.route_backward(f["dweights"], logits, zero_dim),
                 lambda: taot.dispatch_map(ids[None], pos, ids, zero_dim, 1),
                 lambda: taot.dispatch_map(zero_dim, pos, ids, ids[None], 1)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: taot.add_rms_norm(x, None, 1e-6), lambda: taot.add_rms_norm(x, 1.0, 1e-6),
                 lambda: taot.add_rms_norm_backward(x, x, f["rstd"], None), lambda: taot.add_rms_norm_backward(None, x, f["rstd"], w),
                 lambda: taot.add_rms_norm_backward(x, x, f["rstd"], w, workspace=1 << 20),
                 lambda: taot.route_backward(f["dweights"], logits, None), lambda: taot.route_backward(None, logits, ids),
                 lambda: taot.dispatch_rows(x, None), lambda: taot.combine_rows(y, None),
                 lambda: taot.combine_rows_backward(x, y, pos, None)):
        with pytest.raises(TypeError):
            call()


def _stand_in(index):
    return types.SimpleNamespace(get_device=lambda: index, device_index=index, requires_grad=False)


def test_tensors_of_several_devices(monkeypatch):
    """The checks alone, on the CPU: one device for all tensors and the stream."""
    monkeypatch.setattr(taot, "_devices", 2)
    a, b = _stand_in(0), _stand_in(1)
    taot._inputs("f", "x w", None, a, a)
    taot._inputs("f", "x w", a, a, None)
    with pytest.raises(ValueError, match="w is on cuda:1, x on cuda:0"):
        taot._inputs("f", "x y w", None, a, None, b)
    with pytest.raises(ValueError, match="the stream is of cuda:1"):
        taot._inputs("f", "x", b, a)
    taot._on(a, "out", torch.device("cuda:0"))
    with pytest.raises(ValueError, match="out is on cuda:1"):
        taot._on(b, "out", torch.device("cuda:0"))


@pytest.mark.parametrize("device,current", [(0, 0), (1, 0), (2, 1)])
def test_a_launch_goes_to_the_tensors_device(monkeypatch, device, current):
    """On the CPU, with a library that notes the device that is current when it is called."""
    now, seen = [current], []

    @contextlib.contextmanager
    def switch(d):
        was, now[0] = now[0], d.index
        yield
        now[0] = was

    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: now[0], raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: 100 + i, raising=False)
    monkeypatch.setattr(torch.cuda, "device", switch)
    fake = types.SimpleNamespace(f=lambda *a: seen.append((now[0], a)) or 0)
    monkeypatch.setattr(taot, "lib", lambda: fake)
    monkeypatch.setattr(taot, "_devices", 3)
    taot._launch("f", torch.device("cuda", device), None, 1, 2)
    taot._launch("f", torch.device("cuda", device), types.SimpleNamespace(cuda_stream=7), 3)
    assert seen == [(device, (1, 2, 100 + device)), (device, (3, 7))] and now == [current]
