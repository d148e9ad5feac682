"""The binding of the microscaled 4-bit entry points without a GPU."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_training_needs_no_private_name_of_torch():
    """The network module imports where torch does not give the current stream as a number."""
    code = ("import torch\n"
            "for name in ('_cuda_getCurrentRawStream', '_cuda_getDevice'):\n"
            "    if hasattr(torch._C, name): delattr(torch._C, name)\n"
            "from paper_2106_05373_amd import mx, pipeline\n"
            "class Current:\n"
            "    def __init__(self, device): self.cuda_stream = 100 + device\n"
            "torch.cuda.current_stream = Current\n"
            "assert mx._raw_stream(3) == 103 and mx._current_device is torch.cuda.current_device\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr


def _tensor(device, *shape):
    """A tensor that says it is on a GPU that is not there."""
    import torch

    class Elsewhere(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return device

    return torch.zeros(shape).as_subclass(Elsewhere)


def test_a_layer_runs_on_its_own_device_whichever_is_current(monkeypatch):
    import contextlib
    import types
    import pytest
    import torch
    from paper_2106_05373_amd import bcpnn, mx
    current, calls = [0], []

    @contextlib.contextmanager
    def device(index):
        before, current[0] = current[0], index
        yield
        current[0] = before

    def entry(*args):
        calls.append(current[0])
        return 0

    for name in ("bcpnn_mx_from_layer", "bcpnn_mx_forward", "bcpnn_mx_readout", "bcpnn_mx_predict"):
        monkeypatch.setattr(mx.lib, name, entry)
    for name in ("_forward", "_readout", "_predict"):
        monkeypatch.setattr(mx, name, entry, raising=False)
    monkeypatch.setattr(mx, "_current_device", lambda: current[0])
    monkeypatch.setattr(mx.torch.cuda, "device", device)
    stream = types.SimpleNamespace(device_index=1, cuda_stream=7)
    trained = types.SimpleNamespace(_h=None, cfg=bcpnn.default_config(8, 2, 3, 4, 16), stream=stream)
    x, y, s, z = _tensor(1, 5, 16), _tensor(1, 5, 12), _tensor(1, 5, 12), _tensor(0, 5, 12)
    win, one = _tensor(1, 5, 3).int(), _tensor(1, 5).int()
    layer = mx.Layer.of(trained)
    layer.forward(x, y)
    layer.forward(x, y, s)
    layer.readout(x, win)
    layer.predict_with(layer, x, y, one)
    assert calls == [1] * 5 and current == [0]
    for args in ((_tensor(0, 5, 16), y, s), (x, z, s), (x, y, z)):
        with pytest.raises(ValueError):
            layer.forward(*args)
    with pytest.raises(ValueError):
        layer.readout(x, _tensor(0, 5, 3).int())
    with pytest.raises(ValueError):
        layer.predict_with(layer, x, z, one)
    with pytest.raises(TypeError):
        layer.forward(torch.zeros(5, 16), y)
    assert len(calls) == 5
