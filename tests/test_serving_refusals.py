"""What the serving entry points refuse, on the CPU: their argument checks over a stub runtime (tests/serving_refusals.cpp), and the
checks of the Python binding."""
import os
import shutil
import subprocess

import pytest
import torch

import paper_2604_13327_amd as etc
import serving_ref as ref

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2604_13327_amd", "csrc")
HIP = "/opt/rocm/include"


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(HIP), reason="no compiler or HIP headers")
def test_argument_checks(tmp_path):
    exe = tmp_path / "serving_refusals"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           "-I", CSRC, "-I", HIP, "-o", str(exe), os.path.join(HERE, "serving_refusals.cpp")])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr


def test_create_refuses_before_any_device_call():
    for change in ({"d": 96}, {"nq": 5, "nkv": 2}, {"page": 12}, {"vocab": -1}):
        with pytest.raises(etc.EtcError) as e:
            etc.Serving(ref.shape(**change), 1, 1, 1)
        assert e.value.status == -1
    for limits in ((0, 1, 1), (1, 0, 1), (1, 1, 0), (2000, 1, 1)):
        with pytest.raises(etc.EtcError):
            etc.Serving(ref.shape(), *limits)


def test_binding_takes_gpu_tensors_only():
    from paper_2604_13327_amd.binding import _tensor
    with pytest.raises(ValueError, match="current GPU"):
        _tensor(torch.zeros(3), "x", ("float32",), (3,))


def test_binding_checks(monkeypatch):
    from paper_2604_13327_amd import binding

    class Fake:
        """A CPU tensor that says it is on the GPU."""
        def __init__(self, t):
            self.t, self.is_cuda, self.device = t, True, type("D", (), {"index": 0})
        def __getattr__(self, name):
            return getattr(self.t, name)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    t = torch.zeros(4, 6)
    assert binding._tensor(Fake(t), "x", ("float32",), (4, 6)) == t.data_ptr()
    assert binding._tensor(Fake(t[:, :3]), "x", ("float32",), (None, 3), strided=True) == t.data_ptr()
    for bad, kw in ((t.double(), {}), (t[:3], {}), (t.t().contiguous().t(), {}), (t[:, None], {}), (t[:, ::2], {"shape": (4, 3), "strided": True})):
        with pytest.raises(ValueError):
            binding._tensor(Fake(bad), "x", ("float32",), kw.pop("shape", (4, 6)), **kw)
