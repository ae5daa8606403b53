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


class OnGpu:
    """A CPU tensor that says it is on GPU 0."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


def test_binding_checks():
    from paper_2604_13327_amd.binding import _rows, _tensor
    f32 = (torch.float32,)
    t = torch.zeros(4, 6)
    assert _tensor(OnGpu(t), "x", f32, (4, 6), 0) == t.data_ptr()
    for bad in (t, OnGpu(t.double()), OnGpu(t[:3]), OnGpu(torch.zeros(6, 4).t()), OnGpu(t[:, None]), OnGpu(torch.zeros(4, 12)[:, ::2])):
        with pytest.raises(ValueError):
            _tensor(bad, "x", f32, (4, 6), 0)
    with pytest.raises(ValueError):
        _tensor(OnGpu(t), "x", f32, (4, 6), 1)
    wide = torch.zeros(4, 9)
    assert _rows(OnGpu(wide[:, 1:4]), "x", f32, (4, 3), 0) == (wide.data_ptr() + 4, 9)
    assert _rows(OnGpu(wide[:1, :3]), "x", f32, (1, 3), 0)[1] >= 3
    for bad in (wide[:, :3], OnGpu(wide[:, ::3]), OnGpu(wide[:, :4]), OnGpu(wide[:, :3].int())):
        with pytest.raises(ValueError):
            _rows(bad, "x", f32, (4, 3), 0)
