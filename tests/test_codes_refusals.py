"""What the entry points of the cache of codes and of the scores refuse, on the CPU (tests/codes_refusals.cpp), and what the Python
binding does; a library from before they were there loads."""
import os
import shutil
import subprocess
from types import SimpleNamespace

import pytest
import torch

import paper_2604_13327_amd as etc
import serving_ref as ref
from paper_2604_13327_amd import binding

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(HERE, "..", "paper_2604_13327_amd", "csrc")
HIP = "/opt/rocm/include"


@pytest.mark.skipif(shutil.which("g++") is None or not os.path.isdir(HIP), reason="no compiler or HIP headers")
def test_argument_checks(tmp_path):
    exe = tmp_path / "codes_refusals"
    subprocess.check_call(["g++", "-O1", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-fsanitize=undefined", "-fno-sanitize-recover=all",
                           "-I", CSRC, "-I", HIP, "-o", str(exe), os.path.join(HERE, "codes_refusals.cpp")])
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0 and out.stdout == "ok\n", out.stdout + out.stderr


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no compiler")
def test_library_of_the_first_serving_operators_loads(tmp_path):
    """One that the front end generated before there were codes and scores."""
    newer = ("etc_serving_append_codes", "etc_serving_attention_codes", "etc_serving_score")
    src = tmp_path / "old.c"
    src.write_text("".join(f"int {name}(void) {{ return 0; }}\n" for name in binding.EXPORTS if name not in newer))
    subprocess.check_call(["gcc", "-shared", "-fPIC", "-o", str(tmp_path / "libold.so"), str(src)])
    L = binding.load_library(str(tmp_path / "libold.so"))
    assert L.etc_serving_sample.argtypes and not any(hasattr(L, name) for name in newer)


class OnGpu:
    """A CPU tensor that says it is on GPU 0."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)

    def get_device(self):
        return 0


def _serving(vocab=50):
    """The binding without a handle: calls end in a list."""
    s = object.__new__(etc.Serving)
    called = []
    s._h, s._device, s.shape = None, 0, ref.shape(4, 2, 64, vocab=vocab)
    s._L = SimpleNamespace(etc_serving_append_codes="append", etc_serving_attention_codes="attention", etc_serving_score="score")
    s._i32, s._f32, s._bf16, s._float = (torch.int32,), (torch.float32,), (torch.bfloat16,), (torch.bfloat16, torch.float32)
    s._code = {torch.bfloat16: 0, torch.float32: 1}
    s._f8, s._e8 = (torch.float8_e4m3fn,), (torch.float8_e8m0fnu, torch.uint8)
    s._call = lambda fn, io, stream: called.append((fn, io))
    return s, called


def _z(*shape, dtype=torch.int32):
    return OnGpu(torch.zeros(*shape, dtype=torch.uint8).to(dtype) if dtype != torch.float8_e8m0fnu else torch.zeros(*shape, dtype=torch.uint8).view(dtype))


def test_binding_checks():
    s, called = _serving()
    bf, f8, e8, f32 = torch.bfloat16, torch.float8_e4m3fn, torch.float8_e8m0fnu, torch.float32
    q, k, v, slots, out = _z(3, 256, dtype=bf), _z(3, 128, dtype=bf), _z(3, 128, dtype=bf), _z(3), _z(3, 4, 64, dtype=bf)
    kp, vp, ks, vs = _z(5, 16, 2, 64, dtype=f8), _z(5, 16, 2, 64, dtype=f8), _z(5, 2, dtype=e8), _z(5, 2, dtype=torch.uint8)
    good = [q, k, v, slots, slots, out, kp, vp, ks, vs]
    s.append_codes(*good)
    assert called[-1][0] == "append" and called[-1][1].append.n_pages == 5 and called[-1][1].k_scale == ks.data_ptr() and called[-1][1].append.k_pages == kp.data_ptr()
    for at, bad in ((6, _z(5, 16, 2, 64, dtype=bf)), (7, _z(5, 16, 2, 64, dtype=torch.uint8)), (8, _z(4, 2, dtype=e8)), (9, _z(5, 2, dtype=f32)), (8, ks.t), (3, _z(4)), (5, q)):
        with pytest.raises(ValueError):
            s.append_codes(*[bad if i == at else x for i, x in enumerate(good)])
    table, lens, indptr = _z(2, 9), _z(2), _z(3)
    good = [out, _z(3, 4, 64, dtype=bf), indptr, lens, table, kp, vp, ks, vs]
    s.attention_codes(*good)
    assert called[-1][0] == "attention" and called[-1][1].attention.n_seqs == 2 and called[-1][1].v_scale == vs.data_ptr()
    for at, bad in ((5, _z(5, 16, 2, 64, dtype=bf)), (6, _z(5, 8, 2, 64, dtype=f8)), (7, _z(2, 5, dtype=e8)), (8, _z(5, 2)), (2, _z(2))):
        with pytest.raises(ValueError):
            s.attention_codes(*[bad if i == at else x for i, x in enumerate(good)])
    logits, tokens, lp = _z(3, 50, dtype=f32), _z(3), _z(3, dtype=f32)
    ids, tops = _z(3, 7), _z(3, 7, dtype=f32)
    s.score(logits, tokens, lp, entropy_out=lp, top_ids=ids, top_logprobs=tops)
    assert called[-1][0] == "score" and called[-1][1].n_top == 7 and called[-1][1].row_stride == 50
    s.score(OnGpu(torch.zeros(3, 99, dtype=bf)[:, 3:53]), entropy_out=lp)
    assert called[-1][1].row_stride == 99 and called[-1][1].n_top == 0 and called[-1][1].tokens is None
    for kw in ({"tokens": _z(4)}, {"logprob_out": _z(3)}, {"entropy_out": _z(3, 1, dtype=f32)}, {"top_ids": tops}, {"top_ids": ids, "top_logprobs": _z(3, 6, dtype=f32)}):
        with pytest.raises(ValueError):
            s.score(logits, **{"tokens": tokens, "logprob_out": lp, **kw})
    with pytest.raises(ValueError):
        s.score(_z(3, 51, dtype=f32), tokens, lp)
    assert len(called) == 4


@pytest.mark.parametrize("missing", [(), ("float8_e8m0fnu",), ("float8_e8m0fnu", "float8_e4m3fn")])
def test_a_torch_without_types_of_8_bits(monkeypatch, missing):
    """A handle is made and its other operators work; scales may be bytes; what needs a type that is not there is refused."""
    calls = []
    names = [n for n in binding.EXPORTS if n.startswith("etc_serving_")]
    stub = SimpleNamespace(**{n: (lambda *a, n=n: calls.append(n) or 0) for n in names})
    monkeypatch.setattr(binding, "lib", lambda: stub)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    bf, f8 = torch.bfloat16, torch.float8_e4m3fn
    q, k, slots, out = _z(3, 256, dtype=bf), _z(3, 128, dtype=bf), _z(3), _z(3, 4, 64, dtype=bf)
    pool, codes, scale = _z(5, 16, 2, 64, dtype=bf), _z(5, 16, 2, 64, dtype=f8), _z(5, 2, dtype=torch.uint8)
    logits, entropy, out2, one, table = _z(3, 50, dtype=torch.float32), _z(3, dtype=torch.float32), _z(3, 4, 64, dtype=bf), _z(1), _z(1, 5)
    indptr = _z(2)
    for name in missing:
        monkeypatch.delattr(torch, name)
    s = etc.Serving(ref.shape(4, 2, 64, vocab=50), max_seqs=1, max_tokens=3, max_kv_len=9)
    stream = SimpleNamespace(cuda_stream=None)
    s.append(q, k, k, slots, slots, out, pool, pool, stream=stream)
    s.score(logits, entropy_out=entropy, stream=stream)
    assert calls[-2:] == ["etc_serving_append", "etc_serving_score"]
    many = len(calls)
    if "float8_e4m3fn" in missing:
        with pytest.raises(ValueError, match="k_pages"):
            s.append_codes(q, k, k, slots, slots, out, codes, codes, scale, scale, stream=stream)
        with pytest.raises(ValueError, match="k_pages"):
            s.attention_codes(out, out2, indptr, one, table, codes, codes, scale, scale, stream=stream)
        assert len(calls) == many
    else:
        s.append_codes(q, k, k, slots, slots, out, codes, codes, scale, scale, stream=stream)
        assert calls[many:] == ["etc_serving_append_codes"]
    s.close()
