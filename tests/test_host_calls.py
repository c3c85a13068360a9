"""The two ways a Python call reaches the library, the extension and ctypes: the same arguments arrive, the same calls are refused, and neither a missing C
compiler nor another interpreter's extension stands in the way.  No GPU: the library's functions are replaced by some that take notes."""
import ctypes as C
import importlib.machinery
import importlib.util
import os
import subprocess
import sys
import sysconfig

import pytest
import torch

import paper_1911_05146_b200 as hpf
from paper_1911_05146_b200 import binding, build

TYPES = (torch.float32, torch.bfloat16, torch.float16, torch.int32, torch.uint8)
HERE_DEVICE = -1                # what get_device() of a CPU tensor says: these stand for tensors on the current device


class Marshaller:
    def __init__(self, kind, device=HERE_DEVICE, status=0):
        self.seen = []
        self.functions = [C.CFUNCTYPE(C.c_int, *binding._SIGNATURES["hpf_" + n])(lambda *a, n=n: self.seen.append((n, a)) or status) for n in binding._CALLS]
        if kind == "ctypes":
            self.calls = binding._CtypesCalls()
        else:
            path = build.calls()
            loader = importlib.machinery.ExtensionFileLoader("_calls", path)
            self.calls = importlib.util.module_from_spec(importlib.util.spec_from_loader("_calls", loader))
            loader.exec_module(self.calls)
        self.refusals = []

        def refused(status, what, tensor):
            self.refusals.append((status, what))
            raise hpf.HpfError(status, what)
        self.calls.setup(refused, lambda: device, lambda d: 4096 + d, TYPES, tuple(C.cast(f, C.c_void_p).value for f in self.functions))


def _arguments(name, dtype=torch.bfloat16, grad=torch.float32):
    """One tensor of its own for every tensor that a call takes, and numbers that differ."""
    wanted = {"t": dtype, "g": grad, "i": torch.int32, "f": torch.float32, "s": torch.uint8}
    out, number = [], 3
    for s in binding._CALLS[name].split():
        arg, _, kind = s.partition(":")
        if not arg:
            continue
        if kind:
            out.append(torch.zeros(5 + len(out), dtype=wanted[kind]))
        elif arg in ("temperature", "alpha"):
            out.append(0.5 + number)
            number += 1
        else:
            out.append(number)
            number += 1
    return out + [None]


KINDS = ["c", "ctypes"]


@pytest.mark.parametrize("name", list(binding._CALLS))
@pytest.mark.parametrize("dtype", TYPES[:3])
def test_the_same_arguments_arrive(name, dtype):
    args = _arguments(name, dtype)
    for stream in (None, 77, type("Stream", (), {"cuda_stream": 78})()):
        args[-1] = stream
        both = []
        for kind in KINDS:
            m = Marshaller(kind)
            getattr(m.calls, name)(*args)
            both += m.seen
        assert both[0] == both[1]
    # what the library must get, from the order of its own arguments
    tensors = [a for a in args if isinstance(a, torch.Tensor)]
    got = both[0][1]
    assert [p for p in got if isinstance(p, int) and p > 1 << 20] == [t.data_ptr() for t in tensors]
    assert got[-1] == 78 and TYPES.index(dtype) in got
    if "scratch" in binding._CALLS[name]:
        assert got[-2] == tensors[-1].numel()


@pytest.mark.parametrize("name", list(binding._CALLS))
def test_missing_tensors_are_null(name):
    args = _arguments(name)
    for i in range(1, len(args) - 1):
        if isinstance(args[i], torch.Tensor):
            both = []
            for kind in KINDS:
                m = Marshaller(kind)
                getattr(m.calls, name)(*[None if j == i else a for j, a in enumerate(args)])
                both += m.seen
            assert both[0] == both[1] and any(v is None for v in both[0][1][:-1])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(binding._CALLS))
def test_the_same_calls_are_refused(name, kind):
    m = Marshaller(kind)
    args, names = _arguments(name), [s.partition(":")[0] for s in binding._CALLS[name].split() if s[0] != ":"]
    call = getattr(m.calls, name)
    for i, a in enumerate(args[:-1]):
        if isinstance(a, torch.Tensor):
            with pytest.raises(hpf.HpfError):
                call(*[torch.zeros(9, dtype=torch.float64) if j == i else b for j, b in enumerate(args)])
            assert m.refusals[-1] == (binding.ERR_INVALID, names[i])
        elif isinstance(a, int):
            with pytest.raises(OverflowError):
                call(*[1 << 70 if j == i else b for j, b in enumerate(args)])
            if names[i] not in ("rows", "ld", "ld_d", "ld_x", "ld_y"):
                with pytest.raises(OverflowError):
                    call(*[(1 << 31) if j == i else b for j, b in enumerate(args)])
        if isinstance(a, (int, float)):
            with pytest.raises(TypeError):
                call(*["3" if j == i else b for j, b in enumerate(args)])
    with pytest.raises(TypeError):
        call(*args[:-1])
    assert not m.seen
    other = Marshaller(kind, device=0)
    with pytest.raises(hpf.HpfError):
        getattr(other.calls, name)(*args)
    assert other.refusals == [(binding.ERR_INVALID, names[0])] and not other.seen


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("name", list(binding._CALLS))
def test_a_status_of_the_library_raises(name, kind):
    m = Marshaller(kind, status=-2)
    with pytest.raises(hpf.HpfError):
        getattr(m.calls, name)(*_arguments(name))
    assert m.refusals == [(-2, "")] and len(m.seen) == 1


def test_the_extension_is_named_after_its_interpreter():
    assert build.CALLS.endswith(sysconfig.get_config_var("EXT_SUFFIX")) and sysconfig.get_config_var("SOABI") in build.CALLS


@pytest.mark.parametrize("how", ["compiler", "headers"])
def test_the_library_needs_no_c_compiler_and_no_python_headers(how, tmp_path, monkeypatch):
    hpf.lib()                                                # the library is there and fresh
    monkeypatch.setattr(build, "CALLS", str(tmp_path / "_calls.so"))
    if how == "compiler":
        monkeypatch.setenv("CC", "/nowhere/cc")
    else:
        monkeypatch.setattr(build.sysconfig, "get_paths", lambda: {"include": str(tmp_path)})
    compiled = []
    monkeypatch.setattr(build, "_build_library", lambda verbose: compiled.append(verbose))
    with pytest.warns(UserWarning, match="marshalled by ctypes"):
        assert build.build() == build.LIB
    assert not compiled                                      # nothing of the library is compiled again for want of the extension
    with pytest.warns(UserWarning):
        assert build.calls() is None
    assert os.listdir(tmp_path) == []


def test_the_binding_falls_back(monkeypatch):
    monkeypatch.setattr(binding, "_calls", None)
    monkeypatch.setattr(build, "calls", lambda force=False: None)
    monkeypatch.setattr(torch.cuda, "init", lambda: None)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: HERE_DEVICE, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda d: 0, raising=False)
    assert isinstance(binding._fast(), binding._CtypesCalls)
    x = torch.zeros(1, 4)
    hpf.logprobs_fwd(x, None, None, None, None, None, None, 0, 4, 4)                     # an empty batch, in the real library
    with pytest.raises(hpf.HpfError) as e:
        hpf.logprobs_fwd(x, None, None, None, None, None, None, 1, 4, 3)
    assert e.value.status == binding.ERR_INVALID and "row stride" in str(e.value)


def test_an_extension_out_of_date_is_not_used(tmp_path, monkeypatch):
    """Compiled from an older py_calls.c and with no compiler to do it again: its calls may not be the library's any more."""
    old = tmp_path / "_calls.so"
    old.write_bytes(b"")
    os.utime(old, (1, 1))
    monkeypatch.setattr(build, "CALLS", str(old))
    monkeypatch.setenv("CC", "/nowhere/cc")
    with pytest.warns(UserWarning):
        assert build.calls() is None


def test_two_processes_may_compile_it_at_once(tmp_path):
    code = ("import sys; sys.path.insert(0, %r)\n"
            "from paper_1911_05146_b200 import build\n"
            "build.CALLS = %r\n"
            "assert build.calls(force=True) == build.CALLS\n") % (os.path.dirname(os.path.dirname(os.path.abspath(__file__))), str(tmp_path / "_calls.so"))
    both = [subprocess.Popen([sys.executable, "-c", code]) for _ in range(2)]
    assert [p.wait(300) for p in both] == [0, 0]
    assert os.listdir(tmp_path) == ["_calls.so"]
