"""Host side of the routing and 8-bit operators: a missing extension module, scratch sizes, arguments that are refused before
anything is allocated or launched."""
import ctypes
import os
import shutil
import subprocess
import sys

import pytest


@pytest.fixture(scope="module")
def mok():
    from paper_2609_36070_b200 import build
    build.build()
    from paper_2609_36070_b200 import mok
    return mok


def test_the_layer_imports_without_the_extension_module(mok, tmp_path):
    """... and the operators bound in it say how to build it."""
    from paper_2609_36070_b200 import build
    package = tmp_path / "paper_2609_36070_b200"
    package.mkdir()
    for name in os.listdir(build.PKG):
        if name.endswith(".py") or name == "libmok.so":
            shutil.copy(os.path.join(build.PKG, name), package)
    code = """
from paper_2609_36070_b200 import mok
assert mok.mok_i8_experts_workspace_bytes(4, 64, 64, 4, 2) > 0 and callable(mok.mok_moe_forward)
for call in (mok.mok_gate, mok.mok_gate_backward, mok.mok_i8_quantize, mok.mok_i8_linear, mok.mok_i8_matmul, mok.mok_i8_experts):
    try:
        call(None, 1)
    except ImportError as e:
        assert "paper_2609_36070_b200.build" in str(e)
    else:
        raise AssertionError(call)
"""
    env = {**os.environ, "PYTHONPATH": str(tmp_path)}
    done = subprocess.run([sys.executable, "-c", code], cwd=tmp_path, env=env, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr


def test_the_extension_module_is_rebuilt_for_another_torch(mok, tmp_path, monkeypatch):
    from paper_2609_36070_b200 import build
    calls = []

    def compiler(cmd, check):
        calls.append(cmd)
        open(cmd[cmd.index("-o") + 1], "w").close()

    monkeypatch.setattr(build, "BINDING", str(tmp_path / "_binding.so"))
    monkeypatch.setattr(build, "BINDING_FOR", str(tmp_path / "build" / "binding.torch"))
    monkeypatch.setattr(build.subprocess, "run", compiler)
    build.build_binding()
    build.build_binding()
    assert len(calls) == 1                                # up to date
    monkeypatch.setattr("importlib.metadata.version", lambda name: "0.0.1")
    build.build_binding()
    build.build_binding()
    assert len(calls) == 2


@pytest.mark.parametrize("E,k", [(300, 8), (62, 6), (11, 8), (511, 1), (128, 8), (1, 1), (512, 32)])
@pytest.mark.parametrize("H,I", [(2048, 768), (8, 8)])
def test_experts_scratch_never_shrinks_with_the_batch(mok, E, k, H, I):
    """A workspace for T tokens serves every smaller batch, over the thresholds of the tile sizes and of the schedules."""
    sizes = [mok.mok_i8_experts_workspace_bytes(T, H, I, E, k) for T in range(0, 120 * E // k + 40)]
    assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))
    T = 32768 // k
    near = [mok.mok_i8_experts_workspace_bytes(t, H, I, E, k) for t in range(T - 40, T + 40)]
    assert all(a <= b for a, b in zip(near, near[1:]))


def test_argument_names_without_a_utf8_form_are_refused(mok):
    code = """
from paper_2609_36070_b200 import mok
try:
    mok.mok_gate(1, 2, **{chr(0xd800): 3})
except TypeError as e:
    assert "unexpected argument" in str(e)
else:
    raise AssertionError
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    done = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True)
    assert done.returncode == 0, (done.returncode, done.stderr)


class Experts(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("x", "idx", "w", "gu", "gu_scales", "dn", "dn_scales", "dn_max", "add")] +
                [(n, ctypes.c_int64) for n in ("x_stride", "gu_stride", "dn_stride", "add_stride", "out_stride")] +
                [(n, ctypes.c_int32) for n in ("T", "H", "I", "E", "k", "type")] +
                [("out", ctypes.c_void_p), ("workspace", ctypes.c_void_p), ("workspace_bytes", ctypes.c_size_t), ("stream", ctypes.c_void_p)])


def test_scales_that_are_not_aligned_are_refused(mok):
    """(No workspace is given, so that nothing is launched whatever the check of the scales says.)"""
    from paper_2609_36070_b200 import build
    lib, A = ctypes.CDLL(build.LIB), 1 << 20              # A stands for an address
    good = dict(x=A, idx=A, w=A, gu=A, gu_scales=A, dn=A, dn_scales=A, dn_max=A, x_stride=64, gu_stride=64, dn_stride=32, out_stride=64,
                T=8, H=64, I=32, E=4, k=2, type=0, out=A, workspace=None, workspace_bytes=0)
    assert lib.mok_i8_experts(ctypes.byref(Experts(**good))) == mok.MOK_ERR_WORKSPACE
    for name in ("gu_scales", "dn_scales", "dn_max"):
        assert lib.mok_i8_experts(ctypes.byref(Experts(**{**good, name: A + 2}))) == mok.MOK_ERR_ALIGN, name
