"""The in-tree build: the library does without what only the block operators' binding needs."""

from __future__ import annotations

import ctypes
import os

import pytest

from paper_2604_05718_gb300 import build

KERNEL = """
#include <cuda_runtime.h>
__global__ void nothing() {}
extern "C" __attribute__((visibility("default"))) int mpm_small() { return 7; }
"""


@pytest.fixture
def tree(tmp_path, monkeypatch):
    """A source folder with one small .cu, built into its own place."""
    csrc = tmp_path / "csrc"
    csrc.mkdir()
    (csrc / "small.cu").write_text(KERNEL)
    (csrc / "exports.map").write_text("{ global: mpm_*; local: *; };\n")
    monkeypatch.setattr(build, "CSRC", str(csrc))
    monkeypatch.setattr(build, "BUILD", str(tmp_path / "_build"))
    monkeypatch.setattr(build, "LIB", str(tmp_path / "libmpm.so"))
    monkeypatch.setattr(build, "BINDING", str(tmp_path / "_blocks.so"))
    return tmp_path


def fail_on(monkeypatch, reason):
    if reason == "no compiler":
        monkeypatch.setenv("CXX", "/nonexistent/g++")
    elif reason == "does not compile":
        monkeypatch.setenv("CXX", "false")
    else:
        def without_torch(out):
            raise ModuleNotFoundError("No module named 'torch'")
        monkeypatch.setattr(build, "_binding_command", without_torch)


@pytest.mark.parametrize("reason", ["no compiler", "does not compile", "no torch"])
def test_the_library_is_built_where_the_binding_cannot_be(tree, monkeypatch, reason):
    (tree / "_blocks.so").write_bytes(b"of older sources")
    os.utime(tree / "_blocks.so", (1, 1))
    fail_on(monkeypatch, reason)
    with pytest.warns(RuntimeWarning, match="binding"):
        path = build.build()
    assert path == str(tree / "libmpm.so") and ctypes.CDLL(path).mpm_small() == 7
    assert not (tree / "_blocks.so").exists()      # an old one would be handed other entry points


def test_a_kernel_that_does_not_compile_ends_the_build(tree):
    (tree / "csrc" / "small.cu").write_text("this is no program")
    with pytest.raises(RuntimeError, match="command failed"):
        build.build()
    assert not (tree / "libmpm.so").exists()


def test_block_operators_say_that_the_binding_is_missing(monkeypatch):
    from paper_2604_05718_gb300 import blocks

    def missing(name, package):
        raise ImportError(name)

    build.build()
    monkeypatch.setattr(blocks, "_module", None)
    monkeypatch.setattr(blocks.importlib, "import_module", missing)
    with pytest.raises(RuntimeError, match="binding of the block operators"):
        blocks.matmul_mxfp4(blocks.MXFP4(None, None, 1), blocks.MXFP4(None, None, 1))


def test_the_binding_follows_the_torch_it_is_built_for(tree, monkeypatch):
    """Its ABI is that torch's: another one, or another command, builds it again; the same does not."""
    made = []

    def command(out):
        made.append(out)
        return ["sh", "-c", f"echo {len(made)} > '{out}'"]

    monkeypatch.setattr(build, "_binding_command", command)
    version = ["2.0"]
    monkeypatch.setattr(build, "_binding_key", lambda: f"torch {version[0]}", raising=False)
    binding = tree / "_blocks.so"
    build.build()
    assert binding.read_text() == "1\n"
    build.build()
    assert binding.read_text() == "1\n"
    version[0] = "2.1"
    build.build()
    assert binding.read_text() == "2\n"
    build.build()
    assert binding.read_text() == "2\n"


def test_the_binding_key_names_torch(monkeypatch):
    import torch

    key = build._binding_key()
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    assert build._binding_key() != key
