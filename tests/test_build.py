"""The library and the module that calls it on torch tensors are built, found stale and loaded independently of each other."""
import os
import stat
import subprocess
import sys

import pytest

from paper_2510_15312_b200 import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture
def tools(tmp_path, monkeypatch):
    """Compilers that write down that they were called, in the place of the real ones, and other places for what they make."""
    def tool(name, status=0):
        p = tmp_path / name
        p.write_text(f"#!/bin/sh\necho {name} >> {tmp_path}/calls\nwhile [ $# -gt 1 ]; do if [ \"$1\" = -o ] && [ {status} = 0 ]; then echo made > \"$2\"; fi; shift; done\nexit {status}\n")
        p.chmod(p.stat().st_mode | stat.S_IXUSR)
        return str(p)

    class Tools:
        lib, calls_path = str(tmp_path / "lib.so"), str(tmp_path / "calls.so")

        def calls(self):
            done = (tmp_path / "calls").read_text().split() if (tmp_path / "calls").exists() else []
            (tmp_path / "calls").write_text("")
            return sorted(done)

        def use(self, nvcc=0, cxx=0):
            monkeypatch.setenv("NVCC", tool("nvcc", nvcc))
            monkeypatch.setenv("CXX", tool("cxx", cxx))
    t = Tools()
    monkeypatch.setattr(B, "LIB_PATH", t.lib)
    monkeypatch.setattr(B, "TORCH_PATH", t.calls_path)
    # objects are written beside the sources: copies of these
    here = tmp_path / "pkg"
    (here / "csrc").mkdir(parents=True)
    (tmp_path / "include").mkdir()
    for s in B._SOURCES + B._TORCH_SOURCES:
        (here / "csrc" / s).write_text("// " + s)
    (tmp_path / "include" / "sdv.h").write_text("// sdv.h")
    monkeypatch.setattr(B, "_HERE", str(here))
    t.sources = here / "csrc"
    t.use()
    return t


def test_every_source_is_listed():
    have = {f for f in os.listdir(os.path.join(ROOT, "paper_2510_15312_b200", "csrc")) if not f.endswith(".o")}
    assert have == set(B._SOURCES + B._TORCH_SOURCES)


def test_each_is_rebuilt_for_its_own_reasons(tools, monkeypatch):
    import torch
    assert B.build() == tools.lib and tools.calls() == ["cxx", "nvcc", "nvcc", "nvcc"]
    assert B.build() == tools.lib and tools.calls() == []
    (tools.sources / "paged_torch.cpp").write_text("// another")
    B.build()
    assert tools.calls() == ["cxx"]
    (tools.sources / "dense.cuh").write_text("// another")
    B.build()
    assert tools.calls() == ["nvcc"] * 3
    monkeypatch.setattr(torch, "__version__", "0.0")     # another torch
    assert B.build_library() == tools.lib and tools.calls() == []
    B.build()
    assert tools.calls() == ["cxx"]


def test_a_module_that_cannot_be_built_does_not_keep_the_library_from_it(tools):
    tools.use(cxx=1)
    with pytest.raises(subprocess.CalledProcessError):
        B.build()
    assert os.path.exists(tools.lib) and not os.path.exists(tools.calls_path)
    tools.calls()
    assert B.build_library() == tools.lib and tools.calls() == []


def test_a_library_that_cannot_be_built(tools):
    tools.use(nvcc=1)
    with pytest.raises(subprocess.CalledProcessError):
        B.build()
    with pytest.raises(subprocess.CalledProcessError):
        B.build_library()
    assert not os.path.exists(tools.lib)


def python(code):
    out = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr[-2000:]


def test_the_package_does_not_load_torch():
    python("import sys, paper_2510_15312_b200 as p\nassert 'torch' not in sys.modules\np.lib()\np.rope_frequencies(8)\nassert 'torch' not in sys.modules")


def test_the_library_loads_where_there_is_no_torch():
    python("import sys\nsys.modules['torch'] = None\nimport paper_2510_15312_b200 as p\nassert p.lib().sdv_strerror(p.EINVAL)")
