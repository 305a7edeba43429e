"""Where the binding's native part finds the HIP headers, whatever HIPCC is called by."""
import os

import pytest

from paper_2603_19133_amd import build


@pytest.mark.parametrize("name", ["/opt/rocm/bin/hipcc", "hipcc", "no-such-compiler"])
def test_hip_headers_are_found(monkeypatch, name):
    monkeypatch.setattr(build, "HIPCC", name)
    monkeypatch.setenv("PATH", "/opt/rocm/bin" + os.pathsep + os.environ["PATH"])
    monkeypatch.delenv("ROCM_PATH", raising=False)
    path = build.hip_include()
    assert os.path.isabs(path) and os.path.isfile(os.path.join(path, "hip", "hip_runtime_api.h"))


def test_the_native_part_is_compiled_with_them(monkeypatch):
    """The command that build_native would run, by a compiler's bare name."""
    seen = []

    class Done:
        returncode = 0
    monkeypatch.setattr(build, "HIPCC", "hipcc")
    monkeypatch.setenv("PATH", "/opt/rocm/bin" + os.pathsep + os.environ["PATH"])
    monkeypatch.setattr(build.subprocess, "run", lambda cmd, **kw: seen.append(cmd) or Done)
    build.build_native()
    dirs = [a[2:] for a in seen[0] if a.startswith("-I")]
    assert all(os.path.isabs(d) for d in dirs) and any(os.path.isfile(os.path.join(d, "hip", "hip_runtime_api.h")) for d in dirs)
