"""The library without the module of the serving calls (host only)."""
import os
import shutil
import subprocess
import sys

from paper_2502_06786_b200 import binding as mq
from paper_2502_06786_b200 import build

PACKAGE = os.path.dirname(mq.lib_path())


def _copy(tmp_path):
    to = tmp_path / os.path.basename(PACKAGE)
    to.mkdir()
    for f in os.listdir(PACKAGE):
        if f.endswith(".py"):
            shutil.copy(os.path.join(PACKAGE, f), to / f)
    os.symlink(mq.lib_path(), to / "libmatq.so")
    return to


def _run(tmp_path, code):
    return subprocess.run([sys.executable, "-c", code], cwd=tmp_path, env={**os.environ, "PYTHONPATH": str(tmp_path)}, capture_output=True, text=True, timeout=300)


USE = """
from paper_2502_06786_b200 import binding as mq
assert mq.packed_row_bytes(2304, 4) == 1152 and mq.version() >= 100 and mq.gemv_grouped_launches(mq.gemv_group([])) == 0
assert mq.attn_paged_workspace_bytes(1, 1, 8, 2, 128, 1, 64) == 0
import torch
x = torch.zeros(4, 64, dtype=torch.bfloat16)
try:
    mq.quantize_tokens(x)
except ImportError as e:
    assert "_serving" in str(e) and "build" in str(e), e
    print("as told")
"""


def test_the_older_calls_need_the_library_only(tmp_path):
    _copy(tmp_path)
    out = _run(tmp_path, USE)
    assert out.returncode == 0 and out.stdout.strip() == "as told", out.stderr


def test_a_module_for_another_torch_is_told_of_when_it_is_used(tmp_path):
    (_copy(tmp_path) / "_serving.so").write_bytes(b"not a module")
    out = _run(tmp_path, USE)
    assert out.returncode == 0 and out.stdout.strip() == "as told", out.stderr


def test_the_library_alone_is_up_to_date_without_the_module(monkeypatch, tmp_path):
    monkeypatch.setattr(build, "MODULE", str(tmp_path / "missing.so"))
    newest = max(os.path.getmtime(os.path.join(build.CSRC, f)) for f in os.listdir(build.CSRC))
    lib = tmp_path / "libmatq.so"
    lib.write_bytes(b"")
    os.utime(lib, (newest + 1e6, newest + 1e6))
    monkeypatch.setattr(build, "LIB", str(lib))
    assert not build._stale(serving=False) and build._stale()
