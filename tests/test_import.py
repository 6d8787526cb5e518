"""The package without the compiled part of its binding (not built, or built for another
torch): everything but the calls that need it is there, and those say why they are not."""
import os
import shutil
import subprocess
import sys

import pytest

pdn = pytest.importorskip("paper_2604_21100_amd", reason="libpdn.so not built")
torch = pytest.importorskip("torch")

PROGRAM = """
import torch, paper_2604_21100_amd as pdn
n = pdn.pdn_workspace_size(pdn.make_problem(1, 64, 2, 128, 128, gate="scalar"))
assert n > 0 and pdn.pdn_draft_verify_workspace_size(2, 100) > 0 and callable(pdn.pdn_chunk_fwd)
z, i = torch.zeros, torch.zeros(2, dtype=torch.int32)
rows, S = z(2, 2, 64), z(2, 2, 64, 64)
calls = [lambda: pdn.pdn_slot_fwd(rows, rows, rows, z(2, 2), S, precond="identity"),
         lambda: pdn.pdn_slot_draft(rows, rows, rows, z(2, 2), S, z(2, 1, 2, 132), z(2, 2), precond="identity"),
         lambda: pdn.pdn_draft_verify(z(2, 9), i, z(2), z(2))]
for call in calls:
    try:
        call()
    except ImportError as e:
        assert "_pdn_torch" in str(e) and "build" in str(e), e
    else:
        raise AssertionError("no ImportError")
print("fine")
"""


@pytest.mark.parametrize("there", ["missing", "no library"])
def test_without_the_compiled_binding(tmp_path, there):
    at = os.path.dirname(os.path.abspath(pdn.__file__))
    new = tmp_path / "paper_2604_21100_amd"
    new.mkdir()
    shutil.copy(os.path.join(at, "__init__.py"), new)
    os.symlink(os.path.join(at, "libpdn.so"), new / "libpdn.so")
    if there != "missing":
        (new / "_pdn_torch.so").write_bytes(b"built for something else")
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=tmp_path, capture_output=True, text=True, timeout=300,
                       env={**os.environ, "PYTHONPATH": str(tmp_path)})
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-2000:]
