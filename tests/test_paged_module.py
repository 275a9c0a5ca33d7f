"""`_paged` belongs to one torch: without it the paged calls raise, and everything else is there."""
import os
import subprocess
import sys

import paper_2510_25600_b200
from paper_2510_25600_b200 import build

ROOT = os.path.dirname(os.path.dirname(paper_2510_25600_b200.__file__))
WITHOUT = """
import torch
torch.__version__ = "0.0.0"          # the module of this torch is not built
from paper_2510_25600_b200 import binding as P, paged
assert "sm_100a" in P.purekv_version() and P.purekv_decode_paged_ws_bytes(4, 0, 8, 2, 128) > 0
P.purekv_set_wait_limit_ns(0)
for call in (lambda: P.purekv_append_paged(None, None, None, None, None, None), lambda: P.purekv_decode_paged(torch.zeros(1, 1, 64), torch.zeros(1), None, None, None, out=torch.zeros(1))):
    try:
        call()
    except ImportError as e:
        assert "_paged" in str(e) and e.__cause__ is not None
    else:
        raise SystemExit("a paged call without its module")
"""


def test_another_torch_has_all_calls_but_the_paged_ones():
    subprocess.run([sys.executable, "-c", WITHOUT], check=True, cwd=ROOT)


def test_a_torch_without_cuda_builds_the_rest(tmp_path, monkeypatch, capsys):
    monkeypatch.setattr(build, "_TORCH", str(tmp_path))
    monkeypatch.setattr(build, "PAGED", str(tmp_path / "_paged.so"))
    monkeypatch.setattr(build, "_stale", lambda target, deps: target == build.PAGED)   # (nothing else is compiled here)
    assert build.build() == build.LIB
    assert not os.path.exists(build.PAGED) and "_paged" in capsys.readouterr().err
