"""The Python binding's use of torch, checked without a GPU."""
import os
import subprocess
import sys
import types

from paper_2502_01681_b200 import dg4

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WITHOUT_TORCH = """
import sys
sys.modules["torch"] = None                     # importing it raises
from paper_2502_01681_b200 import dg4
assert dg4.load().dg4_status_string(dg4.DG4_OK)
try:
    dg4.dg4_graph_create([1, 1, 2], [0], [0, 1], 1)
except dg4.Dg4Error as e:
    assert e.status == dg4.DG4_ERR_NOT_SORTED
else:
    raise AssertionError("a malformed circuit was taken")
assert dg4.desc(8, dg4.DG4_BF16, 0.25).heads == 8
"""


def test_the_library_loads_and_checks_circuits_without_torch():
    out = subprocess.run([sys.executable, "-c", WITHOUT_TORCH], cwd=ROOT, capture_output=True, text=True)
    assert out.returncode == 0, out.stderr


def test_current_stream_with_and_without_the_raw_handle(monkeypatch):
    cuda = types.SimpleNamespace(current_device=lambda: 3,
                                 current_stream=lambda: types.SimpleNamespace(cuda_stream=41))
    fake = types.SimpleNamespace(_C=types.SimpleNamespace(), cuda=cuda)
    monkeypatch.setattr(dg4, "_torch_module", fake)
    assert dg4._stream(None) == 41
    fake._C._cuda_getCurrentRawStream = lambda device: 100 + device
    assert dg4._stream(None) == 103
    assert dg4._stream(types.SimpleNamespace(cuda_stream=7)) == 7 and dg4._stream(9) == 9
