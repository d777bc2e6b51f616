"""The training calls' argument checks that need no GPU: null handles at the C ABI, and what the binding refuses before it
reaches the library."""
import ctypes
import os
import re
from types import SimpleNamespace

import pytest
import torch

from paper_2502_01681_b200 import dg4

BF16 = torch.bfloat16


def test_null_handles_are_refused():
    lib = dg4.load()
    d = ctypes.byref(dg4.desc(8, dg4.DG4_BF16, 0.25))
    inv = dg4.DG4_ERR_INVALID_ARG
    assert lib.dg4_glu_fwd(None, d, None, 128, None, None, None, 512, 0, None, 0, None, 128, None) == inv
    assert lib.dg4_glu_bwd(None, d, None, 128, None, None, None, 512, 0, None, 128, None, 128, None, None, None, None, 0, None) == inv
    assert lib.dg4_add_norm_fwd(None, d, None, 128, None, 128, None, None, 1e-5, None, 128, None, 128, None) == inv
    assert lib.dg4_norm_bwd(None, d, None, 128, None, 1e-5, None, 128, None, 128, None, 128, None, None, None, 0, None) == inv
    assert lib.dg4_glu_bwd_workspace_bytes(None, d, 512) == 0
    assert lib.dg4_norm_bwd_workspace_bytes(None, d) == 0


def test_activations_match_the_header():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    text = open(os.path.join(root, "include", "dg4.h")).read()
    for name in ("SILU", "GELU", "RELU"):
        assert int(re.search(r"DG4_ACT_%s = (\d+)" % name, text).group(1)) == getattr(dg4, "DG4_ACT_" + name)


def test_weights_and_vectors_are_checked_before_the_library_is_reached():
    g, d = SimpleNamespace(handle=None), dg4.desc(8, dg4.DG4_BF16, 0.25)
    x = torch.zeros((1, 128), dtype=BF16)
    w, wd = torch.zeros((64, 128), dtype=BF16), torch.zeros((128, 64), dtype=BF16)
    bad = [(w, w, w), (w, torch.zeros((72, 128), dtype=BF16), wd), (w.float(), w, wd), (w, w, wd),          # the last: not on the GPU
           (torch.zeros((64, 256), dtype=BF16)[:, :128], w, wd)]
    for weights in bad:
        with pytest.raises(ValueError):
            dg4.dg4_glu_fwd(g, d, x, *weights, dg4.DG4_ACT_SILU, None, x)
        with pytest.raises(ValueError):
            dg4.dg4_glu_bwd(g, d, x, *weights, dg4.DG4_ACT_SILU, x, x, None, None, None)
    for vec in (torch.ones(128), torch.ones(64), torch.ones(128, dtype=torch.float64)):                     # the first: not on the GPU
        with pytest.raises(ValueError):
            dg4.dg4_add_norm_fwd(g, d, x, None, vec, None, 1e-5, None, x)
        with pytest.raises(ValueError):
            dg4.dg4_norm_bwd(g, d, x, vec, 1e-5, x, None, x, None, None)
