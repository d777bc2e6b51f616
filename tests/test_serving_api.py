"""The serving calls' argument checks that need no GPU: null handles at the C ABI, and what the binding refuses before
it reaches the library."""
import ctypes

import pytest
import torch

from paper_2502_01681_b200 import dg4


def test_null_handles_are_refused():
    lib = dg4.load()
    d = dg4.desc(8, dg4.DG4_BF16, 0.25)
    inv = dg4.DG4_ERR_INVALID_ARG
    p = ctypes.byref(d)
    assert lib.dg4_qkv_project_adapters(None, p, None, 128, None, None, None, None, 128, None, 128, None, 128, None) == inv
    assert lib.dg4_out_project_adapters(None, p, None, 128, None, None, None, None, 128, None, 128, None) == inv
    assert lib.dg4_kv8_write(None, p, None, 128, None, 128, None, 288, None, 0, None) == inv
    assert lib.dg4_kv8_read(None, p, None, 288, None, 128, None, 128, None, 0, None) == inv
    assert lib.dg4_sparse_attn_kv8_fwd(None, p, None, 128, None, 288, None, 128, None, 0, None) == inv
    assert lib.dg4_norm_gate_fwd(None, p, None, 128, None, 128, 1.0, None, 0, None, None, None, None, None, 1e-5, None, 128,
                                 None, 128, None) == inv


def test_segments_and_adapters_refuse_what_the_kernels_cannot_read():
    i, bf, f = torch.int32, torch.bfloat16, torch.float32
    with pytest.raises(ValueError):
        dg4.segments(torch.zeros(2, dtype=torch.int64), torch.zeros(1, dtype=i))
    with pytest.raises(ValueError):
        dg4.segments(torch.zeros(2, dtype=i), torch.zeros(1, dtype=i))              # not on the GPU
    for a, b, s in (((2, 16, 64), (2, 384, 16), 2), ((2, 16, 128), (2, 256, 16), 2), ((2, 16, 128), (2, 384, 8), 2),
                    ((2, 16, 128), (3, 384, 16), 2), ((2, 16, 128), (2, 384, 16), 2)):
        with pytest.raises(ValueError):
            dg4.adapters(torch.zeros(a, dtype=bf), torch.zeros(b, dtype=bf), torch.zeros(s, dtype=f))


def test_row_bytes_match_the_header():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dg4.h")).read()
    assert int(re.search(r"#define DG4_KV8_ROW_BYTES (\d+)", text).group(1)) == dg4.DG4_KV8_ROW_BYTES
    assert int(re.search(r"DG4_FLAG_RMS_NORM = (\d+)", text).group(1)) == dg4.DG4_FLAG_RMS_NORM


def test_node_lists_and_vectors_are_checked_before_the_library_is_reached():
    for bad in (torch.zeros(3, dtype=torch.int64), torch.zeros(3, dtype=torch.int32), torch.zeros((2, 2), dtype=torch.int32)):
        for call in (dg4.dg4_kv8_write, dg4.dg4_kv8_read, dg4.dg4_sparse_attn_kv8_fwd):
            with pytest.raises(ValueError):
                call(None, None, None, None, None, nodes=bad)
    from types import SimpleNamespace
    with pytest.raises(ValueError):
        dg4.dg4_norm_gate_fwd(SimpleNamespace(handle=None), dg4.desc(8, dg4.DG4_BF16, 0.25), torch.zeros((1, 128)), torch.zeros((1, 128)), 1.0, torch.ones((1, 128)), None,
                              (torch.ones(128), None), None, 1e-5, None, None)
