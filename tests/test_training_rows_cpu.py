"""What the binding asks of the training calls' tensors before a kernel reads or writes them: type, rows, width, inner stride and
device.  No GPU: stand-ins for CUDA tensors, and a library that only notes that it was reached."""
import types

import pytest
import torch

from paper_2502_01681_b200 import dg4

BF16, F32 = torch.bfloat16, torch.float32
N, D_FF = 300, 64


class Fake:
    """A CUDA tensor as far as the binding looks at it."""
    def __init__(self, shape, dtype=BF16, device=0, strides=None):
        self.meta = torch.empty(shape, dtype=dtype, device="meta")
        if strides is not None:
            self.meta = torch.empty_strided(shape, strides, dtype=dtype, device="meta")
        self.shape, self.dtype, self.index = self.meta.shape, dtype, device
        self.is_cuda, self.device = device >= 0, f"cuda:{device}" if device >= 0 else "cpu"
        self.stride, self.numel, self.dim = self.meta.stride, self.meta.numel, self.meta.dim
        self.is_contiguous, self.element_size = self.meta.is_contiguous, self.meta.element_size

    def get_device(self):
        return self.index

    def data_ptr(self):
        return 4096


@pytest.fixture
def reached(monkeypatch):
    calls = []

    class Library:
        def __getattr__(self, name):
            return lambda *args: calls.append((name, args)) or dg4.DG4_OK
    monkeypatch.setattr(dg4, "load", lambda: Library())
    monkeypatch.setattr(dg4, "_stream", lambda *args: 0)
    return calls


def handle():
    return types.SimpleNamespace(handle=None, info=types.SimpleNamespace(n_nodes=N, device=0))


def rows(dtype=BF16):
    return Fake((N, 128), dtype)


def weights():
    return [Fake((D_FF, 128)), Fake((D_FF, 128)), Fake((128, D_FF))]


def glu_fwd(t, ws=None):
    dg4.dg4_glu_fwd(handle(), dg4.desc(8, dg4.DG4_BF16, 0.25, residual=True), t["X"], *weights(), 0, t["H_res"], t["Y"])


def glu_bwd(t, ws=None):
    dg4.dg4_glu_bwd(handle(), dg4.desc(8, dg4.DG4_BF16, 0.25), t["X"], *weights(), 0, t["dY"], t["dX"], *weights(), ws)


def add_norm(t, ws=None, tag=dg4.DG4_BF16):
    vec = Fake((128,), F32)
    dg4.dg4_add_norm_fwd(handle(), dg4.desc(8, tag, 0.25), t["X"], t["R"], vec, vec, 1e-5, t["Z"], t["Y"])


def norm_bwd(t, ws=None, tag=dg4.DG4_BF16):
    vec = Fake((128,), F32)
    dg4.dg4_norm_bwd(handle(), dg4.desc(8, tag, 0.25), t["Z"], vec, 1e-5, t["dY"], t["D_res"], t["dZ"], vec, vec, ws)


CALLS = [(glu_fwd, ("X", "H_res", "Y")), (glu_bwd, ("X", "dY", "dX")), (add_norm, ("X", "R", "Z", "Y")),
         (norm_bwd, ("Z", "dY", "D_res", "dZ"))]
BAD = {"short": lambda: Fake((N - 1, 128)), "narrow": lambda: Fake((N, 64)), "wide": lambda: Fake((N, 256)), "type": lambda: Fake((N, 128), F32),
       "half": lambda: Fake((N, 128), torch.float16), "host": lambda: Fake((N, 128), BF16, -1), "another GPU": lambda: Fake((N, 128), BF16, 1),
       "inner stride": lambda: Fake((N, 128), BF16, 0, (256, 2)), "transposed": lambda: Fake((N, 128), BF16, 0, (1, N)),
       "one axis": lambda: Fake((N * 128,)), "three axes": lambda: Fake((N, 1, 128))}


@pytest.mark.parametrize("call,names", CALLS)
def test_rows_that_a_call_can_take_reach_the_library(call, names, reached):
    call({name: rows() for name in names})
    call({name: Fake((N, 128), BF16, 0, (1000, 1)) for name in names})                   # rows further apart
    call({name: Fake((N + 77, 128)) for name in names})                                  # a larger buffer
    call({name: rows() for name in names}, Fake((100,), torch.uint8))
    call({name: rows() for name in names}, Fake((0,), torch.uint8, -1))                  # no workspace needed, an empty one given
    assert len(reached) == 5
    assert all(name[4:] in ("glu_fwd", "glu_bwd", "add_norm_fwd", "norm_bwd") for name, _ in reached)
    assert sum(arg == 1000 for arg in reached[1][1]) == len(names) and sum(arg == 1000 for arg in reached[0][1]) == 0


@pytest.mark.parametrize("bad", BAD)
@pytest.mark.parametrize("call,names", CALLS)
def test_rows_that_a_kernel_would_read_or_write_past_their_end_are_refused(call, names, bad, reached):
    for name in names:
        with pytest.raises(dg4.Dg4Error) as e:
            call({**{other: rows() for other in names}, name: BAD[bad]()})
        assert e.value.status == dg4.DG4_ERR_INVALID_ARG and e.value.detail.startswith(name + " is")
    assert not reached


@pytest.mark.parametrize("call,names", CALLS[2:])
def test_a_norm_s_rows_are_of_the_descriptor_s_type(call, names, reached):
    call({name: rows(F32) for name in names}, None, dg4.DG4_F32)
    assert len(reached) == 1
    for name in names:                                                   # 16-bit rows would be read and written to twice their length
        with pytest.raises(dg4.Dg4Error):
            call({**{other: rows(F32) for other in names}, name: rows(BF16)}, None, dg4.DG4_F32)
    assert len(reached) == 1


def test_a_residual_that_is_not_asked_for_is_not_looked_at(reached):
    dg4.dg4_glu_fwd(handle(), dg4.desc(8, dg4.DG4_BF16, 0.25), rows(), *weights(), 0, Fake((1, 128)), rows())
    assert len(reached) == 1


def test_workspaces_weights_and_vectors_elsewhere_are_refused(reached):
    g, d = handle(), dg4.desc(8, dg4.DG4_BF16, 0.25)
    for ws in (Fake((100,), torch.uint8, -1), Fake((100,), torch.uint8, 1), Fake((100,), torch.uint8, 0, (0,)), Fake((100,), torch.uint8, 0, (2,))):
        for call, names in (CALLS[1], CALLS[3]):
            with pytest.raises(dg4.Dg4Error) as e:
                call({name: rows() for name in names}, ws)
            assert e.value.status == dg4.DG4_ERR_INVALID_ARG
    for i in range(3):
        w = weights()
        w[i] = Fake(w[i].shape, BF16, 1)
        with pytest.raises(ValueError):
            dg4.dg4_glu_fwd(g, d, rows(), *w, 0, None, rows())
        with pytest.raises(ValueError):
            dg4.dg4_glu_bwd(g, d, rows(), *weights(), 0, rows(), rows(), *w, None)
    vec, far = Fake((128,), F32), Fake((128,), F32, 1)
    for vecs in ((far, vec), (vec, far)):
        with pytest.raises(ValueError):
            dg4.dg4_add_norm_fwd(g, d, rows(), None, *vecs, 1e-5, None, rows())
        with pytest.raises(ValueError):
            dg4.dg4_norm_bwd(g, d, rows(), vec, 1e-5, rows(), None, rows(), *vecs, None)
    assert not reached
