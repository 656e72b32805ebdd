"""The binding of the token-row operators with tensors on several GPUs, which it tells apart before
any call: a kernel of one GPU must not be given another's memory."""

import pytest
import torch

from paper_2008_00325_amd import umap_rows as R


class On:
    """A contiguous tensor on GPU `gpu`, as far as the binding looks at one."""

    def __init__(self, gpu, *shape, dtype=torch.float32):
        self.gpu, self.shape, self.dtype = gpu, shape, dtype
        self.device = f"cuda:{gpu}"
        self.is_cuda = True

    def get_device(self):
        return self.gpu

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (self.shape[1], 1)

    def numel(self):
        return torch.Size(self.shape).numel()

    def element_size(self):
        return self.dtype.itemsize

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 40


@pytest.fixture
def two_gpus(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch.cuda, "device_count", lambda: 2)
    if hasattr(R, "_only"):
        monkeypatch.setattr(R, "_only", -2)

    def no_call(*args):
        raise AssertionError("the library was called")

    R.lib()
    for name in ("umap_rows_lookup", "umap_rows_lookup_grad", "umap_rows_norm", "umap_rows_norm_grad"):
        monkeypatch.setitem(R._call, name, no_call)


def calls():
    """Each call with its tensors by name."""
    f32, i32, u8 = torch.float32, torch.int32, torch.uint8
    yield R.umap_rows_lookup, dict(table=(9, 8, torch.int8), ids=(4, i32), out=(4, 8, f32), table_scales=(9, f32))
    yield R.umap_rows_lookup_grad, dict(dout=(4, 8, f32), ids=(4, i32), grad=(9, 8, f32), workspace=(9999, u8))
    yield R.umap_rows_norm, dict(x=(9, 8, f32), y=(4, 8, torch.int8), weight=(8, f32), residual=(4, 8, f32), h=(4, 8, f32),
                                 ids=(4, i32), y_scales=(4, f32))
    yield R.umap_rows_norm_grad, dict(dy=(4, 8, f32), h=(4, 8, f32), dx=(4, 8, f32), weight=(8, f32), dh=(4, 8, f32),
                                      dweight=(8, f32), workspace=(9999, u8))


@pytest.mark.parametrize("call,tensors", calls(), ids=lambda x: getattr(x, "__name__", ""))
def test_tensors_on_another_gpu_are_refused(two_gpus, call, tensors):
    def given(other=None, at=1):
        return {name: On(at if name == other else 0, *t[:-1], dtype=t[-1]) for name, t in tensors.items()}

    with pytest.raises(AssertionError, match="the library was called"):
        call(**given())
    for name in tensors:
        with pytest.raises(ValueError, match="lies on GPU 1, the current one is 0"):
            call(**given(name))
        with pytest.raises(ValueError, match="must be a GPU tensor"):
            call(**given(name, -1))


def test_all_on_a_gpu_that_is_not_the_current_one(two_gpus):
    with pytest.raises(ValueError, match="lies on GPU 1, the current one is 0"):
        R.umap_rows_lookup(On(1, 9, 8), None, On(1, 4, 8))
