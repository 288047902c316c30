"""Calls of the 8-bit helpers with tensors of another GPU than the current one are refused before anything is allocated
or launched (a launch goes to the current device).  Without a GPU: stand-ins for the tensors, and for the current device."""
import pytest
import torch


class OnSecondGpu:
    """What the helpers ask of a tensor on cuda:1."""

    def __init__(self, *shape, dtype=torch.bfloat16):
        self.shape, self.dtype, self.device = torch.Size(shape), dtype, torch.device("cuda", 1)

    def dim(self):
        return len(self.shape)

    def stride(self):
        return (self.shape[1], 1)

    def is_contiguous(self):
        return True

    def element_size(self):
        return self.dtype.itemsize

    def get_device(self):
        return 1

    def data_ptr(self):
        return 1 << 40


@pytest.fixture()
def ds(monkeypatch):
    from paper_1905_13298_gb300 import build
    build.build_library()
    import paper_1905_13298_gb300 as ds
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    return ds


def _matrix(ds, rows, cols):
    return ds.F8Matrix(OnSecondGpu(rows, cols, dtype=torch.float8_e4m3fn),
                       OnSecondGpu(rows, -(-cols // 128), dtype=torch.float32))


def test_tensors_of_another_gpu_are_refused(ds):
    x, q, v = OnSecondGpu(4, 256), _matrix(ds, 4, 256), lambda n: OnSecondGpu(n, dtype=torch.float32)
    w = ds.PackedShiftWeights(OnSecondGpu(4096, dtype=torch.uint8), ds.ds_weights(n_out=4, k_red=256))
    for call in (lambda: ds.quantize_f8(x), lambda: ds.quantize_f8(q, "tiles"), lambda: ds.linear_f8(q, q),
                 lambda: ds.expand_shift_weights_f8(w), lambda: ds.rmsnorm_f8(x, v(256)),
                 lambda: ds.rmsnorm_f8_backward(x, x, v(4), v(256)), lambda: ds.gated_f8(x, 128),
                 lambda: ds.gated_f8_backward(q, OnSecondGpu(4, 128))):
        with pytest.raises(ValueError, match="is on cuda:1, the current device is cuda:0"):
            call()


def test_tensors_of_the_current_gpu_are_not(ds, monkeypatch):
    """With their device current the same stand-ins pass the checks, up to the allocation that fails here."""
    if torch.cuda.is_available():
        pytest.skip("a GPU would allocate")
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    with pytest.raises((AssertionError, RuntimeError)):
        ds.linear_f8(_matrix(ds, 4, 256), _matrix(ds, 4, 256))


def test_tensors_of_a_matrix_cannot_be_replaced(ds):
    """Its descriptor holds their addresses: others would be passed over, and the memory of the first ones lost."""
    m = _matrix(ds, 4, 256)
    q, scale = m.q, m.scale
    with pytest.raises(AttributeError):
        m.q = OnSecondGpu(4, 256, dtype=torch.float8_e4m3fn)
    with pytest.raises(AttributeError):
        m.scale = OnSecondGpu(4, 2, dtype=torch.float32)
    assert m.q is q and m.scale is scale
