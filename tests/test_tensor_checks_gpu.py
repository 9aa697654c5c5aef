"""The binding's tensor checks in C++ (csrc/tensors.cpp) against what torch's own methods say: the same tensors pass,
with the same addresses and strides."""
import pytest
import torch

from paper_2606_22968_amd import binding

pytestmark = pytest.mark.gpu


class Sub(torch.Tensor):
    pass


@pytest.fixture(scope="module")
def ext(gpu):
    from paper_2606_22968_amd import _tensors
    assert binding._address is _tensors.address and binding._row_address is _tensors.rows
    return _tensors


def tensors():
    x = torch.zeros((6, 4, 64), dtype=torch.bfloat16, device="cuda")
    rows = torch.zeros((6, 8, 64), dtype=torch.bfloat16, device="cuda")
    yield from (x, x.cpu(), x.float(), x[1:], x[:, 1:3], x[:1], x[:0], x[:, :1], x[:, :, :32], x.transpose(0, 1), x[0],
                x[:, None], rows[:, 2:6], rows[:, :0], rows[::2], rows.flip(0), x.as_subclass(Sub),
                torch.nn.Parameter(x), x.expand(6, 4, 64), x[:1].expand(6, 4, 64), torch.zeros((), device="cuda"),
                torch.zeros(5, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.uint8, device="cuda"),
                torch.zeros(5, dtype=torch.uint8), x.to_sparse(), None, 3, [x])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32, torch.int32, torch.uint8])
@pytest.mark.parametrize("ndim", [-1, 0, 1, 3])
def test_addresses(ext, dtype, ndim):
    for t in tensors():
        for device in (0, 1):
            want = None
            if type(t) in (torch.Tensor, torch.nn.Parameter) and t.layout is torch.strided and t.dtype is dtype and t.is_contiguous() and \
                    t.device == torch.device("cuda", device) and (ndim < 0 or t.dim() == ndim):
                want = t.data_ptr()
            assert ext.address(t, dtype, ndim, device) == want


def test_rows(ext):
    for t in tensors():
        want = None
        if type(t) in (torch.Tensor, torch.nn.Parameter) and t.layout is torch.strided and t.dtype is torch.bfloat16 and t.is_cuda and \
                t.dim() == 3 and t.stride(2) == 1 and (t.stride(1) == t.shape[2] or t.shape[1] <= 1):
            n, h, d = t.shape
            want = (t.data_ptr(), t.stride(0) if n > 1 else h * d, n, h, d)
        assert ext.rows(t, 0) == want
        assert ext.rows(t, 1) is None


def test_parameters_and_subclasses_pass_all_the_same(gpu):
    x = torch.zeros((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    for t in (torch.nn.Parameter(x), x.as_subclass(Sub)):
        assert binding._need(t, torch.bfloat16, "x", 3, 0) == x.data_ptr()
        assert binding._rows(t, "x", 0) == (x.data_ptr(), 128, 2, 2, 64)
    with pytest.raises(ValueError):
        binding._need(x, torch.bfloat16, "x", 3, 1)


def test_wrong_calls(ext):
    for args in ((), (None,), (None, 3, 1, 0), (None, torch.uint8, "a", 0)):
        with pytest.raises(TypeError):
            ext.address(*args)
    with pytest.raises(TypeError):
        ext.rows(None)
