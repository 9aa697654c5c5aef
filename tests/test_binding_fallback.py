"""The binding where its shortcuts (module _marshal) are not there: the checks of tensors that it then makes itself, and
that every call works."""
import importlib.util
import inspect
import sys

import pytest
import torch

import paper_2606_22968_amd as package
from paper_2606_22968_amd import binding

NAME = "paper_2606_22968_amd._marshal"


@pytest.fixture(scope="module")
def plain(mocap_lib):
    """The binding's module once more, loaded while _marshal cannot be imported."""
    with pytest.MonkeyPatch.context() as m:
        m.setitem(sys.modules, NAME, None)
        m.delattr(package, "_marshal", raising=False)
        spec = importlib.util.spec_from_file_location("paper_2606_22968_amd.binding_plain", binding.__file__)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
    assert module._marshal is None
    return module


class Sub(torch.Tensor):
    pass


def tensors(device):
    x = torch.zeros((6, 4, 64), dtype=torch.bfloat16, device=device)
    rows = torch.zeros((6, 8, 64), dtype=torch.bfloat16, device=device)
    yield from (x, x.float(), x[1:], x[:, 1:3], x[:1], x[:0], x[:, :1], x[:, :, :32], x.transpose(0, 1), x[0], x[:, None],
                rows[:, 2:6], rows[:, :0], rows[::2], x.as_subclass(Sub), torch.nn.Parameter(x), x[:1].expand(6, 4, 64),
                torch.zeros((), device=device), torch.zeros(5, dtype=torch.int32, device=device), x.to_sparse(), None, 3, [x])


def check_tensors(plain, device, index):
    """_need and _rows take what they should, and refuse everything else as a TypeError or ValueError."""
    for t in tensors(device):
        strided = isinstance(t, torch.Tensor) and t.layout is torch.strided
        for dtype in (torch.bfloat16, torch.float32, torch.int32):
            for ndim in (None, 0, 1, 3):
                for at in (index, index + 1):
                    good = strided and t.dtype is dtype and t.is_contiguous() and (ndim is None or t.dim() == ndim) and at == index
                    if good:
                        assert plain._need(t, dtype, "t", ndim, at) == t.data_ptr()
                    else:
                        with pytest.raises((TypeError, ValueError)):
                            plain._need(t, dtype, "t", ndim, at)
        good = strided and t.dtype is torch.bfloat16 and t.dim() == 3 and t.stride(2) == 1 and \
            (t.shape[1] <= 1 or t.stride(1) == t.shape[2])
        if good:
            n, h, d = t.shape
            assert tuple(plain._rows(t, "t", index)) == (t.data_ptr(), t.stride(0) if n > 1 else h * d, n, h, d)
        else:
            with pytest.raises((TypeError, ValueError)):
                plain._rows(t, "t", index)
        with pytest.raises((TypeError, ValueError)):
            plain._rows(t, "t", index + 1)


def test_tensor_checks_on_the_cpu(plain, monkeypatch):
    """A CPU tensor's device is -1.  (_require asks for a GPU tensor; here it does for a tensor of this device.)"""
    source, scope = inspect.getsource(plain._require), dict(vars(plain))
    assert "is_cuda" in source
    exec(source.replace("is_cuda", "is_cpu"), scope)
    monkeypatch.setattr(plain, "_require", scope["_require"])
    check_tensors(plain, "cpu", -1)


@pytest.mark.gpu
def test_tensor_checks(gpu, plain):
    check_tensors(plain, "cuda", 0)
    with pytest.raises(ValueError):
        plain._need(torch.zeros(3), torch.float32, "t", 1, 0)


@pytest.mark.gpu
def test_every_call(gpu, plain):
    """The calls of mocap_cache.h, with the same results as through the shortcuts, and their refusals."""
    from test_marshal_gpu import calls

    def run(module, name, four, args, outputs):
        store = module.Kv4Store(3, 64, 2, 64, fill=0x41) if four else module.KvStore(3, 64, 2, 64, fill=1.0)
        for x in outputs:
            x.fill_(7.0)
        args = [module.Rope(a.inv_freq, a.interleaved) if isinstance(a, binding.Rope) else a for a in args]
        getattr(module, name)(store, *args)
        pools = [getattr(store, p) for p in ("k_pool", "v_pool", "k_scale", "v_scale") if hasattr(store, p)]
        return [x.clone() for x in (*outputs, *pools)]

    for name, four, args, outputs in calls():
        for a, b in zip(run(binding, name, four, args, outputs), run(plain, name, four, args, outputs)):
            assert torch.equal(a, b), name
    store = plain.Kv4Store(3, 64, 2, 64, fill=0)
    k, table = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    with pytest.raises(plain.MocapError):
        plain.mocap_kv4_append(store, table, 190, k, k)
    for bad in (k.cpu(), k[0], k.transpose(0, 1), k[..., ::2]):
        with pytest.raises(ValueError):
            plain.mocap_kv4_append(store, table, 0, bad, bad)
