"""The binding's shortcuts in C++ (csrc/marshal.cpp): tensor checks against what torch's own methods say, and whole calls
against the binding's long way."""
import pytest
import torch

from paper_2606_22968_amd import binding

pytestmark = pytest.mark.gpu


class Sub(torch.Tensor):
    pass


@pytest.fixture(scope="module")
def ext(gpu):
    from paper_2606_22968_amd import _marshal
    binding.load_library()  # whose calls the shortcuts are bound to
    assert binding._address is _marshal.address and binding._row_address is _marshal.rows
    return _marshal


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


def calls():
    """(name, store's kind, arguments, outputs) of an ordinary call of each kind."""
    def rand(*shape):
        return torch.randn(shape, generator=torch.Generator().manual_seed(len(shape) + shape[0])).to(torch.bfloat16).cuda()

    h_q, h_kv, d = 4, 2, 64
    table = torch.tensor([2, 0, 1], dtype=torch.int32, device="cuda")
    tables, lens = table.repeat(2, 1), torch.tensor([70, 0], dtype=torch.int32, device="cuda")
    rope = binding.Rope(torch.ones(d // 2, device="cuda"), True)
    rows = rand(20, h_q + 2 * h_kv, d)
    q, k, v = rows[:, :h_q], rows[:, h_q:h_q + h_kv], rows[:, h_q + h_kv:]
    two, out2 = [x[:2] for x in (q, k, v)], torch.empty((2, h_q, d), dtype=torch.bfloat16, device="cuda")
    out = torch.empty((20, h_q, d), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    loaded = [torch.empty((2, 5, h_kv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    o2, lse2 = torch.empty_like(out2), torch.empty((2, h_q), device="cuda")
    dense, o, lse = rand(20, h_q, d), torch.empty_like(out), torch.empty((h_q, 20), device="cuda")
    for four in (False, True):
        name = "kv4_append" if four else "rope_append"
        yield f"mocap_{name}", four, (table, 3, k, v, rope, None, q, out), (out,)
        yield f"mocap_{name}", four, (table, 3, k, v, None, 9, None, None), ()
        name = "kv4_decode_append" if four else "decode_rope_append"
        yield f"mocap_{name}", four, (tables, lens, two[1], two[2], rope, lens, two[0], out2), (out2,)
    yield "mocap_kv4_load", True, (tables, lens, *loaded), tuple(loaded)
    yield "mocap_kv4_decode_attn", True, (tables, lens, dense[:2].contiguous(), 192, 0.1, o2, lse2, ws, 100, 3), (o2, lse2)
    yield "mocap_kv4_decode_attn", True, (tables, lens, dense[:2].contiguous(), 192, 0.1, o2, lse2, None, 0, 0), (o2, lse2)
    yield "mocap_kv4_chunk_attn", True, (table, dense, 50, 0.1, o, lse, ws, 0, 0, 3), (o, lse)


def test_calls_take_the_shortcut_and_do_the_same(ext, monkeypatch):
    def run(name, four, args, outputs, shortcut):
        store = binding.Kv4Store(3, 64, 2, 64, fill=0x41) if four else binding.KvStore(3, 64, 2, 64, fill=1.0)
        with monkeypatch.context() as m:
            if not shortcut:
                m.setattr(binding, "_marshal", None)
            for x in outputs:
                x.fill_(7.0)
            getattr(binding, name)(store, *args)
        pools = [getattr(store, p) for p in ("k_pool", "v_pool", "k_scale", "v_scale") if hasattr(store, p)]
        return [x.clone() for x in (*outputs, *pools)]

    for name, four, args, outputs in calls():
        store = binding.Kv4Store(3, 64, 2, 64, fill=0x41) if four else binding.KvStore(3, 64, 2, 64, fill=1.0)
        assert getattr(ext, name)(store, *args, binding._stream_on(None, 0), 0) == 0, name
        for a, b in zip(run(name, four, args, outputs, True), run(name, four, args, outputs, False)):
            assert torch.equal(a, b), name


def test_unusual_arguments_take_the_long_way(ext):
    """Every argument in turn replaced by what the shortcut does not take: it answers None, having done nothing."""
    for name, four, args, outputs in calls():
        store = binding.Kv4Store(3, 64, 2, 64, fill=0x41) if four else binding.KvStore(3, 64, 2, 64, fill=1.0)
        stream = binding._stream_on(None, 0)
        call = getattr(ext, name)
        for x in outputs:
            x.fill_(7.0)
        for i, arg in enumerate(args):
            wrong = [object(), "3", 1 << 70]
            if isinstance(arg, torch.Tensor):
                wrong += [arg.cpu(), arg.as_subclass(Sub)]
                # (A workspace is any contiguous tensor.)
                wrong += [arg[::2]] if arg.dtype is torch.uint8 else [arg.double(), arg[None]]
            if isinstance(arg, (int, float)) and arg is not True:
                wrong += [None, 1.5 if isinstance(arg, int) else 3] if not (arg == 9) else [1.5]
            for x in wrong:
                assert call(store, *args[:i], x, *args[i + 1:], stream, 0) is None, (name, i, x)
        assert call(object(), *args, stream, 0) is None and call(store, *args, stream, 1) is None
        assert call(store, *args, "x", 0) is None and call(store, *args, stream, None) is None
        other = binding.KvStore(3, 64, 2, 64, fill=1.0) if four else binding.Kv4Store(3, 64, 2, 64, fill=1)
        assert call(other, *args, stream, 0) is None
        for p in ("k_pool", "v_pool") + (("k_scale", "v_scale") if four else ()):
            good = getattr(store, p)
            for bad in (good.cpu(), good.float(), good[..., ::2], good[0], None):
                setattr(store, p, bad)
                assert call(store, *args, stream, 0) is None, (name, p)
            setattr(store, p, good)
        for p in ("h_kv", "head_dim", "block_size", "num_blocks"):
            good = getattr(store, p)
            for bad in ("2", 2.0, 1 << 40):
                setattr(store, p, bad)
                assert call(store, *args, stream, 0) is None, (name, p)
            setattr(store, p, good)
        with pytest.raises(TypeError):
            call(store, *args)
        torch.cuda.synchronize()
        assert all((x == 7.0).all() for x in outputs)


def test_statuses_raise(ext):
    store = binding.Kv4Store(3, 64, 2, 64, fill=0)
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    table = torch.zeros(3, dtype=torch.int32, device="cuda")
    assert ext.mocap_kv4_append(store, table, 190, k, k, None, None, None, None, binding._stream_on(None, 0), 0) == 1
    with pytest.raises(binding.MocapError) as e:
        binding.mocap_kv4_append(store, table, 190, k, k)
    assert e.value.status == 1 and "mocap_kv4_append" in str(e.value)
    with pytest.raises(ValueError):
        ext.bind("mocap_nothing", 1)
