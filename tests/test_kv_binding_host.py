"""What the cache calls refuse of device tensors, decided before the library is called (no GPU needed: the tensors are
fake ones, which have a device, a type and a shape, and no memory)."""
import pytest

torch = pytest.importorskip("torch")
from torch._subclasses.fake_tensor import FakeTensorMode  # noqa: E402

import paper_2408_04323_amd as S  # noqa: E402


def _fake(*shape, dtype=torch.int32, device="cuda:0"):
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device=device)


@pytest.fixture(autouse=True)
def no_call(monkeypatch):
    """A check that is missing ends in a call, and that fails the test."""
    S._kv or S._kv_setup()

    class Watched:
        def __getattr__(self, name, module=S._kv):
            def call(*args):
                got = getattr(module, name)(*args)
                assert got is None, f"{name} reached the library"
                return got
            return call
    monkeypatch.setattr(S, "_kv", Watched())


ASSIGN = dict(context_len=(4,), new_len=(4,), block_table=(4, 2), free_blocks=(3,))


def _assign(change=None, out=None, **more):
    t = {name: _fake(*shape) for name, shape in ASSIGN.items()}
    t.update(change or {})
    return S.kv_assign(**t, block_size=16, max_tokens=8, out=out or _batch(), stream=0, **more)


def _batch(**change):
    b = S.KVBatch.__new__(S.KVBatch)
    b.num_seqs, b.max_tokens = 4, 8
    b.query_start, b.seq_len, b.positions, b.counts = _fake(5), _fake(4), _fake(8), _fake(4)
    b.slots = _fake(8, dtype=torch.int64)
    for name, t in change.items():
        setattr(b, name, t)
    return b


def test_results_on_the_host_are_refused():
    with pytest.raises(ValueError, match="out.query_start must be a device tensor"):
        _assign(out=S.KVBatch(4, 8, device="cpu"))


@pytest.mark.parametrize("name,shape,dtype,what", [
    ("query_start", (4,), torch.int32, "5 elements"), ("seq_len", (5,), torch.int32, "4 elements"),
    ("positions", (7,), torch.int32, "8 elements"), ("positions", (8,), torch.int64, "int32"), ("slots", (8,), torch.int32, "int64"),
    ("slots", (4,), torch.int64, "8 elements"), ("counts", (3,), torch.int32, "4 elements"), ("seq_len", (4,), torch.float32, "int32")])
def test_results_of_another_shape_or_type_are_refused(name, shape, dtype, what):
    with pytest.raises(ValueError, match=f"out.{name} must .*{what}"):
        _assign(out=_batch(**{name: _fake(*shape, dtype=dtype)}))


def test_results_with_gaps_are_refused():
    with pytest.raises(ValueError, match="out.positions must be contiguous"):
        _assign(out=_batch(positions=_fake(16)[::2]))


@pytest.mark.parametrize("name", list(ASSIGN))
def test_slots_from_two_devices_are_refused(name):
    if name == "context_len":
        change = {n: _fake(*shape, device="cuda:1") for n, shape in ASSIGN.items() if n != name}
        what = "new_len"
    else:
        change, what = {name: _fake(*ASSIGN[name], device="cuda:1")}, name
    with pytest.raises(ValueError, match=f"{what} must be on the device of the others"):
        _assign(change)


@pytest.mark.parametrize("name,shape,dtype", [("query_start", 5, torch.int32), ("seq_len", 4, torch.int32),
                                              ("positions", 8, torch.int32), ("slots", 8, torch.int64), ("counts", 4, torch.int32)])
def test_results_on_another_device_are_refused(name, shape, dtype):
    with pytest.raises(ValueError, match=f"out.{name} must be on the device of the others"):
        _assign(out=_batch(**{name: _fake(shape, dtype=dtype, device="cuda:1")}))


def _half(*shape, device="cuda:0"):
    return _fake(*shape, dtype=torch.bfloat16, device=device)


@pytest.mark.parametrize("name", ["v", "slots", "k_cache", "v_cache"])
def test_writes_across_devices_are_refused(name):
    t = dict(k=_half(3, 2, 64), v=_half(3, 2, 64), slots=_fake(3, dtype=torch.int64), k_cache=_half(4, 2, 16, 64), v_cache=_half(4, 2, 16, 64))
    t[name] = _fake(*t[name].shape, dtype=t[name].dtype, device="cuda:1")
    with pytest.raises(ValueError, match=f"{name} must be on the device of the others"):
        S.kv_write(**t, stream=0)


@pytest.mark.parametrize("name", ["k_cache", "v_cache", "block_table", "query_start", "seq_len", "out", "workspace"])
def test_attention_across_devices_is_refused(name):
    t = dict(q=_half(3, 4, 64), k_cache=_half(4, 2, 16, 64), v_cache=_half(4, 2, 16, 64), block_table=_fake(2, 3), query_start=_fake(3),
             seq_len=_fake(2), out=_half(3, 4, 64), workspace=_fake(4096, dtype=torch.uint8))
    t[name] = _fake(*t[name].shape, dtype=t[name].dtype, device="cuda:1")
    with pytest.raises(ValueError, match=f"{name} must be on the device of the others"):
        S.kv_attention(**t, max_new_len=2, max_seq_len=9, stream=0)
