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
    return S.kv_assign(**t, block_size=16, max_tokens=8, out=out, stream=0, **more)


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
