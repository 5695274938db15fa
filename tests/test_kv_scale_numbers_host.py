"""A tensor of one element is a number as a scale, whatever its dimensions, and no scale of blocks (no GPU needed: the tensors are
fake ones, which have a device, a type and a shape, and no memory)."""
import pytest

torch = pytest.importorskip("torch")
from torch._subclasses.fake_tensor import FakeTensorMode  # noqa: E402

import paper_2408_04323_amd as S  # noqa: E402


def _fake(*shape, dtype=torch.int32, device="cuda:0"):
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device=device)


def _half(*shape):
    return _fake(*shape, dtype=torch.bfloat16)


def _f8(*shape):
    return _fake(*shape, dtype=torch.float8_e4m3fn)


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


def _attend(cache, k_scale, v_scale, **change):
    t = dict(out=_half(3, 5, 64))
    t.update(change)
    heads = 2 * cache.shape[1]
    return S.kv_attention(_half(3, heads, 64), cache, cache, _fake(2, 3), _fake(3), _fake(2), 2, 9, k_scale=k_scale, v_scale=v_scale,
                          workspace=_fake(4096, dtype=torch.uint8), stream=0, **t)


def _append(cache, k_scale, v_scale):
    k = _half(3, cache.shape[1], 64)
    return S.kv_append(k, k, None, _fake(3, dtype=torch.int64), cache, cache, k_scale=k_scale, v_scale=v_scale, out=_half(3, 5, 64), stream=0)


NUMBERS = {"cpu": lambda: torch.tensor([[0.5]]), "device": lambda: _fake(1, 1, dtype=torch.float32), "double": lambda: torch.tensor([[0.5]]).double(),
           "three dimensions": lambda: torch.tensor([[[0.5]]])}


@pytest.mark.parametrize("number", list(NUMBERS))
@pytest.mark.parametrize("cache", [lambda: _f8(4, 2, 16, 64), lambda: _half(4, 2, 16, 64), lambda: _half(1, 1, 16, 64), lambda: _f8(4, 1, 16, 64),
                                   lambda: _f8(1, 2, 16, 64)], ids=["f8", "bf16", "bf16-1x1", "f8-4x1", "f8-1x2"])
def test_one_element_is_a_number(number, cache):
    """What is wrong is the output, and that is what the error says."""
    n, c = NUMBERS[number](), cache()
    for pair in ((n, 0.5), (0.5, n), (n, n)):
        with pytest.raises(ValueError, match="out must"):
            _attend(c, *pair)
        with pytest.raises(ValueError, match="out needs queries"):
            _append(c, *pair)


def test_one_block_and_head():
    """There, two float32 tensors on the device are its scales; anything else of one element is a number."""
    c, ok = _f8(1, 1, 16, 64), _fake(1, 1, dtype=torch.float32)
    gaps = _fake(4, 1, dtype=torch.float32)
    for other in (0.5, torch.tensor([[0.5]]), _fake(1, 1, dtype=torch.float64), _fake(1, dtype=torch.float32)):
        with pytest.raises(ValueError, match="out must"):
            _attend(c, ok, other)
    with pytest.raises(ValueError, match="v_scale must be on the device"):
        _attend(c, ok, _fake(1, 1, dtype=torch.float32, device="cuda:1"), out=_half(3, 2, 64))
    with pytest.raises(ValueError, match="k_scale must be .blocks, kv_heads."):
        _attend(c, gaps, ok, out=_half(3, 2, 64))
    with pytest.raises(ValueError, match="both be numbers"):
        _attend(c, gaps, 0.5, out=_half(3, 2, 64))
