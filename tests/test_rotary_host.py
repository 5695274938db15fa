"""Frequencies of rotations, and refusals of the rotation and append calls, decided before anything is launched (no GPU
needed; device tensors are fake ones, which have a device, a type and a shape, and no memory)."""
import ctypes as C
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2408_04323_amd as S
from oracle import rotary as R
from paper_2408_04323_amd._native import LIB_PATH, lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
INVALID, UNSUPPORTED, NO_MEMORY = -1, -4, -5
BUF = (C.c_uint8 * 4096)()
P = (C.addressof(BUF) + 63) & ~63
NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("args", [
    (128,), (2,), (64, 1e6), (1024, 500000.0), (20, 10000.0), (128, 10000.0, "linear", 8.0), (64, 1e4, "base", 4.0),
    (128, 1e4, "ramp", 16.0, 4096), (64, 1e4, "ramp", 40.0, 4096, 1.0, 32.0), (128, 5e5, "bands", 8.0, 8192, 1.0, 4.0),
    (32, 1e4, "ramp", 2.0, 100, 0.5, 0.6), (128, 1e4, "bands", 1.0, 8192, 1.0, 4.0), (96, 1e4, "ramp", 1.0, 4096)], ids=str)
def test_frequencies_match_the_oracle(args):
    got, m = S.rotary_frequencies(*args)
    want, wm = R.frequencies(*args)
    np.testing.assert_allclose(got, want, rtol=1e-14)
    assert m == pytest.approx(wm, rel=1e-15)


@pytest.mark.parametrize("change", [
    dict(dim=0), dict(dim=3), dict(dim=-2), dict(dim=1026), dict(base=1.0), dict(base=NAN), dict(base=INF), dict(scaling=5), dict(scaling=-1),
    dict(scaling=1, factor=0.5), dict(scaling=1, factor=INF), dict(scaling=2, factor=NAN), dict(scaling=2, dim=2), dict(scaling=3, length=0.0),
    dict(scaling=4, length=INF), dict(scaling=4, low=0.0), dict(scaling=3, low=2.0, high=2.0), dict(scaling=3, high=NAN), dict(freqs=None),
    dict(magnitude=None)], ids=str)
def test_frequencies_refuse(change):
    f, m = (C.c_double * 1024)(), C.c_double()
    a = dict(dim=64, base=1e4, scaling=0, factor=2.0, length=4096.0, low=1.0, high=32.0, freqs=f, magnitude=C.byref(m))
    a.update(change)
    assert lib().scoot_rotary_frequencies(*a.values()) == INVALID
    assert lib().scoot_last_error().decode().startswith("rotary: ")
    with pytest.raises(ValueError, match="scaling"):
        S.rotary_frequencies(64, scaling="other")


@pytest.mark.parametrize("dim", [-2 ** 40, -1, 0, 63, 1026, 2 ** 32 + 64, 2 ** 50])
def test_sizes_that_are_none(dim):
    """Sizes that pass 32 bits are not taken for what is left of them."""
    with pytest.raises(S.ScootError, match="dim must be even"):
        S.rotary_frequencies(dim)


ROTATE = dict(x=P, type=1, num_tokens=4, num_heads=2, head_dim=64, x_token_stride=128, x_head_stride=64, positions=P, freqs=P, rotary_dim=64,
              interleaved=0, magnitude=1.0, reverse=0, out=P, out_token_stride=128, out_head_stride=64, stream=None)
APPEND = dict(q=P, num_heads=4, q_token_stride=256, q_head_stride=64, q_out=P, q_out_token_stride=256, q_out_head_stride=64, k=P, v=P, type=1,
              num_tokens=4, num_kv_heads=2, head_dim=64, k_token_stride=128, k_head_stride=64, v_token_stride=128, v_head_stride=64,
              positions=P, slots=P, freqs=P, rotary_dim=64, interleaved=0, magnitude=1.0, k_cache=P, v_cache=P, cache_type=1, num_blocks=4,
              block_size=16, k_scale=1.0, v_scale=1.0, k_scales=None, v_scales=None, stream=None)
F8 = dict(cache_type=2, k_scales=P, v_scales=P + 64)


def _refused(fn, args, status, **change):
    a = dict(args)
    a.update(change)
    assert fn(*a.values()) == status, change
    assert lib().scoot_last_error().decode().split(":")[0] in ("rotate", "kv append", "kv rotation", "kv cache", "kv attention"), change


@pytest.mark.parametrize("change,status", [
    (dict(type=2), INVALID), (dict(num_tokens=-1), INVALID), (dict(num_tokens=2 ** 31), INVALID), (dict(num_heads=0), INVALID),
    (dict(num_heads=1025), INVALID), (dict(head_dim=60), UNSUPPORTED), (dict(head_dim=1032), UNSUPPORTED), (dict(head_dim=0), UNSUPPORTED),
    (dict(rotary_dim=66), INVALID), (dict(rotary_dim=63), INVALID), (dict(rotary_dim=-2), INVALID), (dict(interleaved=2), INVALID),
    (dict(magnitude=NAN), INVALID), (dict(magnitude=INF), INVALID), (dict(x_token_stride=-1), INVALID), (dict(out_head_stride=2 ** 32), INVALID),
    (dict(x=None), INVALID), (dict(out=None), INVALID), (dict(positions=None), INVALID), (dict(freqs=None), INVALID), (dict(x=P + 1), INVALID),
    (dict(freqs=P + 4), INVALID), (dict(positions=P + 2), INVALID)], ids=str)
def test_rotate_refuses(change, status):
    _refused(lib().scoot_rotate, ROTATE, status, **change)


@pytest.mark.parametrize("change,status", [
    (dict(type=2), INVALID), (dict(cache_type=0), INVALID), (dict(num_kv_heads=0), INVALID), (dict(num_heads=-1), INVALID),
    (dict(num_heads=1025), INVALID), (dict(head_dim=68), UNSUPPORTED), (dict(rotary_dim=65), INVALID), (dict(rotary_dim=128), INVALID),
    (dict(rotary_dim=0), INVALID), (dict(interleaved=-1), INVALID), (dict(magnitude=INF), INVALID), (dict(num_tokens=2 ** 31), INVALID),
    (dict(num_tokens=-3), INVALID), (dict(block_size=12), INVALID), (dict(num_blocks=-1), INVALID), (dict(k_token_stride=-1), INVALID),
    (dict(v_head_stride=2 ** 32), INVALID), (dict(q_token_stride=-8), INVALID), (dict(q_out_head_stride=-8), INVALID), (dict(q=None), INVALID),
    (dict(q_out=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(slots=None), INVALID), (dict(positions=None), INVALID),
    (dict(freqs=None), INVALID), (dict(k_cache=None), INVALID), (dict(v_cache=P + 8), INVALID), (dict(k=P + 1), INVALID), (dict(q_out=P + 1), INVALID),
    (dict(slots=P + 4), INVALID), (dict(k_scale=2.0), INVALID), (dict(cache_type=2, k_scale=0.0), INVALID), (dict(cache_type=2, v_scale=NAN), INVALID),
    (dict(cache_type=2, k_scale=2.0 ** -101), INVALID), (dict(cache_type=2, v_scale=2.0 ** 101), INVALID), (dict(F8, k_scales=None), INVALID), (dict(F8, v_scales=None), INVALID), (dict(F8, cache_type=1), INVALID), (dict(F8, k_scale=2.0), INVALID),
    (dict(F8, k_scales=P + 2), INVALID), (dict(F8, v_scales=P), INVALID)], ids=str)
def test_append_refuses(change, status):
    _refused(lib().scoot_kv_append, APPEND, status, **change)


def test_attention_with_scales_refuses():
    a = dict(q=P, type=1, num_tokens=4, num_heads=4, num_kv_heads=2, head_dim=64, q_token_stride=256, q_head_stride=64, k_cache=P, v_cache=P,
             num_blocks=4, block_size=16, block_table=P, max_blocks=4, table_stride=4, query_start=P, seq_len=P, num_seqs=2, max_new_len=2,
             max_seq_len=9, scale=0.1, window=0, k_scales=P, v_scales=P, out=P, out_token_stride=256, out_head_stride=64, workspace=None,
             workspace_bytes=0, stream=None)
    for change, status in ((dict(k_scales=None), INVALID), (dict(v_scales=None), INVALID), (dict(v_scales=P + 2), INVALID), (dict(type=2), INVALID),
                           (dict(head_dim=96), UNSUPPORTED), (dict(scale=NAN), INVALID), (dict(scale=3e38), INVALID), (dict(q=P + 8), INVALID)):
        _refused(lib().scoot_kv_attention_scaled, a, status, **change)
    assert lib().scoot_kv_attention_scaled(*dict(a, num_tokens=0, k_scales=None).values()) == 0


def test_the_kernels_way_to_divide_by_the_pairs():
    """Row i / pairs as (i + 1/2) times a float reciprocal that may be off by one unit: the whole quotient for every number of
    pairs and every row that a workgroup's cosines and sines have."""
    for pairs in range(1, 513):
        i = np.arange(300 * pairs)
        for by in (np.nextafter(np.float32(1) / np.float32(pairs), np.float32(d)) for d in (0, 2)):
            assert np.array_equal(((i.astype(np.float32) + np.float32(0.5)) * by).astype(np.int64), i // pairs), pairs


def test_empty_calls_launch_nothing():
    assert lib().scoot_rotate(*dict(ROTATE, num_tokens=0).values()) == 0
    assert lib().scoot_kv_append(*dict(APPEND, num_tokens=0).values()) == 0
    assert lib().scoot_kv_append(*dict(APPEND, num_blocks=0, num_heads=0, q=None, q_out=None, k_cache=None).values()) == 0


def test_no_exception_leaves_a_call(tmp_path):
    """The calls return a status where the library's host memory runs out (tests/rotary_alloc_check.cpp, built here)."""
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no host C++ compiler")
    exe = str(tmp_path / "rotary_alloc_check")
    subprocess.run([cxx, "-O1", "-g", "-std=c++17", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "rotary_alloc_check.cpp"), "-o", exe, "-ldl"], check=True)
    env = dict(os.environ, HIP_VISIBLE_DEVICES="-1", ROCR_VISIBLE_DEVICES="-1")  # no launch may come of it
    r = subprocess.run([exe, LIB_PATH], capture_output=True, text=True, env=env, timeout=120)
    assert r.returncode == 0, (r.returncode, r.stdout, r.stderr[-500:])
    lines = [line.split(" ", 3) for line in r.stdout.splitlines()]
    assert [x[0] for x in lines] == ["scoot_rotate", "scoot_kv_append", "scoot_kv_append", "scoot_kv_attention_scaled"]
    for name, thrown, status, message in lines:
        assert int(thrown) > 0 and int(status) == NO_MEMORY and "allocation" in message, (name, thrown, status, message)


# ------------------------------------------------------------------- the binding
torch = pytest.importorskip("torch")
from torch._subclasses.fake_tensor import FakeTensorMode  # noqa: E402


def _fake(*shape, dtype=torch.int32, device="cuda:0"):
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device=device)


def _half(*shape, device="cuda:0"):
    return _fake(*shape, dtype=torch.bfloat16, device=device)


@pytest.fixture
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


def _rotary(pairs=32, **more):
    return S.Rotary(_fake(pairs, dtype=more.pop("dtype", torch.float64), **more))


def _rotate(**change):
    t = dict(x=_half(3, 4, 64), positions=_fake(3), rotary=_rotary(), out=_half(3, 4, 64))
    t.update(change)
    return S.rotate(**t, stream=0)


@pytest.mark.parametrize("change,what", [
    (lambda: dict(x=torch.zeros(3, 4, 64, dtype=torch.bfloat16)), "x must be a device tensor"), (lambda: dict(x=_fake(3, 4, 64, dtype=torch.float32)), "x must be float16"),
    (lambda: dict(x=_half(3, 4, 128)[..., ::2]), "contiguous in its last"), (lambda: dict(x=_half(3, 64)), r"must be \(tokens"),
    (lambda: dict(positions=_fake(4)), "positions must have 3"), (lambda: dict(positions=_fake(3, dtype=torch.int64)), "positions must be int32"),
    (lambda: dict(positions=torch.zeros(3, dtype=torch.int32)), "positions must be a device"), (lambda: dict(positions=_fake(6)[::2]), "positions must be contiguous"),
    (lambda: dict(positions=_fake(3, device="cuda:1")), "positions must be on the device"), (lambda: dict(rotary=None), "must be a Rotary"),
    (lambda: dict(rotary=_rotary(33)), "more pairs than a head"), (lambda: dict(rotary=_rotary(dtype=torch.float32)), "float64"),
    (lambda: dict(rotary=_rotary(device="cuda:1")), "freqs must be on the device"), (lambda: dict(rotary=S.Rotary([1.0])), "float64 device tensor"),
    (lambda: dict(out=_half(3, 4, 32)), "out must be"), (lambda: dict(out=_half(2, 4, 64)), "out must have x's"), (lambda: dict(out=_half(3, 4, 64, device="cuda:1")), "out must be on the device"),
    (lambda: dict(out=_fake(3, 4, 64, dtype=torch.float16)), "out must have x's")])
def test_rotate_of_other_tensors_is_refused(no_call, change, what):
    with pytest.raises(ValueError, match=what):
        _rotate(**change())


def _scales(*shape, **more):
    return _fake(*(shape or (4, 2)), dtype=more.pop("dtype", torch.float32), **more)


def _f8(*shape):
    return _fake(*(shape or (4, 2, 16, 64)), dtype=torch.float8_e4m3fn)


def _append(**change):
    t = dict(k=_half(3, 2, 64), v=_half(3, 2, 64), positions=_fake(3), slots=_fake(3, dtype=torch.int64), k_cache=_half(4, 2, 16, 64),
             v_cache=_half(4, 2, 16, 64), rotary=_rotary(), q=_half(3, 4, 64), out=_half(3, 4, 64))
    t.update(change)
    return S.kv_append(**t, stream=0)


def _in_8():
    return dict(k_cache=_f8(), v_cache=_f8(), k_scale=_scales(), v_scale=_scales())


@pytest.mark.parametrize("change,what", [
    (lambda: dict(k=_half(3, 3, 64)), "k must be"), (lambda: dict(v=_half(2, 2, 64)), "v must have"), (lambda: dict(slots=_fake(3)), "slots must be"),
    (lambda: dict(slots=_fake(4, dtype=torch.int64)), "slots must have 3"), (lambda: dict(positions=None), "positions must be a device tensor"),
    (lambda: dict(positions=_fake(2)), "positions must have 3"), (lambda: dict(rotary=_rotary(40)), "more pairs"), (lambda: dict(rotary="yes"), "must be a Rotary"),
    (lambda: dict(rotary=None), "queries need a rotary"), (lambda: dict(q=None), "out needs queries"), (lambda: dict(q=_half(3, 4, 32)), "q must be"),
    (lambda: dict(q=_half(2, 4, 64)), "q must have"), (lambda: dict(q=_fake(3, 4, 64, dtype=torch.float16)), "q must have"), (lambda: dict(out=_half(3, 5, 64)), "out must"),
    (lambda: dict(k_scale=_scales(), v_scale=_scales()), "need a float8"), (lambda: dict(_in_8(), v_scale=1.0), "both be numbers"),
    (lambda: dict(_in_8(), k_scale=_scales(4, 3)), "k_scale must be"), (lambda: dict(_in_8(), v_scale=_scales(dtype=torch.float64)), "v_scale must be float32"),
    (lambda: dict(_in_8(), v_scale=_scales(2, 4).t()), "v_scale must be contiguous"), (lambda: dict(_in_8(), k_scale=torch.ones(4, 2)), "k_scale must be a device"),
    (lambda: dict(_in_8(), k_scale=_scales(device="cuda:1")), "k_scale must be on the device")])
def test_append_of_other_tensors_is_refused(no_call, change, what):
    with pytest.raises(ValueError, match=what):
        _append(**change())


@pytest.mark.parametrize("name", ["v", "positions", "slots", "k_cache", "v_cache", "q", "out"])
def test_append_across_devices_is_refused(no_call, name):
    shape, dtype = {"v": ((3, 2, 64), torch.bfloat16), "positions": ((3,), torch.int32), "slots": ((3,), torch.int64), "q": ((3, 4, 64), torch.bfloat16),
                    "out": ((3, 4, 64), torch.bfloat16)}.get(name, ((4, 2, 16, 64), torch.bfloat16))
    with pytest.raises(ValueError, match=f"{name} must be on the device of the others"):
        _append(**{name: _fake(*shape, dtype=dtype, device="cuda:1")})


@pytest.mark.parametrize("change,what", [
    (lambda: dict(k_scale=_scales(4, 3)), "k_scale must be"), (lambda: dict(v_scale=_scales(dtype=torch.float16)), "v_scale must be float32"), (lambda: dict(v_scale=0.5), "both be numbers"),
    (lambda: dict(v_scale=_scales(device="cuda:1")), "v_scale must be on the device"), (lambda: dict(k_cache=_half(4, 2, 16, 64), v_cache=_half(4, 2, 16, 64)), "need a float8")])
def test_attention_with_other_scales_is_refused(no_call, change, what):
    t = dict(q=_half(3, 4, 64), block_table=_fake(2, 3), query_start=_fake(3), seq_len=_fake(2), out=_half(3, 4, 64), workspace=_fake(4096, dtype=torch.uint8), **_in_8())
    t.update(change())
    with pytest.raises(ValueError, match=what):
        S.kv_attention(**t, max_new_len=2, max_seq_len=9, stream=0)


@pytest.mark.parametrize("number", [np.float32(0.5), torch.tensor(0.5), torch.tensor([0.5])], ids=str)
def test_numbers_of_other_kinds_are_no_scales_of_blocks(no_call, number):
    """What is wrong is the output, and that is what the error says."""
    with pytest.raises(ValueError, match="out must"):
        _append(k_cache=_f8(), v_cache=_f8(), k_scale=number, v_scale=0.5, out=_half(3, 5, 64))
    with pytest.raises(ValueError, match="out must"):
        S.kv_attention(_half(3, 4, 64), _f8(), _f8(), _fake(2, 3), _fake(3), _fake(2), 2, 9, k_scale=number, v_scale=0.5, out=_half(3, 5, 64),
                       workspace=_fake(4096, dtype=torch.uint8), stream=0)


@pytest.mark.parametrize("stream", [0, 4096])
def test_a_given_stream_and_host_tensors_are_refused(stream):
    x, f = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(32, dtype=torch.float64)
    with pytest.raises(ValueError, match="device"):
        S.rotate(x, torch.zeros(3, dtype=torch.int32), S.Rotary(f), stream=stream)
    cache = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        S.kv_append(x, x, torch.zeros(3, dtype=torch.int32), torch.zeros(3, dtype=torch.int64), cache, cache, rotary=S.Rotary(f), q=x, stream=stream)
