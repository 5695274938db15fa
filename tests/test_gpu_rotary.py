"""Rotations by position on the GPU against the float64 oracle, within the bound of their roundings."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402
from oracle import rotary as R  # noqa: E402
from rotary_cases import pair_size, rotate_bound  # noqa: E402
from test_gpu_kv_cache import TYPES, dev, f64  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


def check(got, x, positions, freqs, magnitude, interleaved, reverse, kind):
    """Rows of negative positions are not looked at."""
    live = np.asarray(positions) >= 0
    want = R.rotate(x[live], np.asarray(positions)[live], freqs, magnitude, interleaved, reverse)
    off = np.abs(got[live] - want)
    bound = rotate_bound(x[live], want, len(freqs), interleaved, magnitude, kind)
    bad = ~(off <= bound)
    assert not bad.any(), f"{bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0].tolist()}, most {np.nanmax(off / bound):.3g} bounds"


# tokens, heads, dim, turned: pieces of eight, single elements, parts of a head, heads past 256 threads
SHAPES = [(1, 1, 8, 8), (1, 40, 128, 128), (3, 9, 64, 64), (65, 5, 64, 32), (7, 48, 128, 64), (33, 3, 192, 64), (300, 2, 80, 32), (17, 4, 96, 24),
          (5, 3, 72, 6), (9, 2, 1024, 1024), (2, 3, 1024, 1022), (4, 6, 40, 40), (11, 1024, 8, 2), (2500, 9, 256, 256), (40, 3, 24, 0), (6, 2, 48, 40)]


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_rotate_matches_oracle(shape, kind, interleaved):
    tokens, heads, dim, turned = shape
    say("rotate", shape, kind, interleaved)
    rng = np.random.default_rng(tokens + dim + turned)
    x = dev(rng.standard_normal((tokens, heads, dim)) * np.exp(rng.uniform(-4, 4, (tokens, 1, 1))), TYPES[kind])
    pos = rng.integers(0, 1 << 17, tokens)
    freqs = R.frequencies(turned, 10000.0)[0] if turned else np.zeros(0)
    rot = S.Rotary(dev(freqs, torch.float64), 1.0 if turned < dim else 1.21, interleaved)
    for reverse in (False, True):
        got = S.rotate(x, dev(pos, torch.int32), rot, reverse=reverse)
        check(f64(got), f64(x), pos, freqs, rot.magnitude, interleaved, reverse, kind)
        assert torch.equal(got[..., turned:], x[..., turned:])


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shape", [(13, 5, 128, 128), (9, 3, 64, 32), (21, 2, 192, 64), (3, 2, 1024, 1022)], ids=str)
def test_rotate_of_strided_rows_and_in_place(shape, interleaved):
    """Rows inside a fused projection, aligned to 16 bytes and not; results into others; and a part of every head in place."""
    tokens, heads, dim, turned = shape
    say("rotate strided", shape, interleaved)
    rng = np.random.default_rng(dim)
    pos, freqs = rng.integers(0, 5000, tokens), R.frequencies(turned)[0]
    rot = S.Rotary(dev(freqs, torch.float64), 1.0, interleaved)
    for start in (8, 3):
        fused = dev(rng.standard_normal((tokens, heads * dim + 31)), torch.bfloat16)
        fused = torch.cat([fused, fused[:, :9]], 1)[:, :heads * dim + 32]
        x = fused[:, start:start + heads * dim].view(tokens, heads, dim)
        res = torch.full((tokens, heads + 1, dim + 16), 7.0, dtype=torch.bfloat16, device=DEV)
        out = res[:, 1:, 8:8 + dim]
        assert S.rotate(x, dev(pos, torch.int32), rot, out=out) is out
        check(f64(out), f64(x), pos, freqs, 1.0, interleaved, False, "bf16")
        want = out.clone()
        res[:, 1:, 8:8 + dim] = 7.0
        assert (res == 7.0).all()
        before = fused.clone()
        S.rotate(x, dev(pos, torch.int32), rot, out=x)
        assert torch.equal(x, want)
        fused[:, start:start + heads * dim] = before[:, start:start + heads * dim]
        assert torch.equal(fused, before)
        if turned % 8:
            continue  # no head of its own
        # The last `turned` elements of every head: a view, in place.
        tail = x[..., dim - turned:]
        want = S.rotate(tail.contiguous(), dev(pos, torch.int32), rot)
        head = x[..., :dim - turned].clone()
        S.rotate(tail, dev(pos, torch.int32), rot, out=tail)
        assert torch.equal(tail, want) and torch.equal(x[..., :dim - turned], head)


def test_rows_of_negative_positions_stay():
    rng = np.random.default_rng(3)
    x = dev(rng.standard_normal((70, 6, 64)), torch.float16)
    pos = rng.integers(-5, 50, 70)
    pos[[0, 69]] = [-1, -2 ** 31]
    rot = S.rotary_create(64)
    out = torch.full_like(x, 3.0)
    S.rotate(x, dev(pos, torch.int32), rot, out=out)
    assert (out[dev(pos < 0, torch.bool)] == 3.0).all() and (pos < 0).sum() > 3
    check(f64(out), f64(x), pos, f64_freqs(rot), 1.0, False, False, "f16")


def test_nothing_to_turn_copies_every_row():
    """Without pairs the positions are not looked at."""
    x = dev(np.random.default_rng(4).standard_normal((5, 3, 40)), torch.bfloat16)
    none = S.Rotary(torch.zeros(0, dtype=torch.float64, device=DEV))
    assert torch.equal(S.rotate(x, dev([-1, 0, -7, 3, 2 ** 31 - 1], torch.int32), none), x)


def f64_freqs(rot):
    return rot.freqs.cpu().numpy()


@pytest.mark.parametrize("most", [2 ** 20, 2 ** 31 - 1])
def test_far_positions(most):
    """The angle is a product in double, as the oracle's; frequencies above 1, negative and zero, too."""
    rng = np.random.default_rng(5)
    x = dev(rng.standard_normal((64, 4, 64)), torch.float16)
    pos = np.concatenate([most - rng.integers(0, 1000, 62), [0, most]])
    freqs = np.concatenate([R.frequencies(32)[0], [0.0, -0.5, 2.0, 6.5, 100.0, 1e-9, np.pi, np.pi / 2], rng.uniform(0, 1, 8)])
    got = S.rotate(x, dev(pos, torch.int32), S.Rotary(dev(freqs, torch.float64)))
    # Angles of up to 2^38 radians: 2^-53 of that, once in the product (the same on both sides) and in the oracle's cosine.
    check(f64(got), f64(x), pos, freqs, 1.0, False, False, "f16")


def test_values_that_are_not_finite_stay_in_their_pairs():
    x = torch.ones(2, 3, 64, dtype=torch.bfloat16, device=DEV)
    x[0, 0, 3], x[0, 1, 40], x[1, 2, 50], x[1, 0, 0] = float("nan"), float("inf"), float("-inf"), 3e38
    rot = S.Rotary(dev(R.frequencies(32)[0], torch.float64))  # of 64 elements 32: pairs (i, i + 16)
    got = S.rotate(x, dev([5, 7], torch.int32), rot)
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[0, 0, [3, 19]] = True
    bad[0, 1, 40] = bad[1, 2, 50] = True
    assert torch.equal(~torch.isfinite(got), bad)
    assert got[0, 1, 40] == float("inf") and got[1, 2, 50] == float("-inf")


def test_reverse_is_the_gradient_and_turns_back():
    """Against differences: rotate is linear, so (y(x + d) - y(x)) . g over a large d is the gradient's product with d, up to
    the roundings of the two results and of the gradient."""
    rng = np.random.default_rng(6)
    x, d, g = (dev(rng.standard_normal((40, 4, 128)), torch.float16) for _ in range(3))
    pos = dev(rng.integers(0, 4096, 40), torch.int32)
    rot = S.rotary_create(128, scaling="ramp", factor=8.0, length=512)
    grad = S.rotate(g, pos, rot, reverse=True)
    both = (x + d)
    step = f64(both) - f64(x)
    rise = f64(S.rotate(both, pos, rot)) - f64(S.rotate(x, pos, rot))
    got, want = (rise * f64(g)).sum((1, 2)), (step * f64(grad)).sum((1, 2))
    size = rot.magnitude * 2.0 * 2.0 ** -11 * ((np.abs(f64(both)) + np.abs(f64(x)) + np.abs(step)) * 1.0)
    # Each result is off by 2^-11 of itself, at most of |a| + |b|; 1.5 for those of a pair's partner.
    slack = 1.5 * (size.reshape(40, 4, 2, 64).sum(2, keepdims=True).repeat(2, 2).reshape(40, 4, 128) * (np.abs(f64(g)) + np.abs(f64(grad)))).sum((1, 2))
    assert (np.abs(got - want) <= slack).all()
    plain = S.rotary_create(128)
    back = S.rotate(S.rotate(x, pos, plain), pos, plain, reverse=True)
    y = pair_size(f64(x), 64, False)
    assert (np.abs(f64(back) - f64(x)) <= 2 * 2.0 ** -11 * y + 2.0 ** -11 * np.abs(f64(x)) + 1e-6 * y).all()


def test_on_another_stream_and_twice_the_same_bits():
    rng = np.random.default_rng(7)
    x, pos = dev(rng.standard_normal((500, 8, 128)), torch.bfloat16), dev(rng.integers(0, 9999, 500), torch.int32)
    rot = S.rotary_create(128)
    want = S.rotate(x, pos, rot)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for i in range(10):
        got = S.rotate(x, pos, rot, stream=side.cuda_stream)
        junk = torch.full((1 << 21,), float("nan"), device=DEV)
        side.synchronize()
        assert torch.equal(got, want), i
        del junk
    assert torch.equal(S.rotate(x, pos, rot, stream=0), want)


def test_no_tokens():
    rot = S.rotary_create(64)
    got = S.rotate(torch.empty(0, 4, 64, dtype=torch.float16, device=DEV), dev([], torch.int32), rot)
    assert got.shape == (0, 4, 64)
