"""Attention over blocks whose scales are far apart, row by row: a row's result is as near to the float64 oracle's as the
blocks that this row sees, at the weights that it gives them, allow.  Blocks that it does not see, because they come later or lie
before its window, have no part in its bound, and neither has the largest scale of the cache."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402
from oracle import kv_cache as kv  # noqa: E402
from test_gpu_kv_cache import BITS, _attend_inputs, _check, dev, f64  # noqa: E402
from test_gpu_kv_scaled import _call, _reference, say  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _case(lens, d, kind="bf16", hq=4, hkv=2, bs=16, window=0, scale=None):
    return dict(lens=lens, kind=kind, cache="f8", hq=hq, hkv=hkv, d=d, bs=bs, window=window, scale=scale, hints=None, stale=0.0)


def _inputs(c, exponents, seed=0):
    """Scales of the values 2^exponents(request, block, blocks of the request, head) and of the keys 0.02; every block is held."""
    s = _attend_inputs(c, seed)
    blocks, hkv = s["k"].shape[:2]
    e = np.zeros((blocks, hkv))
    for r, (a, n) in enumerate(c["lens"]):
        held = -(-(a + n) // c["bs"])
        for i in range(held):
            for h in range(hkv):
                e[s["table"][r, i], h] = exponents(r, i, held, h)
    s["ks"], s["vs"] = torch.full((blocks, hkv), 0.02, device=DEV), dev(np.exp2(e), torch.float32)
    return s, e


def _row_top(c, s):
    """The largest |value| that each row sees, (tokens, heads, 1)."""
    v = np.abs(f64(s["v"])).max(-1) * f64(s["vs"])[:, :, None]
    top = np.zeros((int(s["start"][-1]), c["hq"], 1))
    for r, (a, n) in enumerate(c["lens"]):
        at = np.arange(a + n)
        size = v[s["table"][r, at // c["bs"]], :, at % c["bs"]]  # (keys, kv heads)
        for j in range(n):
            first = max(0, a + j + 1 - c["window"]) if c["window"] else 0
            seen = size[first:a + j + 1].max(0)
            top[int(s["start"][r]) + j, :, 0] = np.repeat(seen, c["hq"] // c["hkv"])
    return top


def _row_bound(c, s, ref, top):
    """The oracle's bound, weights to 11 bits, and those that are lost below 2^-25 of the largest times the row's own largest value
    `top`; beside it what a scale's logarithm adds (2^-24 of the scores, and 2^-21)."""
    out, spread, reach = ref
    keys = max(a + n for a, n in c["lens"])
    more = (3 * 2.0 ** -24 * reach[..., None] + 2.0 ** -21) * (spread + np.abs(out))
    return kv.attention_bound(out, spread, reach, keys, c["d"], BITS[c["kind"]], 11, top) + more


FORMS = {"few": ([(21, 6), (3, 1)], 8, 2), "few_parts": ([(6300, 6)], 8, 2), "tiles": ([(0, 150), (70, 40)], 16, 4), "tiles_far": ([(300, 100)], 16, 4),
         "tiles_parts": ([(4500, 60)], 16, 4)}


@pytest.mark.parametrize("d,kind", [(64, "f16"), (128, "bf16"), (192, "bf16"), (256, "f16")])
@pytest.mark.parametrize("far", [20, 30, 60, 128])
@pytest.mark.parametrize("form", list(FORMS))
def test_later_blocks_have_no_part_in_earlier_rows(form, far, d, kind):
    """The last block of every request, which its first new tokens do not see, has values 2^far times as large."""
    say("rows, later", form, far, d, kind)
    lens, bs, hq = FORMS[form]
    c = _case(lens, d, kind, hq=hq, bs=bs)
    low = -64 if far > 60 else -far // 2 if kind == "bf16" else -6
    high = low + far if kind == "bf16" or far <= 20 else low + 20
    if high - low < far:
        high = low + far  # beyond half precision: those rows are infinite in the reference's type, and are left out
    s, _ = _inputs(c, lambda r, i, held, h: high if i == held - 1 else low)
    got, ref = f64(_call(c, s)), _reference(c, s)
    bound = _row_bound(c, s, ref, _row_top(c, s))
    # Numbers that are none of the result's type: below half of its smallest step, or above its largest.
    tiny, most = (2.0 ** -25, 65504.0) if kind == "f16" else (2.0 ** -134, 3.38e38)
    ok = np.abs(ref[0]) + bound < most
    assert ok[int(s["start"][0])].all() and ok.any(-1).any(0).all()
    _check(np.where(ok, got, 0), np.where(ok, ref[0], 0), np.where(ok, bound + tiny, 1))


@pytest.mark.parametrize("d,kind", [(64, "bf16"), (128, "f16"), (192, "f16"), (256, "bf16")])
@pytest.mark.parametrize("lens,window,bs", [([(300, 8)], 5, 8), ([(300, 60), (90, 1)], 40, 16), ([(5000, 70)], 300, 8), ([(900, 2)], 100, 32)])
def test_blocks_before_the_window_have_no_part(lens, window, bs, d, kind):
    """Blocks that the first new tokens see, and the last ones do not, are 2^40 times as large."""
    say("rows, window", lens, window, bs, d, kind)
    c = _case(lens, d, kind, hq=2, bs=bs, window=window)
    s, _ = _inputs(c, lambda r, i, held, h: 34 if (i + 1) * bs <= lens[r][0] + lens[r][1] - window else -6)
    got, ref = f64(_call(c, s)), _reference(c, s)
    bound = _row_bound(c, s, ref, _row_top(c, s))
    ok = np.abs(ref[0]) + bound < (65504.0 if kind == "f16" else 3e38)
    assert ok[-1].all()
    _check(np.where(ok, got, 0), np.where(ok, ref[0], 0), np.where(ok, bound + 2.0 ** -25, 1))


@pytest.mark.parametrize("share", [0.25, 0.5, 1.0])
@pytest.mark.parametrize("far", [(-64, 64), (-20, 20), (-30, 0), (0, 18)])
@pytest.mark.parametrize("lens,d", [([(600, 1)], 64), ([(6000, 1)], 128), ([(600, 40)], 64), ([(3000, 40)], 128), ([(300, 90)], 256), ([(2000, 2)], 192)])
def test_large_blocks_of_small_weights(lens, d, far, share):
    """Blocks of large values whose weights are as much smaller (share 1), or less so: both kinds count, and no weight is lost,
    however small it is."""
    say("rows, weights", lens, d, far, share)
    c = _case(lens, d)
    rng = np.random.default_rng(d)
    s, e = _inputs(c, lambda r, i, held, h: rng.choice(far), 7)
    k = s["k"].float() * 0.25
    k[..., 0] = 0.0
    k[torch.as_tensor(e == far[0], device=DEV), :, 0] = 64.0  # says how heavy a block is
    q = s["q"].float()
    q[..., 0] = share * (far[1] - far[0]) * np.log(2.0) * d ** 0.5 / (64 * 0.02)
    s.update(k=k.to(s["k"].dtype), q=q.to(torch.bfloat16))
    got, ref = f64(_call(c, s)), _reference(c, s)
    _check(got, ref[0], _row_bound(c, s, ref, 0.0))


@pytest.mark.parametrize("spread", [0, 6, 14, 15, 16, 17, 21, 22])
@pytest.mark.parametrize("lens,d", [([(150, 1)], 64), ([(9000, 3)], 128), ([(0, 70)], 128), ([(4700, 40)], 64), ([(90, 40)], 192), ([(40, 90)], 256)])
def test_every_code_at_every_distance(lens, d, spread):
    """All 254 codes, the smallest ones among them, with equal weights, in blocks that are `spread` octaves apart: few, then one
    that comes late, after all others were done, for some heads larger and for some smaller."""
    say("rows, codes", lens, d, spread)
    c = _case(lens, d, "bf16", scale=0.0)
    s, _ = _inputs(c, lambda r, i, held, h: (spread if (i == held - 1) == (h == 0) else 0) - 7)
    codes = torch.arange(s["v"].numel(), device=DEV) * 37 % 256
    codes[(codes & 127) == 127] = 1
    s["v"] = codes.to(torch.uint8).view(torch.float8_e4m3fn).view(s["v"].shape)
    got, ref = f64(_call(c, s)), _reference(c, s)
    # The same weight for every key: nothing of it is rounded.  What is left: the sums in float, and the result's rounding.
    out, size, _ = ref
    keys = max(a + n for a, n in c["lens"])
    _check(got, out, 2.0 ** -8 * np.abs(out) + 1.05 * (keys + 8) * 2.0 ** -24 * (size + np.abs(out)))


@pytest.mark.parametrize("lens,d", [([(50, 100)], 64), ([(60, 7)], 128), ([(4500, 50)], 128), ([(100, 40)], 256)])
def test_values_that_are_no_numbers_beside_blocks_far_apart(lens, d):
    say("rows, not numbers", lens, d)
    a, n = lens[0]
    c = _case(lens, d, hq=2)
    s, _ = _inputs(c, lambda r, i, held, h: 20 if i == held - 1 else -20)
    at, head, dim = a + n // 2, 1, d - 3
    v = s["v"].float()
    v[int(s["table"][0, at // 16]), head, at % 16, dim] = float("nan")
    ref = _reference(c, s)
    bound = _row_bound(c, s, ref, _row_top(c, s))
    got = f64(_call(c, dict(s, v=v.to(s["v"].dtype))))
    nan = np.zeros_like(got, dtype=bool)
    nan[n // 2:, head, dim] = True
    assert (np.isnan(got) == nan).all()
    _check(np.where(nan, ref[0], got), ref[0], bound)


@pytest.mark.parametrize("lens,d", [([(50, 100)], 64), ([(60, 7)], 128), ([(4500, 50)], 128), ([(9000, 1)], 192)])
def test_blocks_far_apart_twice_are_the_same_bits(lens, d):
    c = _case(lens, d, hq=2)
    s, _ = _inputs(c, lambda r, i, held, h: 20 if i % 3 == 2 else -20)
    a, b = _call(c, s), _call(c, s)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))


@pytest.mark.parametrize("kind", ["bf16", "f16"])
@pytest.mark.parametrize("lens,d,window", [([(200, 1), (90, 5)], 64, 0), ([(300, 60), (40, 1)], 128, 45), ([(5000, 40)], 64, 700), ([(130, 70)], 192, 0),
                                           ([(220, 40)], 256, 60)])
def test_missing_blocks_and_any_scales_far_apart(lens, d, window, kind):
    """Scales of any fraction, 2^-10 to 2^18 for halves of the blocks; entries that name no block inside what rows see, and, before
    the window, blocks whose scales are no numbers."""
    say("rows, missing", lens, d, window, kind)
    c = _case(lens, d, kind, window=window)
    rng = np.random.default_rng(d)
    s, _ = _inputs(c, lambda r, i, held, h: rng.choice([-10, 18]) + rng.uniform(-1, 1) if kind == "bf16" else rng.choice([-14, 3]) + rng.uniform(-1, 1))
    held_by = [s["table"][r, i] for r, (a, n) in enumerate(lens) for i in range(-(-(a + n) // 16))]
    junk = min(set(range(s["k"].shape[0])) - set(held_by))
    top = np.abs(f64(s["v"])).max() * f64(s["vs"]).max()
    for r, (a, n) in enumerate(lens):
        held = -(-(a + n) // 16)
        if held > 6:
            s["table"][r, held // 2] = rng.choice([-1, s["k"].shape[0], 2 ** 31 - 1])
            s["table"][r, held - 2] = -1
        if window:
            s["table"][r, :max(0, a + 1 - window) // 16] = junk
    ref = _reference(c, s)
    bound = _row_bound(c, s, ref, top)
    for x in (s["k"], s["v"]):
        x.view(torch.uint8)[junk] = 0x7f  # no number
    s["ks"][junk], s["vs"][junk] = float("nan"), float("inf")
    got = f64(_call(c, s))
    ok = np.abs(ref[0]) + bound < (65504.0 if kind == "f16" else 3e38)
    assert ok[-1].all()
    _check(np.where(ok, got, 0), np.where(ok, ref[0], 0), np.where(ok, bound + 2.0 ** -25, 1))


@pytest.mark.parametrize("tokens,d,length", [(1, 64, 700), (4, 128, 5000), (40, 64, 300), (40, 256, 300), (40, 128, 4000)])
def test_fractions_of_scales_beside_large_scores(tokens, d, length):
    """Values' scales that are no powers of two beside scores of any size: every third key has the same score x, the others
    1.5 x (x negative) or 0.5 x, whose weights are below 2^-1000 of theirs or, for the smallest x, as the oracle's softmax says.
    What is off: the weights' rounding (2^-11) and the logarithm of a scale (2^-21), the result's rounding (2^-8), sums in float,
    and, with scores below 2^11, at which a scale's logarithm is added to them, 2^-13 of the weights."""
    say("rows, fractions", tokens, d, length)
    blocks = -(-length // 16)
    g = torch.Generator(device=DEV).manual_seed(3)
    codes = torch.randn(blocks, 1, 16, d, generator=g, device=DEV).mul_(50).clamp_(-448, 448).to(torch.float8_e4m3fn)
    vs = (torch.rand(blocks, 1, generator=g, device=DEV) * 4 - 2).exp2_()
    ks = torch.randint(-3, 4, (blocks, 1), generator=g, device=DEV).float().exp2_()
    third = torch.arange(blocks * 16, device=DEV) % 3 == 0
    v = (codes.double() * vs[:, :, None, None].double()).view(-1, d)
    mean = ((v * third[:, None]).cumsum(0) / third.cumsum(0)[:, None])[:length]
    size_of = ((v.abs() * third[:, None]).cumsum(0) / third.cumsum(0)[:, None])[:length]
    table = torch.arange(blocks, dtype=torch.int32, device=DEV)[None]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for size in (1.4e3, 1e4, 1e6, 2e7, 3e7, 1.1e8, 3e9, 1e15, 1e30, 1e37):
        for sign in (-1.0, 1.0):
            k = torch.zeros(blocks * 16, d, device=DEV)
            k[:, 1] = 16.0 * torch.where(third, 1.0, 1.5 if sign < 0 else 0.5)
            k = (k.view(blocks, 1, 16, d) / ks[:, :, None, None]).to(torch.float8_e4m3fn)
            q = torch.zeros(tokens, 2, d, dtype=torch.bfloat16, device=DEV)
            q[..., 1] = sign * min(size / 16, 3e36)
            n = min(tokens, length)
            scale = size / (float(q[0, 0, 1].abs()) * 16.0)
            got = S.kv_attention(q, k, codes, table, i32(0, tokens), i32(length), tokens, length, scale=scale, k_scale=ks, v_scale=vs)
            off = (got[tokens - n:].double() - mean[length - n:, None]).abs()
            weights = 2 * (2.0 ** -11 + 2.0 ** -21 + (2.0 ** -13 if size < 2048 else 0.0)) + length * 2.0 ** -23
            bound = 2.0 ** -8 * mean[length - n:, None].abs() + weights * size_of[length - n:, None] * 1.01
            assert (off <= bound).all(), (size, sign, float((off / bound).max()))
