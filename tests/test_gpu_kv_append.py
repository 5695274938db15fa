"""Appends on the GPU against the float64 oracle: queries and keys within the bound of their roundings, values and scales
exactly, and what a growing scale makes of earlier values exactly."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402
from oracle import kv_cache as kv  # noqa: E402
from oracle import rotary as R  # noqa: E402
from rotary_cases import BITS, TINY, pair_size, turned_bound  # noqa: E402
from test_gpu_kv_cache import TYPES, dev, f64  # noqa: E402
from test_gpu_rotary import check as check_turned  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


def _case(lens, kind="bf16", cache=None, scales=None, hq=4, hkv=2, d=64, turned=None, pairs=False, bs=16, odd=0, queries=True):
    """``lens``: (context, new) of the requests.  ``scales``: one, two (powers of two) or any numbers per block and head;
    ``odd``: rows that start off 16 bytes."""
    return dict(lens=lens, kind=kind, cache=cache or kind, scales=scales, hq=hq, hkv=hkv, d=d, turned=d if turned is None else turned,
                pairs=pairs, bs=bs, odd=odd, queries=queries)


CASES = {
    "one": _case([(0, 1)]),
    "decode": _case([(i * 37 % 300, 1) for i in range(70)], hq=32, hkv=8, d=128, kind="f16"),
    "chunk": _case([(5, 100), (0, 33), (17, 1)], hq=7, hkv=1, d=128, turned=64),
    "wide": _case([(9, 40)], hq=2, hkv=1, d=256, pairs=True, bs=32),
    "odd_rows": _case([(9, 40), (3, 3)], hq=3, hkv=2, d=64, odd=1, bs=8),
    "odd_pairs": _case([(9, 40), (3, 3)], hq=3, hkv=2, d=80, turned=20, bs=8, kind="f16"),
    "keys_alone": _case([(9, 40)], queries=False),
    "nothing_turned": _case([(9, 40)], queries=False, turned=0, kind="f16"),
    "f8": _case([(5, 100), (0, 1)], cache="f8", scales="one", hq=8, hkv=2, d=128),
    "f8_odd": _case([(5, 20), (0, 1)], cache="f8", scales="one", hq=3, hkv=5, d=24, turned=10, kind="f16", pairs=True),
    "f8_nothing_turned": _case([(5, 20)], cache="f8", scales="one", turned=0, queries=False),
    "blocks_one": _case([(0, 1)], cache="f8", scales="two"),
    "blocks_decode": _case([(i * 37 % 300, 1) for i in range(70)], cache="f8", scales="two", hq=32, hkv=8, d=128),
    "blocks_decode_any": _case([(i * 29 % 200, 1 + i % 3) for i in range(40)], cache="f8", scales="any", hq=4, hkv=4, d=64, kind="f16"),
    "blocks_chunk": _case([(5, 100), (0, 33), (17, 1), (30, 0)], cache="f8", scales="two", hq=8, hkv=2, d=128),
    "blocks_chunk_any": _case([(5, 100), (0, 33), (17, 2)], cache="f8", scales="any", hq=5, hkv=5, d=64, bs=8, kind="f16"),
    "blocks_32": _case([(5, 100), (50, 70), (17, 2)], cache="f8", scales="two", hq=10, hkv=2, d=192, turned=64, bs=32),
    "blocks_256": _case([(300, 500), (17, 2)], cache="f8", scales="two", hq=2, hkv=1, d=64, bs=256),
    "blocks_256_wide": _case([(100, 300)], cache="f8", scales="two", hq=1, hkv=1, d=256, bs=256),
    "blocks_1024": _case([(3, 20), (0, 9)], cache="f8", scales="two", hq=1, hkv=2, d=1024, bs=8),
    "blocks_1024_of_64": _case([(3, 90)], cache="f8", scales="any", hq=1, hkv=1, d=1024, bs=64),
    "blocks_pairs": _case([(3, 90)], cache="f8", scales="two", hq=2, hkv=2, d=128, turned=72, pairs=True),
    "blocks_single_elements": _case([(3, 90), (11, 1)], cache="f8", scales="any", hq=2, hkv=3, d=72, turned=6, bs=8, kind="f16"),
    "blocks_odd_rows": _case([(3, 90), (11, 1)], cache="f8", scales="two", hq=2, hkv=3, d=64, odd=3, bs=32),
    "blocks_odd_wide": _case([(3, 30)], cache="f8", scales="two", hq=2, hkv=1, d=1024, odd=1, bs=16, pairs=True),
    "blocks_nothing_turned": _case([(3, 90), (11, 1)], cache="f8", scales="two", turned=0, queries=False, hkv=9),
    "blocks_many": _case([(i % 23, 1 + 60 * (i % 40 == 7)) for i in range(2500)], cache="f8", scales="two", hq=2, hkv=1, d=64, bs=8),
}


def _inputs(c, seed):
    rng = np.random.default_rng(seed)
    lens, bs, hq, hkv, d = c["lens"], c["bs"], c["hq"] if c["queries"] else 0, c["hkv"], c["d"]
    tokens = sum(n for _, n in lens)
    x = rng.standard_normal((tokens, (hq + 2 * hkv) * d + 8)) * np.exp(rng.uniform(-1.5, 1.5, (tokens, 1)))
    x = dev(x, TYPES[c["kind"]])
    at = lambda i, n: x[:, c["odd"] + i * d:c["odd"] + (i + n) * d].view(tokens, n, d)  # noqa: E731
    s = dict(q=at(0, hq) if hq else None, k=at(hq, hkv), v=at(hq + hkv, hkv))
    need = [-(-(a + n) // bs) for a, n in lens]
    order = rng.permutation(sum(need) + 3)
    pos, slots, first = [], [], 0
    for (a, n), m in zip(lens, need):
        p = np.arange(a, a + n)
        pos.append(p)
        slots.append(order[first + p // bs] * bs + p % bs)
        first += m
    s["pos"], s["slots"] = np.concatenate(pos), np.concatenate(slots)
    total = len(order)
    codes = kv.round_e4m3(rng.standard_normal((2, total, hkv, bs, d)) * 90)
    s["k_cache"], s["v_cache"] = (dev(y, torch.float32).to(TYPES[c["cache"]]) for y in codes)
    s["k_scale"], s["v_scale"] = (0.03, 0.7) if c["scales"] == "one" else (1.0, 1.0)
    if c["scales"] in ("two", "any"):
        for name in ("k_scale", "v_scale"):
            e = rng.uniform(-10, -6, (total, hkv))
            s[name] = dev(np.exp2(np.floor(e) if c["scales"] == "two" else e), torch.float32)
    pairs = c["turned"] // 2
    s["freqs"] = R.frequencies(c["turned"])[0] if pairs else np.zeros(0)
    s["rotary"] = S.Rotary(dev(s["freqs"], torch.float64), 1.1, c["pairs"]) if pairs else None
    return s


def _call(s, **more):
    args = dict(rotary=s["rotary"], k_scale=s["k_scale"], v_scale=s["v_scale"], q=s["q"])
    args.update(more)
    return S.kv_append(s["k"], s["v"], dev(s["pos"], torch.int32), dev(s["slots"], torch.int64), s["k_cache"], s["v_cache"], **args)


def _clone(s):
    return {k: v.clone() if k in ("k_cache", "v_cache", "k_scale", "v_scale") and torch.is_tensor(v) else v for k, v in s.items()}


def _check(c, s, before, got):
    """What the call made of `before`: s after it, and the queries."""
    pairs, il = c["turned"] // 2, c["pairs"]
    mag = s["rotary"].magnitude if pairs else 1.0
    slots = np.where(s["pos"] >= 0, s["slots"], -1) if pairs else s["slots"]
    if s["q"] is not None:
        check_turned(f64(got), f64(s["q"]), s["pos"], s["freqs"], mag, il, False, c["kind"])
    for name in ("k", "v"):
        x = f64(s[name])
        turns = name == "k" and pairs > 0
        y = R.rotate(x, s["pos"], s["freqs"], mag, il) if turns else x
        off = turned_bound(pair_size(x, pairs, il), mag) if turns else np.zeros_like(x)
        cache, old = f64(s[name + "_cache"]), f64(before[name + "_cache"])
        stored = kv.write(y, slots, old, lambda z: z)
        slack = kv.write(off, slots, np.zeros_like(old), lambda z: z)
        new = kv.write(np.ones_like(x), slots, np.zeros_like(old), lambda z: z) > 0
        if c["cache"] != "f8":
            bound = np.where(new, slack + (2.0 ** -BITS[c["kind"]] * (np.abs(stored) + slack) + TINY[c["kind"]]) * turns, 0)
            assert (np.abs(cache - stored) <= bound).all(), name
            continue
        if c["scales"] == "one":
            scale, codes = np.float32(s[name + "_scale"]), np.where(new, stored / float(np.float32(s[name + "_scale"])), old)
        else:
            codes, scale, _ = R.append_scaled(y, slots, old, before[name + "_scale"].cpu().numpy())
            np.testing.assert_array_equal(s[name + "_scale"].cpu().numpy(), scale, err_msg=name)
            scale = scale[:, :, None, None].astype(np.float64)
        np.testing.assert_array_equal(np.where(new, 0, cache), np.where(new, 0, codes), err_msg=name)  # earlier and other values
        if turns:
            # The float that is rounded to 8 bits is off by the turn's bound and one division (2^-24).
            codes = np.clip(codes, -448, 448)
            near = (slack / scale + 2.0 ** -24 * np.abs(codes)) * 1.01
            step = 2.0 ** -4 * (np.abs(codes) + near) + 2.0 ** -10
            assert (np.abs(cache - codes) <= np.where(new, step + near, 0)).all(), name
        else:
            exact = kv.round_e4m3((stored.astype(np.float32) / np.float32(scale)).astype(np.float64))
            np.testing.assert_array_equal(np.where(new, cache, 0), np.where(new, exact, 0), err_msg=name)


@pytest.mark.parametrize("name", list(CASES))
def test_append_matches_oracle(name):
    c = CASES[name]
    say("append", name)
    s = _inputs(c, len(name))
    before = _clone(s)
    _check(c, s, before, _call(s))


@pytest.mark.parametrize("name", ["decode", "blocks_decode", "blocks_chunk", "blocks_odd_rows", "f8"])
def test_append_without_queries_and_twice(name):
    """Keys and values alone are the same bits; a second call on what the first one left changes nothing."""
    c = CASES[name]
    say("append twice", name)
    s = _inputs(c, 3)
    t = _clone(s)
    q = _call(s)
    assert _call(t, q=None) is None
    first = _clone(s)
    again = _call(s)
    assert torch.equal(q, again)
    for k in ("k_cache", "v_cache"):
        assert torch.equal(s[k].view(torch.uint8), t[k].view(torch.uint8)) and torch.equal(s[k].view(torch.uint8), first[k].view(torch.uint8))
    if torch.is_tensor(s["k_scale"]):
        assert torch.equal(s["k_scale"], t["k_scale"]) and torch.equal(s["v_scale"], first["v_scale"])


@pytest.mark.parametrize("name", ["chunk", "f8", "blocks_chunk", "blocks_256", "blocks_decode_any", "odd_rows"])
def test_tokens_that_are_skipped(name):
    """Negative positions skip a token whole, slots outside the cache only its key and value; its neighbours' blocks are then
    runs of their own."""
    c = CASES[name]
    say("append skipped", name)
    s = _inputs(c, 4)
    rng = np.random.default_rng(1)
    n = len(s["pos"])
    slots = s["k_cache"].shape[0] * c["bs"]
    last = max(0, n - 1)  # whole tails of requests, so that a block's tokens stay rows in a row
    ends = np.cumsum([m for _, m in c["lens"]])
    for i, e in enumerate(ends):
        if i % 2 == 0:
            s["slots"][max(0, e - 3):e] = [-1, slots, 2 ** 40][-min(3, e):]
        else:
            s["pos"][max(ends[i - 1], e - 2):e] = -1
    before = _clone(s)
    out = torch.full_like(s["q"], 5.0)
    assert _call(s, out=out) is out
    assert (out[dev(s["pos"] < 0, torch.bool)] == 5.0).all()
    _check(c, s, before, out)
    assert last >= 0 and rng is not None


def test_queries_in_place():
    c = CASES["blocks_chunk"]
    s = _inputs(c, 5)
    t = _clone(s)
    want = _call(t)
    q = s["q"].clone()
    assert _call(s, q=q, out=q) is q and torch.equal(q, want)


@pytest.mark.parametrize("d,bs", [(64, 8), (128, 16), (256, 256)])
def test_a_scale_over_steps(d, bs):
    """Token after token into one block, each larger than those before, then smaller ones: the scale is the oracle's after
    every step, and values that were stored stay what they were until they fall below the format's normal range."""
    say("growing", d, bs)
    rng = np.random.default_rng(d)
    kc, vc = (torch.zeros(3, 2, bs, d, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
    ks, vs = torch.full((3, 2), float("nan"), device=DEV), torch.full((3, 2), -1.0, device=DEV)
    codes, scales = f64(vc), vs.cpu().numpy()
    held = np.zeros((2, bs, d))
    for j in range(min(bs, 24)):
        size = 2.0 ** (j - 5) if j < 12 else 2.0 ** (4 - j)
        k, v = (dev(size * rng.standard_normal((1, 2, d)), torch.bfloat16) for _ in range(2))
        slot = dev([bs + j], torch.int64)
        S.kv_append(k, v, None, slot, kc, vc, k_scale=ks, v_scale=vs)
        codes, scales, fresh = R.append_scaled(f64(v), [bs + j], codes, scales)
        codes = np.where(fresh[:, None, :, None], kv.round_e4m3(codes), codes)
        np.testing.assert_array_equal(vs.cpu().numpy(), scales)
        np.testing.assert_array_equal(f64(vc)[1], codes[1])
        held[:, j] = f64(v)[0]
        now = f64(vc)[1] * scales[1][:, None, None]
        # Rounded once on its way in (2^-4 of itself, or half a smallest step, 2^-10 E), and by half a smallest step of the new
        # scale at each growth.  Scales at least double: E + E / 2 + E / 4 + ... < 2 E.
        assert (np.abs(now - held)[:, :j + 1] <= 2.0 ** -4 * np.abs(held[:, :j + 1]) + 2 * 2.0 ** -10 * scales[1][:, None, None]).all()
    assert torch.isnan(ks[[0, 2]]).all() and (vs[[0, 2]] == -1.0).all() and torch.isfinite(ks[1]).all()


@pytest.mark.parametrize("turned", [0, 64])
def test_values_that_are_not_finite(turned):
    """NaN is kept, infinities are limited; neither counts for the scale.  Zeros get the least scale, the largest a limit."""
    x = torch.zeros(4, 1, 64, dtype=torch.bfloat16, device=DEV)
    x[0, 0, :4] = torch.tensor([float("nan"), float("inf"), float("-inf"), 100.0])
    x[2] = 3e38
    x[3, 0, 5] = float("inf")
    kc, vc = (torch.zeros(4, 1, 16, 64, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
    ks, vs = (torch.ones(4, 1, device=DEV) for _ in range(2))
    rot = S.rotary_create(64) if turned else None
    S.kv_append(x, x, dev([0, 0, 0, 0], torch.int32), dev([0, 16, 32, 48], torch.int64), kc, vc, rotary=rot, k_scale=ks, v_scale=vs)
    for c, s in ((kc, ks), (vc, vs)):
        assert s[:, 0].tolist() == [0.25, 2.0 ** -64, 2.0 ** 64, 2.0 ** -64]
        got = c[:, 0, 0].float()
        assert torch.isnan(got[0, 0]) and got[0, 3] == 384.0  # 400 is halfway between 384 (1.100 2^8, even) and 416 (1.101 2^8)
        assert (got[1] == 0).all() and (got[2].abs() == 448).all()
        if c is vc or not turned:
            assert got[0, 1] == 448 and got[0, 2] == -448 and got[3, 5] == 448


def test_a_cache_past_32_bits():
    """Offsets of more than 2^31 elements, with scales and without."""
    say("append far")
    blocks = 2 ** 31 // (2 * 16 * 64) + 8
    slots = dev([blocks * 16 - 2, blocks * 16 - 1, 0, (blocks - 3) * 16 + 5], torch.int64)
    k, v = torch.randn(2, 4, 2, 64, device=DEV).to(torch.bfloat16)
    pos = dev([3, 4, 0, 77], torch.int32)
    rot = S.rotary_create(64)
    small = dev([32 + 14, 32 + 15, 0, 16 + 5], torch.int64)
    for scaled in (False, True):
        t = torch.float8_e4m3fn if scaled else torch.bfloat16
        far, near = (torch.zeros(2, n, 2, 16, 64, dtype=t, device=DEV) for n in (blocks, 3))
        fs, ns = (torch.ones(2, n, 2, device=DEV) for n in (blocks, 3))
        more = lambda s: dict(k_scale=s[0], v_scale=s[1]) if scaled else {}  # noqa: E731
        S.kv_append(k, v, pos, slots, far[0], far[1], rotary=rot, **more(fs))
        S.kv_append(k, v, pos, small, near[0], near[1], rotary=rot, **more(ns))
        for i in range(2):
            assert torch.equal(far[i][[0, blocks - 3, blocks - 1]].view(torch.uint8), near[i].view(torch.uint8))
            assert torch.equal(fs[i][[0, blocks - 3, blocks - 1]], ns[i])
        del far


def test_append_agrees_with_rotate_and_write():
    """One call, or the three that it stands for: the same bits in a 16-bit cache."""
    rng = np.random.default_rng(9)
    qkv = dev(rng.standard_normal((90, 12, 128)), torch.bfloat16)
    pos, slots = dev(np.arange(90) + 7, torch.int32), dev(np.arange(90) + 39, torch.int64)
    rot = S.rotary_create(128, base=5e5)
    a, b = (torch.zeros(2, 9, 2, 16, 128, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    q = S.kv_append(qkv[:, 8:10], qkv[:, 10:], pos, slots, a[0], a[1], rotary=rot, q=qkv[:, :8])
    turned = S.rotate(qkv[:, :10], pos, rot)
    S.kv_write(turned[:, 8:], qkv[:, 10:], slots, b[0], b[1])
    assert torch.equal(q, turned[:, :8]) and torch.equal(a, b)


def test_a_tensor_of_one_element_is_a_number():
    """For the append and for the attention over what it stored."""
    rng = np.random.default_rng(10)
    x = dev(rng.standard_normal((20, 8, 64)), torch.bfloat16)
    pos, slots = dev(np.arange(20), torch.int32), dev(np.arange(20), torch.int64)
    table, start, length = dev([[0, 1]], torch.int32), dev([0, 20], torch.int32), dev([20], torch.int32)
    got = []
    for number in (0.25, np.float32(0.25), torch.tensor(0.25), torch.tensor([0.25])):
        c = torch.zeros(2, 2, 2, 16, 64, dtype=torch.float8_e4m3fn, device=DEV)
        q = S.kv_append(x[:, 4:6], x[:, 6:], pos, slots, c[0], c[1], rotary=S.rotary_create(64), k_scale=number, v_scale=number, q=x[:, :4])
        out = S.kv_attention(q, c[0], c[1], table, start, length, 20, 20, k_scale=number, v_scale=number)
        got.append((c.view(torch.uint8), out))
    for c, out in got[1:]:
        assert torch.equal(c, got[0][0]) and torch.equal(out, got[0][1])


def test_no_tokens():
    z = torch.empty(0, 2, 64, dtype=torch.bfloat16, device=DEV)
    c = torch.zeros(2, 3, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
    assert S.kv_append(z, z, dev([], torch.int32), dev([], torch.int64), c[0], c[1], rotary=S.rotary_create(64), q=z).shape == (0, 2, 64)
