"""Attention over a cache with scales of blocks and heads, against the float64 oracle on what the blocks stand for: in every
form of the kernel (tests/kv_cases.py), with windows, missing blocks, blocks that hold anything where nothing is seen, scales
far apart, and scores of any size."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv_cases  # noqa: E402
import paper_2408_04323_amd as S  # noqa: E402
from oracle import kv_cache as kv  # noqa: E402
from test_gpu_kv_cache import ATTEND, BITS, TYPES, _attend_inputs, _check, dev, f64  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
FORMS = {n: c for n, c in kv_cases.CASES.items() if c["cache"] == "f8"}
FORMS.update({n: c for n, c in ATTEND.items() if c["cache"] == "f8" or n in ("hints_small", "hints_large", "mixed_many", "decode_long", "block_edges",
                                                                            "decode_group_of_130", "window_one", "window_wide", "draft_tokens")})


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


def _inputs(c, seed, spread=3.0, two=False):
    """_attend_inputs in 8 bits with scales spread over 2^+-spread, and where no request's token lies codes and scales of
    anything: NaN, infinities, zeros, negative and huge numbers."""
    rng = np.random.default_rng(seed)
    s = _attend_inputs(dict(c, cache="f8"), seed)
    blocks, hkv = s["k"].shape[:2]
    e = rng.uniform(-spread, spread, (2, blocks, hkv))
    held = np.zeros(blocks, dtype=bool)
    for r, (a, n) in enumerate(c["lens"]):
        held[s["table"][r, :-(-(a + n) // c["bs"])]] = True
    junk = rng.choice([np.nan, np.inf, -np.inf, 0.0, -1.0, 1e38, 1e-45, 5.0], (2, blocks, hkv))
    scales = np.where(held[:, None], np.exp2(np.round(e) if two else e) * 0.02, junk)
    s["ks"], s["vs"] = (dev(x, torch.float32) for x in scales)
    return s


def _call(c, s, **more):
    hints = c["hints"] or (max(n for _, n in c["lens"]), max(a + n for a, n in c["lens"]))
    args = dict(max_new_len=hints[0], max_seq_len=hints[1], scale=c["scale"], window=c["window"], k_scale=s["ks"], v_scale=s["vs"])
    args.update(more)
    return S.kv_attention(s["q"], s["k"], s["v"], dev(s["table"], torch.int32), dev(s["start"], torch.int32), dev(s["seq"], torch.int32), **args)


def _reference(c, s):
    with np.errstate(invalid="ignore"):
        k, v = (f64(s[n]) * f64(s[n + "s"])[:, :, None, None] for n in ("k", "v"))
    return kv.attention(f64(s["q"]), k, v, s["table"], s["start"], s["seq"], c["d"] ** -0.5 if c["scale"] is None else c["scale"], c["window"])


def _bound(c, s, ref):
    """The oracle's bound with what scales add.  A score's scale is a product of two floats (2^-24 of the score, twice).  A
    value's scale is 2^e f; log2 f goes into the weight's exponent beside m, which is log2(e) times the largest score, less 6:
    rounded to 2^-24 of that, (1.45 reach + 8) 2^-24, times ln 2 of the weight; the logarithm itself and the reciprocal of f are
    off by 2^-22: (3 * 2^-24 reach + 2^-21) in all.  Values at less than 2^-15 of the largest scale are off by at most
    2^-25 * 2^6 * 2^e for the largest scale's exponent e (it may be up to 2^6 above the reference), less than 2^-25 of 448 times
    the largest scale, and so are weights below the normal range."""
    out, spread, reach = ref
    vs = f64(s["vs"])
    top = 448.0 * max(float(vs[np.isfinite(vs) & (vs > 0) & (vs < 1e30)].max()), 1e-30)
    keys = max(a + n for a, n in c["lens"])
    more = (3 * 2.0 ** -24 * reach[..., None] + 2.0 ** -21) * (spread + np.abs(out)) + 2.0 ** -25 * top
    return kv.attention_bound(out, spread, reach, keys, c["d"], BITS[c["kind"]], 11, top) + more


@pytest.mark.parametrize("name", list(FORMS))
def test_every_form_matches_the_oracle(name):
    say("scaled", name)
    c = FORMS[name]
    s = _inputs(c, len(name), two=len(name) % 2 == 0)
    got, ref = f64(_call(c, s)), _reference(c, s)
    assert np.isfinite(ref[0]).all()
    _check(got, ref[0], _bound(c, s, ref))


@pytest.mark.parametrize("name", [n for n, c in kv_cases.CASES.items() if c["cache"] == "f8" and c["kind"] == "bf16"])
def test_every_form_with_a_window_and_missing_blocks(name):
    say("scaled, window", name)
    c = dict(FORMS[name], window=45)
    s = _inputs(c, len(name))
    rng = np.random.default_rng(1)
    # Blocks before the window have gone to others, or nowhere; some inside it are missing, too.
    for r, (a, n) in enumerate(c["lens"]):
        gone = max(0, a + 1 - 45) // c["bs"]
        s["table"][r, :gone] = rng.choice([-1, s["k"].shape[0], 2 ** 31 - 1, int(s["table"].max())], gone)
        if a > 200:
            s["table"][r, a // c["bs"]] = -1
    got, ref = f64(_call(c, s)), _reference(c, s)
    _check(got, ref[0], _bound(c, s, ref))


@pytest.mark.parametrize("name", [n for n, c in kv_cases.CASES.items() if c["cache"] == "f8" and c["kind"] == "f16"])
def test_one_scale_for_all_is_the_call_with_one_scale(name):
    """Powers of two for every block: weights and sums are those of one scale, and so are the bits."""
    say("scaled, one", name)
    c = FORMS[name]
    s = _attend_inputs(c, 3)
    shape = s["k"].shape[:2]
    one = dict(s, ks=0.03125, vs=0.0625)
    many = dict(s, ks=torch.full(shape, 0.03125, device=DEV), vs=torch.full(shape, 0.0625, device=DEV))
    a, b = _call(c, one), _call(c, many)
    assert torch.equal(a.view(torch.int16), b.view(torch.int16))
    assert torch.equal(b.view(torch.int16), _call(c, many).view(torch.int16))


@pytest.mark.parametrize("far", [(-64, 64), (-20, 20), (-40, 0), (0, 40)])
@pytest.mark.parametrize("lens,d", [([(600, 1)], 64), ([(6000, 1)], 128), ([(600, 40)], 64), ([(3000, 40)], 128), ([(300, 90)], 256), ([(2000, 2)], 192)])
def test_scales_far_apart(lens, d, far):
    """Blocks of tiny values that take most of the weight, beside blocks of huge ones that take little: the tiny ones count in
    the softmax's sum, whatever their values' scale is."""
    say("scaled, far", lens, d, far)
    c = dict(lens=lens, kind="bf16", hq=4, hkv=2, d=d, bs=16, window=0, scale=None, hints=None, stale=0.0)
    s = _attend_inputs(dict(c, cache="f8"), 7)
    rng = np.random.default_rng(d)
    blocks = s["k"].shape[0]
    e = rng.choice(far, (blocks, 2))
    s["vs"] = dev(np.exp2(e), torch.float32)
    # The first element of every key says how heavy its block is: 2^10 for those of small scales.
    k = s["k"].float() * 0.25
    k[..., 0] = 0.0
    small = torch.as_tensor(e == far[0], device=DEV)
    k[small, :, 0] = 64.0
    q = s["q"].float()
    q[..., 0] = 10 * np.log(2.0) * d ** 0.5 / (64 * 0.02)
    s.update(k=k.to(s["k"].dtype), q=q.to(torch.bfloat16), ks=torch.full((blocks, 2), 0.02, device=DEV))
    got, ref = f64(_call(c, s)), _reference(c, s)
    _check(got, ref[0], _bound(c, s, ref))


def test_blocks_of_zeros_count():
    """A block of zeros with the least scale, as an append leaves it, takes its share of the softmax."""
    for tokens in (1, 40):
        c = dict(lens=[(100, tokens)], kind="f16", hq=4, hkv=2, d=128, bs=16, window=0, scale=0.0, hints=None, stale=0.0)
        s = _inputs(c, 1)
        zero = s["table"][0, 1]
        v = s["v"].float()
        v[zero] = 0.0
        s["v"] = v.to(s["v"].dtype)
        s["vs"][zero] = 2.0 ** -64
        got, ref = f64(_call(c, s)), _reference(c, s)
        _check(got, ref[0], _bound(c, s, ref))


@pytest.mark.parametrize("tokens,d,length", [(1, 64, 700), (4, 128, 5000), (40, 64, 300), (40, 256, 300), (40, 128, 4000)])
def test_large_scores_have_a_softmax(tokens, d, length):
    """Scores up to the largest float over blocks of unlike scales, powers of two: every third key has the score x, the others
    1.5 x (x negative) or 0.5 x, so the result is the mean of every third value, up to the rounding of the weights (2^-11), of
    the result (2^-8) and of sums in float.  (Other scales' fractions are lost beside such scores, as the interface says.)"""
    say("scaled, large scores", tokens, d, length)
    blocks, kind = -(-length // 16), torch.bfloat16
    g = torch.Generator(device=DEV).manual_seed(1)
    codes = torch.randn(blocks, 1, 16, d, generator=g, device=DEV).mul_(50).clamp_(-448, 448).to(torch.float8_e4m3fn)
    vs = torch.randint(-5, 6, (blocks, 1), generator=g, device=DEV).float().exp2_()
    ks = torch.randint(-3, 4, (blocks, 1), generator=g, device=DEV).float().exp2_()
    third = torch.arange(blocks * 16, device=DEV) % 3 == 0
    v = (codes.double() * vs[:, :, None, None].double()).view(-1, d)
    mean = ((v * third[:, None]).cumsum(0) / third.cumsum(0)[:, None])[:length]
    size_of = ((v.abs() * third[:, None]).cumsum(0) / third.cumsum(0)[:, None])[:length]
    table = torch.arange(blocks, dtype=torch.int32, device=DEV)[None]
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    for size in (1e5, 3e7, 1.1e8, 7e8, 3e9, 1e15, 1e30, 1e37):
        for sign in (-1.0, 1.0):
            k = torch.zeros(blocks * 16, d, device=DEV)
            k[:, 1] = 16.0 * torch.where(third, 1.0, 1.5 if sign < 0 else 0.5)
            k = (k.view(blocks, 1, 16, d) / ks[:, :, None, None]).to(torch.float8_e4m3fn)
            q = torch.zeros(tokens, 2, d, dtype=kind, device=DEV)
            q[..., 1] = sign * min(size / 16, 3e36)
            n = min(tokens, length)
            scale = size / (float(q[0, 0, 1].abs()) * 16.0)
            got = S.kv_attention(q, k, codes.view_as(codes), table, i32(0, tokens), i32(length), tokens, length, scale=scale, k_scale=ks, v_scale=vs)
            off = (got[tokens - n:].double() - mean[length - n:, None]).abs()
            bound = 2.0 ** -8 * mean[length - n:, None].abs() + (2 * 2.0 ** -11 + length * 2.0 ** -23) * size_of[length - n:, None] * 1.01
            assert (off <= bound).all(), (size, sign, float((off / bound).max()))


@pytest.mark.parametrize("name", ["few-128-bf16-f8-one each", "tiles-64-bf16-f8-many", "tiles_parts-256-bf16-f8-one each", "few_parts-192-bf16-f8-many"])
def test_values_that_are_not_finite_stay_with_their_rows(name):
    say("scaled, not finite", name)
    c = dict(FORMS[name], stale=0.0)
    s = _inputs(c, 2)
    clean = _call(c, s)
    r = len(c["lens"]) - 2
    a, n = c["lens"][r]
    j = n // 2
    at, head, dim = a + j, c["hkv"] - 1, c["d"] - 3
    x = s["v"].float()
    x[int(s["table"][r, at // c["bs"]]), head, at % c["bs"], dim] = float("nan")
    got = _call(c, dict(s, v=x.to(s["v"].dtype)))
    nan, first, g = torch.zeros_like(got, dtype=torch.bool), int(s["start"][r]), c["hq"] // c["hkv"]
    nan[first + j:first + n, head * g:(head + 1) * g, dim] = True
    assert torch.equal(torch.isnan(got), nan)
    others = ~nan
    others[first:first + n] = False
    assert torch.equal(got[others], clean[others])
    ref = _reference(c, s)
    _check(np.where(nan.cpu().numpy(), ref[0], f64(got)), ref[0], _bound(c, s, ref))


@pytest.mark.parametrize("lens,d", [([(20, 3), (0, 2), (0, 4), (700, 1), (9, 0)], 64), ([(0, 150), (70, 33), (5, 1)], 128), ([(4500, 40), (0, 3)], 128),
                                    ([(6000, 1), (3, 1)], 192)])
def test_infinite_scores_and_rows_that_see_nothing(lens, d):
    """A row whose scores are all -inf is no number; one that sees nothing is zero."""
    c = dict(lens=lens, kind="bf16", hq=4, hkv=2, d=d, bs=16, window=0, scale=None, hints=None, stale=0.0)
    s = _inputs(c, 8)
    k = s["k"].float()
    k[..., 0] = -k[..., 0].abs() - 1.0
    s["k"] = k.to(s["k"].dtype)
    s["seq"][1] = max(0, lens[1][1] - 1)  # its first token stands before the cache's start
    bad = torch.zeros(s["q"].shape[:2], dtype=torch.bool, device=DEV)
    bad[::3, 1] = True
    s["q"][..., 0] = torch.where(bad, torch.full_like(s["q"][..., 0], float("inf")), s["q"][..., 0])
    got = _call(c, s)
    none = torch.zeros_like(bad)
    none[int(s["start"][1])] = bool(s["seq"][1] < lens[1][1])
    lost = bad & ~none
    nan = torch.isnan(got)
    assert torch.equal(nan.all(-1), lost) and torch.equal(nan.any(-1), lost)
    assert (got[none] == 0).all()


def test_a_cache_past_32_bits():
    """The last block of a cache of more than 2^32 bytes; scales by block and head."""
    say("scaled, far block")
    blocks = 2 ** 32 // (2 * 16 * 64) + 8
    kc = torch.zeros(blocks, 2, 16, 64, dtype=torch.float8_e4m3fn, device=DEV)
    vc = torch.zeros_like(kc)
    ks, vs = (torch.full((blocks, 2), float("nan"), device=DEV) for _ in range(2))
    g = torch.Generator(device=DEV).manual_seed(4)
    for x in (kc, vc):
        x[blocks - 1] = torch.randn(2, 16, 64, generator=g, device=DEV).mul_(60).to(x.dtype)
    ks[blocks - 1], vs[blocks - 1] = torch.tensor([0.02, 0.01], device=DEV), torch.tensor([0.3, 0.07], device=DEV)
    q = torch.randn(20, 4, 64, generator=g, device=DEV).to(torch.bfloat16)
    for tokens in (1, 16):
        n = min(tokens, 16)
        out = S.kv_attention(q[:n], kc, vc, dev([[blocks - 1]], torch.int32), dev([0, n], torch.int32), dev([16], torch.int32), n, 16, k_scale=ks, v_scale=vs)
        k, v = (f64(x[-1:]) * f64(y[-1:])[:, :, None, None] for x, y in ((kc, ks), (vc, vs)))
        ref = kv.attention(f64(q[:n]), k, v, np.array([[0]]), [0, n], [16], 64 ** -0.5)
        bound = kv.attention_bound(*ref, 16, 64, 8, 11, 448 * 0.3) + 1e-5 * np.abs(ref[0])
        _check(f64(out), ref[0], bound)


# Sizes as in perf/more_operators.py: (requests, new, context, hq, hkv, d, block, type)
LARGE = {"decode": (48, 1, 32767, 64, 8, 128, 32, "bf16"), "mixed": (40, 60, 3395, 28, 4, 128, 8, "f16"), "long": (1, 1024, 31744, 32, 8, 128, 16, "bf16")}


@pytest.mark.parametrize("name", list(LARGE))
def test_values_without_a_mean_at_full_size(name):
    """48 rows of a full-sized call."""
    say("scaled, large", name)
    requests, new, ctx, hq, hkv, d, bs, kind = LARGE[name]
    rng = np.random.default_rng(len(name))
    lens = [(int(rng.integers(ctx // 4, ctx + 1)), int(rng.integers(max(1, new // 2), new + 1))) for _ in range(requests)]
    lens[0] = (ctx, new)
    need = [-(-(a + n) // bs) for a, n in lens]
    order = rng.permutation(sum(need))
    table = np.full((requests, max(need)), -1)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    g = torch.Generator(device=DEV).manual_seed(len(name))
    k, v = (torch.randn(len(order), hkv, bs, d, generator=g, device=DEV).mul_(90).clamp_(-448, 448).to(torch.float8_e4m3fn) for _ in range(2))
    ks, vs = (torch.randn(len(order), hkv, generator=g, device=DEV).exp_().mul_(0.011) for _ in range(2))
    start = np.concatenate([[0], np.cumsum([n for _, n in lens])])
    q = torch.randn(int(start[-1]), hq, d, generator=g, device=DEV).to(TYPES[kind])
    out = S.kv_attention(q, k, v, dev(table, torch.int32), dev(start, torch.int32), dev([a + n for a, n in lens], torch.int32),
                         max(n for _, n in lens), max(a + n for a, n in lens), k_scale=ks, v_scale=vs)
    rows = rng.integers(0, start[-1], 48)
    rows[:2] = [0, start[-1] - 1]
    for t in rows.tolist():
        r = int(np.searchsorted(start, t, side="right")) - 1
        h = int(rng.integers(0, hq))
        kh, length = h // (hq // hkv), lens[r][0] + (t - int(start[r])) + 1
        blocks = dev(table[r, :-(-length // bs)], torch.int64)
        one = lambda x, y: (f64(x.view(torch.uint8)[blocks, kh].view(x.dtype)) * f64(y[blocks, kh])[:, None, None]).reshape(1, 1, -1, d)[:, :, :length]  # noqa: E731
        kx, vx = one(k, ks), one(v, vs)
        ref = kv.attention(f64(q[t:t + 1, h:h + 1]), kx, vx, np.array([[0]]), [0, 1], [length], d ** -0.5)
        c = dict(lens=[(length - 1, 1)], d=d, kind=kind)
        _check(f64(out[t:t + 1, h:h + 1]), ref[0], _bound(c, dict(vs=vs[blocks, kh]), ref))
