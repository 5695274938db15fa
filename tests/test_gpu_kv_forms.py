"""Every form of the attention kernel against the float64 oracle (tests/kv_cases.py; that each case takes the form that it is
there for is checked on the host), with windows and with values that are not finite; and rows of calls of the size of a
loaded engine's, with values of no mean, where rounded weights do not average out."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import kv_cases  # noqa: E402
import paper_2408_04323_amd as S  # noqa: E402
from oracle import kv_cache as kv  # noqa: E402
from test_gpu_kv_cache import BITS, TYPES, _attend_inputs, _bound, _call, _check, _reference, dev, f64  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def say(*a):
    print("[case]", *a, flush=True)
    sys.stdout.flush()


@pytest.mark.parametrize("name", list(kv_cases.CASES))
def test_every_form_matches_the_oracle(name):
    say("form", name)
    c = kv_cases.CASES[name]
    s = _attend_inputs(c, seed=len(name))
    got, ref = f64(_call(c, s)), _reference(c, s)
    assert np.isfinite(ref[0]).all()
    _check(got, ref[0], _bound(c, s, ref))


@pytest.mark.parametrize("name", [n for n, c in kv_cases.CASES.items() if not c["form"][3] and c["kind"] == "bf16"])
def test_every_form_with_a_window(name):
    say("form, window", name)
    c = dict(kv_cases.CASES[name], window=45)
    s = _attend_inputs(c, seed=len(name))
    got, ref = f64(_call(c, s)), _reference(c, s)
    _check(got, ref[0], _bound(c, s, ref))


@pytest.mark.parametrize("name", [n for n, c in kv_cases.CASES.items() if c["kind"] == "bf16"])
def test_every_form_keeps_values_that_are_not_finite_apart(name):
    """A NaN in the value of a new token reaches the rows from that token on, in its key head and dimension, and no other."""
    say("form, not finite", name)
    c = dict(kv_cases.CASES[name], stale=0.0)
    s = _attend_inputs(c)
    clean = _call(c, s)
    r = len(c["lens"]) - 2
    a, n = c["lens"][r]
    j = n // 2  # the query that stands at the bad token
    at, head, dim = a + j, c["hkv"] - 1, c["d"] - 3
    x = s["v"].float()
    x[int(s["table"][r, at // c["bs"]]), head, at % c["bs"], dim] = float("nan")
    got = _call(c, dict(s, v=x.to(s["v"].dtype)))
    nan, first = torch.zeros_like(got, dtype=torch.bool), int(s["start"][r])
    g = c["hq"] // c["hkv"]
    nan[first + j:first + n, head * g:(head + 1) * g, dim] = True
    assert torch.equal(torch.isnan(got), nan)
    others = ~nan
    others[first:first + n] = False  # the same request's rows may be summed in another order
    assert torch.equal(got[others], clean[others])
    off = (got.float() - clean.float()).abs()[~nan].max()
    assert off <= 8 * 2.0 ** -BITS["bf16"], off  # values of at most about 4, rounded once more or less


# Sizes as in perf/operators.py, and its other shapes: (requests, new, context, hq, hkv, d, block, type, cache)
LARGE = {
    "decode": (256, 1, 4095, 32, 8, 128, 16, "bf16", "bf16"),
    "decode_f8": (48, 1, 32767, 64, 8, 128, 32, "bf16", "f8"),
    "mixed": (40, 60, 3395, 28, 4, 128, 8, "f16", "f16"),
    "prefill": (4, 4096, 0, 32, 8, 128, 16, "bf16", "bf16"),
    "long": (1, 1024, 64512, 32, 8, 64, 16, "bf16", "bf16"),
    "long_192": (2, 500, 9000, 12, 4, 192, 16, "f16", "f16"),
    "long_256": (2, 500, 9000, 8, 1, 256, 32, "bf16", "bf16"),
}


@pytest.mark.parametrize("name", list(LARGE))
def test_values_without_a_mean_at_full_size(name):
    """48 rows of a full-sized call.  The bound is the oracle's: with bfloat16 weights each is off by up to 2^-9 of itself,
    independently, and the values do not cancel that."""
    say("large", name)
    requests, new, ctx, hq, hkv, d, bs, kind, cache = LARGE[name]
    rng = np.random.default_rng(len(name))
    lens = [(int(rng.integers(ctx // 4, ctx + 1)) if ctx else 0, int(rng.integers(max(1, new // 2), new + 1))) for _ in range(requests)]
    lens[0] = (ctx, new)
    need = [-(-(a + n) // bs) for a, n in lens]
    order = rng.permutation(sum(need))
    table = np.full((requests, max(need)), -1)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    g = torch.Generator(device=DEV).manual_seed(len(name))
    k, v = (torch.randn(len(order), hkv, bs, d, generator=g, device=DEV) for _ in range(2))
    ks, vs = (0.03, 0.05) if cache == "f8" else (1.0, 1.0)
    k, v = (x.div_(y).clamp_(-448, 448).to(TYPES[cache]) if cache == "f8" else x.to(TYPES[cache]) for x, y in ((k, ks), (v, vs)))
    start = np.concatenate([[0], np.cumsum([n for _, n in lens])])
    q = torch.randn(int(start[-1]), hq, d, generator=g, device=DEV).to(TYPES[kind])
    out = S.kv_attention(q, k, v, dev(table, torch.int32), dev(start, torch.int32), dev([a + n for a, n in lens], torch.int32),
                         max(n for _, n in lens), max(a + n for a, n in lens), k_scale=ks, v_scale=vs)
    rows = rng.integers(0, start[-1], 48)
    rows[:2] = [0, start[-1] - 1]
    for t in rows.tolist():
        r = int(np.searchsorted(start, t, side="right")) - 1
        a, n = lens[r]
        h = int(rng.integers(0, hq))
        kh, length = h // (hq // hkv), a + (t - int(start[r])) + 1
        blocks = dev(table[r, :-(-length // bs)], torch.int64)
        one = lambda x, scale: f64(x.view(torch.uint8)[blocks, kh].view(x.dtype).reshape(1, -1, d)[:, :length])[:, None] * scale  # noqa: E731
        kx, vx = one(k, ks), one(v, vs)
        ref = kv.attention(f64(q[t:t + 1, h:h + 1]), kx, vx, np.array([[0]]), [0, 1], [length], d ** -0.5)
        bound = kv.attention_bound(*ref, length, d, BITS[kind], 11 if cache == "f8" else BITS[kind], np.abs(vx).max())
        _check(f64(out[t:t + 1, h:h + 1]), ref[0], bound)


@pytest.mark.parametrize("d,cache", [(64, "bf16"), (128, "f8"), (256, "bf16")])
@pytest.mark.parametrize("hints", [(5000, 100000), (20, 100000), (5000, 1), (1, 100000), (17, 1)])
def test_hints_far_from_the_lengths(hints, d, cache):
    """More than 16 rows of a request, announced as more and as fewer tokens than there are: parts that stay empty, tiles
    with all keys in one part, tiles taken sixteen rows at a time."""
    say("hints", hints, d, cache)
    c = dict(lens=[(40, 20), (20, 1), (700, 30), (0, 0), (3, 2)], kind="bf16", cache=cache, hq=8, hkv=2, d=d, bs=16, window=0, scale=None,
             hints=hints, stale=float("nan"))
    s = _attend_inputs(c, seed=d)
    got, ref = f64(_call(c, s)), _reference(c, s)
    _check(got, ref[0], _bound(c, s, ref))
