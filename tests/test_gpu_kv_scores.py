"""Scores that are not finite or very large.  A row that sees keys, all of them with scores of -inf, has no softmax, and a row
that sees nothing is zero.  The two differ in nothing but what they see, so both stand side by side here, in every way that
the keys are gone through: few rows and tiles, in one part and in several, with windows and with blocks that are missing."""
import sys

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f8": torch.float8_e4m3fn}

CASES = {  # (cached, new) of every request; more
    "few": ([(20, 3), (0, 2), (0, 4), (700, 1), (9, 0)], {}),
    "few_short": ([(0, 1), (3, 1), (40, 2)], dict(d=128, kind="f16")),
    "few_of_many": ([(13 * i % 70, 1 + i % 3) for i in range(40)], dict(hkv=8, hq=8)),
    "few_parts": ([(9000, 2), (40, 1)], dict(d=256, hkv=1, hq=4)),
    "few_parts_of_many": ([(3000, 1)] * 20 + [(7, 2)] * 20, dict(hkv=8, hq=16)),
    "few_f8": ([(100, 2), (3, 1)], dict(cache="f8", d=128)),
    "few_f8_parts": ([(6000, 1), (3, 1)], dict(cache="f8", hq=8, hkv=1, d=192)),
    "few_window": ([(500, 2), (9, 1)], dict(window=40)),
    "tiles": ([(0, 150), (70, 33), (5, 1)], dict(d=128, kind="f16")),
    "tiles_of_many": ([(i % 60, 1 + 30 * (i % 3 == 0)) for i in range(40)], dict(hkv=8, hq=8)),
    "tiles_parts": ([(4500, 40), (0, 3)], dict(d=128, hkv=1)),
    "tiles_wide": ([(30, 70)], dict(d=256)),
    "tiles_192": ([(30, 70), (1400, 40)], dict(d=192, hq=6)),
    "tiles_f8": ([(100, 60)], dict(cache="f8")),
    "tiles_window": ([(300, 90), (0, 40)], dict(window=37)),
}


def _inputs(lens, kind="bf16", cache=None, hq=4, hkv=2, d=64, bs=16, window=0, seed=0):
    """All first elements of the keys are negative, so an infinite one of a query gives -inf with every key."""
    rng = np.random.default_rng(seed)
    cache = cache or kind
    need = [-(-(a + n) // bs) for a, n in lens]
    order = rng.permutation(sum(need) + 2)
    table = np.full((len(lens), max(need) + 1), -1)
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = order[at:at + n]
        at += n
    kc, vc = rng.standard_normal((2, len(order), hkv, bs, d))
    kc[..., 0] = -1.0 - np.abs(kc[..., 0])
    tokens = sum(n for _, n in lens)
    q = rng.standard_normal((tokens, hq, d))
    bad = rng.random((tokens, hq)) < 0.4
    if bad.shape[0] > 2:
        bad[:, 0], bad[1] = True, True  # a head of all tokens, all heads of a token
    q[..., 0] = np.where(bad, 0.5, q[..., 0])
    put = lambda x, t: torch.as_tensor(x, dtype=torch.float32).to(TYPES[t]).to(DEV)  # noqa: E731
    return dict(q=put(q, kind), k=put(kc, cache), v=put(vc, cache), table=table, bad=bad, window=window, lens=lens, bs=bs,
                start=np.concatenate([[0], np.cumsum([n for _, n in lens])]), seq=np.array([a + n for a, n in lens]))


def _call(s, q):
    i32 = lambda x: torch.as_tensor(np.asarray(x)).to(torch.int32).to(DEV)  # noqa: E731
    return S.kv_attention(q, s["k"], s["v"], i32(s["table"]), i32(s["start"]), i32(s["seq"]), max(n for _, n in s["lens"]),
                          max(a + n for a, n in s["lens"]), window=s["window"])


def _sees(s):
    """Tokens that see a key, from the definition."""
    got = []
    blocks = s["k"].shape[0]
    for r, (_, n) in enumerate(s["lens"]):
        for j in range(n):
            p = int(s["seq"][r]) - n + j
            keys = range(max(0, p - s["window"] + 1) if s["window"] else 0, p + 1)
            got.append(any(0 <= s["table"][r, b] < blocks for b in {k // s["bs"] for k in keys}))
    return np.array(got)


def _check(s):
    sees = _sees(s)
    clean = _call(s, s["q"])
    q = s["q"].clone()
    bad = torch.as_tensor(s["bad"], device=DEV)
    q[..., 0] = torch.where(bad, torch.full_like(q[..., 0], INF), q[..., 0])
    got = _call(s, q)
    lost = bad & torch.as_tensor(sees, device=DEV)[:, None]
    nan = torch.isnan(got)
    assert torch.equal(nan.all(-1), lost) and torch.equal(nan.any(-1), lost)
    assert torch.equal(got[~lost], clean[~lost])
    assert (got[torch.as_tensor(~sees, device=DEV)] == 0).all()
    return sees


@pytest.mark.parametrize("name", list(CASES))
def test_rows_of_infinite_scores_are_no_numbers(name):
    print("[case] scores", name, flush=True)
    sys.stdout.flush()
    lens, more = CASES[name]
    assert _check(_inputs(lens, seed=len(name), **more)).all()


@pytest.mark.parametrize("name", list(CASES))
def test_rows_that_see_nothing_beside_them(name):
    """Requests with fewer tokens than they ask for, and blocks that are missing: all of some request's, some of the others'."""
    print("[case] scores, missing", name, flush=True)
    lens, more = CASES[name]
    s = _inputs(lens, seed=len(name), **more)
    rng = np.random.default_rng(1)
    s["table"][rng.random(s["table"].shape) < 0.5] = -1
    s["table"][0] = [-1, s["k"].shape[0], 2 ** 31 - 1, -7][:s["table"].shape[1]] + [-1] * max(0, s["table"].shape[1] - 4)
    if len(lens) > 1:
        s["seq"][1] = max(0, lens[1][1] - 1)  # its first token stands before the cache's start
    sees = _check(s)
    assert not sees.all()


@pytest.mark.parametrize("d,length", [(64, 16), (64, 700), (128, 5000), (256, 300)])
@pytest.mark.parametrize("tokens", [1, 4, 40])
@pytest.mark.parametrize("kind", ["bf16", "f16"])
def test_large_scores_have_a_softmax(kind, tokens, d, length):
    """Scores up to the largest float, where a float's steps are far larger than what a softmax tells apart.  Every third key
    has the score x, the others 1.5 x (x negative) or 0.5 x (positive), 70,000 and more apart: the result is the mean of the
    every-third values that a row sees, up to the rounding of these values' mean (|v| < 5) and of a sum in float."""
    print("[case] large scores", kind, tokens, d, length, flush=True)
    t, blocks = TYPES[kind], -(-length // 16)
    g = torch.Generator(device=DEV).manual_seed(1)
    v = torch.randn(blocks, 1, 16, d, generator=g, device=DEV).clamp_(-5, 5).to(t)
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    third = torch.arange(blocks * 16, device=DEV) % 3 == 0
    flat = v.view(-1, d).double() * third[:, None]
    mean = (flat.cumsum(0) / third.cumsum(0)[:, None])[:length]
    table = torch.arange(blocks, dtype=torch.int32, device=DEV)[None]
    bits = 9 if kind == "bf16" else 12
    for size, at in ((1e5, 1.0), (3e7, 1.0), (1.1e8, 1.0), (1.9e8, 1.0), (7e8, 3e4), (3e9, 3e4), (1e15, 3e4), (1e30, 1e10), (1e37, 1e10), (2.2e38, 1e10)):
        if kind == "f16" and size > 1e9:
            continue
        for sign in (-1.0, 1.0):
            k = torch.zeros(blocks * 16, d, device=DEV)
            k[:, 1] = at * torch.where(third, 1.0, 1.5 if sign < 0 else 0.5)
            q = torch.zeros(tokens, 2, d, dtype=t, device=DEV)
            q[..., 1] = sign * min(size / at, 6e4 if kind == "f16" else 3e38)
            kc = k.to(t).view(blocks, 1, 16, d)
            n = min(tokens, length)
            scale = size / (float(q[0, 0, 1].abs()) * float(kc[0, 0, 0, 1]))
            got = S.kv_attention(q, kc, v, table, i32(0, tokens), i32(length), tokens, length, scale=scale)
            off = (got[tokens - n:].double() - mean[length - n:, None]).abs().max()
            assert off <= 5 * (2.0 ** -bits + length * 2.0 ** -23), (size, sign, float(off))
