"""The bounds of a step's attention tell mistakes: results of zero, of queries that were not turned, and plain means fail them."""
import numpy as np
import pytest

import step_bounds
from oracle import kv_cache as kv
from oracle import rotary as R

HQ, HKV, D, BS = 8, 2, 128, 16


def _to_bf16(x):
    e = np.exp2(np.floor(np.log2(np.abs(np.where(x == 0, 1, x)))) - 7)
    return np.round(x / e) * e


@pytest.mark.parametrize("context,new", [(0, 40), (43, 1), (90, 5), (17, 130)])
def test_wrong_results_fail(context, new):
    rng = np.random.default_rng(context)
    freqs, _ = R.frequencies(D, scaling="bands", factor=4.0, length=64, low=1.0, high=4.0)
    n = context + new
    x = _to_bf16(rng.standard_normal((n, HQ + 2 * HKV, D)) * np.exp(rng.uniform(-1, 1)))
    pos = np.arange(n)
    turned = _to_bf16(R.rotate(x[:, :HQ], pos, freqs))[context:]
    blocks = -(-n // BS)
    held = np.zeros((2, blocks, HKV, BS, D))
    for i, y in enumerate((R.rotate(x[:, HQ:HQ + HKV], pos, freqs), x[:, HQ + HKV:])):
        codes, scales, _ = R.append_scaled(y, pos, held[i], np.ones((blocks, HKV)))
        held[i] = kv.round_e4m3(codes) * scales[:, :, None, None]
    table, start, seq = np.arange(blocks)[None], [0, new], [n]
    attend = lambda q, scale: kv.attention(q, held[0], held[1], table, start, seq, scale)  # noqa: E731
    ref = attend(turned, D ** -0.5)
    v = np.abs(held[1]).transpose(0, 2, 1, 3).reshape(-1, HKV, D).max(-1)
    top = np.repeat(np.maximum.accumulate(v)[context:n], HQ // HKV, 1)[..., None]
    bound = step_bounds.attention_bound(ref, n, D, top)

    def fails(got):
        return (np.abs(got - ref[0]) > bound).any(-1)
    assert not fails(_to_bf16(ref[0])).any()
    assert fails(np.zeros_like(ref[0])).all()
    later = pos[context:] > 0  # the first token sees one key, whose weight is 1
    assert fails(attend(_to_bf16(x[context:, :HQ]), D ** -0.5)[0])[later].mean() > 0.95
    assert fails(attend(turned, 0.0)[0])[later].mean() > 0.95
