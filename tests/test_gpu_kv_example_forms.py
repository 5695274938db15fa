"""The example's step with rotations and with a cache of 8 bits: its results against the oracle on what the cache holds,
over steps of growing, ending and new requests, and a short tuning run."""
import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402
from oracle import kv_cache as kv  # noqa: E402
from oracle import rotary as R  # noqa: E402
from test_gpu_kv_cache import _check, f64  # noqa: E402

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("tune_cache_step", os.path.join(ROOT, "examples", "tune_cache_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("turns,scaled", [(True, False), (False, True), (True, True)])
def test_steps_of_a_changing_batch(ex, turns, scaled):
    rotary = S.rotary_create(ex.DIM, base=5e5) if turns else None
    step = ex.CacheStep(16, 2048, rotary=rotary, scaled=scaled)
    gen = torch.Generator(device="cuda").manual_seed(6)
    plan = [([40, 17], []), ([1, 30], []), ([1, 1, 100], [1]), ([1, 1], []), ([0, 1, 5], [0]), ([1, 1, 64, 9], [])]
    for new, done in plan:
        step.add(len(new) - len(step.context))
        pos = np.concatenate([np.arange(c, c + n) for c, n in zip(step.context, new)])
        qkv = torch.randn(sum(new), ex.HEADS + 2 * ex.KV_HEADS, ex.DIM, generator=gen, device="cuda").to(torch.bfloat16)
        q = qkv[:, :ex.HEADS]
        out = step.run(new, qkv)
        if turns:
            q = S.rotate(q, torch.tensor(pos, dtype=torch.int32, device="cuda"), rotary)
        k, v = f64(step.k_cache), f64(step.v_cache)
        if scaled:
            k, v = (x * f64(s)[:, :, None, None] for x, s in ((k, step.k_scale), (v, step.v_scale)))
        start = np.concatenate([[0], np.cumsum(new)])
        table = step.table.cpu().numpy()
        ref = kv.attention(f64(q), k, v, table, start, step.context, ex.DIM ** -0.5)
        _check(f64(out), ref[0], kv.attention_bound(*ref, max(step.context), ex.DIM, 8, 11 if scaled else 8, np.abs(v).max()))
        # The last token's keys of every request, within the cache's rounding.
        for i, n in enumerate(new):
            if n:
                at = step.context[i] - 1
                x = f64(qkv[start[i + 1] - 1:start[i + 1], ex.HEADS:ex.HEADS + ex.KV_HEADS])
                want = R.rotate(x, [at], f64(rotary.freqs))[0] if turns else x[0]
                block = table[i, at // 16]
                step_of = 2.0 ** -10 * (f64(step.k_scale)[block][:, None] if scaled else 0)  # half the smallest step
                assert (np.abs(k[block, :, at % 16] - want) <= (2.0 ** -4 if scaled else 2.0 ** -7) * np.abs(want) + step_of + 2.0 ** -20).all()
        if done:
            step.remove(done)


def test_a_short_tuning_run(ex):
    X, Y, valid, best = ex.tune(2, 2, n_requests=8, pool=4096, rotary=S.rotary_create(ex.DIM), scaled=True)
    assert best >= 0 and valid[best] and Y[best, 0] < 0 < Y[best, 1]
