"""The example that evaluates configurations on the cache operators: a step's result against the oracle after several
steps of growing, ending and new requests, and a short tuning run."""
import importlib.util
import os

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from oracle import kv_cache as kv  # noqa: E402

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ex():
    spec = importlib.util.spec_from_file_location("tune_cache_step", os.path.join(ROOT, "examples", "tune_cache_step.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


def test_steps_of_a_changing_batch(ex):
    """Every request's last step sees exactly the keys and values that its own steps wrote, whatever blocks they got."""
    step = ex.CacheStep(16, 2048)
    gen = torch.Generator(device="cuda").manual_seed(5)
    heads = ex.HEADS + 2 * ex.KV_HEADS
    plan = [([40, 17], []), ([1, 30], []), ([1, 1, 100], [1]), ([1, 1], []), ([0, 1, 5], [0]), ([1, 1, 64, 9], [])]
    seen, names, fresh = {}, [], 0  # per request: its keys and values so far
    for new, done in plan:
        while len(names) < len(new):
            step.add(1)
            names.append(fresh)
            seen[fresh] = []
            fresh += 1
        tokens = sum(new)
        qkv = torch.randn(tokens, heads, ex.DIM, generator=gen, device="cuda").to(torch.bfloat16)
        out = step.run(new, qkv).float().cpu().numpy().astype(np.float64)
        host = qkv.float().cpu().numpy().astype(np.float64)
        at = 0
        for i, n in enumerate(new):
            seen[names[i]].append(host[at:at + n, ex.HEADS:])
            kvs = np.concatenate(seen[names[i]])
            length = len(kvs)
            if n:
                # the oracle on one dense block
                k = kvs[None, :, :ex.KV_HEADS].transpose(0, 2, 1, 3)
                v = kvs[None, :, ex.KV_HEADS:].transpose(0, 2, 1, 3)
                ref = kv.attention(host[at:at + n, :ex.HEADS], k, v, np.array([[0]]), [0, n], [length], ex.DIM ** -0.5)
                bound = kv.attention_bound(*ref, length, ex.DIM, 8, 8, np.abs(v).max())
                assert (np.abs(out[at:at + n] - ref[0]) <= bound).all()
            at += n
        if done:
            step.remove(done)
            names = [x for i, x in enumerate(names) if i not in done]
    held = sum(step.blocks_of(c) for c in step.context)
    assert step.free.numel() + held == 2048 // 16
    assert len(torch.unique(step.free)) == step.free.numel()


def test_a_full_cache_is_a_crash(ex):
    knobs = {"max-num-seqs": 64, "max-num-batched-tokens": 4096, "block-size": 16, "enable-chunked-prefill": True}
    assert ex.evaluate(knobs, [(500, 4)] * 8, cache_tokens=1024) is None
    got = ex.evaluate(knobs, [(500, 4)] * 8, cache_tokens=8192)
    assert got is not None and got[0] > 0 and got[1] > 0


def test_a_short_tuning_run(ex):
    X, Y, valid, best = ex.tune(3, 2, n_requests=12, pool=4096)
    assert X.shape == (6, 9) and len(valid) == 6
    assert best >= 0 and valid[best] and Y[best, 0] < 0 < Y[best, 1]
