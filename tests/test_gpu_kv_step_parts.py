"""A serving step with rotations and scales of blocks, part by part and step by step: the queries and the cache's keys and values
against float64 on the step's vectors, and every step's attention against float64 on what the cache holds then."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import rotary_cases as B  # noqa: E402
import step_bounds  # noqa: E402
from oracle import kv_cache as kv  # noqa: E402
from oracle import rotary as R  # noqa: E402
from test_gpu_kv_cache import _check, f64  # noqa: E402
from test_gpu_kv_rotated_step import BLOCKS, BS, D, HKV, HQ, STEPS, Engine  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", [0, 3])
@pytest.mark.parametrize("steps", [STEPS, [(100, 0, 1), (1, 90, 1), (1, 1, 1), (30, 2, 200), (1, 1, 1), (1, 0, 1)]], ids=["mixed", "chunks"])
def test_every_part_of_every_step(steps, seed):
    e = Engine(steps, seed)
    freqs = e.rotary.freqs.cpu().numpy()
    seen = [[] for _ in range(3)]  # the requests' rows, of all steps so far
    for i, new in enumerate(steps):
        e.run(i)
        x, at, n = f64(e.qkv[i]), 0, sum(new)
        table = e.table.cpu().numpy()
        cache = [f64(c) * f64(s)[:, :, None, None] for c, s in ((e.kc, e.ks), (e.vc, e.vs))]
        scales = [f64(s) for s in (e.ks, e.vs)]
        top = np.zeros((n, HQ, 1))
        for r in range(3):
            rows = x[at:at + new[r]]
            pos = np.arange(len(seen[r]), len(seen[r]) + new[r])
            want = R.rotate(rows[:, :HQ], pos, freqs)
            _check(f64(e.q[i][at:at + new[r]]), want, B.rotate_bound(rows[:, :HQ], want, D // 2, False, 1.0, "bf16"))
            seen[r] += list(rows)
            if not seen[r]:
                continue
            all_rows, where = np.array(seen[r]), np.arange(len(seen[r]))
            block, slot = table[r, where // BS], where % BS
            assert ((block >= 0) & (block < BLOCKS)).all()
            keys = all_rows[:, HQ:HQ + HKV]
            turned = R.rotate(keys, where, freqs)
            _check(cache[0][block, :, slot], turned, step_bounds.key_bound(keys, turned, D // 2, scales[0][block][:, :, None]))
            values = all_rows[:, HQ + HKV:]
            _check(cache[1][block, :, slot], values, 2.0 ** -4 * np.abs(values) + 2 * 2.0 ** -10 * scales[1][block][:, :, None])
            largest = np.maximum.accumulate(np.abs(cache[1][block, :, slot]).max(-1))
            top[at:at + new[r], :, 0] = np.repeat(largest[pos], HQ // HKV, 1)
            at += new[r]
        b = e.batch[i]
        ref = kv.attention(f64(e.q[i][:n]), *cache, table, b.query_start.cpu().numpy(), b.seq_len.cpu().numpy(), D ** -0.5)
        _check(f64(e.out[i][:n]), ref[0], step_bounds.attention_bound(ref, int(b.seq_len.max()), D, top))
