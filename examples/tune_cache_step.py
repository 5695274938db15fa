"""Tunes an inference engine's cache step where it runs: suggestions from the
library, evaluations on the library's own cache operators.

The evaluator is the attention part of an engine's step for one layer: a
scheduler with the knobs max-num-seqs, max-num-batched-tokens, block-size and
enable-chunked-prefill of the space in workloads/synth.py takes synthetic
requests through kv_assign (blocks and slots), kv_write (keys and values into
the cache) and kv_attention (prompt chunks and single tokens over the cache),
and measures generated tokens per second and the 99th percentile of the step
time.  With --rotary the vectors are turned by their positions on the way, and
with --cache f8 the cache holds 8-bit floats with a scale per block and head
(kv_append in the place of kv_write).  A configuration whose step runs out of blocks counts as crashed, which
the feasibility forest learns.  The other knobs do not act on one layer of one
GPU and are searched along.

    python examples/tune_cache_step.py --rounds 6 --parallel 2
"""
import argparse
import os
import sys
import time

import numpy as np
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2408_04323_amd as scoot  # noqa: E402
from workloads.synth import VLLM_MAX_MODEL_LEN, sobol_table, vllm_decode, vllm_space  # noqa: E402

HEADS, KV_HEADS, DIM = 32, 8, 128


def requests(n, seed=0):
    """(prompt, answer) lengths: log-normal prompts, short answers."""
    rng = np.random.default_rng(seed)
    prompt = np.clip(np.exp(rng.normal(5.5, 1.0, n)), 16, VLLM_MAX_MODEL_LEN - 256).astype(int)
    return list(zip(prompt.tolist(), rng.integers(8, 96, n).tolist()))


class CacheStep:
    """The cache of one layer and the requests that run in it.  ``rotary``
    turns queries and keys by their positions; a ``scaled`` cache holds 8-bit
    floats with a scale per block and head."""

    def __init__(self, block_size, cache_tokens, device="cuda", rotary=None, scaled=False):
        self.bs = int(block_size)
        blocks = cache_tokens // self.bs
        shape = (blocks, KV_HEADS, self.bs, DIM)
        self.rotary, self.scaled = rotary, scaled
        dtype = torch.float8_e4m3fn if scaled else torch.bfloat16
        self.k_cache = torch.zeros(shape, dtype=dtype, device=device)
        self.v_cache = torch.zeros(shape, dtype=dtype, device=device)
        self.k_scale = torch.ones(shape[:2], device=device) if scaled else 1.0
        self.v_scale = torch.ones(shape[:2], device=device) if scaled else 1.0
        self.free = torch.randperm(blocks, device=device).to(torch.int32)
        self.cols = -(-VLLM_MAX_MODEL_LEN // self.bs)
        self.table = torch.full((0, self.cols), -1, dtype=torch.int32, device=device)
        self.context = []  # cached tokens of the running requests, in the table's order
        self.device = device

    def add(self, n):
        self.table = torch.cat([self.table, self.table.new_full((n, self.cols), -1)])
        self.context += [0] * n

    def blocks_of(self, tokens):
        return -(-tokens // self.bs)

    def run(self, new, qkv):
        """One step: ``new[i]`` tokens of request i, whose queries, keys and
        values are the rows of ``qkv`` (tokens, HEADS + 2 KV_HEADS, DIM).
        Returns the attention's result, or None if the cache is full."""
        taken = sum(self.blocks_of(c + n) - self.blocks_of(c) for c, n in zip(self.context, new))
        if taken > self.free.numel():
            return None
        tokens = sum(new)
        lens = torch.tensor([self.context, new], dtype=torch.int32).to(self.device)
        batch = scoot.kv_assign(lens[0], lens[1], self.table, self.free, self.bs, tokens)
        q, k, v = qkv[:tokens, :HEADS], qkv[:tokens, HEADS:HEADS + KV_HEADS], qkv[:tokens, HEADS + KV_HEADS:]
        if self.rotary is None and not self.scaled:
            scoot.kv_write(k, v, batch.slots, self.k_cache, self.v_cache)
        else:
            turned = scoot.kv_append(k, v, batch.positions, batch.slots, self.k_cache, self.v_cache, self.rotary, self.k_scale,
                                     self.v_scale, q=None if self.rotary is None else q)
            q = q if turned is None else turned
        self.context = [c + n for c, n in zip(self.context, new)]
        out = scoot.kv_attention(q, self.k_cache, self.v_cache, self.table, batch.query_start, batch.seq_len,
                                 max_new_len=max(new), max_seq_len=max(self.context), k_scale=self.k_scale, v_scale=self.v_scale)
        self.free = self.free[taken:]
        return out

    def remove(self, done):
        """The requests at the places ``done`` end: their blocks become free."""
        gone = set(done)
        back = [self.table[i, :self.blocks_of(self.context[i])] for i in done]
        self.free = torch.cat([self.free] + back)
        keep = [i for i in range(len(self.context)) if i not in gone]
        self.table = self.table[torch.tensor(keep, dtype=torch.int64, device=self.device)]
        self.context = [self.context[i] for i in keep]


def evaluate(knobs, work, cache_tokens=1 << 16, device="cuda", **of_step):
    """(generated tokens per second, 99th percentile of the step time in
    seconds) of serving ``work`` under ``knobs``; None if the cache ran full."""
    budget, seats = int(knobs["max-num-batched-tokens"]), int(knobs["max-num-seqs"])
    step = CacheStep(knobs["block-size"], cache_tokens, device, **of_step)
    gen = torch.Generator(device=device).manual_seed(1)
    qkv = torch.randn(budget, HEADS + 2 * KV_HEADS, DIM, generator=gen, device=device).to(torch.bfloat16)
    waiting, running, times, made = list(work), [], [], 0  # running: [prompt tokens left, answer tokens left]
    while waiting or running:
        room = budget - sum(1 for r in running if r[0] == 0)
        new = [1 if r[0] == 0 else 0 for r in running]
        for i, r in enumerate(running):  # prompts under way
            n = min(r[0], max(0, room))
            new[i] += n
            room -= n
        first = len(running)
        while waiting and len(running) < seats and room > 0:
            prompt, answer = waiting[0]
            if not knobs["enable-chunked-prefill"] and prompt > room:
                break
            waiting.pop(0)
            n = min(prompt, room)
            running.append([prompt, answer])
            new.append(n)
            room -= n
        step.add(len(running) - first)
        torch.cuda.synchronize()
        t = time.perf_counter()
        if step.run(new, qkv) is None:
            return None
        torch.cuda.synchronize()
        times.append(time.perf_counter() - t)
        done = []
        for i, (r, n) in enumerate(zip(running, new)):
            if r[0] > 0:
                r[0] -= n
            elif n:
                r[1] -= 1
                made += 1
                if r[1] == 0:
                    done.append(i)
        if done:
            step.remove(done)
            running = [r for r in running if r[1] > 0]
    return made / sum(times), float(np.quantile(times, 0.99))


def tune(rounds, parallel, n_requests=64, cache_tokens=1 << 16, pool=16384, say=print, **of_step):
    """Algorithm 1 with measured evaluations: (X, Y, valid, best row)."""
    sp = vllm_space()
    poly, vinit = sobol_table(sp["d"])
    space = dict(levels=sp["levels"], poly=poly, vinit=vinit, A=sp["A"], b=sp["b"])
    work = requests(n_requests)
    X, Y, valid, delta, c = np.zeros((0, sp["d"])), np.zeros((0, 2)), np.zeros(0, dtype=np.uint8), 0.5, 0
    for t in range(rounds):
        x, _, _ = scoot.suggest(X, Y, valid, space, k=parallel, delta=delta, pool_size=pool, pool_skip=1 + t * pool, t=t + 1)
        knobs = vllm_decode(x)
        bad = False
        for i in range(len(x)):
            kn = {name: col[i] for name, col in knobs.items()}
            got = evaluate(kn, work, cache_tokens, **of_step)
            bad = bad or got is None
            y = (0.0, 0.0) if got is None else (-got[0], got[1])
            X, Y, valid = np.vstack([X, x[i]]), np.vstack([Y, y]), np.append(valid, np.uint8(got is not None))
            say(f"round {t}: seqs {kn['max-num-seqs']:5d} tokens {kn['max-num-batched-tokens']:5d} block {kn['block-size']:2d} "
                f"chunked {int(kn['enable-chunked-prefill'])}: "
                + ("crashed" if got is None else f"{got[0]:8.0f} tokens/s, p99 step {got[1] * 1e3:.2f} ms"))
        if t:
            delta, c = scoot.delta_update(delta, c, k=parallel, any_invalid=bad)
    best = int(np.argmin(np.where(valid != 0, Y[:, 0], np.inf))) if valid.any() else -1
    return X, Y, valid, best


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--rounds", type=int, default=6)
    ap.add_argument("--parallel", type=int, default=2)
    ap.add_argument("--requests", type=int, default=64)
    ap.add_argument("--cache-tokens", type=int, default=1 << 16)
    ap.add_argument("--rotary", type=float, metavar="BASE", help="turn queries and keys by their positions")
    ap.add_argument("--cache", choices=("bf16", "f8"), default="bf16")
    a = ap.parse_args()
    rotary = None if a.rotary is None else scoot.rotary_create(DIM, base=a.rotary)
    X, Y, valid, best = tune(a.rounds, a.parallel, a.requests, a.cache_tokens, rotary=rotary, scaled=a.cache == "f8")
    if best < 0:
        print("no configuration ran")
        return 1
    print("most tokens/s:", {k: v[0].item() for k, v in vllm_decode(X[best:best + 1]).items()},
          f"{-Y[best, 0]:.0f} tokens/s, p99 step {Y[best, 1] * 1e3:.2f} ms")
    return 0


if __name__ == "__main__":
    sys.exit(main())
