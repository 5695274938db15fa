"""A serving step with rotations and scales of blocks, as an engine runs it: slots, an append that turns queries and keys,
attention over the cache in 8 bits.  Several steps, eagerly, on a stream of their own and captured."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402
from oracle import kv_cache as kv  # noqa: E402
from oracle import rotary as R  # noqa: E402
from test_gpu_kv_cache import _check, dev, f64  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
HQ, HKV, D, BS, BLOCKS, COLS = 8, 2, 128, 16, 96, 24


class Engine:
    """Three requests; a step brings a prompt, a chunk of it, or single tokens."""

    def __init__(self, steps, seed=0):
        rng = np.random.default_rng(seed)
        self.steps, self.qkv = steps, []
        for new in steps:
            self.qkv.append(dev(rng.standard_normal((sum(new) + 3, HQ + 2 * HKV, D)) * np.exp(rng.uniform(-1, 1)), torch.bfloat16))
        self.rotary = S.rotary_create(D, scaling="bands", factor=4.0, length=64, low=1.0, high=4.0)
        self.order = dev(rng.permutation(BLOCKS), torch.int32)
        self.kc, self.vc = (torch.zeros(BLOCKS, HKV, BS, D, dtype=torch.float8_e4m3fn, device=DEV) for _ in range(2))
        self.ks, self.vs = (torch.ones(BLOCKS, HKV, device=DEV) for _ in range(2))
        self.table = torch.full((3, COLS), -1, dtype=torch.int32, device=DEV)
        self.context = [torch.tensor(np.sum(steps[:i], 0) if i else np.zeros(3), dtype=torch.int32).to(DEV) for i in range(len(steps))]
        self.new = [torch.tensor(n, dtype=torch.int32).to(DEV) for n in steps]
        self.batch = [S.KVBatch(3, sum(n) + 3, DEV) for n in steps]
        self.q = [torch.zeros(sum(n) + 3, HQ, D, dtype=torch.bfloat16, device=DEV) for n in steps]
        self.out = [torch.zeros_like(q) for q in self.q]
        self.taken = [sum(-(-int(sum(s[r] for s in steps[:i])) // BS) for r in range(3)) for i in range(len(steps))]
        most = max(max(n) for n in steps)
        self.space = torch.empty(max(1, max(S.kv_attention_workspace(sum(n) + 3, HQ, HKV, D, 3, most, BS * COLS) for n in steps)), dtype=torch.uint8,
                                 device=DEV)

    def state(self):
        return self.kc, self.vc, self.ks, self.vs, self.table

    def run(self, i):
        b, x = self.batch[i], self.qkv[i]
        S.kv_assign(self.context[i], self.new[i], self.table, self.order[self.taken[i]:], BS, x.shape[0], out=b)
        S.kv_append(x[:, HQ:HQ + HKV], x[:, HQ + HKV:], b.positions, b.slots, self.kc, self.vc, rotary=self.rotary, k_scale=self.ks,
                    v_scale=self.vs, q=x[:, :HQ], out=self.q[i])
        S.kv_attention(self.q[i], self.kc, self.vc, self.table, b.query_start, b.seq_len, max(self.steps[i]), BS * COLS, k_scale=self.ks,
                       v_scale=self.vs, out=self.out[i], workspace=self.space)


STEPS = [(40, 3, 0), (1, 70, 17), (1, 1, 1), (5, 1, 130), (1, 1, 1)]


def test_steps_match_the_oracle():
    """The attention of every step against float64 on the exact keys and values: what lies between is the cache's 8 bits,
    off by 2^-4 of a value, or half a smallest step of its block's scale for each time that it grew (less than 2 * 2^-10 E in
    all, E <= 2 / 448 of the block's largest), and the softmax of scores that are off by q . (k' - k)."""
    e = Engine(STEPS)
    keys, values = [[[] for _ in range(3)] for _ in range(2)]
    freqs = e.rotary.freqs.cpu().numpy()
    for i, new in enumerate(STEPS):
        e.run(i)
        x, at = f64(e.qkv[i]), 0
        for r in range(3):
            pos = np.arange(len(keys[r]), len(keys[r]) + new[r])
            rows = x[at:at + new[r]]
            keys[r] += list(R.rotate(rows[:, HQ:HQ + HKV], pos, freqs))
            values[r] += list(rows[:, HQ + HKV:])
            q = R.rotate(rows[:, :HQ], pos, freqs)
            got = f64(e.out[i][at:at + new[r]])
            k, v = np.array(keys[r]).reshape(-1, HKV, D), np.array(values[r]).reshape(-1, HKV, D)
            for j, p in enumerate(pos):
                for h in range(HQ):
                    kh, vh = k[:p + 1, h // (HQ // HKV)], v[:p + 1, h // (HQ // HKV)]
                    s = D ** -0.5 * (kh @ q[j, h])
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    # Off in keys and values, element by element; largest of all blocks for a block's largest.
                    dk = 2.0 ** -4 * np.abs(kh) + 2 * 2.0 ** -10 * 2 / 448 * np.abs(k).max()
                    dv = 2.0 ** -4 * np.abs(vh) + 2 * 2.0 ** -10 * 2 / 448 * np.abs(v).max()
                    ds = D ** -0.5 * (dk @ np.abs(q[j, h])) + 2.0 ** -8 * D ** -0.5 * (np.abs(kh) @ np.abs(q[j, h]))  # and the query's rounding
                    want, spread = w @ vh, w @ np.abs(vh)
                    off = np.expm1(2 * ds.max()) * (spread + w @ dv) + w @ dv + 2.0 ** -7 * (spread + np.abs(want))
                    assert (np.abs(got[j, h] - want) <= off).all(), (i, r, j, h)
            at += new[r]
        assert (e.out[i][sum(new):] == 0).all() and (e.q[i][sum(new):] == 0).all()  # rows of no request
        held = f64(e.vc) * f64(e.vs)[:, :, None, None]
        for r in range(3):  # the cache holds the values to 8 bits
            t = e.table[r].cpu().numpy()
            for p, val in enumerate(values[r]):
                b = t[p // BS]
                big = 2 * 2.0 ** -10 * f64(e.vs)[b][:, None]
                assert (np.abs(held[b, :, p % BS] - val) <= 2.0 ** -4 * np.abs(val) + big).all(), (r, p)


def test_attention_of_a_step_is_that_of_what_the_cache_holds():
    e = Engine(STEPS, seed=3)
    for i in range(len(STEPS)):
        e.run(i)
    i = len(STEPS) - 2
    f = Engine(STEPS, seed=3)
    for j in range(i + 1):
        f.run(j)
    k, v = (f64(c) * f64(s)[:, :, None, None] for c, s in ((f.kc, f.ks), (f.vc, f.vs)))
    b, n = f.batch[i], sum(STEPS[i])
    ref = kv.attention(f64(f.q[i]), k, v, f.table.cpu().numpy(), b.query_start.cpu().numpy(), b.seq_len.cpu().numpy(), D ** -0.5)
    bound = kv.attention_bound(*(x[:n] for x in ref), BS * COLS, D, 8, 11, 448 * float(f.vs.max()))
    _check(f64(f.out[i][:n]), ref[0][:n], bound)
    assert torch.equal(e.out[i], f.out[i])  # the same bits again


def test_steps_in_graphs():
    """Two steps captured, each into a graph of its own that shares cache and workspace with the other, replayed in turn on the
    stream that they were captured on, with eager work in between."""
    eager = Engine(STEPS, seed=5)
    want = []
    for i in range(len(STEPS)):
        eager.run(i)
        want.append([x.clone() for x in (*eager.state(), eager.out[i], eager.q[i])])
    e = Engine(STEPS, seed=5)
    start = [x.clone() for x in e.state()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in range(len(STEPS)):
            e.run(i)
    side.synchronize()
    for got, ref in zip((*e.state(), e.out[-1], e.q[-1]), want[-1]):
        assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8))
    graphs = []
    for i in range(len(STEPS)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            e.run(i)
        graphs.append(g)
    for turn in range(3):
        for x, x0 in zip(e.state(), start):
            x.copy_(x0)
        for i, g in enumerate(graphs):
            e.out[i].zero_()
            e.q[i].zero_()
            if turn == 1:
                torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for got, ref in zip((*e.state(), e.out[i], e.q[i]), want[i]):
                assert torch.equal(got.view(torch.uint8), ref.view(torch.uint8)), (turn, i)


def test_a_step_on_a_stream_that_is_not_current():
    """Every call named the same stream: results, workspaces and made queries belong to it."""
    e = Engine(STEPS, seed=6)
    for i in range(3):
        e.run(i)
    f = Engine(STEPS, seed=6)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    s = side.cuda_stream
    for i in range(3):
        x = f.qkv[i]
        b = S.kv_assign(f.context[i], f.new[i], f.table, f.order[f.taken[i]:], BS, x.shape[0], stream=s)
        q = S.kv_append(x[:, HQ:HQ + HKV], x[:, HQ + HKV:], b.positions, b.slots, f.kc, f.vc, rotary=f.rotary, k_scale=f.ks, v_scale=f.vs,
                        q=x[:, :HQ], stream=s)
        out = S.kv_attention(q, f.kc, f.vc, f.table, b.query_start, b.seq_len, max(STEPS[i]), BS * COLS, k_scale=f.ks, v_scale=f.vs, stream=s)
        junk = torch.full((1 << 20,), float("nan"), device=DEV)  # takes freed memory of the current stream
        side.synchronize()
        n = sum(STEPS[i])
        assert torch.equal(q[:n], e.q[i][:n]) and torch.equal(out[:n], e.out[i][:n]), i
        del junk


@pytest.mark.skipif(not torch.cuda.is_available() or torch.cuda.device_count() < 2, reason="needs a second GPU")
def test_calls_on_a_device_that_is_not_current():
    g, got = torch.Generator().manual_seed(3), []
    qkv = torch.randn(70, 12, 64, generator=g).to(torch.bfloat16)
    torch.cuda.set_device(0)
    for at in ("cuda:0", "cuda:1"):
        x, rot = qkv.to(at), S.rotary_create(64, device=at)
        kc, vc = torch.zeros(2, 16, 2, 16, 64, device=at).to(torch.float8_e4m3fn)
        ks, vs = torch.ones(2, 16, 2, device=at)
        pos, slots = torch.arange(70, dtype=torch.int32, device=at), torch.arange(70, device=at)
        q = S.kv_append(x[:, 8:10], x[:, 10:], pos, slots, kc, vc, rotary=rot, k_scale=ks, v_scale=vs, q=x[:, :8])
        got.append([t.cpu() for t in (q, S.rotate(x, pos, rot), kc.view(torch.uint8), vs)])
        assert torch.cuda.current_device() == 0
    assert all(torch.equal(a, b) for a, b in zip(*got))
