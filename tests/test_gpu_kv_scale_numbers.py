"""Scales that are tensors of one element are numbers; of a cache of one block and one head they may be that block's."""
import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _cache(blocks, heads, dtype, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return [torch.randn(blocks, heads, 16, 64, generator=g, device=DEV).mul_(3).to(dtype) for _ in range(2)]


def _attend(q, k, v, blocks, **scales):
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)  # noqa: E731
    return S.kv_attention(q, k, v, i32(*range(blocks))[None], i32(0, q.shape[0]), i32(16 * blocks), q.shape[0], 16 * blocks, **scales)


@pytest.mark.parametrize("shape", [(), (1,), (1, 1), (1, 1, 1)])
@pytest.mark.parametrize("at", ["cpu", DEV])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float8_e4m3fn])
def test_attention_takes_a_number_of_any_shape(dtype, at, shape):
    k, v = _cache(3, 2, dtype)
    q = torch.randn(2, 4, 64, generator=torch.Generator(device=DEV).manual_seed(2), device=DEV).to(torch.bfloat16)
    ks, vs = (torch.full(shape, x, device=at) for x in (0.5, 0.25)) if dtype is torch.float8_e4m3fn else (torch.ones(shape, device=at) for _ in range(2))
    want = _attend(q, k, v, 3, k_scale=float(ks), v_scale=float(vs))
    for pair in ((ks, vs), (ks, float(vs)), (float(ks), vs)):
        assert torch.equal(_attend(q, k, v, 3, k_scale=pair[0], v_scale=pair[1]), want)


def test_appends_take_a_number_of_any_shape():
    g = torch.Generator(device=DEV).manual_seed(3)
    x = torch.randn(5, 2, 64, generator=g, device=DEV).to(torch.bfloat16)
    slots = torch.arange(5, device=DEV)
    want = _cache(3, 2, torch.float8_e4m3fn)
    S.kv_append(x, x, None, slots, *want, k_scale=0.5, v_scale=0.25)
    for at in ("cpu", DEV):
        got = _cache(3, 2, torch.float8_e4m3fn)
        S.kv_append(x, x, None, slots, *got, k_scale=torch.tensor([[0.5]], device=at), v_scale=torch.tensor([[0.25]], device=at))
        assert all(torch.equal(a.view(torch.uint8), b.view(torch.uint8)) for a, b in zip(got, want))


def test_scales_of_one_block_and_head():
    """Updated in place by an append, and read by attention without a copy to the host (inside a graph)."""
    g = torch.Generator(device=DEV).manual_seed(4)
    x = torch.randn(16, 1, 64, generator=g, device=DEV).mul_(1000).to(torch.bfloat16)
    q = torch.randn(16, 3, 64, generator=g, device=DEV).to(torch.bfloat16)
    k, v = _cache(1, 1, torch.float8_e4m3fn)
    ks, vs = torch.ones(1, 1, device=DEV), torch.ones(1, 1, device=DEV)
    S.kv_append(x, 2 * x, None, torch.arange(16, device=DEV), k, v, k_scale=ks, v_scale=vs)
    need = 2.0 ** torch.ceil(torch.log2(x.float().abs().max() / 448))
    assert float(ks) == float(need) and float(vs) == 2 * float(need)
    one = _attend(q, k, v, 1, k_scale=float(ks), v_scale=float(vs), scale=1e-4)
    assert torch.equal(_attend(q, k, v, 1, k_scale=ks, v_scale=vs, scale=1e-4), one)
    table, start, length = (torch.tensor(n, dtype=torch.int32, device=DEV) for n in ([[0]], [0, 16], [16]))
    out = torch.zeros_like(q)
    space = torch.empty(max(1, S.kv_attention_workspace(16, 3, 1, 64, 1, 16, 16)), dtype=torch.uint8, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        S.kv_attention(q, k, v, table, start, length, 16, 16, scale=1e-4, k_scale=ks, v_scale=vs, out=out, workspace=space)
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, one)
