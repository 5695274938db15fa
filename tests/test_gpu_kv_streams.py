"""Cache calls on the default stream named by its handle, 0: in order with what is queued there."""
import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _ints(*v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def test_handle_0_is_the_default_stream():
    t = torch.zeros(1, device=DEV)
    with torch.cuda.stream(torch.cuda.Stream()):
        with S._kv_on(0, t):
            assert torch.cuda.current_stream().cuda_stream == 0
        side = torch.cuda.current_stream().cuda_stream
        assert side != 0
    with S._kv_on(side, t):
        assert torch.cuda.current_stream().cuda_stream == side


def test_a_step_on_handle_0_is_in_order():
    """Lengths, vectors and queries are still being made on the default stream when the calls are issued, and their results
    are used there at once: everything a step reads and writes has to be ordered by that stream alone."""
    print("[case] stream 0 in order", flush=True)
    g = torch.Generator(device=DEV).manual_seed(3)
    qkv = torch.randn(70, 12, 64, generator=g, device=DEV).to(torch.bfloat16)
    slow = torch.randn(4096, 4096, generator=g, device=DEV)
    lengths, want = _ints(60, 10), None
    for late in (False, True):
        ctx, new, live = _ints(0, 0), _ints(0, 0), torch.zeros_like(qkv)
        table = torch.full((2, 8), -1, dtype=torch.int32, device=DEV)
        free = torch.arange(16, dtype=torch.int32, device=DEV)
        kc, vc = torch.zeros(2, 16, 2, 16, 64, dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        if late:
            x = slow
            for _ in range(20):
                x = torch.mm(x, slow).mul_(1e-2)  # some ten milliseconds in front
        new.copy_(lengths)
        live.copy_(qkv)
        b = S.kv_assign(ctx, new, table, free, 16, 70, stream=0)
        S.kv_write(live[:, 8:10], live[:, 10:], b.slots, kc, vc, stream=0)
        out = S.kv_attention(live[:, :8], kc, vc, table, b.query_start, b.seq_len, 60, 60, stream=0)
        got = (out + 0, b.slots + 0, b.seq_len + 0, kc + 0)
        if late:
            assert all(torch.equal(a, w) for a, w in zip(got, want))
        else:
            torch.cuda.synchronize()
            want = got
    assert want[2].tolist() == [60, 10] and torch.isfinite(want[0]).all() and (want[0] != 0).any()


@pytest.mark.skipif(not torch.cuda.is_available() or torch.cuda.device_count() < 2, reason="needs a second GPU")
def test_a_step_on_a_device_that_is_not_current():
    """Streams and kernels are those of the tensors' device."""
    g = torch.Generator().manual_seed(3)
    qkv, got = torch.randn(70, 12, 64, generator=g).to(torch.bfloat16), []
    torch.cuda.set_device(0)
    for at in ("cuda:0", "cuda:1"):
        lens = torch.tensor([[0, 0], [60, 10]], dtype=torch.int32, device=at)
        table, free = torch.full((2, 8), -1, dtype=torch.int32, device=at), torch.arange(16, dtype=torch.int32, device=at)
        kc, vc = torch.zeros(2, 16, 2, 16, 64, dtype=torch.bfloat16, device=at)
        x = qkv.to(at)
        b = S.kv_assign(lens[0], lens[1], table, free, 16, 70)
        S.kv_write(x[:, 8:10], x[:, 10:], b.slots, kc, vc)
        got.append(S.kv_attention(x[:, :8], kc, vc, table, b.query_start, b.seq_len, 60, 60).cpu())
        assert torch.cuda.current_device() == 0
    assert torch.equal(*got)
