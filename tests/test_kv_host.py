"""Refusals of the key/value cache calls, decided before anything is launched (no GPU needed)."""
import ctypes as C

import numpy as np
import pytest

import paper_2408_04323_amd as S
from paper_2408_04323_amd._native import lib

INVALID, UNSUPPORTED = -1, -4
BUF = (C.c_uint8 * 4096)()
P = (C.addressof(BUF) + 63) & ~63

ASSIGN = dict(context_len=P, new_len=P, num_seqs=2, block_size=16, block_table=P, max_blocks=4, table_stride=4,
              free_blocks=P, num_free=3, max_tokens=8, query_start=P, seq_len=P, positions=P, slots=P, counts=P, stream=None)
WRITE = dict(k=P, v=P, type=1, num_tokens=4, num_kv_heads=2, head_dim=64, k_token_stride=128, k_head_stride=64,
             v_token_stride=128, v_head_stride=64, slots=P, k_cache=P, v_cache=P, cache_type=1, num_blocks=4, block_size=16,
             k_scale=1.0, v_scale=1.0, stream=None)
ATTEND = dict(q=P, type=1, num_tokens=4, num_heads=4, num_kv_heads=2, head_dim=64, q_token_stride=256, q_head_stride=64,
              k_cache=P, v_cache=P, cache_type=1, num_blocks=4, block_size=16, block_table=P, max_blocks=4, table_stride=4,
              query_start=P, seq_len=P, num_seqs=2, max_new_len=2, max_seq_len=9, scale=0.1, window=0, k_scale=1.0, v_scale=1.0,
              out=P, out_token_stride=256, out_head_stride=64, workspace=None, workspace_bytes=0, stream=None)


def _refused(fn, args, status, **change):
    a = dict(args)
    a.update(change)
    assert fn(*a.values()) == status, change
    assert lib().scoot_last_error().decode().startswith("kv "), change


@pytest.mark.parametrize("change", [
    dict(num_seqs=-1), dict(num_seqs=2 ** 20 + 1), dict(block_size=12), dict(block_size=4), dict(block_size=512), dict(block_size=0),
    dict(block_size=-16), dict(max_blocks=-1), dict(max_blocks=2 ** 30, table_stride=2 ** 30), dict(table_stride=3),
    dict(table_stride=2 ** 40), dict(num_free=-1), dict(max_tokens=-1), dict(max_tokens=2 ** 31), dict(context_len=None),
    dict(new_len=None), dict(block_table=None), dict(free_blocks=None), dict(query_start=None), dict(seq_len=None),
    dict(positions=None), dict(slots=None), dict(counts=None)], ids=str)
def test_assign_refuses(change):
    _refused(lib().scoot_kv_assign, ASSIGN, INVALID, **change)


@pytest.mark.parametrize("change,status", [
    (dict(type=2), INVALID), (dict(type=7), INVALID), (dict(cache_type=0), INVALID), (dict(cache_type=3), INVALID),
    (dict(num_kv_heads=0), INVALID), (dict(num_kv_heads=1025), INVALID), (dict(head_dim=60), UNSUPPORTED),
    (dict(head_dim=0), UNSUPPORTED), (dict(head_dim=1032), UNSUPPORTED), (dict(block_size=24), INVALID), (dict(num_blocks=-1), INVALID),
    (dict(num_blocks=2 ** 31), INVALID), (dict(num_tokens=-1), INVALID), (dict(num_tokens=2 ** 31), INVALID),
    (dict(k_token_stride=-1), INVALID), (dict(v_head_stride=2 ** 32), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID),
    (dict(slots=None), INVALID), (dict(k_cache=None), INVALID), (dict(v_cache=None), INVALID), (dict(k=P + 1), INVALID),
    (dict(k_cache=P + 8), INVALID), (dict(k_scale=0.5), INVALID), (dict(cache_type=2, k_scale=0.0), INVALID),
    (dict(cache_type=2, v_scale=float("nan")), INVALID), (dict(cache_type=2, v_scale=float("inf")), INVALID)], ids=str)
def test_write_refuses(change, status):
    _refused(lib().scoot_kv_write, WRITE, status, **change)


@pytest.mark.parametrize("change,status", [
    (dict(type=2), INVALID), (dict(cache_type=0), INVALID), (dict(num_heads=3), INVALID), (dict(num_heads=0), INVALID),
    (dict(num_heads=2048), INVALID), (dict(head_dim=96), UNSUPPORTED), (dict(head_dim=512), UNSUPPORTED), (dict(block_size=48), INVALID),
    (dict(num_tokens=-1), INVALID), (dict(num_seqs=-1), INVALID), (dict(num_seqs=2 ** 20 + 1), INVALID), (dict(max_new_len=-1), INVALID),
    (dict(max_seq_len=2 ** 31), INVALID), (dict(window=-1), INVALID), (dict(scale=float("nan")), INVALID), (dict(scale=-1.0), INVALID),
    (dict(max_blocks=-1), INVALID), (dict(max_blocks=5), INVALID), (dict(table_stride=2 ** 40), INVALID),
    (dict(q_token_stride=-8), INVALID), (dict(q_token_stride=257), INVALID), (dict(out_head_stride=68), INVALID), (dict(q=P + 2), INVALID),
    (dict(out=P + 8), INVALID), (dict(k_cache=P + 8), INVALID), (dict(q=None), INVALID), (dict(out=None), INVALID),
    (dict(k_cache=None), INVALID), (dict(block_table=None), INVALID), (dict(query_start=None), INVALID), (dict(seq_len=None), INVALID),
    (dict(v_scale=2.0), INVALID), (dict(cache_type=2, k_scale=-1.0), INVALID)], ids=str)
def test_attention_refuses(change, status):
    _refused(lib().scoot_kv_attention, ATTEND, status, **change)


def test_empty_calls_launch_nothing():
    w, a = dict(WRITE), dict(ATTEND)
    for change in (dict(num_tokens=0), dict(num_blocks=0)):
        assert lib().scoot_kv_write(*{**w, **change}.values()) == 0
    for change in (dict(num_tokens=0), dict(num_seqs=0)):
        assert lib().scoot_kv_attention(*{**a, **change}.values()) == 0


def test_workspace_bytes():
    assert S.kv_attention_workspace(0, 8, 2, 128, 0, 0, 0) >= 0
    # one long request on an empty GPU is split along its keys, a large batch is not
    assert S.kv_attention_workspace(8192, 32, 8, 128, 2, 4096, 4096) % 16 == 0
    for bad in (dict(heads=3), dict(head_dim=80), dict(num_seqs=-1), dict(window=-2)):
        args = dict(tokens=4, heads=4, kv_heads=2, head_dim=64, num_seqs=2, max_new_len=2, max_seq_len=9, window=0)
        args.update(bad)
        with pytest.raises(S.ScootError):
            S.kv_attention_workspace(**args)


def test_a_short_workspace_is_refused():
    args = dict(ATTEND)
    args.update(num_tokens=1, num_seqs=1, num_heads=8, num_kv_heads=1, head_dim=128, max_new_len=1, max_seq_len=65536, max_blocks=4096,
                table_stride=4096)
    need = S.kv_attention_workspace(1, 8, 1, 128, 1, 1, 65536)
    if need == 0:
        pytest.skip("these sizes are not split")
    _refused(lib().scoot_kv_attention, args, INVALID, workspace=None, workspace_bytes=0)
    _refused(lib().scoot_kv_attention, args, INVALID, workspace=P, workspace_bytes=need - 1)
    _refused(lib().scoot_kv_attention, args, INVALID, workspace=P + 8, workspace_bytes=need)


def test_binding_refuses_host_tensors_and_wrong_shapes():
    torch = pytest.importorskip("torch")
    z = torch.zeros(4, dtype=torch.int32)
    with pytest.raises(ValueError, match="device"):
        S.kv_assign(z, z, torch.zeros(4, 2, dtype=torch.int32), z, 16, 8)
    k = torch.zeros(3, 2, 64, dtype=torch.bfloat16)
    cache = torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device"):
        S.kv_write(k, k, torch.zeros(3, dtype=torch.int64), cache, cache)
    with pytest.raises(ValueError, match="device"):
        S.kv_attention(k, cache, cache, torch.zeros(1, 2, dtype=torch.int32), z[:2], z[:1], 1, 1)
    with pytest.raises(ValueError, match="float16"):
        S.kv_attention(k.float(), cache.float(), cache.float(), torch.zeros(1, 2, dtype=torch.int32), z[:2], z[:1], 1, 1)
    assert np.array_equal(z.numpy(), np.zeros(4))


@pytest.mark.parametrize("block_size", [8, 16, 32, 64, 128, 256])
def test_attention_refuses_tables_past_its_key_numbers(block_size):
    """Keys are counted in 32 bits, and strips of 64 of them may start 32 before the last one: such a table's end would
    wrap around."""
    most = (2 ** 31 - 256) // block_size
    fits = dict(ATTEND, block_size=block_size, max_blocks=most, table_stride=most, num_tokens=0)  # no tokens: nothing is launched
    assert lib().scoot_kv_attention(*fits.values()) == 0
    _refused(lib().scoot_kv_attention, ATTEND, INVALID, block_size=block_size, max_blocks=most + 1, table_stride=most + 1, num_tokens=0)


@pytest.mark.parametrize("change", [dict(scale=3e38), dict(scale=1e20, k_scale=1e20, cache_type=2), dict(scale=2.4e38)], ids=str)
def test_attention_refuses_scales_whose_product_overflows(change):
    """A score of 0 would become 0 * inf."""
    _refused(lib().scoot_kv_attention, ATTEND, INVALID, **change)
    fits = dict(ATTEND, num_tokens=0, scale=2.3e38)  # nothing is launched
    assert lib().scoot_kv_attention(*fits.values()) == 0
