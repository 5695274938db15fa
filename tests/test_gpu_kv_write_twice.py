"""Two tokens with one slot: the contract leaves the slot's content open, but each piece of eight elements is one token's,
and no other slot changes."""
import pytest

torch = pytest.importorskip("torch")

import paper_2408_04323_amd as S  # noqa: E402

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("cache", [torch.bfloat16, torch.float8_e4m3fn], ids=["16 bits", "8 bits"])
def test_a_slot_named_twice_holds_pieces_of_its_tokens(cache):
    print("[case] write twice", cache, flush=True)
    tokens, heads, d, bs = 600, 3, 128, 16
    g = torch.Generator(device=DEV).manual_seed(2)
    k, v = torch.randint(-8, 9, (2, tokens, heads, d), generator=g, device=DEV).to(torch.bfloat16)  # exact in both types
    slots = torch.arange(tokens, device=DEV)
    slots[tokens // 2:] = slots[:tokens // 2]  # far apart: other workgroups
    slots[[5, 7]] = slots[[6, 6]]              # and side by side
    kc, vc = (torch.full((tokens // bs + 2, heads, bs, d), 9.0, device=DEV).to(cache) for _ in range(2))
    S.kv_write(k, v, slots, kc, vc)
    for x, c in ((k, kc), (v, vc)):
        got = c.float().transpose(1, 2).reshape(-1, heads, d // 8, 8)
        x = x.float().view(tokens, heads, d // 8, 8)
        for s in set(slots.tolist()):
            mine = x[slots == s]  # tokens of this slot
            assert (mine == got[s]).all(-1).any(0).all(), s
        rest = torch.ones(len(got), dtype=torch.bool, device=DEV)
        rest[slots] = False
        assert (got[rest] == 9).all()
