"""Attention cases that reach every form of the kernel, small ones: for each head dimension and cache type few rows with four
and with eight waves, and tiles, each with the keys in one part and in several, with more workgroups than compute units and with
fewer.  ``form`` is what a case is there for ("few" or "tiles", waves, LDS buffers, several parts)."""

DIMS, TYPES, CACHES = (64, 128, 192, 256), ("bf16", "f16"), ("same", "f8")
# One request of more than 16 rows makes a call one of tiles; the others' few rows go along.
MANY = [(i * 13 % 60, 1) for i in range(7)]


def _lens():
    """(lens, kv_heads): more than 256 items and key heads, and fewer."""
    return {
        "few": MANY + [(300, 3), (0, 2)], "few_parts": MANY + [(6200, 2), (0, 1)],
        "tiles": MANY + [(70, 20), (0, 40)], "tiles_parts": MANY + [(2300, 24), (0, 17)],
    }


def row_bytes(c):
    return c["d"] * (1 if c["cache"] == "f8" else 2)


def cases():
    got = {}
    for d in DIMS:
        for kind in TYPES:
            for cache in CACHES:
                for name, lens in _lens().items():
                    for many in (True, False):
                        wide = d * (1 if cache == "f8" else 2) > 256  # no eight waves
                        tiles, parts = name.startswith("tiles"), name.endswith("parts")
                        if (wide and not tiles and not many) or (d >= 192 and tiles and parts and many):
                            continue  # the same form as its neighbour, or parts that would not pay
                        c = dict(lens=lens if many else lens[5:], kind=kind, cache="f8" if cache == "f8" else kind, hq=33 if many else 4,
                                 hkv=33 if many else 2, d=d, bs=16, window=0, scale=None, hints=None, stale=float("nan"))
                        buffers = 4 if d == 192 and cache == "f8" else 2
                        c["form"] = ("tiles", 4, buffers, parts) if tiles else ("few", 4 if many or wide else 8, 0, parts)
                        got[f"{name}-{d}-{kind}-{c['cache']}-{'many' if many else 'one each'}"] = c
    return got


CASES = cases()


def plan_line(c):
    lens = c["lens"]
    return " ".join(map(str, (sum(n for _, n in lens), c["hq"], c["hkv"], c["d"], 1 if c["cache"] == "f8" else 2, len(lens),
                              max(n for _, n in lens), max(a + n for a, n in lens), c["window"])))
