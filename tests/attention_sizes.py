"""Sizes that together reach every kernel the attention operators' plans choose: prompts as (queries, keys, sequences, heads, key heads,
elements, causal), caches as (requests, longest, heads, key heads, elements, tokens of a page)."""

FORWARD = {
    "bfloat16": [(40, 40, 1, 2, 1, d, True) for d in (20, 64, 90, 128, 200)] + [(600, 600, 1, 2, 2, d, True) for d in (32, 60, 96, 128)] +
                [(2100, 2100, 20, 32, 32, d, True) for d in (16, 64, 96, 128, 256)] + [(70, 1500, 1, 2, 1, d, False) for d in (32, 40, 96, 128, 130)] +
                [(2200, 2200, 2, 64, 1, 32, False), (65, 5000, 1, 4, 4, 64, True)],
    "float32": [(40, 40, 1, 2, 1, d, True) for d in (20, 64, 90, 128, 200)] + [(70, 1500, 1, 2, 1, d, False) for d in (32, 40, 96, 128, 130)],
}
BACKWARD = {
    "bfloat16": [(40, 40, 1, 2, 1, d, True) for d in (20, 64, 90, 128, 200)] + [(700, 700, 1, 4, 2, d, True) for d in (30, 64, 96, 127, 256)] +
                [(2100, 2100, 20, 32, 32, d, True) for d in (16, 64, 96, 128, 256)] + [(1100, 1100, 2, 16, 16, d, False) for d in (32, 64, 96, 128)] +
                [(2100, 2100, 1, 16, 16, d, True) for d in (64, 96, 128)] + [(2100, 2100, 1, 32, 32, d, True) for d in (96, 128)] +
                [(4500, 4500, 1, 16, 16, 128, True), (4500, 4500, 1, 16, 16, 72, True)] + [(90, 150, 2, 4, 2, d, False) for d in (80, 120, 160)],
    "float32": [(40, 40, 1, 2, 1, d, True) for d in (20, 64, 90, 128, 200)] + [(700, 700, 1, 4, 2, d, True) for d in (30, 64, 96, 127, 256)] +
               [(90, 150, 2, 4, 2, d, False) for d in (24, 48, 80, 120, 160)],
}
BACKWARD["bfloat16"] += [(1100, 1100, 1, 8, 2, d, False) for d in (96, 128)]
CACHES = {t: [(3, 100, 2, 1, d, 16) for d in (16, 64, 72, 128, 192)] + [(3, 300, 4, 2, d, 7) for d in (13, 65, 130)] + [(2, 2000, 3, 1, 64, 16), (40, 700, 32, 4, 32, 16)]
          for t in ("bfloat16", "float32")}


def calls():
    """All of them for attention_launches.record."""
    out = [[what, *s, t] for what, sizes in (("forward", FORWARD), ("backward", BACKWARD)) for t, group in sizes.items() for s in group]
    return out + [["paged", *s, t] for t, group in CACHES.items() for s in group]
