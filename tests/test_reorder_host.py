"""Two caches of a reordering share no memory: every pair of arrays, refused on the host."""
import ctypes as C

import paper_2402_06262_b200 as R
from test_decoding_host import INVALID, two_caches

FIELDS = ("K", "V", "s", "q", "n", "pos", "live", "t_next")
S, G, B, d = 2, 2, 16, 64
BYTES = dict(K=S * G * B * d * 2, V=S * G * B * d * 2, live=S * G * 4, t_next=S * G * 4)


def size(f):
    return BYTES.get(f, S * G * B * 4)


def test_caches_that_share_memory_are_refused():
    src = two_caches()
    far = {f: 0x1100000 + 0x100000 * i for i, f in enumerate(FIELDS)}
    call = lambda dst: R.lib().roco_cache_reorder(C.byref(src), C.byref(dst), 0x10000, None)  # noqa: E731
    for theirs in FIELDS:
        for mine in FIELDS:
            at = getattr(src, theirs)
            if theirs == "K" and mine == "K":
                places = (at + 16, at + size("K") - 16, at - size("K") + 16)      # (the same K: in place)
            elif mine in ("K", "V"):
                places = (at, at + size(theirs) // 16 * 16 - 16, at - size(mine) + 16)
            else:
                places = (at, at + size(theirs) - 4, at - size(mine) + 4)
            for x in places:
                assert call(two_caches(**{**far, mine: x})) == INVALID, (theirs, mine, hex(x))
