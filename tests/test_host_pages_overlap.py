"""Host-only: nat_kv_reserve and nat_kv_release refuse arrays that share memory with one that is written, but for counts and lengths in their own places."""
import pytest

import paper_2603_06619_amd as nat

N, WIDTH, PAGES, CAP, BASE = 3, 4, 9, 10, 1 << 40
READ = dict(counts=4, lens=4 * N, change=4 * N)
RESERVE = dict(READ, free=4 * PAGES, table=4 * N * WIDTH, counts_out=8, lens_out=4 * N, start=4 * N, cu=4 * N + 4, slots=8 * CAP, pos=4 * CAP, ws=4 * N)
RELEASE = dict(READ, table=4 * N * WIDTH, free=4 * PAGES, counts_out=8, lens_out=4 * N, ws=4 * N + 4)
UNTOUCHED = {"reserve": {"counts", "lens", "change", "free"}, "release": {"counts", "lens", "change", "table"}}


def reserve(lib, a):
    return lib.nat_kv_reserve(a["table"], WIDTH, N, 16, a["lens"], a["change"], a["free"], PAGES, a["counts"], CAP, a["counts_out"], a["lens_out"], a["start"], a["cu"], a["slots"],
                              a["pos"], a["ws"], 256, None)


def release(lib, a):
    return lib.nat_kv_release(a["table"], WIDTH, N, 16, a["lens"], a["change"], a["free"], PAGES, a["counts"], a["counts_out"], a["lens_out"], a["ws"], 256, None)


@pytest.mark.parametrize("call,sizes", [(reserve, RESERVE), (release, RELEASE)], ids=["reserve", "release"])
def test_each_pair(call, sizes):
    """Every two arrays of which one is written: the second at the first's place, and where their last and first elements meet."""
    lib = nat.load_library()
    invalid = call(lib, dict.fromkeys(sizes, 0))                                     # (NULL pointers)
    apart = {name: BASE + 4096 * i for i, name in enumerate(sizes)}
    tried = 0
    for x in sizes:
        for y in sizes:
            if x == y or {x, y} <= UNTOUCHED[call.__name__]:
                continue
            places = [apart[x], apart[x] + sizes[x] - 4, apart[x] - sizes[y] + 4]
            if (y, x) in (("counts_out", "counts"), ("lens_out", "lens"), ("counts", "counts_out"), ("lens", "lens_out")):
                places = [p for p in places if p != apart[x]]
            if y == "ws":
                places = [p for p in places if p % 256 == 0]
            for at in places:
                assert call(lib, dict(apart, **{y: at})) == invalid, (x, y, at - apart[x])
                tried += 1
    assert tried > 50
