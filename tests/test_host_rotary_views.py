"""Which views the rotary call takes for its results: slices of one tensor, interleaved or not, as long as no element belongs to two of
them.  The answer is compared with one that looks at every element."""
import random

import pytest

from host_calls import run


def elements(first, strides, counts, D):
    """Every element of a view, None if one is in it twice."""
    rows = [first + i * strides[0] + j * strides[1] + k * strides[2] for i in range(counts[0]) for j in range(counts[1]) for k in range(counts[2])]
    all_ = [r + c for r in rows for c in range(D)]
    return set(all_) if len(set(all_)) == len(all_) else None


def disjoint(sizes, views):
    B, L, Hq, Hkv, D = sizes
    sets = [elements(first, s, (B, n, L), D) for (first, *s), n in zip(views, (Hq, Hkv, Hkv))]
    return all(s is not None for s in sets) and not (sets[0] & sets[1] or sets[0] & sets[2] or sets[1] & sets[2])


def fused(B, L, Hq, Hkv, D, layout, room=0):
    """Q, K and V as the slices of one tensor's heads; room: elements between the batches beside them."""
    H = Hq + 2 * Hkv
    b = H * L * D + room
    h, l = (D, H * D) if layout == "tokens" else (L * D, D)
    return [(n * h, b, h, l) for n in (0, Hq, Hq + Hkv)]


@pytest.mark.parametrize("layout", ["tokens", "heads"])
@pytest.mark.parametrize("room", [0, 40])
def test_heads_of_one_tensor(layout, room):
    cases = []
    for Hq, Hkv in [(1, 1), (24, 24), (24, 12), (24, 8), (24, 4), (6, 2), (5, 2), (8, 1), (2, 5)]:
        for B, L in [(1, 9), (2, 9), (3, 1), (1, 1), (2, 33024)]:
            sizes, views = [B, L, Hq, Hkv, 64], fused(B, L, Hq, Hkv, 64, layout, room)
            assert L > 9 or disjoint(sizes, views)
            cases += [[sizes, views], [sizes, [(f - (8 if i == 2 else 0), *s) for i, (f, *s) in enumerate(views)]]]   # V begins inside K
    for i, (case, got) in enumerate(zip(cases, run("rotary_views", cases))):
        assert "must not overlap" in got if i % 2 else got == 0, (case, got)


def test_a_row_that_belongs_to_two_views():
    sizes = (1, 2, 2, 2, 64)
    views = [(0, 0, 320, 192), (128, 0, 320, 192), (4096, 0, 320, 192)]              # element 320 is in the first two
    assert not disjoint(sizes, views)
    assert run("rotary_views", [[sizes, views]]) == ["rotary_heads: K must not overlap Q"]


def test_as_every_element_says():
    rng = random.Random(5)
    cases = []
    while len(cases) < 1500:
        sizes = (rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 4), rng.randint(1, 3), 32)
        B, L, Hq, Hkv, D = sizes
        shared = rng.random() < 0.6
        strides = None
        views = []
        for n in (Hq, Hkv, Hkv):
            if strides is None or not shared:
                order = [(L, 2), (max(Hq, Hkv) if shared else n, 1), (B, 0)]
                rng.shuffle(order)
                strides, step = [0, 0, 0], D * rng.randint(1, 3) + 8 * rng.randint(0, 3)
                for count, place in order:                   # each steps over what the ones before reach, as the call wants it
                    strides[place] = step if count > 1 else 0
                    step = max(step, (count - 1) * step + D + 8 * rng.randint(0, 20) if count > 1 else step)
            views.append((8 * rng.randint(0, 150), *strides))
        if all(elements(f, s, (B, n, L), D) is not None for (f, *s), n in zip(views, (Hq, Hkv, Hkv))):
            cases.append([sizes, views])
    want = [disjoint(*c) for c in cases]
    assert 150 < sum(want) < 1350
    for case, got, fine in zip(cases, run("rotary_views", cases), want):
        assert got == 0 if fine else (got != 0 and "overlap" in got), (case, got)
