"""The oracles of the 4-bit cache and of the page calls, pinned on the CPU."""
import numpy as np
import pytest

from oracle import cache_pages as cp
from oracle import fp4


def test_codes_and_their_rounding():
    """Every value of the format comes back; others go to the nearest, halves to the even code."""
    for k in (-100, -7, 0, 3, 125):
        x = np.zeros((16, 32))
        x[:, 0], x[:, 1] = 6.0, np.concatenate([fp4.VALUES, -fp4.VALUES])
        code, scale = fp4.encode(x * 2.0 ** k)
        assert np.all(scale == k + 127) and np.array_equal(code[:, 1], [0, 1, 2, 3, 4, 5, 6, 7, 8, 9, 10, 11, 12, 13, 14, 15])
        assert np.array_equal(fp4.decode(code, scale), x * 2.0 ** k)
    x = np.zeros((1, 32))
    x[0, :15] = [6.5, .25, .75, 1.25, 1.75, 2.5, 3.5, 5, .2501, .7499, 1.2501, 1.7499, 2.4999, 3.4999, 5.0001]
    assert list(fp4.encode(x)[0][0, :15]) == [7, 0, 2, 2, 4, 4, 6, 6, 1, 1, 3, 3, 4, 5, 7]


def test_scale_is_the_smallest_with_seven():
    rng = np.random.default_rng(0)
    x = rng.normal(size=(400, 32)) * 2.0 ** rng.integers(-60, 60, size=(400, 1))
    code, scale = fp4.encode(x)
    s, top = 2.0 ** (scale[:, 0].astype(float) - 127), np.abs(x).max(axis=1)
    assert np.all(7 * s >= top) and np.all(3.5 * s < top)
    assert np.all(np.abs(fp4.decode(code, scale) - x) <= s[:, None])
    assert fp4.encode(np.full((1, 32), 7.0))[1] == 127 and fp4.encode(np.full((1, 32), 7.001))[1] == 128
    assert fp4.encode(np.zeros((1, 32)))[1] == 27
    code, scale = fp4.encode(np.where(np.arange(64) == 40, np.inf, 1.0)[None])
    assert list(scale[0]) == [125, 255] and not code[0, 32:].any()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("part", [0, 1])
def test_tiles_hold_every_code_once(d, part):
    byte, high, scale = fp4.places(d, part)
    assert sorted((2 * byte + high).reshape(-1)) == list(range(16 * d))
    assert sorted(np.unique(scale)) == list(range(8 * d, 17 * d // 2))
    rng = np.random.default_rng(d)
    code = rng.integers(0, 16, size=(3, 2, 16, d)).astype(np.uint8)
    sc = rng.integers(0, 256, size=(3, 2, 16, d // 32)).astype(np.uint8)
    back = fp4.load(fp4.store(code, sc, part), d, part)
    assert np.array_equal(back[0], code) and np.array_equal(back[1], sc)


def _rows(rng, pool, n):
    ids, rows, at = list(rng.permutation(pool)), [], 5
    for _ in range(n):
        k = int(rng.integers(0, 6))
        rows.append(ids[:5] + ids[at:at + k])
        at += k
    return rows


@pytest.mark.parametrize("seed", range(20))
def test_fork_keeps_every_text_apart(seed):
    """Holders add up; a child reads its parent's tokens; a page that can be appended to has one holder."""
    rng = np.random.default_rng(seed)
    rows = _rows(rng, 80, 6)
    refs = [sum(row.count(p) for row in rows) for p in range(80)]
    lengths = [int(rng.integers(0, 16 * len(r) + 1)) for r in rows]
    parent = [int(rng.integers(-1, 6)) for _ in range(7)]
    room = [int(rng.integers(0, 40)) for _ in parent]
    status, new, lens, after, copies, need, have = cp.fork(rows, lengths, parent, room, refs, 20)
    assert status == 0 and need <= have
    assert after == [sum(row.count(p) for row in new) for p in range(80)]
    content = {p: p for p in range(80)}
    content.update({to: src for src, to in copies})
    assert not {s for s, _ in copies} & {t for _, t in copies}
    for i, p in enumerate(parent):
        assert len(new[i]) == -(-(lens[i] + room[i]) // 16)
        if p >= 0:
            assert lens[i] == lengths[p]
            pages = -(-lens[i] // 16)
            assert [content[q] for q in new[i][:pages]] == rows[p][:pages]
        for q in new[i][lens[i] // 16:]:
            assert after[q] == 1


@pytest.mark.parametrize("seed", range(20))
def test_compact_fills_the_front(seed):
    rng = np.random.default_rng(seed)
    rows = _rows(rng, 70, 5)
    refs = [sum(row.count(p) for row in rows) for p in range(70)]
    status, new, after, moved, copies = cp.compact(rows, refs)
    live = sum(r > 0 for r in refs)
    assert status == 0 and all(r > 0 for r in after[:live]) and not any(after[live:])
    assert after == [sum(row.count(p) for row in new) for p in range(70)]
    came = {to: src for src, to in copies}
    assert [[came.get(p, p) for p in row] for row in new] == rows


def test_forks_that_cannot_be():
    refs = [1, 1, 2, 0]
    rows, lengths = [[0, 2], [1, 2]], [20, 32]
    ok = dict(rows=rows, lengths=lengths, parent=[0], room=[0], refs=refs, to_pages=4)
    assert cp.fork(**ok)[0] == 0
    for change in (dict(parent=[2]), dict(room=[-1]), dict(lengths=[33, 32]), dict(to_pages=1), dict(refs=[1, 1, 1, 0]),
                   dict(rows=[[0, 4], [1, 2]])):
        assert cp.fork(**{**ok, **change})[0] == 2
    assert cp.fork(**{**ok, "room": [45], "to_pages": 9})[0] == 1


def test_error_of_a_value():
    """At most s up to 7 s; above 7 * 2^125, where the scale stays 2^125, at most 2 s, and 6 * 2^125 is what remains."""
    rng = np.random.default_rng(4)
    x = rng.uniform(-1, 1, size=(400, 32)) * 2.0 ** rng.integers(-90, 128, size=(400, 1))
    x[0], x[1], x[2] = np.finfo(np.float32).max, 7 * 2.0 ** 125, np.nextafter(np.float32(7 * 2.0 ** 125), np.float32(np.inf))
    code, scale = fp4.encode(x)
    s = np.repeat(2.0 ** (scale.astype(np.float64) - 127), 32, axis=-1)
    off = np.abs(fp4.decode(code, scale) - x)
    above = np.abs(x) > 7 * 2.0 ** 125
    assert above[0].all() and above[2].all() and not above[1].any()
    assert (off[~above] <= s[~above]).all() and (off[above] <= 2 * s[above]).all() and (off[above] > s[above]).all()
    assert (fp4.decode(code, scale)[above] == 6 * 2.0 ** 125 * np.sign(x[above])).all()
