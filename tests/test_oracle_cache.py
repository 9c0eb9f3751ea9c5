"""Pins of the 8-bit cache's plain definition (oracle/cache.py) to things other than itself. No GPU."""
import numpy as np
import pytest

from oracle import cache as oc


def test_e4m3_numbers_are_torchs():
    torch = pytest.importorskip("torch")
    got = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(got, oc.e4m3_values())


def test_e4m3_rounding_is_torchs():
    torch = pytest.importorskip("torch")
    vals = oc.e4m3_values()
    mid = (vals[1:] + vals[:-1]) / 2                         # ties, exact in float32
    x = np.concatenate([vals, mid, mid * (1 + 2.0 ** -20), mid * (1 - 2.0 ** -20), np.random.default_rng(0).uniform(-448, 448, 2000)]).astype(np.float32)
    x = np.concatenate([x, -x])
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(oc.nearest_code(x, "e4m3"), want)


def test_int8_rounding_and_range():
    x = np.array([0.5, 1.5, -0.5, -2.5, 126.5, 127.4, 200.0, -np.inf, np.inf, np.nan])
    assert oc.nearest_code(x, "int8").tolist() == [0, 2, 0, -2, 126, 127, 127, -127, 127, 0]


@pytest.mark.parametrize("fmt,bound", [("int8", 0.5), ("e4m3", 16.0)])
def test_stored_rows_come_back_within_half_a_step(fmt, bound):
    rng = np.random.default_rng(1)
    c = oc.Cache(1, 2, 64, 4, 1, 4, fmt)
    x = rng.standard_normal((1, 2, 37, 2, 64))
    assert c.reserve([0], [37]) == [37]
    c.store(0, x)
    for w in range(2):
        y = c.rows(0, 0, w)
        step = c.scales[0][:, c.table[0, np.arange(37) // 16], w].T[..., None]
        assert (np.abs(y - x[0, w]) <= bound * step * (1 + 1e-12)).all()


def test_attention_is_softmax_and_a_lone_key_is_its_value():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((3, 4, 8)), rng.standard_normal((3, 2, 8)), rng.standard_normal((3, 2, 8))
    none = np.zeros((0, 2, 8))
    out, lse, _ = oc.attention(q, k, v, none, none, np.eye(3, dtype=bool), 0.3)
    assert np.allclose(out, np.repeat(v, 2, axis=1)) and np.allclose(lse[1, 3], 0.3 * q[1, 3] @ k[1, 1])
    out, lse, _ = oc.attention(q, k, v, none, none, np.zeros((3, 3), bool), 0.3)
    assert (out == 0).all() and (lse == -np.inf).all()
    # the cached half and the pass's half are one sum
    a, la, _ = oc.attention(q, k, v, k, v, np.zeros((3, 3), bool), 0.3)
    b, lb, _ = oc.attention(q, k, v, none, none, np.ones((3, 3), bool), 0.3)
    assert np.allclose(a, b) and np.allclose(la, lb)


def test_rotation_keeps_lengths_and_depends_on_distance():
    rng = np.random.default_rng(3)
    f = 1e4 ** (-np.arange(4) / 4)
    x, y = rng.standard_normal((1, 1, 12)), rng.standard_normal((1, 1, 12))
    for il in (False, True):
        r = lambda z, p: oc.rotate(z, [p], f, 1.0, il)  # noqa: E731
        assert np.allclose(np.linalg.norm(r(x, 77)), np.linalg.norm(x)) and np.array_equal(r(x, 77)[..., 8:], x[..., 8:])
        assert np.allclose((r(x, 9) * r(y, 5)).sum(), (r(x, 104) * r(y, 100)).sum())
    pair = oc.rotate(np.array([[[1.0, 0.0]]]), [1], [np.pi / 2], 2.0, True)
    assert np.allclose(pair, [[[0.0, 2.0]]])


def test_pages_by_hand():
    c = oc.Cache(1, 1, 64, 6, 4, 3, "int8")
    assert c.reserve([1, 0], [20, 16]) == [20, 16]                   # pages 0, 1 and 2
    assert c.table[1, :2].tolist() == [0, 1] and c.table[0, 0] == 2
    c.fork([1], [2])
    assert c.refs.tolist() == [2, 2, 1, 0, 0, 0]
    assert c.reserve([2, 1], [1, 13]) == [1, 13]                     # both leave the shared page 1; 33 tokens need a third
    assert c.table[2].tolist() == [0, 3, -1] and c.table[1].tolist() == [0, 4, 5]
    assert c.refs.tolist() == [2, 0, 1, 1, 1, 1]
    assert c.reserve([0, 3], [17, 1]) == [0, 0]                      # two pages asked, one free; the next finds none left
    c.truncate([1], [16])
    assert c.refs.tolist() == [2, 0, 1, 1, 0, 0] and c.lens.tolist() == [16, 16, 21, 0]
    assert c.compact() == 3 and c.refs.tolist() == [2, 1, 1, 0, 0, 0] and c.table[2].tolist() == [0, 1, -1]


def test_frequencies_of_the_scalings():
    from paper_2503_14153_b200 import SpecError, rotary_frequencies
    f, g = rotary_frequencies(8, 1e4)
    assert g == 1.0 and np.allclose(f, [1, 0.1, 0.01, 0.001])
    assert np.allclose(rotary_frequencies(8, 1e4, "linear", 4.0)[0], np.array(f) / 4)
    n = rotary_frequencies(8, 1e4, "ntk", 4.0)[0]
    assert n[0] == 1.0 and np.isclose(n[-1], f[-1] / 4)              # the fastest pair keeps its pace, the slowest is stretched by the factor
    y, g = rotary_frequencies(64, 1e4, "yarn", 4.0, 8192)
    p = np.array(rotary_frequencies(64, 1e4)[0])
    turns = 8192 * p / (2 * np.pi)
    assert np.isclose(g, 0.1 * np.log(4) + 1) and np.allclose(np.array(y)[turns > 40], p[turns > 40]) and np.allclose(np.array(y)[turns < 0.8], p[turns < 0.8] / 4)
    for bad in (dict(rot=7, base=1e4), dict(rot=8, base=1e4, scaling="x"), dict(rot=8, base=1e4, scaling="yarn", factor=2.0), dict(rot=2, base=1e4, scaling="ntk")):
        with pytest.raises(SpecError):
            rotary_frequencies(**bad)
