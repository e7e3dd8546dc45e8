"""CPU pins of the beam-decode oracle: the quantiser's bounds, the record's
layout, tables, selection and reordering on cases worked out by hand."""
import numpy as np
import pytest

from oracle import beam as ob


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
def test_quantiser_error_is_within_half_a_step(dtype):
    rng = np.random.default_rng(1)
    eps = 2.0 ** -8 if dtype == "bf16" else 2.0 ** -11
    for _ in range(200):
        x = ob.round16(rng.normal(rng.normal(), abs(rng.normal()) + 0.1, 64), dtype)
        c, s, z = ob.quantise(x, dtype)
        back = s * (c - 8.0) + z
        # half a step, what clamping adds (15 steps off by the rounding of s) and the rounding of z
        assert np.abs(back - x).max() <= s * (0.5 + 15 * eps) + eps * abs(z)
        assert c.min() >= 0 and c.max() <= 15


def test_constant_and_non_finite_groups():
    c, s, z = ob.quantise(np.full(64, 1.5), "bf16")
    assert s == 0 and z == 1.5 and (c == 8).all()
    for bad in (np.inf, -np.inf, np.nan):
        x = np.zeros(64)
        x[5] = bad
        _, s, z = ob.quantise(x, "f16")
        assert np.isnan(s) and np.isnan(z)


def test_record_places_are_a_partition():
    seen = np.zeros((ob.RECORD, 2), int)
    for pos in range(16):
        for d in range(64):
            for v in (0, 1):
                byte, nib = ob.code_place(pos, d, v)
                seen[byte, nib] += 1
        for v in (0, 1):
            seen[ob.scale_place(pos, v):][:4] += 1
    assert (seen == 1).all()


def test_cache_round_trip():
    rng = np.random.default_rng(2)
    c = ob.Cache(3, 32, 2, 128, "bf16", fill=0xFF)
    rows = ob.round16(rng.normal(size=(2, 256)), "bf16")
    c.put(37, rows[0], 0)
    c.put(37, rows[1], 1)
    for v in (0, 1):
        want = np.concatenate([s * (k - 8.0) + z for k, s, z in (ob.quantise(g, "bf16") for g in rows[v].reshape(-1, 64))])
        np.testing.assert_array_equal(c.get(37, v), want.astype(np.float32))


def test_attention_closed_forms():
    v = np.array([[1.0, 0], [0, 1], [5, 5]])
    k = np.zeros((3, 2))
    out, _ = ob.attention(np.ones((3, 2)), k, v, 1.0, np.array([[1, 1, 0], [0, 0, 0], [0, 0, 1]], bool))
    np.testing.assert_allclose(out, [[0.5, 0.5], [0, 0], [5, 5]])


def test_page_plan_by_hand():
    t = np.full((3, 4), -1)
    t[0, 0] = 9
    t, off, slots, lens, left, err = ob.page_plan([10, 0, 0], [18, 1, 40], 16, [1, 2, 3, 4], 4, t, 60, 10)
    assert t[0, 1] == 4 and t[1, 0] == 3 and off == [0, 8, 9, 9] and lens == [18, 1, 0] and left == 2
    assert slots[:9] == [9 * 16 + 10 + i for i in range(6)] + [64, 65, 48] and set(slots[9:]) == {-1}
    assert err == (True, False)  # the third request needs three blocks; two are left


def test_selection_by_hand():
    x = np.log(np.array([[0.5, 0.3, 0.1, 0.1], [0.1, 0.2, 0.3, 0.4]]))
    got, _ = ob.beam_select(x, np.array([0.0, -0.1]), np.zeros(4), eos=0)
    assert got["fin_parent"][0] == 0 and got["token"] == [3, 1] and got["parent"] == [1, 0]


def test_reorder_by_hand():
    t = np.array([[1, 10], [1, 11], [2, 12]])
    new, freed, moves = ob.beam_reorder(t, 20, [1, 1, 0], 16)
    assert new.tolist() == [[1, 11], [1, 12], [1, 10]] and freed == [2] and moves == [(11, 12, 4)]
    new, freed, moves = ob.beam_reorder(t, 20, [-1, -1, -1], 16)
    assert (new == -1).all() and freed == [1, 2, 10, 11, 12] and not moves
