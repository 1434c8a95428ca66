"""The plain definitions themselves, on hand-made numbers (no GPU)."""
import numpy as np

import pass_reference as ref


def test_quantise_keeps_extremes_inside_and_takes_ties_to_even():
    x = np.zeros(64, dtype=np.float32)
    x[:5] = [0.0, 15.0, 0.5, 1.5, 2.5]                # scale 1, offset 0: ties at one half
    code, s, z = ref.quantise(x)
    assert (s, z) == (1.0, 0.0) and list(code[:5]) == [0, 15, 0, 2, 2]
    code, s, z = ref.quantise(np.full(64, 0.3, dtype=np.float32))
    assert z <= 0.3 and abs(code[0] * s + z - 0.3) <= s / 2 + 1e-9
    assert np.isnan(ref.quantise(np.array([1.0, np.inf] * 32))[1])
    assert ref.quantise(np.zeros(64))[1:] == (0.0, 0.0)


def test_every_code_has_a_place_of_its_own_in_a_run():
    for D in (64, 128):
        seen = {f(t, c, D) for f in (ref.key_byte, ref.value_byte) for t in range(16) for c in range(D)}
        assert len(seen) == 2 * 16 * D and {a for a, _ in seen} == set(range(16 * D))


def test_cache_round_trip_and_rows():
    rng = np.random.default_rng(1)
    for D in (64, 128):
        cache = np.zeros((3, 2, 32 * (D + 8)), dtype=np.uint8)
        x = rng.normal(size=(2, 2, D)).astype(np.float32)
        for h in range(2):
            ref.cache_put(cache, 32, D, 37, h, x[0, h], x[1, h])
        k, v = ref.cache_rows(cache, 32, D, [37])
        for h in range(2):
            kk, vv = ref.cache_get(cache, 32, D, 37, h)
            assert np.array_equal(kk, k[0, h]) and np.array_equal(vv, v[0, h])
            _, s, _ = ref.quantise(x[0, h])
            assert np.abs(kk - x[0, h]).max() <= s / 2 + 1e-6


def test_plan_takes_gives_back_and_refuses_in_order():
    r = ref.plan(seq=[5, 16, 3], new=[12, 0, 1], count=[1, 3, 1], head=6, tail=8, table=[[0, 9, 9], [1, 2, 3], [4, 9, 9]],
                 ring=[5, 6, 7, 8, 0, 0, 6, 5], page=16, T=14)
    assert r["block_table"][0][:2] == [0, 6] and r["block_count"] == [2, 1, 1] and r["ring_pos"] == [7, 10]
    assert r["free_ring"][:2] == [2, 3] and r["cu_new"] == [0, 12, 12, 13]
    assert r["slot"][:12] == [5 + i for i in range(11)] + [6 * 16] and r["slot"][12:] == [4 * 16 + 3, -1]
    r = ref.plan([0, 0], [40, 16], [0, 0], 0, 2, [[0, 0, 0]] * 2, [1, 2], 16, 99)
    assert r["row_status"] == [ref.NO_BLOCKS] * 2
