"""The oracle of the block formats against the formats' printed properties and closed forms.  CPU only."""
import numpy as np
import pytest
import torch

from oracle import store


def test_code_values():
    assert store.VALUES8[-1] == 448 and store.VALUES8[8] == 2.0 ** -6 and store.VALUES8[1] == 2.0 ** -9
    e4m3 = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(store.VALUES8, e4m3)
    assert np.all(np.diff(store.VALUES4) > 0) and np.all(np.diff(store.VALUES8) > 0)


def test_nearest_is_round_to_nearest_even():
    rng = np.random.default_rng(1)
    v = np.concatenate([rng.uniform(0, 464, 20000), np.abs(rng.standard_normal(20000)), (store.VALUES8[1:] + store.VALUES8[:-1]) / 2])
    v = v.astype(np.float32)
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(store.VALUES8[store.nearest(v, store.VALUES8)], want)
    #  ties of the 4-bit codes, by hand: to the even mantissa
    for a, b in ((0.25, 0), (0.75, 1), (1.25, 1), (1.75, 2), (2.5, 2), (3.5, 4), (5.0, 4)):
        assert store.VALUES4[store.nearest(a, store.VALUES4)] == b
    assert store.nearest(7.0, store.VALUES4) == 8 and store.nearest(6.99, store.VALUES4) == 7
    assert store.nearest(464.0, store.VALUES8) == 126 and store.nearest(464.01, store.VALUES8) == 127


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_scales_are_the_smallest_that_hold_the_block(dtype):
    for most in (1.0, 5.9, 6.0, 6.9, 7.0, 7.1, 448.0, 464.0, 470.0, 3e-5, 60000.0):
        for values, bounds in ((store.VALUES4, store.BOUNDS4[dtype]), (store.VALUES8, store.BOUNDS8[dtype])):
            e = store.scale_exponent(most, values, bounds)
            if e < bounds[1]:
                assert store.nearest(most / 2.0 ** e, values) < len(values)
            if e > bounds[0]:
                assert store.nearest(most / 2.0 ** (e - 1), values) >= len(values)
    assert store.scale_exponent(0.0, store.VALUES4, store.BOUNDS4[dtype]) == store.BOUNDS4[dtype][0]


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
def test_every_value_at_every_scale_is_a_number_of_the_type(dtype):
    t = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    for values, (lo, hi) in ((store.VALUES4, store.BOUNDS4[dtype]), (store.VALUES8, store.BOUNDS8[dtype])):
        for e in (lo, lo + 1, 0, hi - 1, hi):
            v = values * 2.0 ** e
            if values is store.VALUES8:
                v = v[v <= store.MOST8[dtype]]
            assert np.array_equal(torch.from_numpy(v).to(t).double().numpy(), v)


def test_round_trip_of_representable_blocks_and_error_bounds():
    rng = np.random.default_rng(2)
    X = rng.standard_normal((5, 70)) * np.exp(rng.standard_normal((5, 1)) * 4)
    for pack, unpack, half in ((lambda x: store.pack4(x, None, "f32"), store.unpack4, 2.0 ** -2), (lambda x: store.pack8(x, "f32"), store.unpack8, 2.0 ** -4)):
        c, s = pack(X)
        Y = unpack(c, s, 70)
        c2, s2 = pack(Y)
        assert np.array_equal(unpack(c2, s2, 70), Y)
        least = np.repeat(2.0 ** (s.astype(float) - 127), 32, axis=1)[:, :70] * (0.25 if half == 0.25 else 2.0 ** -10)
        # half a step: half the distance of the codes, which is at most `half` of the value, or half the smallest code
        assert np.all(np.abs(X - Y) <= np.maximum(half * np.abs(X), least))


def test_masked_weights_and_bad_values():
    W = np.full((1, 40), 1.0)
    W[0, 3] = np.nan
    M = np.ones((1, 40), dtype=np.uint8)
    M[0, 3] = 0
    c, s = store.pack4(W, M, "f32")
    assert c[0, 3] == 0 and s[0, 0] != 255 and np.all(store.unpack4(c, s, 40)[0, 4:] == 1.0)
    c, s = store.pack4(W, None, "f32")
    assert s[0, 0] == 255 and s[0, 1] != 255 and np.isnan(store.unpack4(c, s, 40)[0, :32]).all()
    c, s = store.pack8(W, "bf16")
    u = store.unpack8(c, s, 40)
    assert np.isnan(u[0, 3]) and np.all(np.delete(u[0], 3) == 1.0)
    assert np.array_equal(store.packed_nibbles(store.nibbles(np.array([[0x21, 0xF3]], dtype=np.uint8))), [[0x21, 0xF3]])
