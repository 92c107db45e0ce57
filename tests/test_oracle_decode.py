"""Pins of oracle/decode.py that do not call back into it: hand-worked values, brute force, closed forms, a library's softmax."""

import numpy as np
import pytest
import scipy.special
import torch

from oracle import decode


def test_e2m1_hand_worked():
    # a block whose largest value is 6 has exponent 0: the grid itself, midpoints to the even code
    x = np.zeros((1, 32))
    x[0, :16] = [6, 5, 4.9, 5.1, 2.5, 3.5, 0.25, 0.75, 1.25, 1.75, -0.25, -0.26, -2.4, 0, -0.0, 0.2]
    codes, exps = decode.to_mxfp4(x)
    assert exps.tolist() == [[127]]
    back = decode.from_mxfp4(codes, exps)[0, :16]
    assert back.tolist() == [6, 4, 4, 6, 2, 4, 0, 1, 1, 2, 0, -0.5, -2, 0, 0, 0]
    assert np.signbit(back[10]) and np.signbit(back[14]) and not np.signbit(back[13])
    assert codes[0, 0] == 7 | 6 << 4            # 6 is code 7 (low half: the first element), 4 is code 6


@pytest.mark.parametrize("top,exponent", [(7.0, 0), (7.0001, 1), (3.5, -1), (3.50001, 0), (6.0, 0), (1.0, -2), (0.0, -127), (2.0 ** -130, -127)])
def test_block_exponent(top, exponent):
    x = np.zeros((1, 32))
    x[0, 9] = -top
    assert decode.block_exponents(x)[0, 0] == exponent


def test_no_element_is_off_by_more_than_half_a_step():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((200, 64)) * 2.0 ** rng.integers(-20, 20, (200, 1))
    codes, exps = decode.to_mxfp4(x)
    back = decode.from_mxfp4(codes, exps)
    scale = np.repeat(2.0 ** (exps.astype(float) - 127), 32, -1)
    mag = np.abs(x) / scale
    step = np.where(mag < 2, 0.5, np.where(mag < 4, 1.0, 2.0))
    assert (np.abs(back - x) <= step / 2 * scale * (1 + 1e-12)).all()
    # brute force over all 16 values
    grid = np.concatenate([decode.E2M1, -decode.E2M1])
    best = np.abs(x[..., None] - grid * scale[..., None]).min(-1)
    assert np.allclose(np.abs(back - x), best, rtol=1e-12, atol=0)


def test_blocks_that_are_not_finite():
    x = np.ones((2, 64))
    x[0, 3], x[1, 40] = np.nan, np.inf
    back = decode.from_mxfp4(*decode.to_mxfp4(x))
    assert np.isnan(back[0, :32]).all() and (back[0, 32:] == 1).all() and (back[1, :32] == 1).all() and np.isnan(back[1, 32:]).all()


def test_e4m3_against_torch():
    bits = np.arange(65536, dtype=np.uint16)
    t = torch.from_numpy(bits.view(np.int16)).view(torch.bfloat16)
    x = t.double().numpy()
    fine = np.abs(x) <= 448
    want = t.to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(decode.to_e4m3(x)[fine], want[fine])
    assert (decode.to_e4m3(x)[np.isfinite(x) & ~fine] & 127 == 126).all() and (decode.to_e4m3(x)[~np.isfinite(x)] & 127 == 127).all()
    codes = np.arange(256, dtype=np.uint8)
    assert np.array_equal(decode.from_e4m3(codes), torch.from_numpy(codes).view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


@pytest.mark.parametrize("T", [1, 3])
def test_attend_against_a_masked_softmax(T):
    rng = np.random.default_rng(T)
    B, Hkv, G, d = 2, 2, 3, 8
    lens, offs = [5, 0, 2, 9], [1, 8, 8, 12]
    k, v = rng.standard_normal((25, d)), rng.standard_normal((25, d))
    q = rng.standard_normal((B, Hkv * G, T, d))
    w0 = rng.random(25)
    out, lse, w, terms, spread = decode.attend(q, k, v, offs, lens, Hkv, T, w0)
    total = np.zeros(25)
    for s, n in enumerate(lens):
        b, h = divmod(s, Hkv)
        for g in range(G):
            x = q[b, h * G + g] @ k[offs[s]:offs[s] + n].T / np.sqrt(d)
            mask = np.arange(n)[None] > n - T + np.arange(T)[:, None]
            x = np.where(mask, -np.inf, x)
            for t in range(T):
                if n - T + t < 0:
                    assert (out[b, h * G + g, t] == 0).all() and lse[b, h * G + g, t] == -np.inf
                    continue
                p = scipy.special.softmax(x[t])
                total[offs[s]:offs[s] + n] += p
                np.testing.assert_allclose(out[b, h * G + g, t], p @ v[offs[s]:offs[s] + n], rtol=1e-12, atol=1e-14)
                np.testing.assert_allclose(lse[b, h * G + g, t], scipy.special.logsumexp(x[t]), rtol=1e-12)
    np.testing.assert_allclose(w, w0 + total, rtol=1e-12)
    # every query that sees a row gives out one unit of weight
    seen = sum(G * sum(n - T + t >= 0 for t in range(T)) for n in lens)
    assert abs((w - w0).sum() - seen) < 1e-10


def test_attend_closed_forms():
    # equal keys: the mean of the values; one key far above the others: its value
    k, v = np.zeros((4, 8)), np.arange(32.0).reshape(4, 8)
    q = np.ones((1, 1, 1, 8))
    out, lse, w, _, _ = decode.attend(q, k, v, [0], [4], 1, 1)
    assert np.allclose(out[0, 0, 0], v.mean(0)) and np.isclose(lse[0, 0, 0], np.log(4)) and np.allclose(w, 0.25)
    k[2] = 100.0
    out, lse, w, _, _ = decode.attend(q, k, v, [0], [4], 1, 1)
    assert np.allclose(out[0, 0, 0], v[2]) and np.isclose(lse[0, 0, 0], 800 / np.sqrt(8)) and np.allclose(w, [0, 0, 1, 0])


def test_evict_hand_worked():
    w = np.array([3.0, 1.0, 3.0, 2.0, 0.5, 9.0, 9.0])
    assert decode.evict_segment(w, 2, 4).tolist() == [0, 2, 5, 6]          # two of the first five, then the last two
    assert decode.evict_segment(w, 2, 3).tolist() == [0, 5, 6]             # equal weights: the lower row
    assert decode.evict_segment(w, 0, 2).tolist() == [5, 6]
    assert decode.evict_segment(w, 3, 1).tolist() == [4, 5, 6]             # a capacity below the window
    assert decode.evict_segment(w, 2, 7).tolist() == list(range(7))
    assert decode.evict_segment(np.array([1.0, np.nan, np.inf, 5.0, 0.0]), 1, 3).tolist() == [1, 2, 4]
    assert decode.evict_segment(np.array([0.0, -0.0, 0.0]), 0, 2).tolist() == [0, 1]
