"""Pins of the paged-cache reference: the tile layout against the other helper's
reading of the header, appending against whole-block quantisation, growth of a
page's scale, and attention against torch in float64."""
import numpy as np
import pytest
import torch

import oracle as O
from gpu_helpers import fp8_tiles_to_rows
from oracle import kv_cache as R


def test_tile_places_are_the_headers_layout():
    tile = np.random.default_rng(0).integers(0, 256, 8192).astype(np.uint8)
    for op, place in ((0, R.K_PLACE), (1, R.V_PLACE)):
        rows, _ = fp8_tiles_to_rows(tile.reshape(1, 1, 1, 8192), 64, op)
        assert np.array_equal(tile[place], rows[0, 0])
        assert np.array_equal(np.sort(place.ravel()), np.arange(8192))


def empty(P, kv, B, mp):
    return (np.zeros((P, kv, 8192), np.uint8), np.ones((P, kv), np.float32),
            np.zeros((P, kv, 8192), np.uint8), np.ones((P, kv), np.float32),
            np.arange(B * mp, dtype=np.int32).reshape(B, mp))


def test_whole_pages_are_the_block_quantisation():
    rng = np.random.default_rng(1)
    x, y = (rng.standard_normal((150, 2, 128)).astype(np.float32) * 10 for _ in range(2))
    x, y = (O.widen_bf16(R.to_bf16_bits(t)).astype(np.float32) for t in (x, y))
    k8, sk, v8, sv, pages = empty(3, 2, 1, 3)
    k8, sk, v8, sv, _ = R.append(x, y, k8, sk, v8, sv, pages, [0, 150], [150])
    for h in range(2):
        for t, code, scale, place in ((x, k8, sk, R.K_PLACE), (y, v8, sv, R.V_PLACE)):
            want, s = O.quantize_fp8_blocks(t[:, h].astype(np.float64), 64)
            got = np.concatenate([code[j, h, place] for j in range(3)])[:150]
            assert np.array_equal(got, want)
            assert np.array_equal(scale[:, h].astype(np.float64), s)


def test_token_by_token_grows_the_scale_exactly():
    rng = np.random.default_rng(2)
    x = rng.integers(1, 9, (70, 1, 128)).astype(np.float32) * 2.0 ** np.arange(70)[:, None, None]
    k8, sk, v8, sv, pages = empty(2, 1, 1, 2)
    for n in range(70):
        k8, sk, v8, sv, _ = R.append(x[n:n + 1], x[n:n + 1], k8, sk, v8, sv, pages, [0, 1], [n + 1])
    # one call over all tokens: the same scales, and the same codes but for
    # values that were rounded more than once on their way below 2^-6
    a8, sa, b8, sb, _ = R.append(x, x, *empty(2, 1, 1, 2)[:4], pages, [0, 70], [70])
    assert np.array_equal(sk, sa) and np.array_equal(sv, sb)
    got, want = (R.e4m3_decode(t[0, 0, R.K_PLACE]) for t in (k8, a8))
    big = np.abs(want) >= 2.0 ** -6
    assert big.any() and np.array_equal(got[big], want[big])
    assert np.abs(got - want).max() <= 2.0 ** -9     # one subnormal step


def test_rotation_is_the_complex_product_and_keeps_the_rest():
    rng = np.random.default_rng(3)
    x = rng.standard_normal((3, 128)).astype(np.float32)
    ang = rng.uniform(0, 7, 32)
    cs = np.stack([np.cos(ang), np.sin(ang)], -1).astype(np.float32)
    y = R.rotate(x, cs)
    z = (x[:, 0:64:2] + 1j * x[:, 1:64:2].astype(np.float64)) * (cs[:, 0] + 1j * cs[:, 1].astype(np.float64))
    assert np.allclose(y[:, 0:64:2], z.real, atol=1e-6) and np.allclose(y[:, 1:64:2], z.imag, atol=1e-6)
    assert np.array_equal(y[:, 64:], x[:, 64:])


def test_exponent_rule():
    for amax, e in ((448.0, 0), (448.0001, 1), (224.0, -1), (0.0, -126), (2.0 ** -140, -126),
                    (2.0 ** 127, 119)):
        assert R.page_exponent(amax) == e


@pytest.mark.parametrize("chunk,window", [(0, 0), (1, 0), (1, 5), (4, 2), (100, 0)])
def test_attention_matches_torch(chunk, window):
    rng = np.random.default_rng(chunk * 10 + window)
    k8, sk, v8, sv, pages = empty(4, 2, 2, 2)
    x, y = (rng.standard_normal((100, 2, 128)).astype(np.float32) for _ in range(2))
    k8, sk, v8, sv, _ = R.append(x, y, k8, sk, v8, sv, pages, [0, 90, 100], [90, 10])
    q = rng.standard_normal((12, 4, 128))
    o, lse = R.attend(q, k8, sk, v8, sv, pages, [0, 9, 12], [90, 10], 0.1, chunk, window)
    for b, (lo, n, length) in enumerate(((0, 9, 90), (9, 3, 10))):
        pos, j = torch.arange(length - n, length)[:, None], torch.arange(length)[None]
        mask = torch.ones(n, length, dtype=torch.bool)
        if chunk:
            mask = j // chunk <= pos // chunk
            if window:
                mask &= j // chunk > pos // chunk - window
        for h in range(4):
            dec = lambda code, s, place: torch.tensor(np.concatenate(
                [R.e4m3_decode(code[p, h // 2, place]) * float(s[p, h // 2]) for p in pages[b]])[:length])
            s = 0.1 * torch.tensor(q[lo:lo + n, h]) @ dec(k8, sk, R.K_PLACE).T
            s = s.masked_fill(~mask, -torch.inf)
            want = torch.softmax(s, -1) @ dec(v8, sv, R.V_PLACE)
            assert np.allclose(o[lo:lo + n, h], want, rtol=1e-10, atol=1e-12)
            assert np.allclose(lse[lo:lo + n, h], torch.logsumexp(s, -1), rtol=1e-12)


def test_rows_without_keys_and_missing_pages():
    k8, sk, v8, sv, pages = empty(2, 1, 1, 2)
    q = np.ones((3, 1, 128))
    o, lse = R.attend(q, k8, sk, v8, sv, np.array([[-1, 7]]), [0, 2], [100], 0.1)
    assert np.array_equal(o[:2], np.zeros((2, 1, 128))) and np.all(np.isneginf(lse[:2]))
    assert np.isnan(o[2]).all()
    o, lse = R.attend(q, k8, sk, v8, sv, pages, [0, 3], [2], 0.1, 1)   # one row before position 0
    assert np.isneginf(lse[0, 0]) and np.isfinite(lse[1:]).all()
