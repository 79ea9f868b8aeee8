"""The served decoding step's oracle (oracle/serving.py) against library routines, hand-worked values and its own invariants."""
import math

import numpy as np
import pytest
import torch

from oracle import serving as sv


def test_codes_are_those_of_the_type():
    lib = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(sv.e4m3_values(), lib)
    # every bf16 value up to 448 rounds as the library's cast does
    x = torch.arange(-32768, 32768, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float()
    x = x[x.abs() <= 448]
    np.testing.assert_array_equal(sv.e4m3_code(x.numpy()), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())
    assert sv.e4m3_code(np.nan) & 127 == 127


@pytest.mark.parametrize("most, scale", [(0.0, 2.0 ** -100), (448.0, 1.0), (449.0, 2.0), (447.0, 1.0), (224.0, 0.5), (224.5, 1.0), (1e-40, 2.0 ** -100),
                                         (3e38, 2.0 ** 110)])
def test_scale_of_a_block(most, scale):
    assert sv.block_scale(most) == scale


def test_turned_is_a_rotation_that_only_the_difference_of_positions_matters_to():
    rng = np.random.default_rng(1)
    q, k = rng.standard_normal((2, 64))
    for m in (1, 77):
        a = sv.turned(q, 1000 + m, 1e4) @ sv.turned(k, 1000, 1e4)
        assert a == pytest.approx(sv.turned(q, m, 1e4) @ k, rel=1e-9)
    # the first pair by one radian per position
    np.testing.assert_allclose(sv.turned(np.eye(64)[0], 3, 1e4)[:2], (math.cos(3), math.sin(3)))


def _filled(rng, lens, new, page=16, hkv=2, dh=64, spare=2):
    held = [-(-(a + b) // page) for a, b in zip(lens, new)]
    n_pages = sum(held) + spare
    table = np.full((len(lens), max(held)), -1, np.int32)
    ids = iter(rng.permutation(n_pages))
    for s, h in enumerate(held):
        table[s, :h] = [next(ids) for _ in range(h)]
    pools = [sv.e4m3_code(np.clip(rng.standard_normal((n_pages, hkv, page, dh)) * 80, -448, 448)) for _ in range(2)]
    scales = [2.0 ** rng.integers(-8, -5, (n_pages, hkv)).astype(np.float64) for _ in range(2)]
    first = np.concatenate(([0], np.cumsum(new)))
    return table, first, pools, scales


def test_append_stores_the_nearest_codes_and_keeps_earlier_tokens():
    rng = np.random.default_rng(2)
    lens, new = [5, 16, 0], [14, 3, 1]
    table, first, (kp, vp), (ks, vs) = _filled(rng, lens, new)
    n = sum(new)
    k, v = rng.standard_normal((2, n, 2, 64))
    _, kp2, vp2, ks2, vs2, exact = sv.cache_append(table, lens, first, None, None, k, v, kp, vp, ks, vs)
    val = sv.e4m3_values()
    for j, (pg, sc) in enumerate(((kp2, ks2), (vp2, vs2))):
        assert len(exact[j]) == n * 2
        for (p, h, o), x in exact[j].items():
            got = val[pg[p, h, o]] * sc[p, h]
            assert np.all(np.abs(got - x) <= np.maximum(np.abs(x) * 2.0 ** -4, sc[p, h] * 2.0 ** -10))
    # sequence 0's five earlier tokens: the same values, rounded to the larger scale
    p = table[0, 0]
    for h in range(2):
        before, after = val[kp[p, h, :5]] * ks[p, h], val[kp2[p, h, :5]] * ks2[p, h]
        assert ks2[p, h] >= ks[p, h]
        assert np.all(np.abs(before - after) <= ks2[p, h] * 2.0 ** -10)
    # nothing else changed
    touched = {int(table[0, 0]), int(table[0, 1]), int(table[1, 1]), int(table[2, 0])}
    for p in set(range(len(kp))) - touched:
        np.testing.assert_array_equal(kp[p], kp2[p])
    np.testing.assert_array_equal(kp[table[2, 0], :, 1:], kp2[table[2, 0], :, 1:])


def test_attention_is_the_librarys_on_the_gathered_rows():
    rng = np.random.default_rng(3)
    lens, new = [40, 0], [3, 2]
    table, first, (kp, vp), (ks, vs) = _filled(rng, lens, new)
    q = rng.standard_normal((5, 4, 64))
    out, lse = sv.cache_attention(table, lens, first, q, kp, vp, ks, vs)
    val = sv.e4m3_values()
    for s in range(2):
        total = lens[s] + new[s]
        kk, vv = (torch.from_numpy(np.concatenate([(val[pg[p]] * sc[p][:, None, None]) for p in table[s] if p >= 0], 1)[:, :total]) for pg, sc in ((kp, ks), (vp, vs)))
        qq = torch.from_numpy(q[first[s]:first[s + 1]]).transpose(0, 1)
        mask = torch.arange(total)[None] <= lens[s] + torch.arange(new[s])[:, None]
        ref = torch.nn.functional.scaled_dot_product_attention(qq, kk.repeat_interleave(2, 0), vv.repeat_interleave(2, 0), attn_mask=mask)
        np.testing.assert_allclose(out[first[s]:first[s + 1]], ref.transpose(0, 1).numpy(), rtol=1e-12, atol=1e-12)
    # a prior result over some tokens joins to the result over all: cut the first sequence's pages in two
    a, al = sv.cache_attention(np.where(np.arange(3) < 1, table, -1), lens, first, q, kp, vp, ks, vs)
    b, bl = sv.cache_attention(np.where(np.arange(3) < 1, -1, table), lens, first, q, kp, vp, ks, vs, prior=a, prior_lse=al)
    np.testing.assert_allclose(b, out, rtol=1e-12, atol=1e-12)
    np.testing.assert_allclose(bl, lse, rtol=1e-12)
    # nothing there: zeros
    z, zl = sv.cache_attention(np.full_like(table, -1), lens, first, q, kp, vp, ks, vs)
    assert np.all(z == 0) and np.all(np.isneginf(zl))


def test_products_with_four_bits():
    rng = np.random.default_rng(4)
    q = rng.integers(0, 16, (6, 64)).astype(np.uint8)
    codes = q[:, 0::2] | (q[:, 1::2] << 4)
    scales, zeros, x, bias = rng.random((6, 2)), rng.integers(0, 16, (6, 2)).astype(np.uint8), rng.standard_normal((3, 64)), rng.standard_normal(6)
    y = sv.w4_linear(x, codes, scales, zeros, bias, group=32)
    for t in range(3):
        for n in range(6):
            ref = bias[n] + sum(x[t, k] * scales[n, k // 32] * (int(q[n, k]) - int(zeros[n, k // 32])) for k in range(64))
            assert y[t, n] == pytest.approx(ref, rel=1e-12)
    np.testing.assert_array_equal(sv.w4_linear(x, codes, scales, np.full((6, 2), 8), None, 32), sv.w4_linear(x, codes, scales, None, None, 32))


@pytest.mark.parametrize("zeros", [False, True])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_weights_as_they_are_laid_out(group, zeros):
    """quantize_w4: every weight is within half a step of its value, whatever the scale was rounded to (a bf16 scale is off by 2^-9, 15 steps of it at most)."""
    from paper_2505_19342_amd import binding as B
    rng = np.random.default_rng(group + zeros)
    w = (rng.standard_normal((5, 256)) * 0.02).astype(np.float32) + (0.01 if zeros else 0.0)
    w[2, :group] = 0.0
    w[3, :group] = np.abs(w[3, :group])
    codes, scales, z = B.quantize_w4(w, group, "bf16", zeros)
    assert codes.shape == (5, 128) and codes.dtype == np.uint8 and (z is not None) == zeros
    back = sv.w4_linear(np.eye(256), codes, scales, z, None, group).T
    step = np.repeat(scales.astype(np.float64), group, 1)
    # with zeros the zero point is rounded too: the two ends may each lose half a step more
    assert np.all(np.abs(back - w) <= step * ((1.0 if zeros else 0.5) + 16 * 2.0 ** -9))
    with pytest.raises(B.AstraError):
        B.quantize_w4(w, 96)
