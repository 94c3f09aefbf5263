"""Pins of the serving-step oracle (fp64 NumPy): every function against another way of writing the definition down."""

import numpy as np
import pytest

import oracle
from oracle import serving_oracle as S


def test_norm_rope_keeps_length_and_reduces_to_its_parts():
    rng = np.random.default_rng(0)
    x = rng.standard_normal((2, 5, 64))
    y = S.norm_rope_rows(x, None, np.arange(5) * 1000, eps=0.0)
    assert np.allclose((y * y).mean(-1), 1.0)                               # a rotation keeps the row's mean square of 1
    w = rng.standard_normal(64)
    assert np.allclose(S.norm_rope_rows(x, w, np.zeros(5), 1e-3), x * w / np.sqrt((x**2).mean(-1, keepdims=True) + 1e-3))
    unit = np.ones((1, 1, 64))
    assert np.allclose(S.norm_rope_rows(unit, None, [7], eps=0.0), oracle.rope_rotate(unit, [7]))


@pytest.mark.parametrize("flags,ptype", [(0, "intermittent"), (oracle.FLAG_NO_REP_ZONE, "contiguous")])
def test_norm_rope_gradients_against_central_differences(flags, ptype):
    rng = np.random.default_rng(1)
    n, c, t, tail, D = 2, 2, 2, 1, 8
    rows = oracle.seq_len(n, c, t, tail, flags)
    q, k = rng.standard_normal((1, 2, rows, D)), rng.standard_normal((1, 1, rows, D))
    wq, wk = 1 + 0.3 * rng.standard_normal((2, D))
    gq, gk = rng.standard_normal(q.shape), rng.standard_normal(k.shape)
    args = dict(tail_read=tail, flags=flags, eps=0.05, position_type=ptype)

    def loss():
        a, b = S.qk_norm_rope(q, k, wq, wk, n, c, t, **args)
        return (a * gq).sum() + (b * gk).sum()

    got = S.qk_norm_rope_bwd(q, k, wq, wk, gq, gk, n, c, t, **args)
    for x, dx in zip((q, k, wq, wk), got):
        flat = x.reshape(-1)
        for i in rng.choice(flat.size, size=min(12, flat.size), replace=False):
            keep, h = flat[i], 1e-6
            flat[i] = keep + h
            hi = loss()
            flat[i] = keep - h
            lo = loss()
            flat[i] = keep
            assert abs((hi - lo) / (2 * h) - dx.reshape(-1)[i]) < 1e-7 * max(1, abs(dx).max())


def test_shared_decode_is_the_plain_decode_over_both_caches():
    rng = np.random.default_rng(2)
    B, H, D, P, lens = 3, 2, 16, 9, [0, 4, 7]
    kp, vp = rng.standard_normal((2, H, P, D))
    k_own = [rng.standard_normal((H, n + 1, D)) for n in lens]
    v_own = [rng.standard_normal((H, n + 1, D)) for n in lens]
    q = rng.standard_normal((B, H, D))
    o, lse, _ = S.decode_attn_shared(q, k_own, v_own, kp, vp)
    for b, n in enumerate(lens):
        kc = np.concatenate([kp, k_own[b], np.zeros((H, 2, D))], 1)[None]
        vc = np.concatenate([vp, v_own[b], np.zeros((H, 2, D))], 1)[None]
        want, wlse, _, _ = oracle.decode_attn(q[b][None, :, None], k_own[b][None, :, n:], v_own[b][None, :, n:], kc, vc, P + n)
        assert np.allclose(o[b], want[0, :, 0]) and np.allclose(lse[b], wlse.reshape(-1))
    # a group of query heads sees its kv head's keys: repeating the kv heads gives the same
    q2 = rng.standard_normal((B, 2 * H, D))
    o2, lse2, _ = S.decode_attn_shared(q2, k_own, v_own, kp, vp)
    o3, lse3, _ = S.decode_attn_shared(q2, [x.repeat(2, 0) for x in k_own], [x.repeat(2, 0) for x in v_own], kp.repeat(2, 0), vp.repeat(2, 0))
    assert np.allclose(o2, o3) and np.allclose(lse2, lse3)


def test_extend_by_hand():
    table = [[5, 9, -1], [-1, -1, -1], [3, -1, -1], [7, 8, 6]]
    # ps 4: 6 of 8 held entries used, 3 new; empty sequence, 5 new; idle; 11 of 12 used, 3 new (two beyond the table)
    got = S.paged_extend([6, 0, -1, 11], [3, 5, 2, 3], [2, 0, 1, 3], [60, 0, 0, 100], [20, 21], None, table, 4, 13)
    tab, rows, pages, held, slots, seq, pos, taken = got
    assert tab.tolist() == [[5, 9, 20], [21, -1, -1], [3, -1, -1], [7, 8, 6]]
    assert rows.tolist() == [0, 3, 8, 8, 11] and pages.tolist() == [0, 1, 3, 3, 3] and taken == 3
    assert held.tolist() == [3, 1, 1, 3]
    assert slots.tolist() == [38, 39, 80, 84, 85, 86, 87, -1, 27, -1, -1, -1, -1]
    assert seq.tolist() == [0, 0, 0, 1, 1, 1, 1, 1, 3, 3, 3, -1, -1]
    assert pos.tolist() == [60, 61, 62, 0, 1, 2, 3, 4, 100, 101, 102, 0, 0]
    # a compress step left the sequence shorter than its pages: none are drawn until they are full again
    assert S.paged_extend([2], [7], [3], None, [20], None, [[1, 2, 3]], 4, 7)[2].tolist() == [0, 0]
