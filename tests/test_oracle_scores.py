"""Pins for the oracle of changed scores and of the norm with axes: the formulas written out pair by pair, and properties
(no change without cap and slopes, distances only, a shift of all positions)."""
import math

import numpy as np
import pytest
import torch

import aspd_workloads as W
from oracle import TokenTable, attend, rotate
from oracle.scores import attend_scored, norm_rotate


def _table(seed, pos_mode="same_seq"):
    wl = W.random_small(seed, dtype="f32", num_q_heads=4, num_kv_heads=2, head_dim=64, batch=2, prefix_range=(0, 30),
                        branch_len_range=(1, 9))
    tt = TokenTable(wl.block_tables, 16, pos_mode=pos_mode)
    tt.append_serial(wl.prefix_len)
    tt.open_parallel(wl.num_branches)
    meta = tt.append_parallel(wl.branch_len)
    return wl, tt, meta, wl.draw_q(meta.NQ)


def test_without_cap_and_slopes_it_is_attention():
    wl, tt, meta, q = _table(1)
    got = attend_scored(tt, meta, q, wl.k_cache, wl.v_cache)
    out, lse = attend(tt, meta, q, wl.k_cache, wl.v_cache)
    assert np.abs(got["out"] - out).max() < 1e-13 and np.abs(got["lse"] - lse).max() < 1e-13
    assert np.array_equal(got["keys"], meta.kv_len)


@pytest.mark.parametrize("cap,bias,mode", [(2.0, False, "same_seq"), (0.0, True, "same_seq"), (1.5, True, "same_max"), (1.0, True, ("fix", 20))])
def test_pair_by_pair(cap, bias, mode):
    wl, tt, meta, q = _table(2, mode)
    slopes = [0.5, 0.25, -0.1, 1.0] if bias else None
    got = attend_scored(tt, meta, q, wl.k_cache, wl.v_cache, softcap=cap, slopes=slopes)
    for r in range(meta.NQ):
        s, i = int(meta.q_seq[r]), int(meta.logical_slot[r])
        for h in range(4):
            total, acc = 0.0, np.zeros(64)
            for j in range(len(tt.pos[s])):
                if not tt.visible_pair(s, i, j):
                    continue
                at = int(tt.physical_slot(s, j))
                x = float(q[r, h].double() @ wl.k_cache[at // 16, h // 2, at % 16].double()) / 8
                x = cap * math.tanh(x / cap) if cap else x
                x += slopes[h] * (tt.pos[s][j] - tt.pos[s][i]) if bias else 0
                total += math.exp(x)
                acc += math.exp(x) * wl.v_cache[at // 16, h // 2, at % 16].double().numpy()
            assert np.abs(got["out"][r, h] - acc / total).max() < 1e-12
            assert abs(got["lse"][r, h] - math.log(total)) < 1e-12


def test_norm_and_axes():
    rng = np.random.default_rng(3)
    x = rng.normal(size=(5, 3, 64))
    pos = rng.integers(0, 5000, size=(5, 32))
    assert np.allclose(norm_rotate(x, pos[:, 0], 1e4), rotate(x, pos[:, 0], 1e4), rtol=0, atol=1e-11)  # (angles: 5000 * 2^-52 each)
    w = rng.normal(size=64)
    y = norm_rotate(x, pos, 1e4, w, 1e-6, 1.0)
    for n in range(5):
        for h in range(3):
            z = [v / math.sqrt(sum(u * u for u in x[n, h]) / 64 + 1e-6) * (1 + w[i]) for i, v in enumerate(x[n, h])]
            for i in range(32):
                phi = int(pos[n, i]) * 1e4 ** (-2 * i / 64)
                assert abs(y[n, h, i] - (z[i] * math.cos(phi) - z[i + 32] * math.sin(phi))) < 1e-10   # (angles: 5000 * 2^-52 each, |z| < 10)
                assert abs(y[n, h, i + 32] - (z[i + 32] * math.cos(phi) + z[i] * math.sin(phi))) < 1e-10
    assert np.array_equal(norm_rotate(x, pos, 0), x)
