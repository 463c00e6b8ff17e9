"""Attention over 8-bit pages where scales, weights and queries lie far apart: no row may cost another one its bits.

Tolerance.  Notation and first terms as at the head of test_gpu_q8; what is left out here is its last term, in the largest product of
weight and scale among all rows.  Weights enter the products as half-precision numbers (a second one, 2^11 times finer, in single
precision) after a power of two has brought the largest product of weight and scale of a column, among the rows of a tile of 32 whose scales lie
within 2^6 of one another, to 1 or more: a weight is off by half a step, 2^-11 of it (2^-21), or of small ones by 2^-25 (2^-36) of that
largest product.  Sums: each tensor-core product adds 16 rows to a sum and may cut it, 4 e; tiles, warps and pieces come on top, n / 16 + 64
additions in all.  So
|err| <= u |out| + (2 L + 2^-20 + 2^-11 [fp32: 2^-21] + 4 (n / 16 + 64) e) sum_r p_r |v_r| + 2^-25 [2^-36] sum_r max_r'(p_r' s_r') |code_r|,
r' in r's tile with a scale within 2^6 of r's."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as orc
from paper_2511_03092_b200 import binding as B
from tests.test_gpu_q8 import DT, E, HALF_STEP, Pages8, config, f64, i32, run_decode

pytestmark = pytest.mark.gpu


def check_near(c, q, slots, out, dtype, reach_terms=None, sums=None):
    """Every output against the definition, by the tolerance above.  reach_terms: how many products a logit is a sum of (d by default); sums: how
    many additions an output takes at most (n / 16 + 64 by default)."""
    hk, hv = c.host()
    table, lengths, cfg = c.table.cpu().numpy(), c.seq_len.tolist(), c.cfg
    g, terms = cfg.n_q_heads // cfg.n_kv_heads, (reach_terms or cfg.d_qk) + 8
    step, least = (2.0 ** -11, 2.0 ** -25) if dtype == "bf16" else (2.0 ** -21, 2.0 ** -36)
    for i, slot in enumerate(slots):
        n = lengths[slot]
        k, there = hk.rows(table[slot], n)
        v, _ = hv.rows(table[slot], n)
        s = np.array([[hv.scales[p, :, o // c.block] for p, o in [hv.place(table[slot], r)]][0] for r in there], dtype=np.float64)
        for u in range(q.shape[1]):
            m = int((there < n - q.shape[1] + 1 + u).sum())
            got = f64(out[i, u])
            if m == 0:
                assert (got == 0).all()
                continue
            tile = there[:m] // 32
            for h in range(cfg.n_q_heads):
                kh, vh, sh, x = k[:m, h // g], v[:m, h // g], s[:m, h // g], f64(q[i, u, h])
                z = (kh @ x) * cfg.softmax_scale
                p = np.exp(z - z.max())
                p /= p.sum()
                want, mass = p @ vh, p @ np.abs(vh)
                L = terms * E * (np.abs(kh) @ np.abs(x)).max() * cfg.softmax_scale + np.abs(kh).sum(axis=1).max() * 2.0 ** -38 * np.abs(x).max() * cfg.softmax_scale
                top = np.zeros(m)
                for t in np.unique(tile):
                    a = np.flatnonzero(tile == t)
                    near = np.abs(np.log2(sh[a])[:, None] - np.log2(sh[a])[None]) <= 6
                    top[a] = np.where(near, (p * sh)[a][None], 0).max(axis=1)
                bound = HALF_STEP[dtype] * np.abs(want) + (2 * L + 2.0 ** -20 + step + 4 * (sums or m / 16 + 64) * E) * mass
                bound = bound + least * (top[:, None] * np.abs(vh) / sh[:, None]).sum(axis=0)
                err = np.abs(got[h] - want)
                assert (err <= bound).all(), f"entry {i}, token {u}, head {h}: {err.max():.3e}, {(err / bound).max():.1f} times the bound"


def fill(c, rows, heads=slice(None), codes=None, scale=None, which=1, slot=0):
    """Codes and scales of some rows of a sequence."""
    pool, scales = c.pools[which].view(torch.uint8), c.scales[which]
    for r in rows:
        p, o = c.table[slot, r // c.page].item(), r % c.page
        if codes is not None:
            pool[p, heads, o] = codes
        if scale is not None:
            scales[p, heads, o // c.block] = scale


def queries(n, q_len, hq, d, dtype, seed=0):
    return torch.randn(n, q_len, hq, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)).to(DT[dtype])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("old,new", [(-8, 120), (-10, 119)])
def test_a_tile_of_far_larger_scales_leaves_what_was_summed_before(old, new, dtype):
    """The last 32 rows have zero codes on a scale more than 2^127 above that of the rows before."""
    cfg = config(4, 2, 64, dtype=dtype)
    c = Pages8(cfg, 32, 32, [384], seed=1, spread=0)
    c.scales[1].fill_(2.0 ** old)
    fill(c, range(352, 384), codes=0, scale=2.0 ** new)
    q = queries(1, 1, 4, 64, dtype)
    out = run_decode(c, q, i32([0]))
    check_near(c, q, [0], out, dtype)
    assert c.bits() == 0
