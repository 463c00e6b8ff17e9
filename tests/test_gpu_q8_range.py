"""Attention over 8-bit pages where scales, weights and queries lie far apart: no row may cost another one its bits.

Tolerance.  Notation and first terms as at the head of test_gpu_q8; what is left out here is its last term, in the largest product of
weight and scale among all rows.  Weights enter the products as half-precision numbers (a second one, 2^11 times finer, in single
precision) after a power of two has brought the largest product of weight and scale of a column, among the rows of a tile of 32 whose scales lie
within 2^6 of one another, to 1 or more: a weight is off by half a step, 2^-11 of it (2^-21), or of small ones by 2^-25 (2^-36) of that
largest product.  Sums: each tensor-core product adds 16 rows to a sum and may cut it, 4 e; tiles, warps and pieces come on top, n / 16 + 64
additions in all.  So
|err| <= u |out| + (2 L + 2^-20 + 2^-11 [fp32: 2^-21] + 4 (n / 16 + 64) e) sum_r p_r |v_r| + 2^-25 [2^-36] sum_r max_r'(p_r' s_r') |code_r|,
r' in r's tile with a scale within 2^6 of r's; and half of the smallest step there is, where an output lies below the normal numbers of its
type: bf16 numbers under 2^-126 are 2^-133 apart, which is 2^-134, of single precision 2^-150 for each addition."""
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
                bound = bound + (2.0 ** -134 if dtype == "bf16" else (sums or m / 16 + 64) * 2.0 ** -150)
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


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("old,new", [(-126, 110), (-100, 60), (60, -100), (110, -126)])
def test_tiles_on_scales_at_both_ends(old, new, dtype):
    """Whole tiles of zero codes on one scale and of ordinary ones on the other, either first."""
    cfg = config(4, 2, 64, dtype=dtype)
    low = min(old, new)
    for rows in (range(352, 384), range(0, 320), range(160, 192)):
        c = Pages8(cfg, 32, 32, [384], seed=1, spread=0)
        c.scales[1].fill_(2.0 ** old)
        fill(c, rows, scale=2.0 ** new)
        fill(c, rows if new > low else [r for r in range(384) if r not in rows], codes=0)
        q = queries(1, 1, 4, 64, dtype)
        check_near(c, q, [0], run_decode(c, q, i32([0])), dtype)
        assert c.bits() == 0


@pytest.mark.parametrize("layout,hq,hkv,d", [("hnd", 8, 2, 128), ("nhd", 2, 2, 64), ("hnd", 5, 1, 80), ("hnd", 2, 2, 256)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len", [1, 4])
@pytest.mark.parametrize("at", [0, 176, 368])
def test_a_block_of_zeros_with_a_far_larger_scale(at, q_len, dtype, layout, hq, hkv, d):
    """Sixteen rows of zero codes, first, in the middle or last, on scales 2^4 to 2^128 above the others'."""
    cfg = config(hq, hkv, d, dtype=dtype)
    c = Pages8(cfg, 64 if at else 8, 16 if at else 8, [384], seed=at + d, layout=layout)
    q = queries(1, q_len, hq, d, dtype, seed=at)
    fill(c, range(at, at + 16), codes=0)
    for up in (4, 8, 12, 16, 20, 24, 40, 128):
        fill(c, range(at, at + 16), scale=2.0 ** (up - 8))
        check_near(c, q, [0], run_decode(c, q, i32([0])), dtype)
    assert c.bits() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("q_len", [1, 3])
def test_scales_that_fall_from_block_to_block(q_len, dtype):
    """Each block's scale 2^9 below that of the block before, all codes in use; weights that grow the other way, so that every block counts."""
    cfg = config(2, 1, 64, dtype=dtype, scale=1.0)
    c = Pages8(cfg, 16, 4, [44], seed=5)
    c.k.view(torch.uint8).zero_()
    c.ks.fill_(1.0)
    for b in range(11):
        fill(c, range(4 * b, 4 * b + 4), scale=2.0 ** (40 - 9 * b))
        for j in range(4):                                  # logits of about 9 ln 2 more each block
            row = torch.zeros(64, dtype=torch.uint8, device="cuda")
            row[0], row[1] = int(orc.encode(6.0 * b)), int(orc.encode(0.24 * b + 0.1 * j))
            fill(c, [4 * b + j], codes=row, which=0)
    q = torch.zeros(1, q_len, 2, 64, dtype=DT[dtype], device="cuda")
    q[..., :2] = 1.0
    check_near(c, q, [0], run_decode(c, q, i32([0])), dtype, reach_terms=2)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_outlier_whose_weight_has_vanished(dtype):
    """One row far larger than the others that almost nobody attends, its neighbours' codes zero on its scale."""
    cfg = config(4, 1, 64, dtype=dtype, scale=1.0)
    for logit, scale in ((-40.0, 2.0 ** 40), (-40.0, 2.0 ** 30), (-80.0, 2.0 ** 100), (-200.0, 2.0 ** 100), (-20.0, 2.0 ** 24)):
        c = Pages8(cfg, 32, 16, [300], seed=2)
        c.ks.fill_(2.0 ** -9)
        fill(c, range(160, 176), codes=0, scale=scale)
        fill(c, [165], codes=int(orc.encode(400.0)))
        row = torch.zeros(64, dtype=torch.uint8, device="cuda")
        row[0] = int(orc.encode(logit))
        fill(c, [165], codes=row, which=0)
        fill(c, range(160, 176), scale=1.0, which=0)
        q = queries(1, 1, 4, 64, dtype, seed=3)
        q[..., 0] = 1.0
        check_near(c, q, [0], run_decode(c, q, i32([0])), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), 3e30])
def test_a_draft_that_was_not_finite_is_taken_back(value, dtype):
    """A draft token with an infinity is appended, attended by its own query alone, and given up; the block keeps its scale."""
    cfg = config(4, 2, 64, dtype=dtype)
    c = Pages8(cfg, 64, 16, [200], seed=4, capacity=256)
    c.table[0, :4] = i32((c.table[0].tolist() + c.free)[:4])
    k, v = (torch.randn(3, 2, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(x)).to(DT[dtype]) for x in (1, 2))
    v[2, :, 5] = value
    q = queries(1, 3, 4, 64, dtype)
    B.snap_paged_q8_append(cfg, c.paged, i32([0]), i32([0, 3]), i32([200]), k, v, *c.cache, c.seq_len, status=c.status)
    out = run_decode(c, q, i32([0]))
    c.seq_len.fill_(202)                                    # the draft is taken back
    check_near(c, q[:, :2], [0], out[:, :2], dtype)
    check_near(c, q, [0], run_decode(c, q, i32([0])), dtype)
    B.snap_paged_q8_append(cfg, c.paged, i32([0]), i32([0, 2]), i32([202]), k[:2].contiguous(), v[:2].contiguous(), *c.cache, c.seq_len,
                           status=c.status)
    check_near(c, q, [0], run_decode(c, q, i32([0])), dtype)
    assert c.bits() == 0


def test_outputs_do_not_follow_the_power_of_other_tiles():
    """A row that has nearly all the weight and codes of zero, as an attention sink has, then rows on ever smaller weights."""
    cfg = config(2, 1, 64, scale=1.0)
    c = Pages8(cfg, 64, 16, [3000], seed=6, spread=0)
    c.k.view(torch.uint8).zero_()
    c.ks.fill_(1.0)
    c.v.view(torch.uint8).copy_(c.v.view(torch.uint8) & 0x7f)
    fill(c, [0], codes=0)
    row = torch.zeros(64, dtype=torch.uint8, device="cuda")
    row[0] = int(orc.encode(40.0))
    fill(c, [0], codes=row, which=0)
    q = torch.zeros(1, 1, 2, 64, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0
    check_near(c, q, [0], run_decode(c, q, i32([0])), "bf16", reach_terms=1)


@pytest.mark.parametrize("n,nats", [(16385, 13.0), (40000, 16.0), (61, 16.0), (700, 20.0)])
def test_single_precision_keeps_small_weights(n, nats):
    """A row of zero codes that has nearly all the weight, as an attention sink has: the output is made of weights of 2^-19 to 2^-29, and is
    as good as it is without that row.  (Each block has the fewest tiles a stretch can have, 5 or 6, or all of a short sequence: a warp
    adds 2 or 6 of them, two products each, four warps join, then 125 pieces or fewer, a warp taking an eighth of them: 40 additions at most.)"""
    cfg = config(2, 1, 64, dtype="f32", scale=1.0)
    c = Pages8(cfg, 64, 64, [n], seed=6, spread=0)
    c.k.view(torch.uint8).zero_()
    c.ks.fill_(1.0)
    c.v.view(torch.uint8).copy_(c.v.view(torch.uint8) & 0x7f)
    fill(c, [0], codes=0)
    row = torch.zeros(64, dtype=torch.uint8, device="cuda")
    row[0] = int(orc.encode(nats))
    fill(c, [0], codes=row, which=0)
    q = torch.zeros(1, 1, 2, 64, dtype=torch.float32, device="cuda")
    q[..., 0] = 1.0 + torch.arange(2, device="cuda") / 32
    check_near(c, q, [0], run_decode(c, q, i32([0])), "f32", reach_terms=1, sums=40)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("size,scale", [(2.0 ** 24, 2.0 ** 120), (2.0 ** 100, 2.0 ** 60), (2.0 ** 60, 2.0 ** 120)])
def test_large_queries_meet_zero_keys_on_large_scales(size, scale, dtype):
    """Keys of zero codes on the scale that a key taken back left: logits of zero, however large the query."""
    cfg = config(4, 1, 64, dtype=dtype)
    c = Pages8(cfg, 32, 16, [150], seed=2)
    c.ks.mul_(1.0 / size)
    fill(c, range(64, 80), codes=0, scale=scale, which=0)
    q = queries(1, 2, 4, 64, dtype) * size
    q[0, 0, 1] /= size                                      # (a column beside it whose logits are next to nothing)
    check_near(c, q, [0], run_decode(c, q, i32([0])), dtype)


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype,hq,hkv,d,dv,page,block", [("bf16", 8, 2, 128, 128, 64, 16), ("f32", 4, 2, 64, 64, 16, 16), ("bf16", 2, 2, 80, 48, 5, 5),
                                                        ("bf16", 2, 2, 256, 256, 16, 8), ("f32", 2, 1, 256, 80, 8, 8)])
@pytest.mark.parametrize("length,q_len", [(100, 4), (64, 2), (65, 3), (130, 45), (3, 5), (7, 70)])
def test_a_value_that_is_not_a_number_reaches_no_token_before_it(length, q_len, dtype, hq, hkv, d, dv, page, block, layout):
    """NaN among the last rows, as a draft may leave it: tokens before that row are as with any other value there, those from it on have a NaN
    in its columns alone, and a token that sees no row has zeros."""
    cfg = config(hq, hkv, d, dv, dtype=dtype, max_seqs=2)
    c = Pages8(cfg, page, block, [length, 40], seed=length, layout=layout)
    q = queries(2, q_len, hq, d, dtype)
    places = [(length - 1, 0, 3), (length - 1, hkv - 1, dv - 1), (max(length - q_len // 2, 0), 0, 3), (max(length - q_len + 1, 0), 0, 17)]
    for r, h, x in places:
        p, o = c.table[0, r // page].item(), r % page
        c.v.view(torch.uint8)[p, h, o, x] = 0x31
    clean = run_decode(c, q, i32([0, 1])).clone()
    assert torch.isfinite(clean.float()).all()
    for r, h, x in places:
        p, o = c.table[0, r // page].item(), r % page
        c.v.view(torch.uint8)[p, h, o, x] = 0xff if x == 17 else 0x7f
    out = run_decode(c, q, i32([0, 1]))
    nan = torch.zeros_like(out, dtype=torch.bool)
    for r, h, x in places:
        for u in range(q_len):
            if r < length - q_len + 1 + u:
                nan[0, u, h * (hq // hkv):(h + 1) * (hq // hkv), x] = True
    assert torch.equal(torch.isnan(out.float()), nan)
    assert torch.equal(out[~nan], clean[~nan])
    assert (out[0, :max(q_len - length, 0)] == 0).all() and c.bits() == 0


@pytest.mark.parametrize("layout,hq,hkv", [("hnd", 8, 2), ("nhd", 8, 2), ("hnd", 8, 1), ("hnd", 16, 1)])
def test_bf16_outputs_are_rounded_once(layout, hq, hkv):
    """Few rows of positive values and exact logits: an output is the exact one's bf16 neighbour, but where that lies next to a border.  What comes
    before the rounding is off by (2 L + 2^-20 + 2^-21 + 4 (n / 16 + 8) e) of it and 2^-24 of the largest product, by the terms of the tolerance above;
    a weight of 11 bits alone is off by 2^-12, eight times that."""
    n, d, g = [2, 3, 5, 8, 9, 31, 33, 40] * 8, 128, hq // hkv
    cfg = config(hq, hkv, d, max_seqs=len(n), scale=1.0)
    c = Pages8(cfg, 64, 64, n, seed=3, spread=0, layout=layout)
    c.v.view(torch.uint8).copy_(c.v.view(torch.uint8) & 0x7f)
    keys = c.k.view(torch.uint8)
    keys[..., 1:] = 0                                       # (one product to a logit, of size 3 at most)
    c.ks.fill_(2.0 ** -7)
    q = torch.zeros(len(n), 1, hq, d, dtype=torch.bfloat16, device="cuda")
    q[..., 0] = 1.0 + torch.arange(hq, device="cuda") / 16
    got, (hk, hv) = f64(run_decode(c, q, i32(list(range(len(n)))))), c.host()
    for i in range(len(n)):
        k, _ = hk.rows(c.table[i].tolist(), n[i])
        v, _ = hv.rows(c.table[i].tolist(), n[i])
        for h in range(hq):
            z = k[:, h // g, 0] * f64(q[i, 0, h, 0])
            p = np.exp(z - z.max())
            want = p @ v[:, h // g] / p.sum()
            off = (2 * 9 * E * np.abs(z).max() + 2.0 ** -20 + 2.0 ** -21 + 4 * (n[i] / 16 + 8) * E) * want + 2.0 ** -24 * (p / p.sum()).max() * v[:, h // g].sum(axis=0)
            half = 2.0 ** (np.floor(np.log2(want)) - 8)
            err = np.abs(got[i, 0, h] - want)
            assert (err <= half + off).all(), f"sequence {i}, head {h}: {((err - half) / off).max():.1f} times what may be left out"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nats", [3.0, 5.0, 40.0])
def test_large_values_over_many_rows(nats, dtype):
    """Values of 2^108 in 3000 rows whose weights grow after the first tile: their sum is of a size of 2^120, and nothing on the way passes 2^128."""
    cfg = config(2, 1, 64, dtype=dtype, scale=1.0)
    c = Pages8(cfg, 64, 64, [3000], seed=6, spread=0)
    c.vs.fill_(2.0 ** 102)
    c.k.view(torch.uint8).zero_()
    c.ks.fill_(1.0)
    row = torch.zeros(64, dtype=torch.uint8, device="cuda")
    row[0] = int(orc.encode(nats))
    for r in range(64, 3000, 5):
        fill(c, range(r, min(r + 4, 3000)), codes=row, which=0)
    q = torch.zeros(1, 1, 2, 64, dtype=DT[dtype], device="cuda")
    q[..., 0] = 1.0
    check_near(c, q, [0], run_decode(c, q, i32([0])), dtype, reach_terms=1)


@pytest.mark.parametrize("layout,hq,hkv,d,q_len", [("hnd", 8, 2, 128, 1), ("nhd", 2, 2, 64, 3), ("hnd", 16, 1, 128, 1), ("nhd", 2, 2, 256, 1)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("by", [4.0, 16.0, 64.0])
def test_weights_that_differ_from_tile_to_tile(by, dtype, layout, hq, hkv, d, q_len):
    """Logits so far apart that most tiles hold next to nothing of a column, each of another one."""
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=2)
    c = Pages8(cfg, 32, 16, [900, 61], seed=3, layout=layout)
    q = queries(2, q_len, hq, d, dtype, seed=1) * by
    check_near(c, q, [0, 1], run_decode(c, q, i32([0, 1])), dtype)
