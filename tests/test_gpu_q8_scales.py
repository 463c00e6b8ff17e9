"""Rows in and out of 8-bit pages whose scales are no powers of two, as another program's may be: each number is rounded once.  The expected
codes and numbers are exact, so nothing is allowed for."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as orc
from paper_2511_03092_b200 import binding as B
from tests.test_gpu_q8 import CODE, DT, Pages8, check_append, config, f64, i32

pytestmark = pytest.mark.gpu

SCALES = [0.7, 6.5, 3.0, 1 / 3, 1.0 + 2.0 ** -23, 2.0 - 2.0 ** -23, 1e-20, 0.9e20, 5e36, 2.0 ** 127 * 1.3]
BORDERS = np.array([(a + b) / 2 for a, b in zip(orc.VALUES[:126], orc.VALUES[1:127])])     # between neighbouring codes: ties


def half_way(values, dtype):
    """The numbers of a type at, just below and just above the given ones."""
    t = torch.from_numpy(values).to(DT[dtype])
    bits = t.view(torch.int16 if dtype == "bf16" else torch.int32)
    return torch.cat([(bits + x).view(DT[dtype]) for x in (-1, 0, 1)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rotated", [False, True])
@pytest.mark.parametrize("kept", [True, False])
def test_appends_to_a_block_whose_scale_is_no_power_of_two(kept, dtype, rotated):
    """Numbers at and around the borders between codes, divided by the scale that the block keeps, rounded once; or numbers for which some of
    the blocks move to the next power of two."""
    heads, d, n = len(SCALES), 128, 11
    cfg = config(heads, heads, d, dtype=dtype)
    c = Pages8(cfg, 16, 16, [5], seed=1, capacity=32)
    scales = torch.tensor(SCALES, dtype=torch.float32)
    for s in c.scales:
        s[c.table[0, 0].item()] = scales.cuda()[:, None]
    k = torch.zeros(n, heads, d, dtype=DT[dtype])
    for h, s in enumerate(scales.double().numpy()):
        x = half_way(np.minimum(BORDERS * s, 3e38 / 1.01), dtype)
        x = torch.cat([x, -x])
        x = x[x.double().abs() <= (448 * 2.0 ** np.floor(np.log2(s)) if kept else 440 * s)]     # (kept: what needs no larger power of two)
        k[:, h] = x[torch.from_numpy(np.random.default_rng(h).integers(0, len(x), n * d))].view(n, d)
        if rotated:                                         # (the scale has to stay what it is)
            k[:, h] /= 2
    k = k.cuda()
    before = c.host()
    rope, freqs = (B.make_rope(rot_dim=32, rot_offset=16), 1 / 10000.0 ** (np.arange(16) / 16)) if rotated else (None, None)
    B.snap_paged_q8_append(cfg, c.paged, i32([0]), i32([0, n]), i32([5]), k, -k, *c.cache, c.seq_len, rope=rope,
                           freqs=torch.from_numpy(freqs).cuda() if rotated else None, status=c.status)
    if rotated and kept:                                    # what turns by its distance, the rest by its codes
        p = c.table[0, 0].item()
        got = c.k.view(torch.uint8)[p, :, 5:].cpu().numpy()
        want = orc.encode(f64(k).transpose(1, 0, 2) / scales.double().numpy()[:, None, None])
        np.testing.assert_array_equal(got[..., :16], want[..., :16])
        np.testing.assert_array_equal(got[..., 48:], want[..., 48:])
    check_append(c, before, [0], [5], [0, n], k, -k, rope, freqs, dtype=dtype)
    for s in c.scales:
        assert torch.equal(s[c.table[0, 0].item(), :, 0].cpu(), scales) == kept or (rotated and not kept)
    assert c.bits() == 0


def test_rows_that_move_from_a_scale_that_is_no_power_of_two():
    """Scales at and around those that bring a code to a border between codes of the larger scale."""
    rng = np.random.default_rng(0)
    heads, d = 300, 64
    code = rng.integers(8, 120, heads)
    ratio = rng.choice(BORDERS[:100], heads) / orc.VALUES[code]
    ratio = ratio / 2.0 ** np.ceil(np.log2(ratio))          # (of old and new scale: less than 1)
    old = torch.from_numpy(ratio.astype(np.float32))
    old = (old.view(torch.int32) + torch.from_numpy(rng.integers(-1, 2, heads).astype(np.int32))).view(torch.float32)
    cfg = config(heads, heads, d, dtype="f32")
    c = Pages8(cfg, 16, 16, [9], seed=1, capacity=16)
    p = c.table[0, 0].item()
    held = rng.integers(0, 127, (heads, 9, d)).astype(np.uint8) | (rng.integers(0, 2, (heads, 9, d)) << 7).astype(np.uint8)
    held[:, :, 0] = code[:, None]
    for pool, scale in zip(c.pools, c.scales):
        pool.view(torch.uint8)[p, :, :9] = torch.from_numpy(held).cuda()
        scale[p, :, 0] = old.cuda()
    x = torch.full((1, heads, d), 448.0, device="cuda")     # (new scale: 1)
    before = c.host()
    B.snap_paged_q8_append(cfg, c.paged, i32([0]), i32([0, 1]), i32([9]), x, x, *c.cache, c.seq_len, status=c.status)
    check_append(c, before, [0], [9], [0, 1], x, x)
    assert torch.equal(c.scales[0][p, :, 0], old.clamp(min=1).cuda()) and c.bits() == 0


def bf16_of(x):
    """Numbers in double precision as the nearest bf16 ones, ties to even, in one rounding (normal numbers)."""
    m, e = np.frexp(x)
    return np.ldexp(np.rint(m * 256), e - 8)


def test_gather_rounds_once():
    """Scales that bring a code next to the border between two bf16 numbers: product and border agree in 24 bits, not in all."""
    rng = np.random.default_rng(0)
    heads, d = 512, 16
    code = rng.choice([x for x in range(8, 127) if x % 8 not in (0, 4)], heads)      # (an odd factor besides powers of two)
    border = (2 * rng.integers(128, 256, heads) + 1) / 512.0
    scale = (border / orc.VALUES[code]).astype(np.float32)
    cfg = config(heads, heads, d)
    c = Pages8(cfg, 16, 16, [3], seed=1)
    p = c.table[0, 0].item()
    c.k.view(torch.uint8)[p, :, :3] = torch.from_numpy(code.astype(np.uint8)).cuda()[:, None, None]
    c.v.view(torch.uint8)[p, :, :3] = torch.from_numpy(code.astype(np.uint8) | 0x80).cuda()[:, None, None]
    for s in c.scales:
        s[p, :, 0] = torch.from_numpy(scale).cuda()
    k, v = (torch.zeros(3, heads, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.snap_paged_q8_gather(cfg, c.paged, i32([0]), i32([0, 3]), i32([0]), *c.cache, k, v, status=c.status)
    want = bf16_of(orc.VALUES[code] * scale.astype(np.float64))[None, :, None]
    twice = f64(torch.from_numpy((orc.VALUES[code] * scale.astype(np.float64)).astype(np.float32)).to(torch.bfloat16))[None, :, None]
    assert (want != twice).any()                            # (rounding to 24 bits first is not the same)
    np.testing.assert_array_equal(f64(k), np.broadcast_to(want, k.shape))
    np.testing.assert_array_equal(f64(v), np.broadcast_to(-want, k.shape))
    assert c.bits() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("positions", [None, 9000])
def test_keys_rotated_in_place_onto_an_uneven_scale(positions, interleaved, dtype):
    """More rows than are rotated at a time, the last of them in the next block; the rotated keys are written over the keys."""
    heads, d, n, first = 6, 64, 60, 7
    cfg = config(2 * heads, heads, d, dtype=dtype, max_seqs=2)
    c = Pages8(cfg, 48, 48, [3, first], seed=1, capacity=96)
    c.table[1, 1] = c.free[0]
    p = c.table[1, 0].item()
    scales = torch.tensor(SCALES[:heads], dtype=torch.float32)
    for s in c.scales:
        s[p] = scales.cuda()[:, None]
    g = torch.Generator(device="cuda").manual_seed(2)
    k, v, q = (torch.randn(n, h, d, device="cuda", generator=g).clamp(-3, 3) for h in (heads, heads, 2 * heads))
    size = torch.exp2(torch.floor(torch.log2(scales))).cuda()[None, :, None] * 64
    k, v, q = (k * size).to(DT[dtype]), (v * size).to(DT[dtype]), q.to(DT[dtype])
    x, before = k.clone(), c.host()
    freqs = 1 / 10000.0 ** (np.arange(32) / 32)
    rope = B.make_rope(rot_dim=64, interleaved=interleaved)
    pos = None if positions is None else [positions + 2 * i for i in range(n)]
    B.snap_paged_q8_append(cfg, c.paged, i32([1]), i32([0, n]), i32([first]), k, v, *c.cache, c.seq_len, rope=rope, freqs=torch.from_numpy(freqs).cuda(),
                           positions=None if pos is None else i32(pos), q=q, q_out=q, k_out=k, status=c.status)
    check_append(c, before, [1], [first], [0, n], x, v, rope, freqs, pos, k, dtype=dtype)
    for s in c.scales:
        assert torch.equal(s[p, :, 0].cpu(), scales)
    assert c.bits() == 0 and c.seq_len.tolist() == [3, first + n]
