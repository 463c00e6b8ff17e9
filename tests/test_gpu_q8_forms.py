"""Attention over 8-bit pages in the forms that the other tests leave out: sequences with pages missing in their middle compared row by row for
every size of page, and two KV heads side by side in a unit (pages stored rows first, at most eight columns for both) over all head sizes,
ways in and numbers of tokens."""
import numpy as np
import pytest
import torch

from paper_2511_03092_b200 import binding as B
from tests.test_gpu_q8 import DT, Pages8, check_decode, config, i32, run_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype,hq,hkv,d,page,block", [("bf16", 8, 2, 128, 64, 16), ("bf16", 4, 2, 64, 8, 8), ("f32", 3, 1, 80, 5, 1), ("f32", 8, 2, 128, 16, 16),
                                                     ("bf16", 32, 2, 128, 32, 32), ("bf16", 2, 2, 256, 48, 16), ("bf16", 2, 2, 80, 16, 4)])
@pytest.mark.parametrize("q_len", [1, 2])
def test_pages_missing_in_the_middle(q_len, dtype, hq, hkv, d, page, block, layout):
    lengths = [3 * page + 2, 300, 6 * page, 0, 20, 40]
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=6)
    c = Pages8(cfg, page, block, lengths, seed=8, layout=layout)
    full = c.table[2, 1].item()                             # a page all of whose rows are there
    c.table[0, 1] = -1
    c.table[1, 0] = 10 ** 6
    c.table[1, 150 // page] = c.k.shape[0]
    c.table[2, :] = -5                                      # nothing of this one is there
    c.table[4, :] = -1                                      # longer than its table, of whose pages one is there
    c.table[4, c.width // 2] = full
    c.seq_len.copy_(i32([lengths[0], lengths[1], lengths[2], -4, c.width * page + 9, 40]))
    g = torch.Generator(device="cuda").manual_seed(2)
    slots = [0, 1, 2, 3, 4, 5, -1, 6, -7, 5]
    q = torch.randn(len(slots), q_len, hq, d, device="cuda", generator=g).to(DT[dtype])
    out = run_decode(c, q, i32(slots))
    assert c.bits() == B.SNAP_DEV_BAD_SLOT | B.SNAP_DEV_BAD_PAGE
    check_decode(c, q, slots, out, dtype)
    for i in (2, 3, 6, 7, 8):
        assert (out[i] == 0).all()
    assert (out[[0, 1, 4, 5, 9]] != 0).any(dim=-1).all()    # (and of these something is attended)


FORMS = [("bf16", 8, 4, 256, 256, 32, 16, 1), ("bf16", 4, 2, 80, 80, 16, 8, 2), ("f32", 2, 2, 64, 64, 32, 32, 4), ("bf16", 2, 2, 192, 256, 16, 4, 3),
         ("bf16", 4, 4, 64, 64, 64, 16, 4), ("bf16", 8, 2, 128, 128, 64, 64, 1), ("f32", 8, 4, 128, 128, 8, 8, 2), ("f32", 2, 2, 256, 256, 16, 16, 2),
         ("f32", 4, 2, 80, 128, 24, 12, 1), ("f32", 2, 2, 208, 144, 8, 2, 3), ("bf16", 6, 2, 128, 64, 5, 5, 1), ("bf16", 2, 2, 256, 256, 3, 1, 4),
         ("f32", 4, 4, 48, 48, 7, 7, 3), ("bf16", 2, 2, 112, 112, 40, 10, 4), ("f32", 6, 2, 64, 32, 16, 16, 1)]


@pytest.mark.parametrize("dtype,hq,hkv,d,dv,page,block,q_len", FORMS)
@pytest.mark.parametrize("lengths", [[0, 1, 2, 3, 31, 32, 33, 255, 383, 384, 385, 700], [9000, 5, 4001]])
def test_two_heads_side_by_side(lengths, dtype, hq, hkv, d, dv, page, block, q_len):
    cfg = config(hq, hkv, d, dv, dtype, max_seqs=len(lengths))
    c = Pages8(cfg, page, block, lengths, seed=d + page, layout="nhd")
    q = (torch.randn(len(lengths), q_len, hq, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)) * 2).to(DT[dtype])
    slots = np.random.default_rng(1).permutation(len(lengths)).tolist()
    out = run_decode(c, q, i32(slots))
    assert c.bits() == 0
    check_decode(c, q, slots, out, dtype)
    assert torch.equal(out, run_decode(c, q, i32(slots)))


@pytest.mark.parametrize("dtype,hq,hkv,d,q_len", [("bf16", 16, 1, 128, 5), ("f32", 12, 2, 64, 7), ("bf16", 8, 2, 256, 9), ("bf16", 32, 1, 64, 33), ("f32", 4, 2, 256, 17)])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
def test_many_columns(layout, dtype, hq, hkv, d, q_len):
    """More columns than a unit holds: query heads of a group times tokens."""
    lengths = [q_len // 2, q_len, 100, 1500]
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=len(lengths))
    c = Pages8(cfg, 16, 8, lengths, seed=q_len, layout=layout)
    q = (torch.randn(len(lengths), q_len, hq, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(4)) * 2).to(DT[dtype])
    out = run_decode(c, q, i32([3, 0, 2, 1]))
    assert c.bits() == 0
    check_decode(c, q, [3, 0, 2, 1], out, dtype)
