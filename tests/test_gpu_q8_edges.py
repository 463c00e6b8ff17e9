"""Calls on the page plan and the 8-bit cache that their documentation allows and everyday use seldom makes: rows of many pages planned by
two launches, more entries than a warp has lanes, entries that are left out between others, many KV heads, first calls inside a capture."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import q8_oracle as orc
from paper_2511_03092_b200 import binding as B
from tests.test_gpu_plan import Step, a_server
from tests.test_gpu_q8 import DT, Pages8, check_append, check_decode, config, f64, i32, run_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("apart", [True, False])
@pytest.mark.parametrize("width", [2500, 2501, 1024, 1025])
def test_plans_of_wide_rows(width, apart):
    """Rows longer than what a block writes at a time, with pages set aside in them; a list that ends between two blocks' parts."""
    rng = np.random.default_rng(width)
    for holes, most in ((True, 9001), (False, 30003)):
        slots, grow, table, length, stack, free = a_server(rng, 60, width, 4, 50, 3 * width, 2 * width, holes=holes, junk=True)
        s = Step(slots, grow, table, length, stack, free, 4, most, apart)
        s.call()
        s.check()


def test_two_graphs_share_the_scratch_of_a_plan():
    rng = np.random.default_rng(9)
    steps = []
    for n in (50, 400):
        slots, grow, table, length, stack, free = a_server(rng, n + 5, 300, 16, n, 2000, 300)
        steps.append(Step(slots, grow, table, length, stack, free, 16, 20000))
    small, large = steps
    small.ws = large.ws
    graphs = []
    for s in (small, large):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.call()
        graphs.append(graph)
    graphs[0].replay(), graphs[1].replay()
    small.check(), large.check()


@pytest.mark.parametrize("entries", [32, 33, 70])
def test_append_among_entries_that_are_left_out(entries):
    """Tokens before the first entry's and behind the last's; entries of no slot, of a slot listed before, out of range, of no tokens; runs
    that begin and end inside blocks."""
    rng = np.random.default_rng(entries)
    seqs = 50
    lengths = rng.integers(0, 60, seqs).tolist()
    cfg = config(4, 2, 64, max_seqs=seqs)
    slots = rng.permutation(seqs)[:entries].tolist() + rng.integers(0, seqs, max(entries - seqs, 0)).tolist()
    slots[3], slots[7], slots[11], slots[20] = -1, slots[2], seqs, -9
    n = rng.integers(0, 40, entries)
    n[5] = 0
    cu = (6 + np.concatenate([[0], np.cumsum(n)])).tolist()
    first = [lengths[s] if 0 <= s < seqs else 0 for s in slots]
    first[9] = -3
    served, seen = [], set()
    for i, s in enumerate(slots):
        if 0 <= s < seqs and s not in seen:
            seen.add(s)                                     # (the first entry of a slot counts, served or not)
            if first[i] >= 0:
                served.append(i)
    full = list(lengths)
    for i in served:
        full[slots[i]] += int(n[i])
    c = Pages8(cfg, 16, 8, full, seed=entries, capacity=112)
    c.seq_len.copy_(i32(lengths))
    g = torch.Generator(device="cuda").manual_seed(entries)
    t = cu[-1] + 9
    k, v = (torch.randn(t, 2, 64, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    k[:6], v[:6], k[cu[-1]:], v[cu[-1]:] = (float("nan"),) * 4
    before = c.host()
    B.snap_paged_q8_append(cfg, c.paged, i32(slots), i32(cu), i32(first), k, v, *c.cache, c.seq_len, status=c.status)
    check_append(c, before, slots, first, cu, k, v, served=served)
    want = list(lengths)
    for i in served:
        if n[i]:
            want[slots[i]] = full[slots[i]]
    assert c.seq_len.tolist() == want
    bits = c.bits()
    assert bits & B.SNAP_DEV_BAD_SLOT and bits & ~(B.SNAP_DEV_BAD_SLOT | B.SNAP_DEV_BAD_PAGE) == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_heads(dtype):
    """More scales of keys in a block of tokens than a CTA's shared memory holds at once; attention and gather over as many heads."""
    heads, lengths = 300, [21, 3]
    cfg = config(heads, heads, 16, dtype=dtype, max_seqs=2)
    c = Pages8(cfg, 8, 1, lengths, seed=1, spread=4)
    g = torch.Generator(device="cuda").manual_seed(3)
    k, v, q = (torch.randn(20, heads, 16, device="cuda", generator=g).to(DT[dtype]) for _ in range(3))
    before = c.host()
    args = (i32([0, 1]), i32([0, 18, 20]), i32([3, 1]))
    B.snap_paged_q8_append(cfg, c.paged, *args, k, v, *c.cache, c.seq_len, status=c.status)
    check_append(c, before, [0, 1], [3, 1], [0, 18, 20], k, v, dtype=dtype)
    x = q[:2].unsqueeze(1).contiguous()
    check_decode(c, x, [1, 0], run_decode(c, x, i32([1, 0])), dtype)
    kb, vb = torch.zeros_like(k), torch.zeros_like(v)
    B.snap_paged_q8_gather(cfg, c.paged, *args, *c.cache, kb, vb, status=c.status)
    for got, cache in zip((kb, vb), c.host()):
        for i, (a, b, row) in enumerate(((0, 18, 3), (18, 20, 1))):
            rows, _ = cache.rows(c.table[i].tolist(), b - a, row)
            np.testing.assert_array_equal(f64(got)[a:b], f64(torch.from_numpy(rows).to(DT[dtype])))
    assert c.bits() == 0


@pytest.mark.parametrize("lengths", [[383, 384, 385, 416] * 30, [384] * 40 + [20000], [1] * 500, [12 * 32 + 1]])
def test_units_around_the_longest_that_stays_whole(lengths):
    cfg = config(4, 2, 64, max_seqs=len(lengths))
    c = Pages8(cfg, 64, 16, lengths, seed=2)
    g = torch.Generator(device="cuda").manual_seed(4)
    q = torch.randn(len(lengths), 1, 4, 64, device="cuda", generator=g).to(torch.bfloat16)
    slots = np.random.default_rng(1).permutation(len(lengths)).tolist()
    check_decode(c, q, slots, run_decode(c, q, i32(slots)), "bf16")
    assert c.bits() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("logit,old,new", [(16.0, 46, -110), (-16.0, -126, 40), (16.0, -126, 100), (-16.0, 100, -126), (0.0, 112, 112)])
def test_weights_and_scales_at_the_ends_of_their_range(logit, old, new, dtype):
    """Rows with scales of 2^old, then one whose weight is 2^184 times theirs, or 2^-184, among rows with scales of 2^new: products of
    weights, scales and what brings them to half precision leave single precision at either end."""
    cfg = config(2, 1, 64, dtype=dtype)
    c = Pages8(cfg, 64, 16, [400], seed=1)
    codes = [x.view(torch.uint8) for x in c.pools]
    codes[0].zero_()
    codes[1].copy_(torch.from_numpy(orc.encode(50 + np.random.default_rng(0).random(codes[1].shape) * 50)).cuda())
    c.scales[0].fill_(1.0)
    c.scales[1].fill_(2.0 ** old)
    row, p = 130, c.table[0].tolist()
    codes[0][p[row // 64], 0, row % 64, 0] = int(orc.encode(logit))
    for r in range(128, 400):
        c.scales[1][p[r // 64], 0, r % 64 // 16] = 2.0 ** new
    if old < -100:                                          # (what the append makes of rows of zeros)
        for r in range(128):
            codes[1][p[r // 64], 0, r % 64] = 0
    q = torch.zeros(1, 1, 2, 64, dtype=DT[dtype], device="cuda")
    q[..., 0] = 64.0
    out = run_decode(c, q, i32([0]))
    assert torch.isfinite(out).all()
    check_decode(c, q, [0], out, dtype)


FIRST = """
import sys
sys.path.insert(0, %r)
import numpy as np, torch
from tests.test_gpu_plan import Step, a_server
from tests.test_gpu_q8 import *
rng = np.random.default_rng(0)
cfg = config(4, 2, 64, max_seqs=2)
c = Pages8(cfg, 16, 8, [700, 40], seed=1)
q = torch.ones(2, 1, 4, 64, device="cuda", dtype=torch.bfloat16)
k = torch.ones(3, 2, 64, device="cuda", dtype=torch.bfloat16)
kb, vb, out = torch.zeros_like(k), torch.zeros_like(k), torch.zeros_like(q)
lists, slots = (i32([1]), i32([0, 3]), i32([37])), i32([1, 0])
ws = torch.empty(B.snap_paged_q8_decode_workspace_bytes(cfg, c.paged, 2, 1), dtype=torch.uint8, device="cuda")
plans = [Step(*a_server(rng, n, 40, 16, n, 500, 60), 16, 4000) for n in (5, 1500)]
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    for s in plans:
        s.call()
    B.snap_paged_q8_append(cfg, c.paged, *lists, k, k, *c.cache, c.seq_len, status=c.status)
    run_decode(c, q, slots, ws=ws, out=out)
    B.snap_paged_q8_gather(cfg, c.paged, *lists, *c.cache, kb, vb, status=c.status)
graph.replay()
for s in plans:
    s.check()
check_decode(c, q, [1, 0], out, "bf16")
assert torch.equal(kb, k) and torch.equal(vb, k) and c.bits() == 0
print("first calls captured")
"""


def test_first_calls_inside_a_capture():
    here = os.path.dirname(os.path.abspath(__file__))
    run = subprocess.run([sys.executable, "-c", FIRST % os.path.dirname(here)], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "first calls captured" in run.stdout, run.stdout + run.stderr
