"""Calls at the edge of what the rotary and paged-cache entry points promise: what of a padded batch is read, what is
left alone, and layouts beside the usual two."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from paper_2511_03092_b200 import binding as B
from tests.test_gpu_paged import DT, Pages, check_decode, check_evict, check_rotation, config, f64, i32, run_decode, run_evict

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------------------
def raw_append(cfg, c, slots, rows, n, k, v, rope=None, freqs=None, positions=None, q=None, q_out=None, k_out=None, weights=None):
    """snap_paged_append by addresses: the buffers need not have n_tokens tokens."""
    at = lambda t: None if t is None else t.data_ptr()  # noqa: E731
    strides = lambda t: (0, 0) if t is None else t.stride()[:2]  # noqa: E731
    rc = B.lib().snap_paged_append(C.byref(cfg), C.byref(c.paged), at(slots), at(rows), n, C.byref(rope) if rope else None, at(freqs),
                                   at(positions), at(q), *strides(q), at(q_out), at(k), *strides(k), at(k_out), at(v), *strides(v), at(c.k),
                                   at(c.v), at(c.table), at(c.seq_len), at(weights), at(c.status), B._stream(None))
    assert rc == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rot", [64, 32, 0])
@pytest.mark.parametrize("by_rows", [True, False])
def test_append_reads_nothing_of_padding(by_rows, rot, dtype):
    """Slot -1 is padding: a batch padded at its end may come in buffers that stop at its last live token.  (The checked
    build raises a bit for a load that belongs to a token without a slot.)"""
    live, padded, hq, hkv, d = 5, 64, 4, 2, 64
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=live)
    c = Pages(cfg, dtype, 16, [48] * live, seed=3)
    start = [0, 7, 15, 16, 40]
    c.seq_len.copy_(i32(start))
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(live, h, d, device="cuda", generator=g).to(DT[dtype]) for h in (hq, hkv, hkv))
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    positions = [9, 100001, 3, 0, 77]
    slots = i32([3, 1, 0, 4, 2] + [-1] * (padded - live))
    order = slots[:live].tolist()
    rows = i32([start[s] for s in order]) if by_rows else None
    freqs = orc.rope_table(rot, 10000.0) if rot else None
    rope = B.make_rope(rot_dim=rot, rot_offset=d - rot) if rot else None
    before = f64(c.k)
    raw_append(cfg, c, slots, rows, padded, k, v, rope=rope, freqs=torch.from_numpy(freqs).cuda() if rot else None,
               positions=i32(positions) if rot else None, q=q, q_out=q_out, k_out=k_out)
    assert c.bits() == 0
    assert c.seq_len.tolist() == [x + 1 for x in start]
    if rot:
        for got, x in ((q_out, q), (k_out, k)):
            check_rotation(f64(got), f64(x), positions, freqs, rot, d - rot, False, 1.0, False, dtype)
    else:
        assert torch.equal(q_out, q) and torch.equal(k_out, k)
    table = c.table.cpu().numpy()
    for i, s in enumerate(order):
        before[table[s, start[s] // 16], :, start[s] % 16] = f64(k_out)[i]
    np.testing.assert_array_equal(f64(c.k), before)


def test_a_slot_listed_again_is_said_so_whatever_its_pages():
    """Next rows: a second listing is skipped as such (SNAP_DEV_BAD_SLOT) and for nothing else, wherever in the call it stands
    and whether or not the row after the first one's has a page."""
    cfg = config(4, 2, 64, max_seqs=4)
    c = Pages(cfg, "bf16", 16, [32, 32, 32, 32], seed=2)
    k = torch.randn(2000, 2, 64, device="cuda").to(torch.bfloat16)
    # the first listing takes the last row there is: the one after it lies past the table
    for others in (1, 1500):
        c.seq_len.copy_(i32([31, 4, 5, 6]))
        c.status.zero_()
        slots = [0] + [-1] * others + [0]
        B.snap_paged_append(cfg, c.paged, i32(slots), None, k[:len(slots)], k[:len(slots)], c.k, c.v, c.table, c.seq_len, status=c.status)
        assert c.bits() == B.SNAP_DEV_BAD_SLOT and c.seq_len.tolist() == [32, 4, 5, 6]
    # no page for the next row: the first listing is skipped for that, the second for being the second
    c.table[1, 1] = -1
    c.seq_len.copy_(i32([0, 20, 0, 0]))
    c.status.zero_()
    B.snap_paged_append(cfg, c.paged, i32([1, 1]), None, k[:2], k[:2], c.k, c.v, c.table, c.seq_len, status=c.status)
    assert c.bits() == B.SNAP_DEV_BAD_SLOT | B.SNAP_DEV_BAD_PAGE and c.seq_len.tolist() == [0, 20, 0, 0]


# ---------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,hq,hkv,d,page", [("bf16", 8, 2, 128, 16), ("bf16", 4, 2, 64, 8), ("bf16", 3, 1, 80, 5), ("f32", 4, 2, 128, 32),
                                                 ("f32", 12, 2, 64, 16), ("bf16", 40, 2, 64, 16)])
def test_weights_of_rows_that_are_left_out_stay(dtype, hq, hkv, d, page):
    """Rows on a page number out of range are not attended: their entries keep what they hold."""
    lengths = [3 * page + 2, 700, 6 * page, 0]
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=4)
    c = Pages(cfg, dtype, page, lengths, seed=8)
    c.table[0, 1] = -1
    c.table[1, 0] = 10 ** 6
    c.table[1, 300 // page] = c.k.shape[0]
    c.table[2, :] = -5                                      # nothing of this one is there
    g = torch.Generator(device="cuda").manual_seed(2)
    q = torch.randn(4, hq, d, device="cuda", generator=g).to(DT[dtype])
    before = torch.rand(c.weights().shape, device="cuda", generator=g)
    for with_in in (True, False):
        w, kept = before.clone(), before + 3.0
        if with_in:
            run_decode(c, q, [0, 1, 2, 3], weights_in=w, weights_out=w)
            other = kept.clone()
            run_decode(c, q, [0, 1, 2, 3], weights_in=before, weights_out=other)
        else:
            run_decode(c, q, [0, 1, 2, 3], weights_out=w)
            other = None
        for slot in range(4):
            _, _, there = c.rows(slot)
            out = np.ones(c.width * page, dtype=bool)
            out[there] = False
            np.testing.assert_array_equal(f64(w)[slot][:, out], f64(before)[slot][:, out])
            if other is not None:
                np.testing.assert_array_equal(f64(other)[slot][:, out], f64(kept)[slot][:, out])
        start = before if with_in else torch.zeros_like(before)
        inside = torch.zeros(w.shape, dtype=torch.bool, device="cuda")
        for slot in range(4):
            inside[slot, :, torch.from_numpy(c.rows(slot)[2]).cuda()] = True
        got = torch.where(inside, w, start)
        check_decode(c, run_decode(c, q, [0, 1, 2, 3]), q, [0, 1, 2, 3], dtype, weights=got, weights_before=start)
    assert c.bits() == B.SNAP_DEV_BAD_PAGE


@pytest.mark.parametrize("dtype,hq,d,page", [("bf16", 4, 128, 16), ("f32", 2, 128, 16), ("f32", 8, 64, 16)])
def test_a_row_of_logit_minus_infinity_is_attended(dtype, hq, d, page):
    """... with weight zero: its entry is written (the old weight, or zero), unlike one that is left out.  A sequence whose every
    logit is -infinity gets zeros, and its weights are written too."""
    cfg = config(hq, 1, d, dtype=dtype, max_seqs=2)
    c = Pages(cfg, dtype, page, [40, 7], seed=8)
    big = 3e38
    q = torch.full((2, hq, d), 2.0, device="cuda").to(DT[dtype])
    c.k[int(c.table[0, 1]), 0, 3] = -big                    # row 19: the sum of its products overflows
    c.k[int(c.table[1, 0]), 0] = -big
    before = torch.rand(c.weights().shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    w = before.clone()
    out = run_decode(c, q, [0, 1], weights_in=before, weights_out=w)
    np.testing.assert_array_equal(f64(w)[1], f64(before)[1])
    assert f64(w)[0, 0, 19] == f64(before)[0, 0, 19] and (f64(out)[1] == 0).all() and np.isfinite(f64(out)).all()
    run_decode(c, q, [0, 1], weights_out=w)
    want = f64(before)
    assert f64(w)[0, 0, 19] == 0 and (f64(w)[1, 0, :7] == 0).all()
    np.testing.assert_array_equal(f64(w)[1, 0, 7:], want[1, 0, 7:])
    assert c.bits() == 0


@pytest.mark.parametrize("dtype,hq,d", [("bf16", 4, 128), ("f32", 4, 128), ("f32", 16, 64)])
def test_weights_carry_a_nan_whatever_piece_it_is_in(dtype, hq, d):
    """One sequence cut into several hundred pieces, the first rows NaN, up to the whole first piece: the outputs and all weights of
    their KV head are NaN."""
    n, page = 50000, 16
    cfg = config(hq, 1, d, dtype=dtype, max_seqs=1)
    c = Pages(cfg, dtype, page, [n], seed=4)
    q = torch.randn(1, hq, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(DT[dtype])
    for p in range(10):
        for half in (slice(0, 8), slice(8, 16)):
            c.k[int(c.table[0, p]), :, half] = float("nan")
            w = c.weights()
            out = run_decode(c, q, [0], weights_out=w)
            assert np.isnan(f64(out)).all() and np.isnan(f64(w)[0, 0, :n]).all(), (p, half)
    assert c.bits() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,dv,page", [(4, 2, 64, 64, 16), (8, 1, 128, 128, 16), (24, 2, 128, 128, 16), (9, 1, 256, 256, 8), (4, 2, 128, 128, 16),
                                              (2, 1, 256, 256, 16), (5, 1, 80, 48, 5), (16, 2, 64, 64, 1)])
def test_a_sequence_of_one_row_returns_its_value_row(hq, hkv, d, dv, page, dtype):
    """Its softmax weight is 1, so nothing is to be rounded: the output holds the value row's bits, the largest finite numbers among them."""
    cfg = config(hq, hkv, d, dv, dtype, max_seqs=3)
    c = Pages(cfg, dtype, page, [1, 1, 1], seed=12)
    top = torch.finfo(DT[dtype]).max
    c.v[int(c.table[1, 0]), :, 0, :4] = torch.tensor([top, -top, top * 0.75, 1e-30], device="cuda").to(DT[dtype])
    q = torch.randn(3, hq, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(DT[dtype])
    out = run_decode(c, q, [2, 0, 1])
    for i, slot in enumerate((2, 0, 1)):
        want = c.v[int(c.table[slot, 0]), :, 0].repeat_interleave(hq // hkv, dim=0)
        assert torch.equal(out[i], want)
    assert c.bits() == 0


@pytest.mark.parametrize("dtype,hq,hkv,d", [("bf16", 4, 2, 128), ("f32", 4, 2, 128), ("f32", 16, 2, 64)])
@pytest.mark.parametrize("n", [1, 3, 128, 129, 700])
def test_batches_of_which_nothing_is_there(n, dtype, hq, hkv, d):
    """Only padding, only empty sequences, both; then one row in the last of them: zeros, but for that one's value row."""
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=n)
    c = Pages(cfg, dtype, 16, [0] * (n - 1) + [1], seed=n)
    q = torch.randn(n, hq, d, device="cuda").to(DT[dtype])
    none = torch.zeros(n, dtype=torch.int32, device="cuda")
    w = c.weights(2.5)
    for slots, seq_len in (([-1] * n, c.seq_len), (list(range(n)), none), ([i if i % 2 else -1 for i in range(n)], none)):
        for keep in (None, w):
            assert (f64(run_decode(c, q, slots, weights_in=keep, weights_out=keep, seq_len=seq_len)) == 0).all()
    assert (f64(w) == 2.5).all()
    out = run_decode(c, q, list(range(n)), weights_out=w)
    assert (f64(out)[:-1] == 0).all()
    assert torch.equal(out[-1], c.v[int(c.table[n - 1, 0]), :, 0].repeat_interleave(hq // hkv, dim=0))
    want = np.full(w.shape, 2.5)
    want[n - 1, :, 0] = hq // hkv
    # a head's only weight is 1, off by what exp2(x - (x + log2 1)) is: nothing but the logit's rounding, which cancels
    np.testing.assert_allclose(f64(w), want, rtol=2.0 ** -20)
    assert c.bits() == 0


def laid_out(c, how):
    """The same cache in other memory: keys and values as views of one pool, one tensor heads first and the other rows first,
    rows with room between them."""
    pages, hkv, page, dqk, dv = *c.k.shape, c.v.shape[3]
    empty = lambda *shape: torch.full(shape, float("nan"), dtype=c.k.dtype, device="cuda")  # noqa: E731
    if how == "one pool":
        pool = empty(pages, 2, hkv, page, max(dqk, dv))
        k, v = pool[:, 0, ..., :dqk], pool[:, 1, ..., :dv]
    elif how == "one pool, rows first":
        pool = empty(pages, page, 2, hkv, max(dqk, dv))
        k, v = pool[:, :, 0, :, :dqk].transpose(1, 2), pool[:, :, 1, :, :dv].transpose(1, 2)
    elif how == "keys heads first, values rows first":
        k, v = empty(pages, hkv, page, dqk), empty(pages, page, hkv, dv).transpose(1, 2)
    elif how == "keys rows first, values heads first":
        k, v = empty(pages, page, hkv, dqk).transpose(1, 2), empty(pages, hkv, page, dv)
    else:
        k, v = empty(pages, hkv, page + 1, dqk + 16)[:, :, :page, :dqk], empty(hkv, pages, page, dv + 48)[..., 16:16 + dv].transpose(0, 1)
    k.copy_(c.k)
    v.copy_(c.v)
    c.k, c.v = k, v
    c.paged = B.make_paged(k, v, c.table)


LAYOUTS = ["one pool", "one pool, rows first", "keys heads first, values rows first", "keys rows first, values heads first", "room between"]


@pytest.mark.parametrize("how", LAYOUTS)
@pytest.mark.parametrize("dtype,hq,hkv,d,dv,page", [("bf16", 8, 2, 128, 128, 16), ("f32", 4, 2, 128, 128, 16), ("bf16", 6, 3, 80, 48, 5),
                                                    ("f32", 12, 2, 64, 64, 24)])
def test_append_attention_and_eviction_in_other_layouts(dtype, hq, hkv, d, dv, page, how):
    sink, recent, topk = 2, 20, 33
    keep, lengths = sink + recent + topk, [300, 40, 55, 56, 1]
    n = len(lengths)
    cfg = config(hq, hkv, d, dv, dtype, max_seqs=2 * n, sink=sink, recent=recent, topk=topk)
    c = Pages(cfg, dtype, page, [x + 2 for x in lengths] + [min(x + 2, keep) for x in lengths], seed=2)
    laid_out(c, how)
    c.seq_len.copy_(i32(lengths + [0] * n))
    g = torch.Generator(device="cuda").manual_seed(4)
    # two tokens a sequence, rotated into their pages
    k, v = (torch.randn(2 * n, hkv, x, device="cuda", generator=g).to(DT[dtype]) for x in (d, dv))
    slots, rows = [i for i in range(n) for _ in range(2)], [x + j for x in lengths for j in range(2)]
    freqs, rope = orc.rope_table(d, 10000.0), B.make_rope(rot_dim=d)
    want_k, want_v, k_out = f64(c.k), f64(c.v), torch.empty_like(k)
    B.snap_paged_append(cfg, c.paged, i32(slots), i32(rows), k, v, c.k, c.v, c.table, c.seq_len, rope=rope, freqs=torch.from_numpy(freqs).cuda(),
                        k_out=k_out, status=c.status)
    check_rotation(f64(k_out), f64(k), rows, freqs, d, 0, False, 1.0, False, dtype)
    table = c.table.cpu().numpy()
    for i, (s, r) in enumerate(zip(slots, rows)):
        want_k[table[s, r // page], :, r % page], want_v[table[s, r // page], :, r % page] = f64(k_out)[i], f64(v)[i]
    np.testing.assert_array_equal(f64(c.k), want_k)
    np.testing.assert_array_equal(f64(c.v), want_v)
    c.lengths = [x + 2 for x in lengths] + [0] * n
    assert c.seq_len.tolist() == c.lengths
    # a step's attention, with the weights that the eviction goes by
    q = torch.randn(n, hq, d, device="cuda", generator=g).to(DT[dtype])
    w = torch.rand(c.weights().shape, device="cuda", generator=g)
    before, live = w.clone(), list(range(n))
    out = run_decode(c, q, live, weights_in=w, weights_out=w)
    check_decode(c, out, q, live, dtype, weights=w, weights_before=before)
    before, k0, v0 = w.clone(), f64(c.k), f64(c.v)
    kept = run_evict(c, live, [n + i for i in live], w, w)
    check_evict(c, live, [n + i for i in live], w, before, kept, k0, v0, set(live))
    assert c.bits() == 0


@pytest.mark.parametrize("dtype,hq,hkv,d", [("f32", 520, 130, 128), ("f32", 136, 34, 256), ("f32", 520, 520, 80), ("bf16", 520, 130, 128),
                                            ("bf16", 600, 40, 64)])
def test_cut_units_of_many_heads_are_joined(dtype, hq, hkv, d):
    """More than 512 query heads in a call: outputs are joined by the borders between the CTAs' stretches."""
    lengths = [1100, 3, 0, 700]
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=len(lengths))
    c = Pages(cfg, dtype, 16, lengths, seed=9)
    g = torch.Generator(device="cuda").manual_seed(6)
    q = torch.randn(4, hq, d, device="cuda", generator=g).to(DT[dtype])
    before = torch.rand(c.weights().shape, device="cuda", generator=g)
    w = before.clone()
    out = run_decode(c, q, [3, 2, 0, 1], weights_in=w, weights_out=w)
    check_decode(c, out, q, [3, 2, 0, 1], dtype, weights=w, weights_before=before)
    assert torch.equal(run_decode(c, q, [3, 2, 0, 1]), out) and c.bits() == 0


@pytest.mark.parametrize("dtype,hq,hkv,d,n,most", [("bf16", 32, 8, 128, 16, 9000), ("bf16", 12, 12, 64, 45, 333), ("f32", 8, 2, 128, 4, 4100),
                                                   ("f32", 16, 2, 64, 20, 3000), ("bf16", 8, 2, 128, 150, 500)])
def test_equal_inputs_give_equal_bits_with_other_calls_between(dtype, hq, hkv, d, n, most):
    """... nothing waited for between the calls: neither what scratch holds nor how the CTAs of one call follow those of the
    one before may show."""
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in rng.integers(0, most + 1, size=n)]
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=n)
    c = Pages(cfg, dtype, 16, lengths, seed=n)
    g = torch.Generator(device="cuda").manual_seed(n)
    qs = [torch.randn(n, hq, d, device="cuda", generator=g).to(DT[dtype]) for _ in range(2)]
    slots = [i32(rng.permutation(n).tolist()) for _ in range(2)]
    ws = torch.full((B.snap_paged_decode_workspace_bytes(cfg, c.paged, n, True),), 0xff, dtype=torch.uint8, device="cuda")
    got = []
    for rep in range(30):
        i = int(rep % 3 == 1)
        out, w = torch.full((n, hq, d), float("nan"), dtype=DT[dtype], device="cuda"), c.weights() if rep % 2 else None
        B.snap_paged_decode_attn(cfg, c.paged, qs[i], slots[i], n, c.k, c.v, c.table, c.seq_len, out, ws, weights_out=w, status=c.status)
        got.append((i, out, w))
    for i in (0, 1):
        outs, ws_ = [o for j, o, _ in got if j == i], [w for j, _, w in got if j == i and w is not None]
        assert all(torch.equal(o, outs[0]) for o in outs) and all(torch.equal(w, ws_[0]) for w in ws_)
    some = [int(x) for x in slots[0][:5]]
    check_decode(c, got[0][1][:5], qs[0], some, dtype)
    assert c.bits() == 0


def test_evictions_replayed_with_other_slots_and_weights():
    """A captured eviction, one after the other without a wait: slots, lengths, weights and tables that kernels just before it
    wrote are the ones it goes by (its copy starts beside its selection, and reads them on every SM)."""
    n, sink, recent, topk, lengths = 6, 2, 30, 60, [300, 90, 250, 500, 93, 420]
    keep = sink + recent + topk
    cfg = config(4, 2, 64, max_seqs=3 * n, sink=sink, recent=recent, topk=topk)
    c = Pages(cfg, "bf16", 16, lengths + [keep] * (2 * n), seed=3)
    g = torch.Generator(device="cuda").manual_seed(8)
    weights = [torch.rand(c.weights().shape, device="cuda", generator=g) for _ in range(2)]
    plans = [([3, 1, 5, 0, 2, 4], [n + i for i in range(n)]), ([0, 4, 2, 5, 3, 1], [2 * n + i for i in range(n)])]
    lens = [i32(lengths + [0] * (2 * n)), i32([x - 40 for x in lengths] + [0] * (2 * n))]
    src, dst, w = i32(plans[0][0]), i32(plans[0][1]), weights[0].clone()
    kept = torch.full((n, 2, keep), -9, dtype=torch.int32, device="cuda")
    ws = torch.empty(B.snap_paged_evict_workspace_bytes(cfg, c.paged, n), dtype=torch.uint8, device="cuda")
    call = lambda: B.snap_paged_evict(cfg, c.paged, src, dst, n, c.k, c.v, c.table, c.seq_len, w, None, ws, kept_rows=kept, status=c.status)  # noqa: E731
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    ids = [(i32(a), i32(b)) for a, b in plans]
    inputs = [(ids[r % 2][0], ids[r % 2][1], lens[r // 2 % 2], weights[r // 3 % 2]) for r in range(12)]
    want = []
    for a, b, ln, wt in inputs:                             # each of them alone, waited for
        for to, x in ((src, a), (dst, b), (c.seq_len, ln), (w, wt)):
            to.copy_(x)
        torch.cuda.synchronize()
        call()
        torch.cuda.synchronize()
        for i, s in enumerate(a.tolist()):
            for h in range(2):
                rows = orc.kept_rows(f64(wt)[s, h], int(ln[s]), sink, recent, topk)
                assert kept[i, h, :len(rows)].tolist() == rows.tolist()
        pages = c.table[b.long(), :-(-keep // 16)].long()
        want.append((kept.clone(), c.seq_len.clone(), c.k[pages], c.v[pages]))
    got = []
    for r in range(240):
        a, b, ln, wt = inputs[r % 12]
        c.k[c.table[b.long(), :-(-keep // 16)].long()] = 0.0
        for to, x in ((w, wt), (c.seq_len, ln), (dst, b), (src, a)):      # the last things before the call
            to.copy_(x)
        graph.replay() if r % 3 else call()
        pages = c.table[b.long(), :-(-keep // 16)].long()
        got.append((kept.clone(), c.seq_len.clone(), c.k[pages], c.v[pages]))
    for r, x in enumerate(got):
        for y, z in zip(x[:2], want[r % 12][:2]):
            assert torch.equal(y, z), r
        for i in range(n):                                  # (rows past a sequence's last are anything)
            rows, b = int(x[1][inputs[r % 12][1][i]]), -(-keep // 16)
            for y, z in zip(x[2:], want[r % 12][2:]):
                mine, its = (t[i].transpose(1, 2).flatten(0, 1)[:rows] for t in (y, z))
                assert torch.equal(mine, its), (r, i)
    assert c.bits() == 0


# ---------------------------------------------------------------------------------------------------------------
# offsets past 32 bits
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rot", [128, 64])
def test_rotation_past_32_bit_offsets(rot):
    """More than 2^31 elements of queries, apart and in place: the first, middle and last tokens."""
    t, h, d = 262150, 64, 128
    cfg = config(h, 1, d)
    rope, freqs = B.make_rope(rot_dim=rot, rot_offset=d - rot), torch.from_numpy(orc.rope_table(rot, 10000.0)).cuda()
    q = torch.empty(t, h, d, dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(1))
    assert q.numel() > 2 ** 31
    pos = torch.arange(t, dtype=torch.int32, device="cuda")
    parts = [slice(0, 7), slice(131069, 131080), slice(t - 9, t)]
    before = [q[s].clone() for s in parts]
    out = torch.empty_like(q)
    B.snap_rope(cfg, rope, freqs, pos, q=q, q_out=out)
    B.snap_rope(cfg, rope, freqs, pos, q=q, q_out=q)
    for s, x in zip(parts, before):
        assert torch.equal(q[s], out[s])
        check_rotation(f64(out[s]), f64(x), pos[s].cpu().numpy(), freqs.cpu().numpy(), rot, d - rot, False, 1.0, False, "bf16")


@pytest.mark.parametrize("dtype,d,pages", [("bf16", 128, 140000), ("f32", 128, 140000)])
def test_append_and_eviction_past_32_bit_offsets(dtype, d, pages):
    """Pools of more than 2^31 elements, tokens further apart than that in their own tensors: what a small cache gives."""
    page, sink, recent, topk, length, hkv = 16, 2, 12, 30, 90, 8
    cfg = config(hkv, hkv, d, dtype=dtype, max_seqs=2, sink=sink, recent=recent, topk=topk)
    c = Pages(cfg, dtype, page, [length + 40, 44], seed=1, spare=0)
    c.lengths = [length, 0]
    c.seq_len.copy_(i32(c.lengths))
    small_k, small_v, small_table = c.k.clone(), c.v.clone(), c.table.clone()
    used = c.k.shape[0]
    far = torch.tensor([(i * 11939) % pages if i % 2 else pages - 1 - i for i in range(used)], dtype=torch.int32, device="cuda")
    assert far.unique().numel() == used
    ks, vs = (torch.empty(pages, hkv, page, d, dtype=DT[dtype], device="cuda") for _ in range(2))
    assert ks.numel() > 2 ** 31
    for new, old in ((ks, small_k), (vs, small_v)):
        new[far.long()] = old
    table = torch.where(small_table >= 0, far[small_table.clamp(min=0).long()], small_table).to(torch.int32).contiguous()
    tokens = 40
    apart = (2 ** 31 // (tokens - 2)) // 64 * 64 + 64       # the last tokens' offsets pass 2^31 elements
    flat = torch.empty(apart * (tokens - 1) + hkv * d, dtype=DT[dtype], device="cuda")
    k = flat.as_strided((tokens, hkv, d), (apart, d, 1))
    k.copy_(torch.randn(tokens, hkv, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)))
    near = k.contiguous()
    slots, rows = i32([0] * tokens), i32(list(range(length, length + tokens)))
    rope, freqs = B.make_rope(rot_dim=d), torch.from_numpy(orc.rope_table(d, 10000.0)).cuda()
    lens = c.seq_len.clone()
    B.snap_paged_append(cfg, c.paged, slots, rows, near, near, c.k, c.v, c.table, c.seq_len, rope=rope, freqs=freqs, status=c.status)
    paged = B.make_paged(ks, vs, table)
    B.snap_paged_append(cfg, paged, slots, rows, k, k, ks, vs, table, lens, rope=rope, freqs=freqs, status=c.status)
    assert torch.equal(lens, c.seq_len) and lens.tolist() == [length + tokens, 0]
    same = lambda: all(torch.equal(x[far.long()].nan_to_num(7.0), y.nan_to_num(7.0)) for x, y in ((ks, c.k), (vs, c.v)))  # noqa: E731
    assert same()
    w = torch.rand(c.weights().shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    c.lengths = [length + tokens, 0]
    before, k0, v0 = w.clone(), f64(c.k), f64(c.v)
    kept = run_evict(c, [0], [1], w, w)
    check_evict(c, [0], [1], w, before, kept, k0, v0, {0})
    other, kept_far = before.clone(), torch.empty_like(kept)
    ws = torch.empty(B.snap_paged_evict_workspace_bytes(cfg, paged, 1), dtype=torch.uint8, device="cuda")
    B.snap_paged_evict(cfg, paged, i32([0]), i32([1]), 1, ks, vs, table, lens, other, other, ws, kept_rows=kept_far, status=c.status)
    assert torch.equal(kept_far, kept) and torch.equal(other, w) and same() and c.bits() == 0


# ---------------------------------------------------------------------------------------------------------------
# under the checked build
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("which", [["tests/test_gpu_paged_edges.py"], ["tests/test_gpu_paged.py", "-k", "decode"]], ids=["these", "attention"])
def test_paged_calls_under_the_checked_build(which):
    """The calls of this file, and attention: units, pieces, pages, logit rows and weights are tested against their arrays."""
    import os
    import subprocess
    import sys
    from paper_2511_03092_b200 import build as snap_build
    if "SNAP_LIBRARY" in os.environ:
        return                                              # (this is that run)
    lib = snap_build.build(debug_bounds=True)
    env = dict(os.environ, SNAP_LIBRARY=os.path.basename(lib))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-m", "pytest", *which, "-m", "gpu", "-q", "-x", "-p", "no:cacheprovider"],
                       cwd=root, env=env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout
