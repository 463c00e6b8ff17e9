"""Rotary positions, the paged cache, its attention and eviction on the GPU against their double-precision definitions.

Tolerances.  u is half a step of the output type (2^-8 bf16, 2^-24 fp32), e = 2^-24.
Rotation: each output is two products and a sum in single precision of a cosine and sine that are themselves off by a
few e (2 ulp of the function, the angle's rounding put back): |err| <= u |y| + 8 e m (|a| + |b|).
Attention: a logit is a sum of d products, off by at most (d + 3) e R (1.4427 for the change of base included), R the
largest scale sum_c |q_c k_c|; a probability then by a factor 1 +- 2 (d + 3) e R to first order (numerator and
denominator), the exponential's own 2^-22 and, bf16, the 2^-16 that its two-number form leaves; sums over n rows add
n e.  So |err| <= u |out| + (2 (d + 3) e R + 2^-20 + 2^-16 [bf16] + 2 n e) sum_r p_r |v_r|, and for a head's weight p the
same factor without the bf16 term."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
from paper_2511_03092_b200 import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
E = 2.0 ** -24


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def i32(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def config(hq, hkv, d, dv=None, dtype="bf16", max_seqs=1, sink=2, recent=8, topk=16):
    return B.make_config(n_q_heads=hq, n_kv_heads=hkv, d_qk=d, d_v=dv or d, dtype=DT[dtype], l_sink=sink, l_recent=recent, topk=topk,
                         l_obs=1, pool_kernel=1, softmax_scale=d ** -0.5, max_seqs=max_seqs)


class Pages:
    """A paged cache whose unused memory is NaN: pools in either layout, a table of shuffled pages."""

    def __init__(self, cfg, dtype, page, lengths, seed=0, layout="hnd", capacity=None, spare=2):
        self.cfg, self.page, rng = cfg, page, np.random.default_rng(seed)
        assert len(lengths) == cfg.max_seqs
        self.width = -(-max(max(lengths), capacity or 1) // page)
        need = [-(-n // page) for n in lengths]
        order = rng.permutation(sum(need) + spare)
        table = np.full((len(lengths), self.width), -1, dtype=np.int32)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        self.free = [int(x) for x in order[at:]]
        self.table = torch.from_numpy(table).cuda()
        self.seq_len = i32(lengths)
        self.lengths = list(lengths)
        g = torch.Generator(device="cuda").manual_seed(seed)
        pools = []
        for d in (cfg.d_qk, cfg.d_v):
            shape = (len(order), cfg.n_kv_heads, page, d) if layout == "hnd" else (len(order), page, cfg.n_kv_heads, d)
            pool = torch.full(shape, float("nan"), dtype=DT[dtype], device="cuda")
            view = pool if layout == "hnd" else pool.transpose(1, 2)
            for i, n in enumerate(lengths):
                for p in range(need[i]):
                    rows = min(page, n - p * page)
                    view[int(table[i, p]), :, :rows] = torch.randn(cfg.n_kv_heads, rows, d, device="cuda", generator=g).to(DT[dtype])
            pools.append(view)
        self.k, self.v = pools
        self.paged = B.make_paged(self.k, self.v, self.table)
        self.status = i32([0])

    def rows(self, slot, length=None):
        n, row = self.lengths[slot] if length is None else length, self.table[slot].cpu().numpy()
        k, there = orc.cache_rows(f64(self.k), row, n)
        return k, orc.cache_rows(f64(self.v), row, n)[0], there

    def weights(self, fill=0.0):
        return torch.full((self.cfg.max_seqs, self.cfg.n_kv_heads, self.width * self.page), fill, device="cuda")

    def bits(self):
        torch.cuda.synchronize()
        return int(self.status.item())


# ---------------------------------------------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------------------------------------------
def check_rotation(got, x, positions, freqs, rot, offset, interleaved, magnitude, inverse, dtype):
    want = orc.rotate(x, positions, freqs, rot, offset, interleaved, magnitude, inverse)
    i = np.arange(rot // 2)
    a, b = (offset + 2 * i, offset + 2 * i + 1) if interleaved else (offset + i, offset + rot // 2 + i)
    reach = np.zeros_like(want)
    reach[..., a] = reach[..., b] = magnitude * (np.abs(x[..., a]) + np.abs(x[..., b]))
    err = np.abs(got - want)
    bound = HALF_STEP[dtype] * np.abs(want) + 8 * E * reach
    bound[reach == 0] = 0                                   # dims that are not rotated: copied
    assert (err <= bound).all(), f"{(err - bound).max():.3e} over the bound"


ROTATIONS = [(8, 2, 128, 128, 0), (5, 5, 64, 32, 32), (4, 1, 80, 80, 0), (4, 2, 80, 40, 0), (3, 1, 48, 6, 5), (2, 2, 16, 2, 1),
             (16, 1, 576, 64, 512), (2, 1, 1024, 1024, 0), (6, 3, 96, 12, 2)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("hq,hkv,d,rot,offset", ROTATIONS)
def test_rope_matches_its_definition(hq, hkv, d, rot, offset, interleaved, dtype):
    cfg = config(hq, hkv, d, min(d, 512), dtype)
    freqs = orc.rope_table(rot, 10000.0)
    for seed, (t, first) in enumerate([(1, 131071), (5, 0), (67, 900001), (700, -350)]):
        rng = torch.Generator().manual_seed(seed)
        fused = torch.randn(t, hq + 2 * hkv, d, generator=rng).to(DT[dtype]).cuda()      # a fused projection: strided views
        q, k = fused[:, :hq], fused[:, hq:hq + hkv]
        x = f64(fused)
        positions = np.random.default_rng(seed).permutation(t) + first
        pos = i32(positions.tolist())
        magnitude, inverse = (1.0, False) if seed % 2 else (1.2079, True)
        rope = B.make_rope(rot_dim=rot, rot_offset=offset, interleaved=interleaved, magnitude=magnitude)
        fr = torch.from_numpy(freqs).cuda()
        q_out = torch.full((hq, t, d), float("nan"), dtype=DT[dtype], device="cuda").transpose(0, 1)   # head-major output
        k_out = torch.full((t, hkv, d), float("nan"), dtype=DT[dtype], device="cuda")
        B.snap_rope(cfg, rope, fr, pos, q=q, k=k, q_out=q_out, k_out=k_out, inverse=inverse)
        args = (positions, freqs, rot, offset, interleaved, magnitude, inverse, dtype)
        check_rotation(f64(q_out), x[:, :hq], *args)
        check_rotation(f64(k_out), x[:, hq:hq + hkv], *args)
        # in place, keys alone first, then the queries: the same bits, and the values beside them untouched
        B.snap_rope(cfg, rope, fr, pos, k=k, k_out=k, inverse=inverse)
        B.snap_rope(cfg, rope, fr, pos, q=q, q_out=q, inverse=inverse)
        assert torch.equal(q, q_out) and torch.equal(k, k_out)
        np.testing.assert_array_equal(f64(fused[:, hq + hkv:]), x[:, hq + hkv:])


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_inverse_is_the_gradient(interleaved):
    """The inverse direction against the formula's transposed map and against differences of the forward call."""
    t, h, d, rot = 9, 3, 64, 48
    cfg, freqs = config(h, 1, d, dtype="f32"), orc.rope_table(rot, 10000.0)
    rope = B.make_rope(rot_dim=rot, rot_offset=8, interleaved=interleaved, magnitude=1.5)
    fr, pos = torch.from_numpy(freqs).cuda(), i32([0, 1, 2, 77, 1000, 65536, 131071, 3, 4])
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn(t, h, d, device="cuda", generator=g) for _ in range(2))
    call = lambda z, inverse=False: (lambda o: (B.snap_rope(cfg, rope, fr, pos, q=z, q_out=o, inverse=inverse), f64(o))[1])(torch.empty_like(z))  # noqa: E731
    dx = call(dy, True)
    check_rotation(dx, f64(dy), pos.cpu().numpy(), freqs, rot, 8, interleaved, 1.5, True, "f32")
    # The map is linear: a difference along v of any length is exact up to rounding, |<dy, R(x + v) - R(x)> - <dx, v>|
    v = torch.randn(t, h, d, device="cuda", generator=g)
    lhs, rhs = (f64(dy) * (call(x + v) - call(x))).sum(), (dx * (f64(x + v) - f64(x))).sum()
    size = (np.abs(f64(dy)) * (np.abs(call(x + v)) + np.abs(call(x)))).sum() + (np.abs(dx) * np.abs(f64(v))).sum()
    assert abs(lhs - rhs) <= 16 * E * 1.5 * size


# ---------------------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("hq,hkv,d,dv,page,rotated", [(8, 2, 128, 128, 16, True), (3, 3, 64, 80, 5, True), (4, 1, 256, 64, 64, False),
                                                      (4, 4, 48, 48, 1, True)])
def test_append_writes_rows_and_nothing_else(hq, hkv, d, dv, page, rotated, layout, dtype):
    lengths = [0, 1, 33, 64, 100]
    cfg = config(hq, hkv, d, dv, dtype, max_seqs=len(lengths))
    c = Pages(cfg, dtype, page, [200] * len(lengths), seed=5, layout=layout)
    c.seq_len.copy_(i32(lengths))
    before_k, before_v = f64(c.k), f64(c.v)
    rope = B.make_rope(rot_dim=d // 2, rot_offset=d // 4, interleaved=layout == "nhd") if rotated else None
    freqs = orc.rope_table(d // 2, 10000.0)
    # ragged prompts, one of them into earlier rows; padding; ids and rows out of range; a page that is not there
    plan = [(0, r) for r in range(37)] + [(2, 33 + r) for r in range(20)] + [(-1, 3), (5, 0), (-7, 2), (4, 7), (1, 200 + page), (3, -1)]
    c.table[3, 150 // page] = 10 ** 6
    plan += [(3, 150), (3, 64)]
    t = len(plan)
    g = torch.Generator(device="cuda").manual_seed(1)
    fused = torch.randn(t, hq + hkv, d, device="cuda", generator=g).to(DT[dtype])
    q, k = fused[:, :hq], fused[:, hq:]
    v = torch.randn(t, hkv, dv, device="cuda", generator=g).to(DT[dtype])
    positions = [1000 + 3 * i for i in range(t)]
    q_out, k_out = (torch.full((t, h, d), 7.0, dtype=DT[dtype], device="cuda") for h in (hq, hkv))
    w = c.weights(3.0)
    B.snap_paged_append(cfg, c.paged, i32([s for s, _ in plan]), i32([r for _, r in plan]), k, v, c.k, c.v, c.table, c.seq_len, rope=rope,
                        freqs=torch.from_numpy(freqs).cuda() if rotated else None, positions=i32(positions) if rotated else None, q=q,
                        q_out=q_out, k_out=k_out, weights=w, status=c.status)
    assert c.bits() == B.SNAP_DEV_BAD_SLOT | B.SNAP_DEV_BAD_PAGE
    done = [i for i, (s, r) in enumerate(plan) if 0 <= s < 5 and 0 <= r < c.width * page and (s, r) != (3, 150)]
    skipped = [i for i in range(t) if i not in done]
    assert (f64(q_out)[skipped] == 7).all() and (f64(k_out)[skipped] == 7).all()
    for got, x in ((q_out, q), (k_out, k)):
        if rotated:
            check_rotation(f64(got)[done], f64(x)[done], np.array(positions)[done], freqs, d // 2, d // 4, layout == "nhd", 1.0, False, dtype)
        else:
            np.testing.assert_array_equal(f64(got)[done], f64(x)[done])
    table, want_w = c.table.cpu().numpy(), np.full(w.shape, 3.0)
    for i in done:                                          # the pages hold what k_out and v say; all else is as before
        s, r = plan[i]
        before_k[table[s, r // page], :, r % page] = f64(k_out)[i]
        before_v[table[s, r // page], :, r % page] = f64(v)[i]
        want_w[s, :, r] = 0.0
    np.testing.assert_array_equal(f64(c.k), before_k)
    np.testing.assert_array_equal(f64(c.v), before_v)
    np.testing.assert_array_equal(f64(w), want_w)
    assert c.seq_len.tolist() == [37, 1, 53, 65, 100]


def test_append_next_rows_grow_the_sequences():
    """rows_dev = None: every token is its sequence's next row at its own position; a slot listed again is skipped."""
    cfg = config(4, 2, 64, dtype="f32", max_seqs=6)
    c = Pages(cfg, "f32", 16, [64] * 6, seed=2)
    c.seq_len.copy_(i32([0, 15, 16, 63, 64, 20]))
    freqs = orc.rope_table(64, 10000.0)
    slots, rope = [3, 0, -1, 2, 1, 0, 4, 2], B.make_rope(rot_dim=64)
    k, v = torch.randn(8, 2, 64, device="cuda"), torch.randn(8, 2, 64, device="cuda")
    before = f64(c.k)
    B.snap_paged_append(cfg, c.paged, i32(slots), None, k, v, c.k, c.v, c.table, c.seq_len, rope=rope, freqs=torch.from_numpy(freqs).cuda(),
                        status=c.status)
    assert c.bits() == B.SNAP_DEV_BAD_SLOT | B.SNAP_DEV_BAD_PAGE       # slots 0 and 2 again; slot 4 is full
    assert c.seq_len.tolist() == [1, 16, 17, 64, 64, 20]
    table = c.table.cpu().numpy()
    got = f64(c.k)
    for i, row in ((0, 63), (1, 0), (3, 16), (4, 15)):
        page = table[slots[i], row // 16]
        check_rotation(got[page, :, row % 16][None], f64(k)[i][None], [row], freqs, 64, 0, False, 1.0, False, "f32")
        got[page, :, row % 16] = before[page, :, row % 16]
    np.testing.assert_array_equal(got, before)


# ---------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------
def run_decode(c, q, slots, weights_in=None, weights_out=None, seq_len=None, stream=None):
    cfg, n = c.cfg, len(slots)
    out = torch.full((n, cfg.n_q_heads, cfg.d_v), float("nan"), dtype=q.dtype, device="cuda")
    need = B.snap_paged_decode_workspace_bytes(cfg, c.paged, n, weights_out is not None)
    ws = torch.full((need,), 0xff, dtype=torch.uint8, device="cuda")          # scratch holds NaN
    B.snap_paged_decode_attn(cfg, c.paged, q, i32(slots), n, c.k, c.v, c.table, c.seq_len if seq_len is None else seq_len, out, ws,
                             weights_in=weights_in, weights_out=weights_out, status=c.status, stream=stream)
    return out


def check_decode(c, out, q, slots, dtype, weights=None, weights_before=None, lengths=None):
    cfg, d = c.cfg, c.cfg.d_qk
    got, want_w, slack_w = f64(out), None, None
    if weights is not None:
        want_w, slack_w = f64(weights_before).copy(), np.zeros(weights.shape)
    for i, slot in enumerate(slots):
        n = (lengths or c.lengths)[slot] if 0 <= slot < cfg.max_seqs else 0
        if n == 0:
            assert (got[i] == 0).all()
            continue
        k, v, there = c.rows(slot, min(n, c.width * c.page))
        o, w, mass, reach = orc.decode(f64(q[i]), k, v, float(np.float32(d ** -0.5)))
        rel = 2 * (d + 3) * E * 1.4427 * reach + 2.0 ** -20 + 2 * len(there) * E
        bound = HALF_STEP[dtype] * np.abs(o) + ((rel + (2.0 ** -16 if dtype == "bf16" else 0.0))[:, None]) * mass
        err = np.abs(got[i] - o)
        assert (err <= bound + 1e-30).all(), f"sequence {i} ({n} rows): {(err / (bound + 1e-30)).max():.2f} of the bound"
        if weights is not None:
            for h in range(cfg.n_kv_heads):
                want_w[slot, h, there] += w[h]
                g = cfg.n_q_heads // cfg.n_kv_heads
                slack_w[slot, h, there] = w[h] * rel[h * g:(h + 1) * g].max() + 2 * E * np.abs(want_w[slot, h, there])
    if weights is not None:
        err = np.abs(f64(weights) - want_w)
        assert (err <= slack_w + 1e-30).all(), f"weights: {(err - slack_w).max():.3e} over the bound"


DECODES = [  # hq, hkv, d, dv, page, layout
    (8, 2, 128, 128, 16, "hnd"), (32, 8, 128, 128, 64, "nhd"), (4, 4, 64, 64, 48, "hnd"), (14, 2, 256, 256, 16, "nhd"),
    (12, 1, 128, 128, 32, "hnd"), (32, 1, 64, 64, 16, "nhd"), (40, 2, 256, 256, 32, "hnd"), (9, 3, 80, 80, 16, "hnd"),
    (6, 1, 128, 64, 8, "nhd"), (2, 1, 48, 96, 5, "hnd"), (16, 2, 64, 64, 1, "nhd"), (11, 1, 192, 256, 24, "hnd"), (5, 5, 16, 16, 7, "hnd"),
    (8, 2, 128, 128, 1, "hnd"), (20, 1, 128, 112, 3, "hnd"), (40, 2, 256, 256, 1, "nhd"), (6, 2, 64, 64, 9, "nhd"), (7, 1, 256, 256, 13, "hnd"),
    (12, 1, 64, 48, 2, "hnd"), (8, 2, 256, 256, 16, "hnd"), (3, 1, 256, 192, 3, "nhd"), (16, 1, 128, 128, 16, "nhd")]
LENGTHS = [0, 1, 15, 16, 17, 31, 333, 0, 2, 1300, 64, 47]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("hq,hkv,d,dv,page,layout", DECODES)
def test_paged_decode_matches_its_definition(hq, hkv, d, dv, page, layout, dtype):
    cfg = config(hq, hkv, d, dv, dtype, max_seqs=len(LENGTHS))
    c = Pages(cfg, dtype, page, LENGTHS, seed=hq * d + page, layout=layout)
    slots = [int(x) for x in np.random.default_rng(1).permutation(len(LENGTHS))]
    slots.insert(3, -1)                                     # a padded batch
    g = torch.Generator(device="cuda").manual_seed(7)
    q = torch.randn(len(slots), hq, d, device="cuda", generator=g).to(DT[dtype])
    q[1::3] *= 6                                            # some sequences look at few rows
    plain = run_decode(c, q, slots)
    check_decode(c, plain, q, slots, dtype)
    before, w = torch.rand(c.weights().shape, device="cuda", generator=g), c.weights()
    w.copy_(before)
    out = run_decode(c, q, slots, weights_in=w, weights_out=w)        # in place
    assert torch.equal(out, plain)
    check_decode(c, out, q, slots, dtype, weights=w, weights_before=before)
    alone = c.weights(5.0)
    run_decode(c, q, slots, weights_out=alone)                        # this step's weights; other entries untouched
    inside = torch.arange(c.width * page, device="cuda") < c.seq_len[:, None, None]
    assert bool((alone.masked_fill(inside, 5.0) == 5.0).all())
    check_decode(c, out, q, slots, dtype, weights=torch.where(inside, alone, torch.zeros_like(alone)), weights_before=c.weights())
    assert c.bits() == 0


@pytest.mark.parametrize("dtype,hq,hkv,d,page", [("bf16", 32, 8, 128, 32), ("f32", 8, 2, 128, 32), ("bf16", 8, 8, 64, 32), ("f32", 16, 2, 96, 32),
                                                 ("bf16", 32, 8, 128, 1), ("bf16", 24, 2, 256, 12), ("f32", 6, 2, 256, 16),
                                                 ("f32", 8, 8, 64, 20)])
def test_paged_decode_of_long_and_single_sequences(dtype, hq, hkv, d, page):
    """One sequence over all CTAs, few tiles per CTA, and many short ones: every way a unit can be cut."""
    for lengths in ([9001], [16 * 37], [5, 20011, 1, 700], [33] * 200):
        cfg = config(hq, hkv, d, dtype=dtype, max_seqs=len(lengths))
        c = Pages(cfg, dtype, page, lengths, seed=len(lengths))
        slots = list(range(len(lengths)))[::-1]
        q = torch.randn(len(slots), hq, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(DT[dtype])
        w = c.weights()
        out = run_decode(c, q, slots, weights_out=w)
        some = slots if len(slots) < 10 else slots[:3]
        check_decode(c, out[:len(some)], q, some, dtype)
        total = f64(w).sum(axis=2)                          # a head's weights sum to one
        np.testing.assert_allclose(total, hq // hkv, rtol=1e-4)
        again = c.weights()
        assert torch.equal(out, run_decode(c, q, slots, weights_out=again)) and torch.equal(w, again)   # equal bits
        assert c.bits() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [31, 45, 64, 97, 128, 129, 300])
def test_paged_decode_of_many_ragged_sequences(n, dtype):
    """Batches around the sizes at which the look-up of sequences changes, lengths of all kinds in every order."""
    rng = np.random.default_rng(n)
    lengths = [int(x) for x in rng.choice([0, 0, 1, 7, 8, 9, 16, 40, 64, 65, 72, 150, 333], size=n)]
    lengths[n // 2] = 2500
    cfg = config(4, 2, 64, dtype=dtype, max_seqs=n)
    c = Pages(cfg, dtype, 16, lengths, seed=n)
    slots = [int(x) for x in rng.permutation(n)]
    q = torch.randn(n, 4, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(n)).to(DT[dtype])
    w = c.weights()
    out = run_decode(c, q, slots, weights_out=w)
    check_decode(c, out, q, slots, dtype, weights=w, weights_before=c.weights())
    assert c.bits() == 0


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("f32", 16), ("bf16", 4)])
def test_paged_decode_leaves_out_what_is_not_there(dtype, page):
    """Pages out of range, lengths past the table, negative lengths, slots out of range and listed twice."""
    cfg = config(8, 2, 64, dtype=dtype, max_seqs=6)
    lengths = [100, 64, 50, 80, 33, 17]
    c = Pages(cfg, dtype, page, lengths, seed=11, capacity=112)
    c.table[0, 48 // page] = -1
    c.table[1, :64 // page] = 10 ** 7                       # nothing of it is there: zeros
    c.table[3, 0] = c.k.shape[0]
    c.seq_len[2] = -5
    pages = c.table[4].clone()
    c.table[4] = c.table[5]                                 # shared pages, and a length past the table (its pages: clamped)
    c.table[4, -(-17 // page):] = pages[-(-17 // page):]
    c.table[4][c.table[4] < 0] = 0
    c.k[0], c.v[0] = 1.0, 2.0
    for x in (c.k, c.v):
        x[torch.isnan(x)] = 0.5
    c.seq_len[4] = 10 ** 9
    slots = [5, 0, 6, 1, 2, 3, 4, -2]
    q = torch.randn(8, 8, 64, device="cuda").to(DT[dtype])
    lens = {0: 100, 1: 64, 2: 0, 3: 80, 4: c.width * page, 5: 17}
    w = c.weights()
    out = run_decode(c, q, slots, weights_out=w)
    assert c.bits() == B.SNAP_DEV_BAD_SLOT | B.SNAP_DEV_BAD_PAGE
    c.lengths = [lens[i] for i in range(6)]
    keep = [0, 1, 2, 4, 5, 6, 7]
    check_decode(c, out[keep], q[keep], [slots[i] for i in keep], dtype)
    assert (f64(out)[3] == 0).all() and (f64(w)[1] == 0).all()
    # listed twice: both rows attend, the first entry's weights count
    c.status.zero_()
    once, twice = c.weights(), c.weights()
    a = run_decode(c, q[:2], [5, 0], weights_out=once)
    two = torch.cat([q[:2], q[2:3]])
    b = run_decode(c, two, [5, 0, 5], weights_out=twice)
    assert c.bits() & B.SNAP_DEV_BAD_SLOT
    check_decode(c, b[2:], two[2:], [5], dtype)
    np.testing.assert_allclose(f64(once), f64(twice), rtol=1e-5, atol=1e-12)
    assert a.shape[0] == 2


def test_paged_decode_past_32_bit_offsets():
    """Pools of more than 2^32 bytes and 2^31 elements: rows at either end of them, bf16 by both kernels and fp32."""
    for dtype, page, d, pages in (("bf16", 16, 128, 140000), ("bf16", 20, 112, 125000), ("f32", 16, 128, 140000)):
        cfg = config(8, 8, d, dtype=dtype, max_seqs=1)
        c = Pages(cfg, dtype, page, [page * 6 - 3], seed=1, spare=0)
        ks, vs = (torch.empty(pages, 8, page, d, dtype=DT[dtype], device="cuda") for _ in range(2))
        assert ks.numel() > 2 ** 31
        far = [pages - 1, 0, pages - 2, 119999, 7, 120001]
        for new, old in ((ks, c.k), (vs, c.v)):
            for i, p in enumerate(far):
                new[p] = old[int(c.table[0, i])]
        small_table, small_k, small_v = c.table.clone(), c.k, c.v
        q = torch.randn(1, 8, d, device="cuda").to(DT[dtype])
        want = run_decode(c, q, [0])
        c.k, c.v, c.table = ks, vs, i32([far])
        c.paged = B.make_paged(ks, vs, c.table)
        assert torch.equal(run_decode(c, q, [0]), want) and c.bits() == 0
        # rows appended there land there
        k1 = torch.randn(1, 8, d, device="cuda").to(DT[dtype])
        B.snap_paged_append(cfg, c.paged, i32([0]), None, k1, k1, ks, vs, c.table, c.seq_len, status=c.status)
        assert torch.equal(ks[120001, :, page - 3], k1[0]) and torch.equal(vs[120001, :, page - 3], k1[0]) and c.bits() == 0
        c.k, c.v, c.table = small_k, small_v, small_table
        del ks, vs


# ---------------------------------------------------------------------------------------------------------------
# eviction
# ---------------------------------------------------------------------------------------------------------------
def run_evict(c, src, dst, w, w_out, want_kept=True):
    cfg, n = c.cfg, len(src)
    kept = torch.full((n, cfg.n_kv_heads, cfg.l_sink + cfg.topk + cfg.l_recent), -9, dtype=torch.int32, device="cuda") if want_kept else None
    ws = torch.full((B.snap_paged_evict_workspace_bytes(cfg, c.paged, n),), 0xff, dtype=torch.uint8, device="cuda")
    B.snap_paged_evict(cfg, c.paged, i32(src), i32(dst), n, c.k, c.v, c.table, c.seq_len, w, w_out, ws, kept_rows=kept, status=c.status)
    return kept


def check_evict(c, src, dst, w, w_before, kept, k_before, v_before, moved):
    """Pools, lengths, weights and kept rows after moving the entries in `moved`; everything else is as before."""
    cfg, page, table = c.cfg, c.page, c.table.cpu().numpy()
    keep = cfg.l_sink + cfg.topk + cfg.l_recent
    want_k, want_v, want_w, want_len = k_before.copy(), v_before.copy(), f64(w_before).copy(), list(c.lengths)
    got_kept = kept.cpu().numpy()
    for i in range(len(src)):
        if i not in moved:
            assert (got_kept[i] == -1).all()
            continue
        n = c.lengths[src[i]]
        want_len[dst[i]] = min(n, keep)
        for h in range(cfg.n_kv_heads):
            rows = orc.kept_rows(f64(w_before)[src[i], h], n, cfg.l_sink, cfg.l_recent, cfg.topk)
            np.testing.assert_array_equal(got_kept[i, h, :len(rows)], rows)
            assert (got_kept[i, h, len(rows):] == -1).all()
            to = np.arange(len(rows))
            a, b = table[src[i], rows // page], table[dst[i], to // page]
            want_k[b, h, to % page] = k_before[a, h, rows % page]
            want_v[b, h, to % page] = v_before[a, h, rows % page]
            want_w[dst[i], h, to] = f64(w_before)[src[i], h, rows]
    np.testing.assert_array_equal(f64(c.k), want_k)
    np.testing.assert_array_equal(f64(c.v), want_v)
    np.testing.assert_array_equal(f64(w), want_w)
    assert c.seq_len.tolist() == want_len


def evict_case(dtype, hkv, d, dv, page, layout, sink, recent, topk, lengths, fill, seed=0):
    n, keep = len(lengths), sink + recent + topk
    cfg = config(2 * hkv, hkv, d, dv, dtype, max_seqs=2 * n, sink=sink, recent=recent, topk=topk)
    c = Pages(cfg, dtype, page, lengths + [min(x, keep) for x in lengths], seed=seed, layout=layout)
    c.lengths = lengths + [0] * n
    c.seq_len.copy_(i32(c.lengths))
    w = c.weights()
    w.copy_(fill(w.shape))
    before, k0, v0 = w.clone(), f64(c.k), f64(c.v)
    src, dst = list(range(n))[::-1], [n + i for i in range(n)][::-1]
    kept = run_evict(c, src, dst, w, w)
    check_evict(c, src, dst, w, before, kept, k0, v0, set(range(n)))
    assert c.bits() == 0


def heavy_tail(shape):
    return torch.rand(shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)) ** 4


def few_values(shape):                                      # ties everywhere, at the threshold too
    return torch.randint(0, 3, shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(2)).float() - 1


def odd_values(shape):                                      # signs, zeros of both signs, infinities, NaN
    g = torch.Generator(device="cuda").manual_seed(4)
    w = torch.randn(shape, device="cuda", generator=g)
    pick = torch.randint(0, 12, shape, device="cuda", generator=g)
    for i, x in enumerate((0.0, -0.0, float("inf"), -float("inf"), float("nan"))):
        w[pick == i] = x
    return w


@pytest.mark.parametrize("fill", [heavy_tail, few_values, odd_values, lambda s: torch.zeros(s, device="cuda")],
                         ids=["heavy", "ties", "odd", "equal"])
@pytest.mark.parametrize("dtype,hkv,d,dv,page,layout,sink,recent,topk", [
    ("bf16", 2, 128, 128, 16, "hnd", 4, 33, 100), ("f32", 3, 80, 48, 5, "nhd", 0, 1, 64), ("bf16", 1, 256, 64, 64, "nhd", 7, 20, 0),
    ("f32", 2, 64, 64, 1, "hnd", 3, 5, 1), ("bf16", 2, 16, 16, 32, "hnd", 0, 200, 333)])
def test_evict_matches_its_definition(dtype, hkv, d, dv, page, layout, sink, recent, topk, fill):
    keep = sink + recent + topk
    lengths = [0, 1, sink + 1, keep - 1, keep, keep + 1, keep + 2, 2 * keep + 3, 700, 1999]
    evict_case(dtype, hkv, d, dv, page, layout, sink, recent, topk, lengths, fill)


@pytest.mark.parametrize("fill", [heavy_tail, few_values], ids=["heavy", "ties"])
@pytest.mark.parametrize("longest", [9000, 380001])
def test_evict_from_long_middles(longest, fill):
    """Middles over a cluster of CTAs, with the keys in shared memory and (past 360 000 rows) without."""
    evict_case("bf16", 1, 16, 16, 64, "hnd", 4, 64, 1500, [longest, 1600, 4000], fill)


def test_evict_skips_what_it_cannot_move():
    cfg = config(4, 2, 64, max_seqs=8, sink=1, recent=4, topk=8)
    lengths = [60, 61, 62, 63]
    c = Pages(cfg, "bf16", 8, lengths + [13] * 4, seed=3)
    c.lengths = lengths + [0] * 4
    c.seq_len.copy_(i32(c.lengths))
    w = torch.rand(c.weights().shape, device="cuda")
    before, k0, v0 = w.clone(), f64(c.k), f64(c.v)
    # moved; onto a source of the call; out of range (each side); an earlier entry's destination; onto itself; moved (a source twice)
    src, dst = [0, 1, -1, 2, 2, 3, 0], [4, 0, 5, 8, 4, 3, 6]
    kept = run_evict(c, src, dst, w, w)
    check_evict(c, src, dst, w, before, kept, k0, v0, {0, 6})
    assert c.bits() == B.SNAP_DEV_BAD_SLOT
    # destination and source pages that are not there: their rows stay out, the rest moves; no weights asked for
    c.status.zero_()
    c.table[7, 0], c.table[1, 7] = -1, 10 ** 6
    k1 = f64(c.k)
    kept = run_evict(c, [1], [7], w, None)
    assert c.bits() == B.SNAP_DEV_BAD_PAGE
    table, rows = c.table.cpu().numpy(), kept.cpu().numpy()
    for h in range(2):
        for r, row in enumerate(rows[0, h]):
            if r >= 8 and row < 56:
                k1[table[7, r // 8], h, r % 8] = k1[table[1, row // 8], h, row % 8]
    np.testing.assert_array_equal(f64(c.k), k1)
    np.testing.assert_array_equal(f64(w)[7], f64(before)[7])


# ---------------------------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,hq,hkv,d,page", [("bf16", 8, 2, 128, 16), ("f32", 6, 3, 64, 8)])
def test_prompt_steps_eviction_steps(dtype, hq, hkv, d, page):
    """A serving run: prompts rotated into their pages and attended, steps that gather weights (captured once and replayed),
    eviction to fresh slots, further steps, against the same run in double precision on the stored values."""
    lengths, sink, recent, topk, steps = [150, 70, 9], 2, 24, 40, 6
    n, keep, cap = len(lengths), sink + recent + topk, 192
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=2 * n, sink=sink, recent=recent, topk=topk)
    c = Pages(cfg, dtype, page, [cap] * (2 * n), seed=9)
    c.k.fill_(float("nan"))
    c.v.fill_(float("nan"))
    c.seq_len.zero_()
    rope = B.make_rope(rot_dim=d, scaling="llama3", base=500000.0, factor=8.0, original_len=64.0)
    freqs, _ = B.snap_rope_table(rope)
    freqs = freqs.cuda()
    g = torch.Generator(device="cuda").manual_seed(0)
    new = lambda t, h: torch.randn(t, h, d, device="cuda", generator=g).to(DT[dtype])  # noqa: E731
    total, w = sum(lengths), c.weights(9.0)
    q, k, v = new(total, hq), new(total, hkv), new(total, hkv)
    slots = i32([i for i, x in enumerate(lengths) for _ in range(x)])
    rows = i32([r for x in lengths for r in range(x)])
    q_out, k_out = torch.empty_like(q), torch.empty_like(k)
    B.snap_paged_append(cfg, c.paged, slots, rows, k, v, c.k, c.v, c.table, c.seq_len, rope=rope, freqs=freqs, q=q, q_out=q_out,
                        k_out=k_out, weights=w, status=c.status)
    # the prompt's own attention takes the rotated queries and keys; its last row is what a step on the pages gives
    cu = np.concatenate([[0], np.cumsum(lengths)]).tolist()
    prompt = torch.empty_like(q)
    B.snap_prefill_attn(cfg, q_out, k_out, v, cu, prompt, status=c.status)
    last = [x - 1 for x in cu[1:]]
    out = run_decode(c, q_out[last].contiguous(), list(range(n)))
    assert c.seq_len.tolist() == lengths + [0] * n
    c.lengths = lengths + [0] * n
    check_decode(c, out, q_out[last], list(range(n)), dtype)
    # two results of the same rows by kernels that each round the output (and one of them its probabilities to bf16)
    np.testing.assert_allclose(f64(out), f64(prompt)[last], atol=2e-2 if dtype == "bf16" else 1e-4)

    ids = i32(list(range(n)))
    position = i32(lengths)
    static = dict(q=new(n, hq), k=new(n, hkv), v=new(n, hkv))
    q_rot, out = torch.empty_like(static["q"]), torch.empty_like(static["q"])
    ws = torch.empty(B.snap_paged_decode_workspace_bytes(cfg, c.paged, n, True), dtype=torch.uint8, device="cuda")

    def step():
        B.snap_paged_append(cfg, c.paged, ids, None, static["k"], static["v"], c.k, c.v, c.table, c.seq_len, rope=rope, freqs=freqs,
                            positions=position, q=static["q"], q_out=q_rot, weights=w, status=c.status)
        B.snap_paged_decode_attn(cfg, c.paged, q_rot, ids, n, c.k, c.v, c.table, c.seq_len, out, ws, weights_in=w, weights_out=w,
                                 status=c.status)
        position.add_(1)

    def check_step(w_before, live):
        before = f64(w_before)
        for i, s in enumerate(live):
            c.lengths[s] += 1
            before[s, :, c.lengths[s] - 1] = 0.0
        assert c.seq_len.tolist() == c.lengths
        check_decode(c, out, q_rot, live, dtype, weights=w, weights_before=torch.from_numpy(before))

    w0 = w.clone()
    step()                                                  # eagerly first
    check_step(w0, [0, 1, 2])
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    saved = [x.clone() for x in (w, c.seq_len, position, c.k, c.v)]
    with torch.cuda.graph(graph, stream=side):
        step()
    for x, y in zip((w, c.seq_len, position, c.k, c.v), saved):
        x.copy_(y)                                          # (capture runs nothing; whatever it did is undone)
    for s in range(steps):
        for name, h in (("q", hq), ("k", hkv), ("v", hkv)):
            static[name].copy_(new(n, h))
        w0 = w.clone()
        graph.replay()
        torch.cuda.synchronize()
        check_step(w0, [0, 1, 2])
    assert position.tolist() == [x + steps + 1 for x in lengths]

    before, k0, v0 = w.clone(), f64(c.k), f64(c.v)
    kept = run_evict(c, [0, 1, 2], [3, 4, 5], w, w)
    check_evict(c, [0, 1, 2], [3, 4, 5], w, before, kept, k0, v0, {0, 1, 2})
    c.lengths[3:] = [min(x, keep) for x in c.lengths[:3]]
    ids.copy_(i32([3, 4, 5]))                               # the captured step goes on over the kept rows
    for s in range(2):
        for name, h in (("q", hq), ("k", hkv), ("v", hkv)):
            static[name].copy_(new(n, h))
        w0 = w.clone()
        graph.replay()
        torch.cuda.synchronize()
        check_step(w0, [3, 4, 5])
    assert c.bits() == 0


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("f32", 16), ("bf16", 8), ("bf16", 3)])
@pytest.mark.parametrize("d", [64, 96])
def test_paged_decode_carries_nan_and_leaves_other_heads_alone(dtype, page, d):
    """A NaN in a row that counts reaches the heads that attend it, over joins too, and no other head."""
    cfg = config(4, 2, d, dtype=dtype, max_seqs=3)
    c = Pages(cfg, dtype, page, [5000, 40, 1], seed=6)
    row = 3333
    c.k[int(c.table[0, row // page]), 1, row % page, 3] = float("nan")
    c.v[int(c.table[1, 5 // page]), 0, 5 % page, 7] = float("nan")
    c.k[int(c.table[2, 0]), 0, 0, 0] = float("nan")
    q = torch.randn(3, 4, d, device="cuda").to(DT[dtype])
    w = c.weights()
    out = f64(run_decode(c, q, [0, 1, 2], weights_out=w))
    assert np.isnan(out[0, 2:]).all() and np.isfinite(out[0, :2]).all()
    assert np.isnan(out[1, :2, 7]).all() and np.isfinite(np.delete(out[1], 7, axis=1)).all() and np.isfinite(out[1, 2:]).all()
    assert np.isnan(out[2, :2]).all() and np.isfinite(out[2, 2:]).all()
    assert np.isnan(f64(w)[0, 1, :5000]).all() and np.isfinite(f64(w)[0, 0]).all() and np.isfinite(f64(w)[1]).all()


def test_calls_on_a_side_stream_and_two_at_once():
    """Two sequences' steps on two streams, each with scratch of its own, equal the same steps one after the other."""
    cfg = config(8, 2, 128, max_seqs=2)
    c = Pages(cfg, "bf16", 16, [5000, 3000], seed=4)
    q = torch.randn(2, 8, 128, device="cuda").to(torch.bfloat16)
    want = [run_decode(c, q[i:i + 1].clone(), [i]) for i in range(2)]
    qs = [q[i:i + 1].clone() for i in range(2)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(run_decode(c, qs[i], [i], stream=s))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])
    assert c.bits() == 0


def test_first_calls_inside_a_capture():
    """Shapes that no call has used before, captured at once: what a call sets up on the host is not a stream operation."""
    cfg = config(6, 2, 32, 48, "bf16", max_seqs=2, sink=1, recent=2, topk=5)
    c = Pages(cfg, "bf16", 8, [30, 8], seed=2)
    c.lengths = [30, 0]
    c.seq_len.copy_(i32(c.lengths))
    q = torch.randn(1, 6, 32, device="cuda").to(torch.bfloat16)
    k, v = torch.randn(1, 2, 32, device="cuda").to(torch.bfloat16), torch.randn(1, 2, 48, device="cuda").to(torch.bfloat16)
    w, out = c.weights(), torch.zeros(1, 6, 48, dtype=torch.bfloat16, device="cuda")
    before = (f64(c.k), f64(c.v))
    ids, src, dst = i32([0]), i32([0]), i32([1])
    rope, freqs = B.make_rope(rot_dim=12, rot_offset=2), torch.from_numpy(orc.rope_table(12, 10000.0)).cuda()
    ws = torch.empty(B.snap_paged_decode_workspace_bytes(cfg, c.paged, 1, True), dtype=torch.uint8, device="cuda")
    ws2 = torch.empty(B.snap_paged_evict_workspace_bytes(cfg, c.paged, 1), dtype=torch.uint8, device="cuda")
    kept = torch.zeros(1, 2, 8, dtype=torch.int32, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.snap_paged_append(cfg, c.paged, ids, None, k, v, c.k, c.v, c.table, c.seq_len, rope=rope, freqs=freqs, weights=w, status=c.status)
        B.snap_paged_decode_attn(cfg, c.paged, q, ids, 1, c.k, c.v, c.table, c.seq_len, out, ws, weights_in=w, weights_out=w, status=c.status)
        B.snap_paged_evict(cfg, c.paged, src, dst, 1, c.k, c.v, c.table, c.seq_len, w, w, ws2, kept_rows=kept, status=c.status)
    torch.cuda.synchronize()
    np.testing.assert_array_equal(f64(c.k), before[0])      # capturing ran nothing
    graph.replay()
    torch.cuda.synchronize()
    c.lengths = [31, 0]
    assert c.seq_len.tolist() == [31, 8] and c.bits() == 0
    check_decode(c, out, q, [0], "bf16")
    for h in range(2):
        np.testing.assert_array_equal(kept.cpu().numpy()[0, h], orc.kept_rows(f64(w)[0, h], 31, 1, 2, 5))


def test_the_paged_calls_under_the_checked_build():
    """Eviction, append and attention once more with the build that tests data-dependent indices (a bad one raises a status
    bit, which these tests require to be clear)."""
    import os
    import subprocess
    import sys
    from paper_2511_03092_b200 import build as snap_build
    lib = snap_build.build(debug_bounds=True)
    env = dict(os.environ, SNAP_LIBRARY=os.path.basename(lib))
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-m", "pytest", "tests/test_gpu_paged.py", "-m", "gpu", "-q", "-x", "-p", "no:cacheprovider",
                        "-k", "evict or append or ragged or together or steps"], cwd=root, env=env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[-2000:]
    assert " passed" in r.stdout
