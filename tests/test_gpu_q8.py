"""The cache in pages of 8-bit numbers on the GPU against its double-precision definitions.

Tolerances.  u is half a step of the output type (2^-8 bf16, 2^-24 fp32), e = 2^-24.
Append: codes and scales of what is not rotated are those of the definition.  A rotated key is off by at most 8 e m (|a| + |b|)
before it is rounded (two products and a sum in single precision, cosines and sines off by a few e), so the number that its code
stands for is at most twice that further from the exact one than the nearest code's; scales do not depend on the rotation.
Attention: a logit is a sum of d products, off by at most (d + 8) e R (a single-precision query enters as two numbers of 11 bits,
2^-22 off; the change of base and two scales), R the largest scale sum_c |q_c k_rc|; a query's smallest parts are cut off 2^-38
below its largest number Q: 2^-38 Q of any.  A probability is then off by a factor 1 +- 2 (that) to first order, the exponential's own 2^-22,
and 2^-11 (bf16: rounded to 11 bits before it multiplies the values) or 2^-21 (fp32: two such numbers); of small ones 2^-31 of the largest
product of probability and scale is cut (2^-25 is half the last step of half precision, the largest is 2^6 or more), times its row's code;
sums over n rows add n e.  So
|err| <= u |out| + (2 L + 2^-20 + 2^-11 [bf16] + 2 n e) sum_r p_r |v_r| + 2^-31 max_r(p_r s_r) sum_r |code_r|."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as porc
from oracle import q8_oracle as orc
from paper_2511_03092_b200 import binding as B

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF_STEP = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
E = 2.0 ** -24
CODE = torch.float8_e4m3fn


def f64(t):
    return t.detach().to("cpu", torch.float64).numpy()


def i32(xs):
    return torch.tensor(xs, dtype=torch.int32, device="cuda")


def config(hq, hkv, d, dv=None, dtype="bf16", max_seqs=1, scale=None):
    return B.make_config(n_q_heads=hq, n_kv_heads=hkv, d_qk=d, d_v=dv or d, dtype=DT[dtype], l_sink=2, l_recent=8, topk=16, l_obs=1, pool_kernel=1,
                         softmax_scale=scale or d ** -0.5, max_seqs=max_seqs)


class Pages8:
    """An 8-bit cache whose unused memory is NaN, codes and scales: pools in either layout, a table of shuffled pages."""

    def __init__(self, cfg, page, block, lengths, seed=0, layout="hnd", capacity=None, spread=2, spare=2):
        self.cfg, self.page, self.block, rng = cfg, page, block, np.random.default_rng(seed)
        self.width = -(-max(max(lengths), capacity or 1) // page)
        need = [-(-n // page) for n in lengths]
        order = rng.permutation(sum(need) + spare)
        table = np.full((len(lengths), self.width), -1, dtype=np.int32)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = order[at:at + n]
            at += n
        self.free = [int(x) for x in order[at:]]
        self.table, self.seq_len, self.lengths = torch.from_numpy(table).cuda(), i32(lengths), list(lengths)
        self.pools, self.scales = [], []
        for d in (cfg.d_qk, cfg.d_v):
            codes = np.full((len(order), cfg.n_kv_heads, page, d), orc.NAN_CODE, dtype=np.uint8)
            scales = np.full((len(order), cfg.n_kv_heads, page // block), np.nan, dtype=np.float32)
            for i, n in enumerate(lengths):
                for p in range(need[i]):
                    rows = min(page, n - p * page)
                    blocks = -(-rows // block)
                    scales[table[i, p], :, :blocks] = 2.0 ** rng.integers(-8 - spread, -8 + spread + 1, (cfg.n_kv_heads, blocks))
                    x = rng.normal(size=(cfg.n_kv_heads, rows, d)) * 100
                    codes[table[i, p], :, :rows] = orc.encode(x)
            t = torch.from_numpy(codes).cuda().view(CODE)
            self.pools.append(t if layout == "hnd" else t.transpose(1, 2).contiguous().transpose(1, 2))
            self.scales.append(torch.from_numpy(scales).cuda())
        self.describe()

    def describe(self):
        (self.k, self.v), (self.ks, self.vs) = self.pools, self.scales
        self.paged = B.make_paged_q8(self.k, self.v, self.table, self.block)
        self.cache = (self.k, self.v, self.ks, self.vs, self.table)
        self.status = i32([0])

    def host(self):
        """The definition's view of both pools, as they are now."""
        return [orc.Cache(c.view(torch.uint8).cpu().numpy(), s.cpu().numpy()) for c, s in zip(self.pools, self.scales)]

    def bits(self):
        torch.cuda.synchronize()
        return int(self.status.item())


# ---------------------------------------------------------------------------------------------------------------
# append
# ---------------------------------------------------------------------------------------------------------------
def nearest_distance(y):
    return np.abs(orc.VALUES[orc.encode(y)] - np.clip(y, -448, 448))


def check_append(c, before, entries, first, cu, k, v, rope=None, freqs=None, positions=None, k_out=None, served=None, dtype="bf16"):
    """Everything the append writes, against the definition run on the cache as it was."""
    table = c.table.cpu().numpy()
    x = [f64(k), f64(v)]
    y, slack = [x[0], x[1]], [np.zeros_like(x[0]), np.zeros_like(x[1])]
    rows = np.zeros(len(x[0]), dtype=np.int64)
    for i in range(len(entries)):
        rows[cu[i]:cu[i + 1]] = np.arange(first[i], first[i] + cu[i + 1] - cu[i])
    factor = 1.0
    if rope is not None:
        pos = rows if positions is None else np.asarray(positions)
        m = rope.magnitude or 1.0
        y[0] = porc.rotate(x[0], pos, freqs, rope.rot_dim, rope.rot_offset, bool(rope.interleaved), m)
        j = np.arange(rope.rot_dim // 2)
        a, b = ((rope.rot_offset + 2 * j, rope.rot_offset + 2 * j + 1) if rope.interleaved else
                (rope.rot_offset + j, rope.rot_offset + rope.rot_dim // 2 + j))
        slack[0][..., a] = slack[0][..., b] = 8 * E * m * (np.abs(x[0][..., a]) + np.abs(x[0][..., b]))
        factor = orc.growth(m)
    written = set()
    for which, (cache, got_codes, got_scales) in enumerate(zip(before, c.pools, c.scales)):
        exact = {}
        for i, slot in enumerate(entries):
            if served is not None and i not in served:
                continue
            done = cache.append(table[slot], first[i], x[which][cu[i]:cu[i + 1]], y[which][cu[i]:cu[i + 1]], factor if which == 0 else 1.0)
            for r in done:
                exact[(slot, r)] = cu[i] + r - first[i]
                written.add(cu[i] + r - first[i])
        np.testing.assert_array_equal(got_scales.cpu().numpy(), cache.scales)
        got = got_codes.view(torch.uint8).cpu().numpy()
        if which == 0 and rope is not None:                 # rotated rows by their distance, the rest by their codes
            for (slot, r), t in exact.items():
                p, o = cache.place(table[slot], r)
                s = cache.scales[p, :, o // c.block][:, None].astype(np.float64)
                want = y[0][t] / s
                off = np.abs(orc.VALUES[got[p, :, o]] - want)
                assert (off <= nearest_distance(want) + 2 * slack[0][t] / s).all(), f"row {r} of slot {slot}: {off.max():.3e}"
                cache.codes[p, :, o] = got[p, :, o]
        np.testing.assert_array_equal(got, cache.codes)
    if k_out is not None:
        t = sorted(written)
        err = np.abs(f64(k_out)[t] - y[0][t])
        assert (err <= (HALF_STEP[dtype] * np.abs(y[0][t]) if rope is not None else 0) + slack[0][t]).all()
    return sorted(written)


SHAPES = [("bf16", 8, 2, 128, 128, 16, 16, True), ("bf16", 3, 3, 64, 80, 5, 1, True), ("f32", 4, 1, 256, 64, 64, 8, False),
          ("f32", 4, 4, 48, 48, 1, 1, True), ("bf16", 6, 2, 80, 128, 48, 48, True), ("f32", 2, 2, 64, 64, 128, 64, True),
          ("bf16", 12, 12, 16, 16, 30, 15, False)]


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype,hq,hkv,d,dv,page,block,rotated", SHAPES)
def test_append_writes_rows_and_nothing_else(dtype, hq, hkv, d, dv, page, block, rotated, layout):
    lengths = [0, 1, 33, 64, 100, 7, 90]
    cfg = config(hq, hkv, d, dv, dtype, max_seqs=len(lengths))
    c = Pages8(cfg, page, block, [200] * len(lengths), seed=5, layout=layout)
    c.seq_len.copy_(i32(lengths))
    rope = B.make_rope(rot_dim=d // 2, rot_offset=d // 4, interleaved=layout == "nhd", magnitude=1.25) if rotated else None
    freqs = porc.rope_table(d // 2, 10000.0)
    c.table[3, 80 // page] = 10 ** 6                        # a page that is not there
    # ragged prompts, one into the middle of the rows there are, one over a bad page, one past the table; nothing to add; padding;
    # ids out of range; a slot listed again; a row below zero
    plan = [(0, 0, 37), (2, 20, 50), (3, 64, 70), (1, 1, 0), (-1, 3, 5), (7, 0, 3), (4, 100, c.width * page - 97), (0, 37, 4), (-9, 0, 2), (5, -3, 6),
            (6, 90, 1)]
    served = [0, 1, 2, 3, 6, 10]
    entries, first, n = ([p[i] for p in plan] for i in range(3))
    cu = np.concatenate([[0], np.cumsum(n)]).tolist()
    t = cu[-1] + 3                                          # padding behind the last
    g = torch.Generator(device="cuda").manual_seed(1)
    size = torch.exp2(torch.randint(-6, 7, (t, 1, 1), device="cuda", generator=g).float())      # rows that raise a scale, and that do not
    fused = (torch.randn(t, hq + hkv, d, device="cuda", generator=g) * size).to(DT[dtype])
    q, k = fused[:, :hq], fused[:, hq:]
    v = (torch.randn(t, hkv, dv, device="cuda", generator=g) * size).to(DT[dtype])
    positions = [1000 + 3 * i for i in range(t)] if layout == "hnd" else None
    q_out, k_out = (torch.full((t, h, d), 7.0, dtype=DT[dtype], device="cuda") for h in (hq, hkv))
    before = c.host()
    B.snap_paged_q8_append(cfg, c.paged, i32(entries), i32(cu), i32(first), k, v, *c.cache, c.seq_len, rope=rope,
                           freqs=torch.from_numpy(freqs).cuda() if rotated else None, positions=i32(positions) if rotated and positions else None,
                           q=q, q_out=q_out, k_out=k_out, status=c.status)
    assert c.bits() == B.SNAP_DEV_BAD_SLOT | B.SNAP_DEV_BAD_PAGE
    written = check_append(c, before, entries, first, cu, k, v, rope, freqs, positions, k_out, served, dtype)
    skipped = [i for i in range(t) if i not in written]
    assert (f64(q_out)[skipped] == 7).all() and (f64(k_out)[skipped] == 7).all()
    assert c.seq_len.tolist() == [37, 1, 70, 134, c.width * page, 7, 91]
    if not rotated:
        np.testing.assert_array_equal(f64(q_out)[written], f64(q)[written])


def test_a_block_filled_row_by_row_holds_what_its_scales_say():
    """One row per call with numbers that grow and shrink: the scale only grows, and rows move to it with at most one rounding
    below the smallest normal code."""
    hkv, d, page, block = 2, 64, 32, 16
    cfg = config(2, hkv, d, dtype="f32", max_seqs=1)
    c = Pages8(cfg, page, block, [1], capacity=64, spare=3)
    c.table[0, :2] = i32(c.free[:2])
    c.ks[:], c.vs[:] = float("nan"), float("nan")           # the scale of a block without rows is not looked at
    g = torch.Generator(device="cuda").manual_seed(3)
    sizes = [0, -4, 3, 3, -10, 9, 0, 12, -30, 30, 2, 1, 0, 40, -60, 5, 1, 2, 3]
    x = torch.randn(len(sizes), hkv, d, device="cuda", generator=g) * torch.exp2(torch.tensor(sizes, device="cuda").float())[:, None, None]
    for r in range(len(sizes)):
        before = c.host()
        B.snap_paged_q8_append(cfg, c.paged, i32([0]), i32([0, 1]), i32([r]), x[r:r + 1], -x[r:r + 1], *c.cache, c.seq_len, status=c.status)
        check_append(c, before, [0], [r], [0, 1], x[r:r + 1], -x[r:r + 1])
    assert c.bits() == 0 and c.seq_len.tolist() == [len(sizes)]
    hk = c.host()[0]
    rows, there = hk.rows(c.table[0].tolist(), len(sizes))
    s = np.repeat(hk.scales[c.table[0, 0].item()], block, axis=1)[:, :len(sizes)].T[..., None]
    assert (np.abs(rows - f64(x)) <= 2.0 ** -4 * np.abs(f64(x)) + 2.0 ** -9 * s).all()


def test_numbers_that_are_not_finite_and_that_are_tiny():
    cfg = config(1, 1, 16, dtype="f32", max_seqs=1)
    c = Pages8(cfg, 16, 4, [1], capacity=48, spare=3)
    c.table[0, :3] = i32(c.free[:3])
    x = torch.zeros(24, 1, 16, device="cuda")
    x[0, 0, 3], x[1, 0, 2] = float("nan"), 5.0              # NaN does not count for the scale
    x[4, 0, 1], x[5, 0, 2], x[6, 0, 0] = float("inf"), -1.0, float("-inf")
    x[8, 0, 0], x[9, 0, 1] = 1e-44, -2e-38                  # below what the smallest scale reaches
    x[12, 0, 0], x[13] = 3.4e38, 1e30
    x[16:20] = float("nan")
    before = c.host()
    B.snap_paged_q8_append(cfg, c.paged, i32([0]), i32([0, 24]), i32([0]), x, x, *c.cache, c.seq_len, status=c.status)
    check_append(c, before, [0], [0], [0, 24], x, x)
    page = c.host()[0]
    assert page.scales[c.table[0, 0].item()][0].tolist() == [2.0 ** -6, 2.0 ** 120, 2.0 ** -126, 2.0 ** 120]
    assert page.scales[c.table[0, 1].item()][0, :2].tolist() == [2.0 ** -126, 2.0 ** -126]
    out = torch.empty_like(x)
    B.snap_paged_q8_gather(cfg, c.paged, i32([0]), i32([0, 24]), i32([0]), *c.cache, out, torch.empty_like(x), status=c.status)
    assert torch.isnan(out[0, 0, 3]) and out[1, 0, 2] == 5.0 and out[4, 0, 1] == float("inf") and out[6, 0, 0] == float("-inf")
    assert torch.isnan(out[16:20]).all() and (out[20:] == 0).all()


def raw_append(cfg, c, slots, cu, first, n, t, k, v, rope=None, freqs=None, q=None, q_out=None, k_out=None):
    """By addresses: the buffers need not have n_tokens tokens."""
    at = lambda x: None if x is None else x.data_ptr()  # noqa: E731
    import ctypes as C
    strides = lambda x: (0, 0) if x is None else x.stride()[:2]  # noqa: E731
    rc = B.lib().snap_paged_q8_append(C.byref(cfg), C.byref(c.paged), at(slots), at(cu), at(first), n, t, C.byref(rope) if rope else None, at(freqs),
                                      None, at(q), *strides(q), at(q_out), at(k), *strides(k), at(k_out), at(v), *strides(v), at(c.k), at(c.v),
                                      at(c.ks), at(c.vs), at(c.table), at(c.seq_len), at(c.status), B._stream(None))
    assert rc == 0


@pytest.mark.parametrize("rot", [64, 0])
def test_append_reads_nothing_of_padding(rot):
    """Room for more tokens and entries than there are, in buffers that stop at the last live token; outputs that are inputs."""
    live, d = 70, 64
    cfg = config(4, 2, d, max_seqs=3)
    c = Pages8(cfg, 16, 8, [100] * 3, seed=3)
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(live, h, d, device="cuda", generator=g).to(torch.bfloat16) for h in (4, 2, 2))
    slots, cu, first = [2, -1, 0, -1], [0, 30, 30, live, live], [11, 5, 20, 0]
    freqs = porc.rope_table(64, 10000.0)
    rope = B.make_rope(rot_dim=64) if rot else None
    before, x = c.host(), k.clone()
    raw_append(cfg, c, i32(slots), i32(cu), i32(first), 4, 4096, k, v, rope, torch.from_numpy(freqs).cuda(), q, q, k)
    check_append(c, before, slots, first, cu, x, v, rope, freqs, None, k, [0, 2])
    assert c.bits() == 0 and c.seq_len.tolist() == [60, 100, 41]


@pytest.mark.parametrize("seqs", [40, 700])
def test_a_step_of_single_tokens(seqs):
    """One token per sequence, queries and keys in place, against a prompt's call token by token."""
    cfg = config(32, 8, 128, max_seqs=seqs)
    rng = np.random.default_rng(seqs)
    lengths = rng.integers(0, 90, seqs).tolist()
    c = Pages8(cfg, 32, 16, [x + 1 for x in lengths], seed=1, capacity=96)
    g = torch.Generator(device="cuda").manual_seed(2)
    q, k, v = (torch.randn(seqs, h, 128, device="cuda", generator=g).to(torch.bfloat16) for h in (32, 8, 8))
    order, freqs = rng.permutation(seqs), porc.rope_table(128, 500000.0)
    first = [lengths[s] for s in order]
    before, x, xq = c.host(), k.clone(), q.clone()
    B.snap_paged_q8_append(cfg, c.paged, i32(order.tolist()), i32(list(range(seqs + 1))), i32(first), k, v, *c.cache, c.seq_len,
                           rope=B.make_rope(rot_dim=128), freqs=torch.from_numpy(freqs).cuda(), q=q, q_out=q, k_out=k, status=c.status)
    check_append(c, before, order.tolist(), first, list(range(seqs + 1)), x, v, B.make_rope(rot_dim=128), freqs, None, k)
    want = porc.rotate(f64(xq), first, freqs, 128)
    reach = np.abs(f64(xq)) + np.abs(np.roll(f64(xq), 64, axis=-1))
    assert (np.abs(f64(q) - want) <= HALF_STEP["bf16"] * np.abs(want) + 8 * E * reach).all()
    assert c.bits() == 0 and c.seq_len.tolist() == [x + 1 for x in lengths]


# ---------------------------------------------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------------------------------------------
def run_decode(c, q, slots, stream=None, ws=None, out=None):
    cfg = c.cfg
    if ws is None:
        ws = torch.full((B.snap_paged_q8_decode_workspace_bytes(cfg, c.paged, q.shape[0], q.shape[1]),), 0xff, dtype=torch.uint8, device="cuda")
    if out is None:
        out = torch.full((*q.shape[:3], cfg.d_v), float("nan"), dtype=q.dtype, device="cuda")
    B.snap_paged_q8_decode_attn(cfg, c.paged, q, slots, *c.cache, c.seq_len, out, ws, status=c.status, stream=stream)
    return out


def check_decode(c, q, slots, out, dtype, lengths=None):
    """Every output against the definition; the rows of a KV head at once."""
    hk, hv = c.host()
    table, lengths = c.table.cpu().numpy(), c.seq_len.tolist() if lengths is None else lengths
    got, x, cfg = f64(out), f64(q), c.cfg
    for i, slot in enumerate(slots):
        n = min(max(lengths[slot], 0), c.width * c.page) if 0 <= slot < cfg.max_seqs else 0
        k, there = hk.rows(table[slot] if n else [], n)
        v, _ = hv.rows(table[slot] if n else [], n)
        s = np.array([[hv.scales[p, :, o // c.block] for p, o in [hv.place(table[slot], r)]][0] for r in there]).reshape(len(there), cfg.n_kv_heads)
        for u in range(q.shape[1]):
            seen = int((there < n - q.shape[1] + 1 + u).sum())
            want, _, mass, reach = porc.decode(x[i, u], k[:seen], v[:seen], cfg.softmax_scale)
            d, g = cfg.d_qk, cfg.n_q_heads // cfg.n_kv_heads
            floor, cut = np.zeros_like(want), np.zeros(cfg.n_q_heads)
            for h in range(cfg.n_q_heads if seen else 0):
                kh, size = k[:seen, h // g], np.abs(x[i, u, h])
                z = (kh @ x[i, u, h]) * cfg.softmax_scale
                p = np.exp(z - z.max())
                codes = np.abs(v[:seen, h // g]) / s[:seen, h // g, None]
                floor[h] = 2.0 ** -31 * (p / p.sum() * s[:seen, h // g]).max() * codes.sum(axis=0)
                cut[h] = np.abs(kh).sum(axis=1).max() * 2.0 ** -38 * size.max() * cfg.softmax_scale
            L = (d + 8) * E * reach + cut
            bound = HALF_STEP[dtype] * np.abs(want) + (2 * L[:, None] + 2.0 ** -20 + (2.0 ** -11 if dtype == "bf16" else 0) + 2 * seen * E) * mass
            bound += floor
            err = np.abs(got[i, u] - want)
            assert (err <= bound).all(), f"entry {i} (slot {slot}, {seen} rows), token {u}: {(err - bound).max():.3e} over {bound.max():.3e}"


CASES = [("bf16", 8, 2, 128, 128, 64, 16, 1), ("bf16", 32, 8, 128, 128, 16, 16, 1), ("f32", 8, 2, 128, 128, 32, 8, 1), ("bf16", 12, 12, 64, 64, 16, 4, 1),
         ("bf16", 4, 2, 80, 80, 5, 5, 1), ("bf16", 7, 1, 256, 256, 48, 16, 1), ("f32", 16, 1, 64, 64, 8, 8, 1), ("f32", 3, 3, 256, 128, 64, 64, 1),
         ("bf16", 40, 2, 64, 128, 1, 1, 1), ("f32", 7, 1, 80, 48, 24, 3, 1), ("bf16", 3, 1, 16, 32, 16, 2, 1), ("bf16", 8, 2, 128, 128, 64, 32, 4),
         ("f32", 4, 2, 64, 64, 16, 16, 3), ("bf16", 14, 2, 128, 64, 128, 128, 8), ("bf16", 2, 2, 80, 80, 40, 20, 17), ("f32", 32, 2, 128, 128, 96, 32, 2)]


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype,hq,hkv,d,dv,page,block,q_len", CASES)
def test_attention_matches_its_definition(dtype, hq, hkv, d, dv, page, block, q_len, layout):
    lengths = [0, 1, 2, page, page + 1, 31, 32, 33, 255, 700]
    cfg = config(hq, hkv, d, dv, dtype, max_seqs=len(lengths))
    c = Pages8(cfg, page, block, lengths, seed=d + page, layout=layout)
    g = torch.Generator(device="cuda").manual_seed(4)
    q = (torch.randn(len(lengths), q_len, hq, d, device="cuda", generator=g) * 2).to(DT[dtype])
    slots = np.random.default_rng(1).permutation(len(lengths)).tolist()
    out = run_decode(c, q, i32(slots))
    assert c.bits() == 0
    check_decode(c, q, slots, out, dtype)
    again = run_decode(c, q, i32(slots))
    assert torch.equal(out, again)
    if q_len == 1:                                          # without the dim of tokens
        flat = torch.empty(len(lengths), hq, dv, dtype=q.dtype, device="cuda")
        ws = torch.empty(B.snap_paged_q8_decode_workspace_bytes(cfg, c.paged, len(lengths)), dtype=torch.uint8, device="cuda")
        B.snap_paged_q8_decode_attn(cfg, c.paged, q[:, 0].contiguous(), i32(slots), *c.cache, c.seq_len, flat, ws)
        assert torch.equal(flat, out[:, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lengths,q_len", [([5124], 1), ([9001, 3, 6000], 1), ([4000, 7777], 5), ([33] * 150, 1), ([700] * 131 + [0, 5000], 2)])
def test_long_and_many_sequences(lengths, q_len, dtype):
    """Sequences that many blocks share, and more of them than a block holds the lengths of."""
    cfg = config(8, 2, 128, dtype=dtype, max_seqs=len(lengths))
    c = Pages8(cfg, 64, 16, lengths, seed=7)
    g = torch.Generator(device="cuda").manual_seed(8)
    q = (torch.randn(len(lengths), q_len, 8, 128, device="cuda", generator=g) * 3).to(DT[dtype])
    slots = list(range(len(lengths)))
    out = run_decode(c, q, i32(slots))
    assert c.bits() == 0
    some = slots if len(slots) < 10 else [0, 1, 64, 127, 128, 129, len(slots) - 2, len(slots) - 1]
    check_decode(c, q[some], some, out[some], dtype)
    if len(slots) >= 10:                                    # the others are whole numbers' worth of finite outputs
        assert torch.isfinite(out.float()).all()


@pytest.mark.parametrize("dtype,hq,hkv,d,page,block", [("bf16", 8, 2, 128, 64, 16), ("bf16", 4, 2, 64, 8, 8), ("f32", 3, 1, 80, 5, 1), ("f32", 8, 2, 128, 16, 16)])
def test_rows_and_sequences_that_are_not_there(dtype, hq, hkv, d, page, block):
    lengths = [3 * page + 2, 300, 6 * page, 0, 20, 40]
    cfg = config(hq, hkv, d, dtype=dtype, max_seqs=6)
    c = Pages8(cfg, page, block, lengths, seed=8)
    c.table[0, 1] = -1
    c.table[1, 0] = 10 ** 6
    c.table[1, 150 // page] = c.k.shape[0]
    c.table[2, :] = -5                                      # nothing of this one is there
    c.seq_len.copy_(i32([lengths[0], lengths[1], lengths[2], -4, c.width * page + 9, 40]))
    c.table[4, :] = c.table[5, 0].item()                    # (as long as the table: the same page again and again, but for what is NaN)
    c.table[4, 1:] = -1
    g = torch.Generator(device="cuda").manual_seed(2)
    slots = [0, 1, 2, 3, 4, 5, -1, 6, -7, 5]
    q = torch.randn(len(slots), 2, hq, d, device="cuda", generator=g).to(DT[dtype])
    out = run_decode(c, q, i32(slots))
    assert c.bits() == B.SNAP_DEV_BAD_SLOT | B.SNAP_DEV_BAD_PAGE
    if 40 >= page:
        check_decode(c, q, slots, out, dtype)
    for i in (2, 3, 6, 7, 8):
        assert (out[i] == 0).all()
    c.status.zero_()
    c.table[2, :] = c.table[5, 0].item()
    run_decode(c, q[6:7], i32([-1]))
    assert c.bits() == 0                                    # padding is nothing to report


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scales_far_apart(dtype):
    """Blocks whose scales differ by up to 2^80, with the weight on the small ones, on the large ones, and on none."""
    hkv, d, page, block = 2, 64, 16, 4
    cfg = config(4, hkv, d, dtype=dtype, max_seqs=3, scale=1.0)
    c = Pages8(cfg, page, block, [130, 67, 40], seed=3)
    rng = np.random.default_rng(5)
    for slot, n in ((0, 130), (1, 67), (2, 40)):
        for b in range(-(-n // block)):
            p, o = c.table[slot, b * block // page].item(), b * block % page // block
            c.vs[p, :, o] = 2.0 ** float(rng.integers(-60, 20))
            c.ks[p, :, o] = 2.0 ** float(rng.integers(-40, -9) if slot < 2 else -120)
    q = torch.randn(3, 1, 4, d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(DT[dtype])
    q[1] *= 2.0 ** -20
    q[0, 0, 0, 5] = 2.0 ** 10                               # numbers of one query far apart as well
    out = run_decode(c, q, i32([0, 1, 2]))
    assert c.bits() == 0
    check_decode(c, q, [0, 1, 2], out, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_row_comes_back_as_it_is(dtype):
    cfg = config(8, 2, 128, dtype=dtype, max_seqs=2)
    c = Pages8(cfg, 64, 16, [1, 1], seed=9, spread=30)
    q = torch.randn(2, 1, 8, 128, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(DT[dtype])
    out = f64(run_decode(c, q, i32([1, 0])))
    for i, slot in enumerate((1, 0)):
        v, _ = c.host()[1].rows(c.table[slot].tolist(), 1)
        np.testing.assert_array_equal(out[i, 0], np.repeat(v[0], 4, axis=0))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_numbers_that_are_not_finite_stay_where_they_are(dtype):
    """A NaN key reaches its KV head's outputs, a NaN value its column; other heads, sequences and earlier rows are as without."""
    cfg = config(4, 2, 64, dtype=dtype, max_seqs=3)
    c = Pages8(cfg, 16, 8, [100, 100, 100], seed=4)
    q = torch.randn(3, 1, 4, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(DT[dtype])
    clean = run_decode(c, q, i32([0, 1, 2])).clone()
    kb, vb = c.k.view(torch.uint8), c.v.view(torch.uint8)
    kb[c.table[0, 3].item(), 1, 5, 7] = 0xff                # NaN key, head 1
    vb[c.table[1, 6].item(), 0, 3, 9] = 0x7f                # NaN value, head 0, column 9
    out = run_decode(c, q, i32([0, 1, 2]))
    assert torch.isnan(out[0, 0, 2:].float()).all() and torch.equal(out[0, 0, :2], clean[0, 0, :2])
    assert torch.isnan(out[1, 0, :2, 9].float()).all() and torch.equal(out[1, 0, 2:], clean[1, 0, 2:]) and torch.equal(out[2], clean[2])
    keep = [x for x in range(64) if x != 9]
    assert torch.equal(out[1, 0, :2, keep], clean[1, 0, :2, keep])
    qn = q.clone()
    qn[2, 0, 1, 0] = float("nan")                           # a NaN query: its own output alone
    out = run_decode(c, qn, i32([0, 1, 2]))
    assert torch.isnan(out[2, 0, 1].float()).all() and torch.equal(out[2, 0, [0, 2, 3]], clean[2, 0, [0, 2, 3]])


def test_pools_past_32_bits():
    """Codes, pages and strides whose offsets pass 2^32."""
    cfg = config(4, 2, 64, max_seqs=2)
    page, pages, stride = 16, 40, 2 ** 27 + 48
    c = Pages8(cfg, page, 4, [300, 77], seed=6, spare=pages - 19 - 5)
    assert c.k.shape[0] == pages
    wide = []
    for t in c.pools:
        big = torch.zeros(stride * pages, dtype=torch.uint8, device="cuda")
        view = big.as_strided((pages, 2, page, 64), (stride, 64 * page, 64, 1))
        view.copy_(t.view(torch.uint8))
        wide.append(view.view(CODE))
    q = torch.randn(2, 1, 4, 64, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).to(torch.bfloat16)
    near = run_decode(c, q, i32([0, 1]))
    kv = [torch.empty(50, 2, 64, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    lists = (i32([0]), i32([0, 50]), i32([250]))
    B.snap_paged_q8_gather(cfg, c.paged, *lists, *c.cache, kv[0], kv[1])
    c.pools = wide
    c.describe()
    assert torch.equal(run_decode(c, q, i32([0, 1])), near)
    B.snap_paged_q8_gather(cfg, c.paged, *lists, *c.cache, kv[2], kv[3])
    assert torch.equal(kv[0], kv[2]) and torch.equal(kv[1], kv[3])
    before = c.host()
    B.snap_paged_q8_append(cfg, c.paged, *lists, kv[0] * 3, kv[1], *c.cache, c.seq_len, status=c.status)
    check_append(c, before, [0], [250], [0, 50], kv[0] * 3, kv[1])
    assert c.bits() == 0


# ---------------------------------------------------------------------------------------------------------------
# gather
# ---------------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype,hkv,d,dv,page,block", [("bf16", 2, 128, 128, 64, 16), ("f32", 3, 80, 16, 5, 5), ("bf16", 1, 64, 256, 16, 1), ("f32", 8, 48, 64, 30, 6)])
def test_gather_reads_rows_back(dtype, hkv, d, dv, page, block, layout):
    lengths = [200, 1, 130]
    cfg = config(hkv, hkv, d, dv, dtype, max_seqs=3)
    c = Pages8(cfg, page, block, lengths, seed=5, layout=layout, spread=20)
    c.table[2, 60 // page] = -1
    plan = [(0, 13, 150), (2, 0, 130), (-1, 0, 4), (0, 0, 200), (1, 0, 1), (1, 0, 0), (3, 0, 5), (0, c.width * page - 2, 0), (2, -1, 3)]
    slots, first, n = ([p[i] for p in plan] for i in range(3))
    cu = np.concatenate([[0], np.cumsum(n)]).tolist()
    t = cu[-1] + 5
    k = torch.full((hkv, t, d), 7.0, dtype=DT[dtype], device="cuda").transpose(0, 1)     # head-major output
    v = torch.full((t, hkv, dv + 16), 7.0, dtype=DT[dtype], device="cuda")[..., :dv]
    B.snap_paged_q8_gather(cfg, c.paged, i32(slots), i32(cu), i32(first), *c.cache, k, v, status=c.status)
    assert c.bits() == B.SNAP_DEV_BAD_SLOT | B.SNAP_DEV_BAD_PAGE
    for got, cache in zip((k, v), c.host()):
        want = np.full(got.shape, 7.0)
        for i in (0, 1, 3, 4):
            rows, there = cache.rows(c.table[slots[i]].tolist(), n[i], first[i])
            want[cu[i] + there - first[i]] = rows
        np.testing.assert_array_equal(f64(got), f64(torch.from_numpy(want).to(DT[dtype])))


# ---------------------------------------------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------------------------------------------
def test_a_server_plans_appends_attends_and_compresses():
    """Prompts planned and appended, steps of one and of three tokens with their drafts taken back, a sequence that ends and
    another in its pages, and a prompt read back for its attention and its compression."""
    hq, hkv, d, page, block, seqs, pool = 8, 2, 128, 16, 8, 4, 60
    cfg = config(hq, hkv, d, max_seqs=seqs)
    c = Pages8(cfg, page, block, [0] * seqs, capacity=400, spare=pool)
    c.ks[:], c.vs[:] = float("nan"), float("nan")
    free, n_free = i32(c.free), i32([pool])
    rope, freqs = B.make_rope(rot_dim=d, base=500000.0), porc.rope_table(d, 500000.0)
    fr = torch.from_numpy(freqs).cuda()
    g = torch.Generator(device="cuda").manual_seed(0)
    truth = {s: [np.zeros((0, hkv, d))] * 2 for s in range(seqs)}       # what was appended, in double precision

    def step(requests, most, attend=True):
        n = len(requests)
        slots, new = i32([s for s, _ in requests]), i32([x for _, x in requests])
        first, cu, ts, tr = i32([0] * n), i32([0] * (n + 1)), i32([0] * most), i32([0] * most)
        ws = torch.empty(B.snap_paged_plan_workspace_bytes(cfg, c.paged, n), dtype=torch.uint8, device="cuda")
        B.snap_paged_plan(cfg, c.paged, slots, new, c.table, c.seq_len, free, n_free, first, cu, ts, tr, ws, status=c.status)
        q, k, v = (torch.randn(most, h, d, device="cuda", generator=g).to(torch.bfloat16) for h in (hq, hkv, hkv))
        raw, ko = k.clone(), torch.empty_like(k)
        B.snap_paged_q8_append(cfg, c.paged, slots, cu, first, k, v, *c.cache, c.seq_len, rope=rope, freqs=fr, q=q, q_out=q, k_out=ko,
                               status=c.status)
        # rope's own call agrees on the keys, rows being positions
        other = torch.empty_like(k)
        B.snap_rope(cfg, rope, fr, tr, k=raw, k_out=other)
        total = int(cu[-1].item())
        assert torch.equal(other[:total], ko[:total])
        for i, (s, x) in enumerate(requests):
            if x < 0:
                truth[s] = [np.zeros((0, hkv, d))] * 2
            a, b, f = int(cu[i].item()), int(cu[i + 1].item()), int(first[i].item())
            truth[s] = [np.concatenate([t[:f], f64(z)[a:b]]) for t, z in zip(truth[s], (ko, v))]
        lens = {x for _, x in requests}
        if attend and len(lens) == 1 and min(lens) > 0:
            ql = lens.pop()
            qs = q[:n * ql].view(n, ql, hq, d)
            out = run_decode(c, qs, slots)
            check_decode(c, qs, [s for s, _ in requests], out, "bf16")
        return q, ts, tr

    step([(0, 130), (2, 77), (1, 40)], 300)
    for _ in range(3):
        step([(2, 1), (0, 1), (1, 1)], 3)
    step([(0, 3), (1, 3), (2, 3)], 9)
    c.seq_len.sub_(i32([2, 0, 3, 0]))                       # drafts taken back: their pages stay with the rows
    step([(0, 2), (1, 2), (2, 2)], 6)
    step([(0, -1), (3, 200), (1, 1)], 201, attend=False)    # one ends, its pages go to another
    step([(0, 21)], 21)
    assert c.bits() == 0
    lens = c.seq_len.tolist()
    held = c.table[c.table >= 0].tolist()
    assert lens == [21, 40 + 3 + 3 + 2 + 1, 77 + 3 + 3 - 3 + 2, 200] and len(set(held)) == len(held) and len(held) + int(n_free.item()) == pool
    for s in range(seqs):                                   # the cache holds what was appended, in 4 bits of precision
        assert len(truth[s][0]) == lens[s]
        for cache, t in zip(c.host(), truth[s]):
            rows, there = cache.rows(c.table[s].tolist(), lens[s])
            scale = np.stack([[cache.scales[p, :, o // block] for p, o in [cache.place(c.table[s].tolist(), r)]][0] for r in there])[..., None]
            assert (np.abs(rows - t) <= (2.0 ** -4 + 2.0 ** -8) * np.abs(t) + 2.0 ** -9 * scale).all()
    # a prompt back as keys and values: its attention and its compression take them
    n = lens[3]
    k, v = (torch.empty(n, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    B.snap_paged_q8_gather(cfg, c.paged, i32([3]), i32([0, n]), i32([0]), *c.cache, k, v, status=c.status)
    q = torch.randn(n, hq, d, device="cuda", generator=g).to(torch.bfloat16)
    attn = torch.empty_like(q)
    B.snap_prefill_attn(cfg, q, k, v, [0, n], attn)
    last = run_decode(c, q[-1:].view(1, 1, hq, d), i32([3]))
    # both within a bf16 step or two of the exact average of numbers of size one
    assert (attn[-1].float() - last[0, 0].float()).abs().max() <= 2.0 ** -6
    lay = B.snap_cache_layout(cfg)
    buf = B.alloc_cache(cfg, lay)
    ws = torch.empty(B.snap_compress_workspace_bytes(cfg, [0, n]), dtype=torch.uint8, device="cuda")
    B.snap_compress(cfg, lay, q[-1:].view(1, hq, 1, d).contiguous(), k, v, [0, n], [0], buf.k_cache, buf.v_cache, buf.seq_len, buf.valid_topk, None, ws,
                    buf.status)
    assert torch.equal(buf.k_cache[0, :, :2], k[:2].transpose(0, 1)) and int(buf.seq_len[0].item()) == n


def test_captured_replayed_and_on_other_streams():
    """Calls captured into a graph and replayed with other inputs; two streams at once with scratch of their own."""
    hq, hkv, d = 8, 2, 64
    cfg = config(hq, hkv, d, max_seqs=5)
    c = Pages8(cfg, 16, 8, [300, 0, 17, 64, 129], seed=2, capacity=320)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(5, 2, hq, d, device="cuda", generator=g).to(torch.bfloat16)
    slots = i32([0, 1, 2, 3, 4])
    eager = run_decode(c, q, slots)
    check_decode(c, q, [0, 1, 2, 3, 4], eager, "bf16")
    ws = [torch.empty(B.snap_paged_q8_decode_workspace_bytes(cfg, c.paged, 5, 2), dtype=torch.uint8, device="cuda") for _ in range(2)]
    outs = [torch.zeros_like(q) for _ in range(2)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(10):
        run_decode(c, q, slots, stream=side, ws=ws[0], out=outs[0])
        run_decode(c, q, slots, ws=ws[1], out=outs[1])
    torch.cuda.synchronize()
    assert torch.equal(outs[0], eager) and torch.equal(outs[1], eager)
    graphs = []
    for _ in range(2):                                      # two graphs that share one scratch, replayed in turn
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            run_decode(c, q, slots, ws=ws[0], out=outs[0])
        graphs.append(graph)
    for lengths, order in (([40, 300, 1, 0, 7], [4, 3, 2, 1, 0]), ([320, 320, 320, 320, 320], [0, 0, 1, -1, 2])):
        c.table[:] = c.table[0].clone()
        c.table[:, 300 // 16:] = c.table[0, :2].clone()
        c.seq_len.copy_(i32([min(x, 299) for x in lengths]))
        slots.copy_(i32(order))
        for graph in graphs:
            outs[0].fill_(float("nan"))
            graph.replay()
            torch.cuda.synchronize()
            check_decode(c, q, order, outs[0], "bf16")
    # the append and the gather, replayed
    k, v = (torch.randn(40, hkv, d, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
    kb, vb = torch.zeros_like(k), torch.zeros_like(v)
    c = Pages8(cfg, 16, 8, [100] * 5, seed=3)
    lists = [i32([1, 3, -1]), i32([0, 9, 40, 40]), i32([50, 7, 0])]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.snap_paged_q8_append(cfg, c.paged, *lists, k, v, *c.cache, c.seq_len, status=c.status)
        B.snap_paged_q8_gather(cfg, c.paged, *lists, *c.cache, kb, vb, status=c.status)
    for entries, cu, first in (([1, 3, -1], [0, 9, 40, 40], [50, 7, 0]), ([4, -1, 0], [0, 1, 1, 39], [63, 0, 21])):
        for t, x in zip(lists, (entries, cu, first)):
            t.copy_(i32(x))
        k.mul_(4)
        before = c.host()
        graph.replay()
        torch.cuda.synchronize()
        check_append(c, before, entries, first, cu, k, v, served=[i for i in range(3) if entries[i] >= 0])
        for got, cache in zip((kb, vb), c.host()):
            for i in range(3):
                if entries[i] >= 0:
                    rows, _ = cache.rows(c.table[entries[i]].tolist(), cu[i + 1] - cu[i], first[i])
                    np.testing.assert_array_equal(f64(got)[cu[i]:cu[i + 1]], rows)
    assert c.bits() == 0
