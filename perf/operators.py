"""Rotary positions, a paged key-value cache with the attention that reads it, and eviction by accumulated attention weight.

Each case is one call of a serving program next to the compressed cache: rotating the queries and keys of a
prompt or a step (``rope``), writing new tokens' rows into the pages of their sequences (``append``), attention
of one new token per sequence over its pages (``decode``, with or without the attention weights that eviction
goes by), and keeping the sinks, the last tokens and the tokens that gathered most weight (``evict``).  With
``own`` false, ``run`` computes them in elementary torch operations; with ``own`` true through the library.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    llama = dict(hq=32, hkv=8, d=128, dtype="bf16")
    return [
        # the queries and keys of one 32k-token prompt, before its attention pass
        dict(name="rope_prompt_32k", op="rope", **llama, tokens=32768, rot=128, offset=0, interleaved=False, scaling="llama3",
             first=0, inverse=False),
        # the gradient of a partly rotated single-precision layer at far positions
        dict(name="rope_f32_partial_grad", op="rope", hq=8, hkv=2, d=128, dtype="f32", tokens=1537, rot=64, offset=0,
             interleaved=True, scaling="yarn", first=100003, inverse=True),
        # one step of 32 sequences: rotate, write key and value to the last page (the smallest call)
        dict(name="append_step_32seq", op="append", **llama, seqs=32, tokens=32, rows=90001, page=16, layout="nhd", rope=True,
             outputs=True),
        # three ragged prompts, rotated on the way into their pages
        dict(name="append_prompts_26k", op="append", **llama, seqs=3, tokens=26003, rows=12000, page=64, layout="hnd", rope=True,
             outputs=True),
        # one sequence at the compressed cache's size: latency
        dict(name="decode_1seq_5k", op="decode", **llama, seqs=1, shortest=5124, longest=5124, page=16, layout="hnd", weights=False),
        # ragged long sequences, uncompressed (the largest call)
        dict(name="decode_16seq_8k_64k", op="decode", **llama, seqs=16, shortest=8192, longest=65536, page=64, layout="nhd", weights=False),
        # many short sequences, one of them still empty: no head is shared
        dict(name="decode_45seq_short", op="decode", hq=12, hkv=12, d=64, dtype="bf16", seqs=45, shortest=0, longest=333, page=16,
             layout="hnd", weights=False),
        # the single-precision configuration
        dict(name="decode_f32_4seq", op="decode", hq=8, hkv=2, d=128, dtype="f32", seqs=4, shortest=2001, longest=4100, page=32,
             layout="hnd", weights=False),
        # steps that gather the weights eviction goes by: one sequence, and a batch
        dict(name="decode_weights_1seq_6k", op="decode", **llama, seqs=1, shortest=6148, longest=6148, page=64, layout="hnd", weights=True),
        dict(name="decode_weights_8seq_16k", op="decode", **llama, seqs=8, shortest=9000, longest=16384, page=64, layout="hnd", weights=True),
        # a full cache is cut back to the compressed cache's size: one sequence after 1024 steps, and long prompts
        dict(name="evict_1seq_6k", op="evict", **llama, seqs=1, shortest=6148, longest=6148, page=64, layout="hnd", sink=4, recent=1024,
             topk=4096),
        dict(name="evict_12seq_32k", op="evict", **llama, seqs=12, shortest=700, longest=32768, page=64, layout="nhd", sink=4,
             recent=1024, topk=4096),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "decode", "decode", "decode", "evict"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    hkv = rng.choice([1, 2, 3, 4, 8])
    c = dict(op=op, hkv=hkv, hq=hkv * rng.choice([1, 2, 4, 4, 7, 8, 16]), d=rng.choice([64, 80, 128, 128, 256]), dtype=dtype)
    token = (c["hq"] + 2 * hkv) * c["d"] * (2 if dtype == "bf16" else 4)          # bytes of a token's queries, keys and values
    row = 2 * hkv * c["d"] * (2 if dtype == "bf16" else 4)                        # bytes of a cache row
    if op == "rope":
        rot = rng.choice([c["d"], c["d"] // 2])
        return dict(c, tokens=_log_int(rng, 1, max(2, min(40000, 400_000_000 // token))), rot=rot,
                    offset=rng.choice([0, c["d"] - rot]), interleaved=rng.random() < 0.5,
                    scaling=rng.choice(["plain", "linear", "llama3", "yarn"]), first=_log_int(rng, 1, 900000), inverse=rng.random() < 0.3)
    c.update(page=rng.choice([1, 8, 16, 16, 32, 48, 64, 128]) if op == "decode" else rng.choice([5, 16, 32, 64]),
             layout=rng.choice(["hnd", "nhd"]))
    if op == "append":
        seqs = rng.randint(1, 40)
        return dict(c, seqs=seqs, tokens=seqs if rng.random() < 0.5 else max(seqs, _log_int(rng, seqs, max(seqs + 1, 400_000_000 // token // 2))),
                    rows=_log_int(rng, 1, 60000), rope=rng.random() < 0.7, outputs=rng.random() < 0.7)
    seqs = _log_int(rng, 1, 48)
    if op == "decode":
        weights = rng.random() < 0.4
        # what the plain form keeps: rows in 32 bits, padded to the longest sequence
        longest = _log_int(rng, 1, max(16, min(60000, 900_000_000 // (seqs * row), 100_000_000 // (seqs * c["hq"]))))
        return dict(c, seqs=seqs, shortest=rng.randint(0, longest), longest=longest, weights=weights)
    seqs = min(seqs, 12)
    longest = _log_int(rng, 10, max(16, min(40000, 400_000_000 // (seqs * row))))
    return dict(c, seqs=seqs, shortest=rng.randint(0, longest), longest=longest, sink=rng.choice([0, 4, 17]),
                recent=_log_int(rng, 1, 1500), topk=rng.choice([0, _log_int(rng, 1, 5000), _log_int(rng, 1, 5000)]))


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _frequencies(rot, scaling):
    """Radians per position of the rot / 2 pairs, in double precision: the handle that a program keeps."""
    base, factor, original = 500000.0, 8.0, 8192.0
    f = base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    if scaling == "linear":
        return f / factor
    if scaling == "llama3":                                 # long waves stretched, short ones kept, a ramp between
        turns = original * f / (2 * math.pi)
        smooth = ((turns - 1.0) / 3.0).clamp(0.0, 1.0)
        return f * (smooth + (1.0 - smooth) / factor)
    if scaling == "yarn":                                   # a linear ramp over the pair's index
        at = lambda n: rot * math.log(original / (n * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), rot - 1)
        ramp = ((torch.arange(rot // 2, dtype=torch.float64) - low) / max(high - low, 1e-3)).clamp(0.0, 1.0)
        return f * ((1.0 - ramp) + ramp / factor)
    return f


def _magnitude(scaling):
    return 0.1 * math.log(8.0) + 1.0 if scaling == "yarn" else 1.0


def _pool(c, pages, g):
    """Key and value pages [pages, heads, rows of a page, d] (stored heads first or rows first), and each KV head's
    direction that some keys and all queries share, so that a few tokens draw most of the attention."""
    shape = (pages, c["hkv"], c["page"], c["d"]) if c["layout"] == "hnd" else (pages, c["page"], c["hkv"], c["d"])
    k = torch.empty(shape, dtype=DTYPES[c["dtype"]], device="cuda").normal_(generator=g)
    v = torch.empty(shape, dtype=DTYPES[c["dtype"]], device="cuda").normal_(generator=g)
    if c["layout"] == "nhd":
        k, v = k.transpose(1, 2), v.transpose(1, 2)
    u = torch.randn(c["hkv"], 1, c["d"], device="cuda", generator=g)
    u = u / u.norm(dim=-1, keepdim=True)
    rank = torch.rand(pages, c["hkv"], c["page"], 1, device="cuda", generator=g) * 4000 + 1
    k.addcmul_((8.0 * rank.pow(-1.1)).to(k.dtype), u.to(k.dtype))
    return k, v, u


def _table(lengths, seqs, page, width, g, pool=0):
    """Page table [seqs, width]: each sequence's pages anywhere in the pool, -1 past its last one; and the pool's size."""
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(max(sum(need), pool) + 3, generator=g, device="cuda").to(torch.int32)
    table = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, int(order.numel())


def _lengths(c, seed):
    r = torch.Generator().manual_seed(seed)
    n = torch.randint(c["shortest"], c["longest"] + 1, (c["seqs"],), generator=r).tolist()
    n[-1] = c["longest"]
    n[0] = c["shortest"] if c["seqs"] > 1 else n[0]
    return n


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g).to(dt)  # noqa: E731
    s = dict(c, dt=dt)
    if c["op"] == "rope":
        t = c["tokens"]
        s.update(q=normal(t, c["hq"], c["d"]), k=normal(t, c["hkv"], c["d"]),
                 positions=torch.arange(c["first"], c["first"] + t, dtype=torch.int32, device="cuda"),
                 freqs=_frequencies(c["rot"], c["scaling"]).cuda(), magnitude=_magnitude(c["scaling"]))
        s.update(q_out=torch.empty_like(s["q"]), k_out=torch.empty_like(s["k"]))
        return s
    if c["op"] == "append":
        t, n, page = c["tokens"], c["seqs"], c["page"]
        each = [t // n + (1 if i < t % n else 0) for i in range(n)]     # a prompt's tokens are consecutive rows
        start = torch.randint(c["rows"] // 2, c["rows"] + 1, (n,), generator=torch.Generator().manual_seed(seed)).tolist()
        width = -(-(max(start) + max(each) + 1) // page)
        table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
        firsts = [b // page for b in start]
        counts = [(b + e - 1) // page - f + 1 for b, e, f in zip(start, each, firsts)]
        most = sum((e - 1) // page + 2 for e in each)
        order = torch.randperm(most, generator=g, device="cuda").to(torch.int32)
        at = 0
        for i in range(n):                                              # the pages of the rows before are elsewhere
            table[i, firsts[i]:firsts[i] + counts[i]] = order[at:at + counts[i]]
            at += counts[i]
        k_pages, v_pages, _ = _pool(c, int(order.numel()), g)
        cat = lambda xs: torch.cat([torch.arange(*x, dtype=torch.int32) for x in xs]).cuda()  # noqa: E731
        s.update(q=normal(t, c["hq"], c["d"]), k=normal(t, c["hkv"], c["d"]), v=normal(t, c["hkv"], c["d"]),
                 rows_dev=cat([(b, b + e) for b, e in zip(start, each)]),
                 slots=torch.cat([torch.full((e,), i, dtype=torch.int32) for i, e in enumerate(each)]).cuda(),
                 seq_len=torch.tensor(start, dtype=torch.int32, device="cuda"), table=table, k_pages=k_pages, v_pages=v_pages,
                 freqs=_frequencies(c["d"], "llama3").cuda(), magnitude=1.0)
        s.update(q_out=torch.empty_like(s["q"]), k_out=torch.empty_like(s["k"]))
        return s
    lengths, page, n = _lengths(c, seed), c["page"], c["seqs"]
    width = max(-(-c["longest"] // page), 1)
    if c["op"] == "decode":
        table, pages = _table(lengths, n, page, width, g)
        k_pages, v_pages, u = _pool(c, pages, g)
        q = torch.randn(n, c["hkv"], c["hq"] // c["hkv"], c["d"], device="cuda", generator=g) + u * math.sqrt(c["d"]) * 0.5
        s.update(q=q.reshape(n, c["hq"], c["d"]).to(dt), table=table, k_pages=k_pages, v_pages=v_pages,
                 slots=torch.randperm(n, generator=g, device="cuda").to(torch.int32),
                 seq_len=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
        s["out"] = torch.empty(n, c["hq"], c["d"], dtype=dt, device="cuda")
        if c["weights"]:
            s["weights_in"] = torch.rand(n, c["hkv"], width * page, device="cuda", generator=g) ** 4
            s["weights_out"] = torch.zeros(n, c["hkv"], width * page, device="cuda")
        return s
    keep = c["sink"] + c["recent"] + c["topk"]
    both = lengths + [min(x, keep) for x in lengths]                    # each sequence, and the slot it is cut back into
    table, pages = _table(both, 2 * n, page, width, g, pool=n * (width + min(width, -(-keep // page))))
    k_pages, v_pages, _ = _pool(c, pages, g)
    s.update(table=table, k_pages=k_pages, v_pages=v_pages, src=torch.arange(n, dtype=torch.int32, device="cuda"),
             dst=torch.arange(n, 2 * n, dtype=torch.int32, device="cuda"),
             seq_len=torch.tensor(lengths + [0] * n, dtype=torch.int32, device="cuda"),
             weights=torch.rand(2 * n, c["hkv"], width * page, device="cuda", generator=g) ** 4 * 30,
             kept=torch.empty(n, c["hkv"], keep, dtype=torch.int32, device="cuda"))
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _rotate(x, cos, sin, rot, offset, interleaved):
    """x [T, H, d]; cos, sin [T, rot / 2]: pair (a, b) becomes (a cos - b sin, b cos + a sin)."""
    y = x.float()
    part = y[..., offset:offset + rot]
    a, b = (part[..., 0::2], part[..., 1::2]) if interleaved else (part[..., :rot // 2], part[..., rot // 2:])
    cos, sin = cos[:, None, :], sin[:, None, :]
    pair = (a * cos - b * sin, b * cos + a * sin)
    turned = torch.stack(pair, dim=-1).flatten(-2) if interleaved else torch.cat(pair, dim=-1)
    return torch.cat([y[..., :offset], turned, y[..., offset + rot:]], dim=-1).to(x.dtype)


def _cos_sin(positions, freqs, magnitude, inverse):
    angle = positions.double()[:, None] * freqs                         # in 64 bits: far positions
    return (angle.cos() * magnitude).float(), (angle.sin() * (-magnitude if inverse else magnitude)).float()


def _plain_rope(s):
    cos, sin = _cos_sin(s["positions"], s["freqs"], s["magnitude"], s["inverse"])
    return [_rotate(x, cos, sin, s["rot"], s["offset"], s["interleaved"]) for x in (s["q"], s["k"])]


def _plain_append(s):
    q, k, page = s["q"], s["k"], s["page"]
    if s["rope"]:
        cos, sin = _cos_sin(s["rows_dev"], s["freqs"], s["magnitude"], False)
        k = _rotate(k, cos, sin, s["d"], 0, False)
        q = _rotate(q, cos, sin, s["d"], 0, False) if s["outputs"] else q
    slots, rows = s["slots"].long(), s["rows_dev"].long()
    pages = s["table"][slots, rows // page].long()
    s["k_pages"][pages, :, rows % page] = k
    s["v_pages"][pages, :, rows % page] = s["v"]
    s["seq_len"].scatter_reduce_(0, slots, s["rows_dev"] + 1, "amax")
    return [s["k_pages"], s["v_pages"], s["seq_len"]] + ([q, k] if s["outputs"] else [])


def _all_rows(pages, table):
    """[n, heads, rows, d] in 32 bits: the rows of a page table's pages in order."""
    x = pages[table.clamp(min=0).long()]                                # [n, width, heads, page, d]
    n, w, h, p, d = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(n, h, w * p, d).float()


def _plain_decode(s):
    slots, n = s["slots"].long(), s["seqs"]
    table, length = s["table"][slots], s["seq_len"][slots]
    k = _all_rows(s["k_pages"], table)
    there = torch.arange(k.shape[2], device=k.device) < length[:, None]
    q = s["q"].float().reshape(n, s["hkv"], -1, s["d"])
    x = (q @ k.transpose(2, 3)) * (1.0 / math.sqrt(s["d"]))
    del k
    x = x.masked_fill(~there[:, None, None], -math.inf)
    p = torch.exp(x - x.amax(dim=-1, keepdim=True).clamp(min=-1e30))    # a sequence with no row: all zero
    p = p / p.sum(dim=-1, keepdim=True).clamp(min=1e-30)
    out = (p @ _all_rows(s["v_pages"], table)).reshape(n, s["hq"], s["d"]).to(s["dt"])
    if not s["weights"]:
        return [out]
    s["weights_out"][slots] = torch.where(there[:, None], s["weights_in"][slots] + p.sum(dim=2), s["weights_out"][slots])
    return [out, s["weights_out"]]


def _plain_evict(s):
    src, dst, page, sink, recent, topk = s["src"].long(), s["dst"].long(), s["page"], s["sink"], s["recent"], s["topk"]
    keep = sink + recent + topk
    length = s["seq_len"][src].long()[:, None, None]
    w = s["weights"][src]                                               # [n, heads, rows]
    row = torch.arange(w.shape[2], device=w.device)
    may = (row >= sink) & (row < length - recent)
    order = torch.sort(w.masked_fill(~may, -math.inf), dim=2, descending=True, stable=True).indices[..., :topk]
    if order.shape[2] < topk:
        order = torch.cat([order, order.new_zeros(*order.shape[:2], topk - order.shape[2])], dim=2)
    r = torch.arange(keep, device=w.device).expand(*w.shape[:2], keep)
    middle = torch.cat([order.sort(dim=2).values, order.new_zeros(*order.shape[:2], 1)], dim=2).gather(2, (r - sink).clamp(0, topk))
    cut = torch.where(r < sink, r, torch.where(r < sink + topk, middle, r - keep + length))
    rows = torch.where(length > keep, cut, r)                           # a sequence within the budget keeps every row
    there = r < length
    i, h, to = there.nonzero(as_tuple=True)
    at = rows[there]
    from_page, to_page = s["table"][src[i], at // page].long(), s["table"][dst[i], to // page].long()
    for pages in (s["k_pages"], s["v_pages"]):
        pages[to_page, h, to % page] = pages[from_page, h, at % page]
    s["weights"][dst[i], h, to] = w[i, h, at]
    s["seq_len"][dst] = length.flatten().clamp(max=keep).int()
    s["kept"].copy_(torch.where(there, rows, -1))
    return [s["k_pages"], s["v_pages"], s["seq_len"], s["weights"], s["kept"]]


# ---------------------------------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------------------------------
def _handles(s):
    """What a program sets up once: the layer's configuration, the pages' description, scratch and status."""
    if "lib" not in s:
        from paper_2511_03092_b200 import binding as B
        cfg = B.make_config(n_q_heads=s["hq"], n_kv_heads=s["hkv"], d_qk=s["d"], d_v=s["d"], dtype=s["dt"], l_sink=s.get("sink", 4),
                            l_recent=s.get("recent", 1024), topk=s.get("topk", 4096), l_obs=1, pool_kernel=1,
                            softmax_scale=1.0 / math.sqrt(s["d"]), max_seqs=s["table"].shape[0] if "table" in s else 1)
        paged = B.make_paged(s["k_pages"], s["v_pages"], s["table"]) if "table" in s else None
        rope = None
        if "freqs" in s:
            rope = B.make_rope(rot_dim=s.get("rot", s["d"]), rot_offset=s.get("offset", 0), interleaved=s.get("interleaved", False),
                               magnitude=s["magnitude"])
        need = 0
        if s["op"] == "decode":
            need = B.snap_paged_decode_workspace_bytes(cfg, paged, s["seqs"], s["weights"])
        elif s["op"] == "evict":
            need = B.snap_paged_evict_workspace_bytes(cfg, paged, s["seqs"])
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        s["lib"] = (B, cfg, paged, rope, ws, torch.zeros(1, dtype=torch.int32, device="cuda"))
    return s["lib"]


def _own(s):
    B, cfg, paged, rope, ws, status = _handles(s)
    if s["op"] == "rope":
        B.snap_rope(cfg, rope, s["freqs"], s["positions"], q=s["q"], k=s["k"], q_out=s["q_out"], k_out=s["k_out"], inverse=s["inverse"])
        return [s["q_out"], s["k_out"]]
    if s["op"] == "append":
        turned = dict(rope=rope, freqs=s["freqs"], positions=s["rows_dev"]) if s["rope"] else {}
        outputs = dict(q=s["q"], q_out=s["q_out"], k_out=s["k_out"]) if s["outputs"] else {}
        B.snap_paged_append(cfg, paged, s["slots"], s["rows_dev"], s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["seq_len"],
                            status=status, **turned, **outputs)
        return [s["k_pages"], s["v_pages"], s["seq_len"]] + ([s["q_out"], s["k_out"]] if s["outputs"] else [])
    if s["op"] == "decode":
        B.snap_paged_decode_attn(cfg, paged, s["q"], s["slots"], s["seqs"], s["k_pages"], s["v_pages"], s["table"], s["seq_len"], s["out"],
                                 ws, weights_in=s.get("weights_in"), weights_out=s.get("weights_out"), status=status)
        return [s["out"]] + ([s["weights_out"]] if s["weights"] else [])
    B.snap_paged_evict(cfg, paged, s["src"], s["dst"], s["seqs"], s["k_pages"], s["v_pages"], s["table"], s["seq_len"], s["weights"],
                       s["weights"], ws, kept_rows=s["kept"], status=status)
    return [s["k_pages"], s["v_pages"], s["seq_len"], s["weights"], s["kept"]]


PLAIN = {"rope": _plain_rope, "append": _plain_append, "decode": _plain_decode, "evict": _plain_evict}


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["op"]](state)


def work(case):
    c, eb = case, 2 if case["dtype"] == "bf16" else 4
    head = c["d"] * eb
    if c["op"] == "rope":
        return dict(bytes=c["tokens"] * ((c["hq"] + c["hkv"]) * 2 * head + 4) + 4 * c["rot"],
                    flops=c["tokens"] * (c["hq"] + c["hkv"]) * 3 * c["rot"])
    if c["op"] == "append":
        heads = 4 * c["hkv"] + (2 * c["hq"] + c["hkv"] if c["outputs"] else 0)
        return dict(bytes=c["tokens"] * (heads * head + 12), flops=c["tokens"] * (c["hkv"] + c["hq"] * c["outputs"]) * 3 * c["d"] * c["rope"])
    mean = (c["shortest"] + c["longest"]) / 2
    if c["op"] == "decode":
        rows = c["seqs"] * mean
        return dict(bytes=rows * c["hkv"] * (2 * head + (8 if c["weights"] else 0)) + c["seqs"] * (2 * c["hq"] * head + 8) + 4 * rows / c["page"],
                    flops=4 * rows * c["hq"] * c["d"])
    keep = c["sink"] + c["recent"] + c["topk"]
    kept = c["seqs"] * c["hkv"] * (mean if c["longest"] <= keep else min(mean, keep))
    return dict(bytes=kept * (4 * head + 8) + 4 * c["seqs"] * c["hkv"] * mean, flops=0)


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _turn64(x, positions, freqs, magnitude, rot, offset, interleaved):
    """Pairs as complex numbers times magnitude * e^(i angle)."""
    y = x.double().clone()
    lo = torch.arange(rot // 2, device=x.device) * (2 if interleaved else 1) + offset
    hi = lo + (1 if interleaved else rot // 2)
    z = torch.complex(y[..., lo], y[..., hi]) * torch.polar(torch.full_like(freqs, magnitude).expand(len(positions), -1),
                                                            torch.outer(positions.double(), freqs))[:, None]
    y[..., lo], y[..., hi] = z.real, z.imag
    return y


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "rope":
        sign = -1 if s["inverse"] else 1
        return [_turn64(x, sign * s["positions"].long(), s["freqs"], s["magnitude"], s["rot"], s["offset"], s["interleaved"])
                for x in (s["q"], s["k"])]
    page = s["page"]
    if s["op"] == "append":
        q, k = s["q"].double(), s["k"].double()
        if s["rope"]:
            q, k = (_turn64(x, s["rows_dev"], s["freqs"], s["magnitude"], s["d"], 0, False) for x in (q, k))
        k_pages, v_pages, lengths = s["k_pages"].double(), s["v_pages"].double(), s["seq_len"].tolist()
        for i in range(s["seqs"]):
            mine = (s["slots"] == i).nonzero().flatten()
            rows = s["rows_dev"][mine].long()
            at = s["table"][i].long()[rows // page]
            for h in range(s["hkv"]):
                k_pages[at, h, rows % page] = k[mine, h]
                v_pages[at, h, rows % page] = s["v"][mine, h].double()
            lengths[i] = max(lengths[i], int(rows.max()) + 1)
        return [k_pages, v_pages, torch.tensor(lengths, dtype=torch.int32, device="cuda")] + ([q, k] if s["outputs"] else [])
    lengths, slots = s["seq_len"].tolist(), s["slots"].tolist() if s["op"] == "decode" else []
    if s["op"] == "decode":
        out = torch.zeros(s["seqs"], s["hq"], s["d"], dtype=torch.float64, device="cuda")
        total = s["weights_out"].double() if s["weights"] else None
        group = s["hq"] // s["hkv"]
        for i, slot in enumerate(slots):
            n = lengths[slot]
            if n == 0:
                continue
            at = s["table"][slot, :-(-n // page)].long()
            for h in range(s["hkv"]):
                k, v = (x[at, h].reshape(-1, s["d"])[:n].double() for x in (s["k_pages"], s["v_pages"]))
                heads = slice(h * group, (h + 1) * group)
                p = torch.softmax(k @ s["q"][i, heads].double().t() / math.sqrt(s["d"]), dim=0)
                out[i, heads] = (v.t() @ p).t()
                if s["weights"]:
                    total[slot, h, :n] = s["weights_in"][slot, h, :n].double() + p.sum(dim=1)
        return [out] + ([total] if s["weights"] else [])
    keep = s["sink"] + s["recent"] + s["topk"]
    s["kept"].fill_(-1)
    for i, n in enumerate(lengths[:s["seqs"]]):
        to = s["seqs"] + i
        s["seq_len"][to] = min(n, keep)
        for h in range(s["hkv"]):
            rows = torch.arange(n, device="cuda")
            if n > keep:
                w = s["weights"][i, h, s["sink"]:n - s["recent"]].double()
                best = torch.argsort(-w, stable=True)[:s["topk"]].sort().values + s["sink"]
                rows = torch.cat([rows[:s["sink"]], best, rows[n - s["recent"]:]])
            new = torch.arange(len(rows), device="cuda")
            a, b = s["table"][i].long()[rows // page], s["table"][to].long()[new // page]
            s["k_pages"][b, h, new % page] = s["k_pages"][a, h, rows % page]
            s["v_pages"][b, h, new % page] = s["v_pages"][a, h, rows % page]
            s["weights"][to, h, new] = s["weights"][i, h, rows]
            s["kept"][i, h, :len(rows)] = rows.int()
    return [s["k_pages"], s["v_pages"], s["seq_len"], s["weights"], s["kept"]]
