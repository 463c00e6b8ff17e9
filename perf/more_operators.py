"""A key-value cache in pages of 8-bit numbers: planning a step's pages, appending to it, attention over it, reading it back.

Each case is one call of a serving program whose cache holds e4m3 numbers with a scale for each block of rows, KV head
and page: handing out the pages of a step and listing its tokens (``plan``), rotating and quantising new tokens' keys
and values on the way into their pages (``append``), attention of the last tokens of each sequence over its pages
(``decode``), and the rows back as dense keys and values, which prompt attention and compression take (``gather``).
With ``own`` false, ``run`` computes them in elementary torch operations; with ``own`` true through the library.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = torch.float8_e4m3fn


def listed():
    llama = dict(hq=32, hkv=8, d=128, dtype="bf16")
    return [
        # a decode step of 32 resident sequences, a token each: a few of them need a new page (the smallest call)
        dict(name="plan_step_32seq", op="plan", seqs=32, shortest=1, longest=8000, new=1, ended=0.0, page=64, width=512, scarce=False),
        # a step of a full server: prompts come in beside sequences that end, all in pages of 16 rows
        dict(name="plan_prompts_300k", op="plan", seqs=75, shortest=0, longest=60000, new=8192, ended=0.3, page=16, width=8192, scarce=True),
        # one step of 32 sequences: rotate, quantise, write a row to the last block
        dict(name="append_step_32seq", op="append", **llama, seqs=32, tokens=32, rows=90001, page=64, block=16, layout="nhd", rope=True,
             outputs=True),
        # three ragged prompts, rotated on the way into their pages
        dict(name="append_prompts_26k", op="append", **llama, seqs=3, tokens=26003, rows=12000, page=64, block=16, layout="hnd", rope=True,
             outputs=True),
        # single precision, keys as they are, a scale for each whole page
        dict(name="append_f32_11seq", op="append", hq=8, hkv=2, d=64, dtype="f32", seqs=11, tokens=4099, rows=700, page=48, block=48,
             layout="hnd", rope=False, outputs=False),
        # one sequence at the compressed cache's size: latency
        dict(name="decode_1seq_5k", op="decode", **llama, seqs=1, shortest=5124, longest=5124, q_len=1, page=64, block=16, layout="hnd"),
        # ragged long sequences (the largest call)
        dict(name="decode_16seq_8k_64k", op="decode", **llama, seqs=16, shortest=8192, longest=65536, q_len=1, page=64, block=64, layout="nhd"),
        # many short sequences, one of them still empty: no head is shared
        dict(name="decode_45seq_short", op="decode", hq=12, hkv=12, d=64, dtype="bf16", seqs=45, shortest=0, longest=333, q_len=1, page=16,
             block=16, layout="hnd"),
        # queries and outputs in single precision
        dict(name="decode_f32_4seq", op="decode", hq=8, hkv=2, d=128, dtype="f32", seqs=4, shortest=2001, longest=4100, q_len=1, page=32,
             block=8, layout="hnd"),
        # several tokens per step: each sees the rows up to its own
        dict(name="decode_4tok_8seq_16k", op="decode", **llama, seqs=8, shortest=9000, longest=16384, q_len=4, page=64, block=32, layout="hnd"),
        # a prompt kept in 8 bits is read back for compression, and ragged parts of short single-precision sequences
        dict(name="gather_prompt_32k", op="gather", **llama, seqs=1, tokens=32768, rows=0, page=64, block=16, layout="hnd"),
        dict(name="gather_f32_23seq", op="gather", hq=8, hkv=2, d=80, dtype="f32", seqs=23, tokens=3001, rows=500, page=16, block=4,
             layout="nhd"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["plan", "append", "append", "decode", "decode", "decode", "gather"])
    page = rng.choice([1, 5, 8, 16, 16, 32, 48, 64, 64, 128])
    if op == "plan":
        seqs = _log_int(rng, 1, 500)
        rows = min(100000, 8_000_000 // seqs, 15000 * page)           # the longest that a sequence can get
        longest = _log_int(rng, 1, rows)
        return dict(op=op, seqs=seqs, shortest=rng.randint(0, longest), longest=longest, new=_log_int(rng, 1, max(1, 400000 // seqs)),
                    ended=rng.choice([0.0, 0.2, 0.5]), page=page, width=-(-(rows + 400000 // seqs) // page) + rng.randint(0, 50),
                    scarce=rng.random() < 0.4)
    dtype = rng.choice(["bf16", "bf16", "f32"])
    hkv = rng.choice([1, 2, 3, 4, 8])
    c = dict(op=op, hkv=hkv, hq=hkv * rng.choice([1, 2, 4, 4, 7, 8, 16]), d=rng.choice([64, 80, 128, 128, 256]), dtype=dtype, page=page,
             block=rng.choice([b for b in range(1, page + 1) if page % b == 0]), layout=rng.choice(["hnd", "nhd"]))
    token = (c["hq"] + 2 * hkv) * c["d"] * (2 if dtype == "bf16" else 4)          # bytes of a token's queries, keys and values
    if op == "decode":
        seqs = _log_int(rng, 1, 48)
        q_len = rng.choice([1, 1, 1, 2, 3, 5, 8])
        # what the plain form keeps: rows in 32 bits, padded to the longest sequence, and every logit
        longest = _log_int(rng, 1, max(16, min(60000, 1_800_000_000 // (seqs * 8 * hkv * c["d"]), 100_000_000 // (seqs * c["hq"] * q_len))))
        return dict(c, seqs=seqs, shortest=rng.randint(0, longest), longest=longest, q_len=q_len)
    seqs = rng.randint(1, 40)
    most = max(seqs + 1, min(30000, 200_000_000 // token))
    if op == "gather":
        return dict(c, seqs=seqs, tokens=max(seqs, _log_int(rng, seqs, most)), rows=_log_int(rng, 1, 20000))
    return dict(c, seqs=seqs, tokens=seqs if rng.random() < 0.5 else max(seqs, _log_int(rng, seqs, most)), rows=_log_int(rng, 1, 60000),
                rope=rng.random() < 0.7, outputs=rng.random() < 0.7)


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _pool(c, pages, g):
    """Key and value pages [pages, heads, rows of a page, d] of e4m3 codes (stored heads first or rows first), their scales
    [pages, heads, blocks of a page], and each KV head's direction that some keys and all queries share, so that a few
    tokens draw most of the attention."""
    shape = (pages, c["hkv"], c["page"], c["d"]) if c["layout"] == "hnd" else (pages, c["page"], c["hkv"], c["d"])
    u = torch.randn(c["hkv"], 1, c["d"], device="cuda", generator=g)
    u = u / u.norm(dim=-1, keepdim=True)
    pools, scales = [], []
    for keys in (True, False):
        # numbers of a size of about one, in blocks whose largest number lies within an octave of the codes' largest
        s = torch.exp2(torch.randint(-8, -5, (pages, c["hkv"], c["page"] // c["block"]), device="cuda", generator=g).float())
        codes = torch.empty(shape, dtype=CODE, device="cuda")
        view = codes if c["layout"] == "hnd" else codes.transpose(1, 2)
        step = max(1, 100_000_000 // (c["hkv"] * c["page"] * c["d"]))
        for at in range(0, pages, step):                               # in parts: single precision takes four times the room
            x = torch.randn(view[at:at + step].shape, device="cuda", generator=g)
            if keys:
                rank = torch.rand(*x.shape[:3], 1, device="cuda", generator=g) * 4000 + 1
                x.addcmul_(8.0 * rank.pow(-1.1), u)
            x /= s[at:at + step].repeat_interleave(c["block"], dim=2)[..., None]
            view[at:at + step] = x.clamp_(-448, 448).to(CODE)
        pools.append(view)
        scales.append(s)
    return (*pools, *scales, u)


def _table(lengths, seqs, page, width, g, pool=0):
    """Page table [seqs, width]: each sequence's pages anywhere in the pool, -1 past its last one; the pages left over; the pool's
    size."""
    need = [-(-n // page) for n in lengths]
    order = torch.randperm(max(sum(need) + 3, pool), generator=g, device="cuda").to(torch.int32)
    table = torch.full((seqs, width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = order[at:at + n]
        at += n
    return table, order[at:].clone(), int(order.numel())


def _lengths(c, seed):
    r = torch.Generator().manual_seed(seed)
    n = torch.randint(c["shortest"], c["longest"] + 1, (c["seqs"],), generator=r).tolist()
    n[-1] = c["longest"]
    n[0] = c["shortest"] if c["seqs"] > 1 else n[0]
    return n


def _prepare_plan(c, seed, g):
    n, page, width = c["seqs"], c["page"], c["width"]
    r = torch.Generator().manual_seed(seed + 1)
    lengths = _lengths(c, seed)
    new = torch.full((n,), 1) if c["new"] == 1 else torch.randint(0, c["new"] + 1, (n,), generator=r)
    new = torch.where(torch.rand(n, generator=r) < c["ended"], -1, new)
    grown = [(-(-(a + b) // page)) - (-(-a // page)) if b > 0 else 0 for a, b in zip(lengths, new.tolist())]
    pool = n * (-(-c["longest"] // page)) + int(1.2 * n * (c["new"] // page + 1)) + 3
    table, free, pages = _table(lengths, n, page, width, g, pool)
    free = free[:int(sum(grown) * (0.6 if c["scarce"] else 1.2)) + 3]   # (other pages are in other hands)
    stack = torch.full((pages,), -1, dtype=torch.int32, device="cuda")
    stack[:len(free)] = free
    i32 = lambda *s: torch.empty(*s, dtype=torch.int32, device="cuda")  # noqa: E731
    most = n * c["new"] + 5                                             # the list has room for any step's tokens
    return dict(pages=pages, most=most, slots=torch.randperm(n, generator=g, device="cuda").to(torch.int32), new=new.int().cuda(),
                table=table, table_out=torch.full_like(table, -1), seq_len=torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                free=stack, n_free=torch.tensor([len(free)], dtype=torch.int32, device="cuda"), n_free_out=i32(1), granted=i32(n), first=i32(n),
                cu=i32(n + 1), token_slots=i32(most), token_rows=i32(most))


def _new_plan(s):
    """The step's counts belong to sequences, as lengths do: of the i-th request is that of its slot."""
    return s["new"][s["slots"].long()]


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(c)
    if c["op"] == "plan":
        s.update(_prepare_plan(c, seed, g))
        s["new"] = _new_plan(s)
        return s
    s["dt"] = dt = DTYPES[c["dtype"]]
    n, page = c["seqs"], c["page"]
    if c["op"] == "decode":
        lengths, width = _lengths(c, seed), max(-(-c["longest"] // page), 1)
        table, _, pages = _table(lengths, n, page, width, g)
        k, v, ks, vs, u = _pool(c, pages, g)
        q = torch.randn(n, c["q_len"], c["hkv"], c["hq"] // c["hkv"], c["d"], device="cuda", generator=g) + u * math.sqrt(c["d"]) * 0.5
        s.update(q=q.reshape(n, c["q_len"], c["hq"], c["d"]).to(dt), table=table, k_pages=k, v_pages=v, k_scales=ks, v_scales=vs,
                 slots=torch.randperm(n, generator=g, device="cuda").to(torch.int32),
                 seq_len=torch.tensor(lengths, dtype=torch.int32, device="cuda"))
        s["out"] = torch.empty_like(s["q"])
        return s
    t = c["tokens"]
    each = [t // n + (1 if i < t % n else 0) for i in range(n)]
    start = torch.randint(c["rows"] // 2, c["rows"] + 1, (n,), generator=torch.Generator().manual_seed(seed)).tolist()
    width = -(-(max(start) + max(each) + 1) // page)
    table = torch.full((n, width), -1, dtype=torch.int32, device="cuda")
    firsts = [b // page for b in start]                                 # the pages of the rows before are elsewhere
    counts = [(b + e - 1) // page - f + 1 for b, e, f in zip(start, each, firsts)]
    order = torch.randperm(sum((e - 1) // page + 2 for e in each), generator=g, device="cuda").to(torch.int32)
    at = 0
    for i in range(n):
        table[i, firsts[i]:firsts[i] + counts[i]] = order[at:at + counts[i]]
        at += counts[i]
    k, v, ks, vs, _ = _pool(c, int(order.numel()), g)
    cu = torch.tensor([0] + each, dtype=torch.int32).cumsum(0).int().cuda()
    s.update(table=table, k_pages=k, v_pages=v, k_scales=ks, v_scales=vs, slots=torch.arange(n, dtype=torch.int32, device="cuda"), cu=cu,
             first=torch.tensor(start, dtype=torch.int32, device="cuda"), seq_len=torch.tensor(start, dtype=torch.int32, device="cuda"))
    normal = lambda h: torch.randn(t, h, c["d"], device="cuda", generator=g).to(dt)  # noqa: E731
    if c["op"] == "append":
        s.update(q=normal(c["hq"]), k=normal(c["hkv"]), v=normal(c["hkv"]),
                 freqs=(500000.0 ** (-torch.arange(0, c["d"], 2, dtype=torch.float64) / c["d"])).cuda())
        s.update(q_out=torch.empty_like(s["q"]), k_out=torch.empty_like(s["k"]))
    else:
        s.update(k=torch.empty(t, c["hkv"], c["d"], dtype=dt, device="cuda"), v=torch.empty(t, c["hkv"], c["d"], dtype=dt, device="cuda"))
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _plain_plan(s):
    slots, n, page = s["slots"].long(), s["new"], s["page"]
    row, length = s["table"][slots], s["seq_len"][slots]                # [requests, width]
    j = torch.arange(row.shape[1], device=row.device)
    held = (row >= 0) & (row < s["pages"])
    ended, length = n < 0, torch.where(n < 0, 0, length)
    # the pages of sequences that end go onto the stack, in order
    back = (held & ended[:, None]).flatten()
    stack = torch.cat([s["free"], s["free"].new_empty(1)])              # one more place, for what does not go back
    place = s["n_free"] + back.cumsum(0) - 1
    stack[torch.where(back, place, s["pages"])] = row.flatten()
    s["free"].copy_(stack[:-1])
    there = s["n_free"] + back.sum()
    # pages that are missing up to each sequence's new length; who gets them; the k-th page granted is the k-th from the top
    fits = ~ended & (length.long() + n <= row.shape[1] * page)
    want = ~held & (j < ((length + n + page - 1) // page)[:, None]) & fits[:, None]
    need = want.sum(dim=1)
    before = need.cumsum(0) - need
    tokens = torch.where(fits, n, 0)
    grant = fits & (tokens.cumsum(0) <= s["most"]) & ((need == 0) | (before + need <= there))
    nth = before[:, None] + want.cumsum(dim=1) - 1
    take = want & grant[:, None]
    page_of = s["free"][torch.where(take, there - 1 - nth, 0)]
    s["table_out"][slots] = torch.where(take, page_of, torch.where(ended[:, None], -1, row))
    s["n_free_out"].copy_(there - torch.where(grant, need, 0).sum())
    s["seq_len"][slots] = length
    # the step's tokens
    granted = torch.where(grant, tokens, 0)
    s["granted"].copy_(granted)
    s["first"].copy_(length)
    s["cu"].zero_()
    s["cu"][1:] = granted.cumsum(0)
    t = torch.arange(s["most"], device=row.device)
    i = torch.searchsorted(s["cu"][1:].long(), t, right=True).clamp(max=len(n) - 1)
    real = t < s["cu"][-1]
    s["token_slots"].copy_(torch.where(real, slots[i], -1))
    s["token_rows"].copy_(torch.where(real, length[i] + t - s["cu"][i], 0))
    return _plan_outputs(s)


def _plan_outputs(s):
    return [s[x] for x in ("table_out", "free", "n_free_out", "seq_len", "granted", "first", "cu", "token_slots", "token_rows")]


def _tokens(s):
    """Of every token of an append or gather: its sequence's entry, its row, the page and the row of the page it is on."""
    t = torch.arange(s["tokens"], device="cuda")
    i = torch.searchsorted(s["cu"].long(), t, right=True) - 1
    row = s["first"].long()[i] + t - s["cu"][i]
    return i, row, s["table"][s["slots"].long()[i], row // s["page"]].long(), row % s["page"]


def _rotate(x, cos, sin):
    """x [T, H, d]: dims i and i + d / 2 are a pair."""
    a, b = x.float().chunk(2, dim=-1)
    cos, sin = cos[:, None, :], sin[:, None, :]
    return torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)


def _scale_for(largest, growth):
    """The power of two whose 448-fold is at least the largest number, a rotation's growth included."""
    mantissa, exponent = torch.frexp(largest * growth)
    e = exponent - 9 + (mantissa > 0.875).int()                         # 448 = 0.875 * 2^9
    return torch.ldexp(torch.ones_like(largest), torch.where(largest > 0, e.clamp(-126, 120), -126))


def _quantised(x, pages, scales, growth, values, s, where):
    """Writes rows `values` (of the inputs x) to their pages; raises the scales of the blocks they are in."""
    i, row, page, off = where
    block, B = off // s["block"], s["block"]
    largest = torch.zeros_like(scales)
    per_token = x.float().abs().amax(dim=-1)                            # [T, heads]
    at = (page[:, None], torch.arange(s["hkv"], device="cuda"), block[:, None])
    flat = (at[0] * s["hkv"] + at[1]) * scales.shape[2] + at[2]
    largest.view(-1).scatter_reduce_(0, flat.flatten(), per_token.flatten(), "amax")
    touched = torch.zeros_like(scales, dtype=torch.bool)
    touched.view(-1)[flat.flatten()] = True
    old = torch.zeros_like(scales)                                      # of blocks that hold rows of their sequence already
    first = s["first"].long()
    begin = first // B * B                                              # the block of a sequence's first new row
    p0, b0 = s["table"][s["slots"].long(), begin // s["page"]].long(), begin % s["page"] // B
    rows = begin[:, None] + torch.arange(B, device="cuda")              # [sequences, B]
    mine = (rows < first[:, None]) & (s["cu"][1:] > s["cu"][:-1])[:, None]
    some = mine.any(dim=1)
    old[p0] = torch.where(some[:, None, None] & (torch.arange(scales.shape[2], device="cuda") == b0[:, None])[:, None], scales[p0], old[p0])
    new = torch.where(touched, torch.maximum(_scale_for(largest, growth), old), scales)
    # what such a block holds, on its new scale
    bytes_, o = pages.view(torch.uint8), begin[:, None] % s["page"] + torch.arange(B, device="cuda")
    held = bytes_[p0[:, None], :, o]                                    # [sequences, B, heads, d]
    ratio = (scales[p0, :, b0] / new[p0, :, b0])[:, None, :, None]
    moved = (held.view(CODE).float() * ratio).to(CODE).view(torch.uint8)
    bytes_[p0[:, None], :, o] = torch.where(mine[:, :, None, None], moved, held)
    scales.copy_(new)
    bytes_[page, :, off] = (values / new[page, :, block][..., None]).clamp(-448, 448).to(CODE).view(torch.uint8)


def _plain_append(s):
    where = _tokens(s)
    k, q, growth = s["k"].float(), s["q"], 1.0
    if s["rope"]:
        angle = where[1].double()[:, None] * s["freqs"]                 # in 64 bits: far positions
        cos, sin = angle.cos().float(), angle.sin().float()
        k, q, growth = _rotate(k, cos, sin), _rotate(q, cos, sin).to(s["dt"]), math.sqrt(2.0)
    _quantised(s["k"], s["k_pages"], s["k_scales"], growth, k, s, where)
    _quantised(s["v"], s["v_pages"], s["v_scales"], 1.0, s["v"].float(), s, where)
    s["seq_len"][s["slots"].long()] = s["first"] + s["cu"][1:] - s["cu"][:-1]
    return [s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["seq_len"]] + ([q, k.to(s["dt"])] if s["outputs"] else [])


def _all_rows(pages, scales, table):
    """[n, heads, rows, d] in 32 bits: the rows of a page table's pages in order."""
    at = table.clamp(min=0).long()
    x = pages.view(torch.uint8)[at].view(CODE).float()                  # [n, width, heads, page, d]
    n, w, h, p, d = x.shape
    x *= scales[at].repeat_interleave(p // scales.shape[2], dim=3)[..., None]
    return x.permute(0, 2, 1, 3, 4).reshape(n, h, w * p, d)


def _plain_decode(s):
    slots, n, ql, hkv = s["slots"].long(), s["seqs"], s["q_len"], s["hkv"]
    table, length = s["table"][slots], s["seq_len"][slots]
    q = s["q"].float().reshape(n, ql, hkv, -1, s["d"]).transpose(1, 2).reshape(n, hkv, -1, s["d"])     # [n, heads, tokens * group, d]
    x = (q @ _all_rows(s["k_pages"], s["k_scales"], table).transpose(2, 3)) * (1.0 / math.sqrt(s["d"]))
    sees = length[:, None] - ql + 1 + torch.arange(ql, device="cuda")   # [n, tokens]: rows before that
    there = torch.arange(x.shape[3], device="cuda") < sees[..., None]
    x = x.view(n, hkv, ql, -1, x.shape[3]).masked_fill(~there[:, None, :, None], -math.inf)
    p = torch.exp(x - x.amax(dim=-1, keepdim=True).clamp(min=-1e30))    # a token that sees no row: all zero
    del x
    p = p / p.sum(dim=-1, keepdim=True).clamp(min=1e-30)
    out = p.flatten(2, 3) @ _all_rows(s["v_pages"], s["v_scales"], table)
    return out.view(n, hkv, ql, -1, s["d"]).transpose(1, 2).reshape(n, ql, s["hq"], s["d"]).to(s["dt"])


def _plain_gather(s):
    _, _, page, off = _tokens(s)
    block = off // s["block"]
    for x, pages, scales in ((s["k"], s["k_pages"], s["k_scales"]), (s["v"], s["v_pages"], s["v_scales"])):
        x.copy_(pages.view(torch.uint8)[page, :, off].view(CODE).float() * scales[page, :, block][..., None])
    return [s["k"], s["v"]]


# ---------------------------------------------------------------------------------------------------------------
# the library's calls
# ---------------------------------------------------------------------------------------------------------------
def _handles(s):
    """What a program sets up once: the layer's configuration, the pages' description, scratch and status."""
    if "lib" not in s:
        from paper_2511_03092_b200 import binding as B
        layer = dict(n_q_heads=s.get("hq", 1), n_kv_heads=s.get("hkv", 1), d_qk=s.get("d", 16), d_v=s.get("d", 16))
        cfg = B.make_config(**layer, dtype=s.get("dt", torch.bfloat16), l_sink=4, l_recent=1024, topk=4096, l_obs=1, pool_kernel=1,
                            softmax_scale=1.0 / math.sqrt(layer["d_qk"]), max_seqs=s["table"].shape[0])
        need, rope = 0, None
        if s["op"] == "plan":
            paged = B.make_page_map(s["page"], s["pages"], s["table"])
            need = B.snap_paged_plan_workspace_bytes(cfg, paged, s["seqs"])
        else:
            paged = B.make_paged_q8(s["k_pages"], s["v_pages"], s["table"], s["block"])
            if s["op"] == "decode":
                need = B.snap_paged_q8_decode_workspace_bytes(cfg, paged, s["seqs"], s["q_len"])
            elif s["op"] == "append" and s["rope"]:
                rope = B.make_rope(rot_dim=s["d"])
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        s["lib"] = (B, cfg, paged, rope, ws, torch.zeros(1, dtype=torch.int32, device="cuda"))
    return s["lib"]


def _own(s):
    B, cfg, paged, rope, ws, status = _handles(s)
    if s["op"] == "plan":
        B.snap_paged_plan(cfg, paged, s["slots"], s["new"], s["table"], s["seq_len"], s["free"], s["n_free"], s["first"], s["cu"],
                          s["token_slots"], s["token_rows"], ws, page_table_out=s["table_out"], n_free_out=s["n_free_out"],
                          granted=s["granted"], status=status)
        return _plan_outputs(s)
    cache = (s["k_pages"], s["v_pages"], s["k_scales"], s["v_scales"], s["table"])
    if s["op"] == "append":
        turned = dict(rope=rope, freqs=s["freqs"]) if s["rope"] else {}
        outputs = dict(q=s["q"], q_out=s["q_out"], k_out=s["k_out"]) if s["outputs"] else {}
        B.snap_paged_q8_append(cfg, paged, s["slots"], s["cu"], s["first"], s["k"], s["v"], *cache, s["seq_len"], status=status, **turned,
                               **outputs)
        return [*cache[:4], s["seq_len"]] + ([s["q_out"], s["k_out"]] if s["outputs"] else [])
    if s["op"] == "decode":
        B.snap_paged_q8_decode_attn(cfg, paged, s["q"], s["slots"], *cache, s["seq_len"], s["out"], ws, status=status)
        return s["out"]
    B.snap_paged_q8_gather(cfg, paged, s["slots"], s["cu"], s["first"], *cache, s["k"], s["v"], status=status)
    return [s["k"], s["v"]]


PLAIN = {"plan": _plain_plan, "append": _plain_append, "decode": _plain_decode, "gather": _plain_gather}


def run(state):
    if own:
        return _own(state)
    return PLAIN[state["op"]](state)


def work(case):
    c = case
    if c["op"] == "plan":
        # every table row is read and written, two numbers for each place in the list of tokens, some for each request
        return dict(bytes=8 * c["seqs"] * c["width"] + 8 * c["seqs"] * c["new"] + 28 * c["seqs"], flops=0)
    eb, head = 2 if c["dtype"] == "bf16" else 4, c["d"]                 # head: bytes of a row of codes
    scales = 4 / c["block"]
    if c["op"] == "decode":
        rows = c["seqs"] * (c["shortest"] + c["longest"]) / 2
        queries = c["seqs"] * c["q_len"] * c["hq"] * c["d"]
        return dict(bytes=rows * c["hkv"] * 2 * (head + scales) + queries * 2 * eb + 8 * c["seqs"] + 4 * rows / c["page"],
                    flops=4 * rows * c["q_len"] * c["hq"] * c["d"])
    rows = c["tokens"] * c["hkv"] * 2 * (head * (1 + eb) + scales)
    if c["op"] == "gather":
        return dict(bytes=rows + 4 * c["tokens"] / c["page"], flops=c["tokens"] * c["hkv"] * 2 * c["d"])
    outputs = c["tokens"] * (2 * c["hq"] + c["hkv"]) * head * eb if c["outputs"] else 0
    return dict(bytes=rows + outputs + 4 * c["tokens"] / c["page"],
                flops=c["tokens"] * c["d"] * (4 * c["hkv"] + 3 * (c["hkv"] + c["hq"] * c["outputs"]) * c["rope"]))


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------------------------------------------
def _turn64(x, positions, freqs):
    """Pairs as complex numbers times e^(i angle)."""
    half = x.shape[-1] // 2
    z = torch.complex(x[..., :half], x[..., half:]) * torch.polar(torch.ones_like(freqs).expand(len(positions), -1),
                                                                  torch.outer(positions.double(), freqs))[:, None]
    return torch.cat([z.real, z.imag], dim=-1)


def _exact_append(s):
    """Sequence by sequence and block by block; codes stay unrounded."""
    q, k, v = (s[x].double() for x in "qkv")
    cu, first, slots, page, B = s["cu"].tolist(), s["first"].tolist(), s["slots"].tolist(), s["page"], s["block"]
    rows = torch.cat([torch.arange(f, f + b - a, device="cuda") for f, a, b in zip(first, cu[:-1], cu[1:])])
    turned, growth = k, 1.0
    if s["rope"]:
        q, turned, growth = _turn64(q, rows, s["freqs"]), _turn64(k, rows, s["freqs"]), math.sqrt(2.0)
    out = []
    table = s["table"].tolist()
    for x, y, pages, scales, f in ((k, turned, s["k_pages"], s["k_scales"], growth), (v, v, s["v_pages"], s["v_scales"], 1.0)):
        big = [x.abs().amax(dim=-1).cpu(), scales.cpu().clone()]        # [T, heads]
        codes = pages.double()
        for i, slot in enumerate(slots):
            a, n = cu[i], cu[i + 1] - cu[i]
            b = first[i] // B
            while b * B < first[i] + n:
                lo, hi = max(b * B, first[i]), min((b + 1) * B, first[i] + n)
                p, at = table[slot][b * B // page], b * B % page
                top = big[0][a + lo - first[i]:a + hi - first[i]].amax(dim=0) * f
                new = torch.tensor([2.0 ** max(-126, min(120, math.ceil(math.log2(t / 448.0)))) if t > 0 else 2.0 ** -126 for t in top.tolist()])
                if lo > b * B:
                    old = big[1][p, :, at // B]
                    new = torch.maximum(new, old)
                    codes[p, :, at:at + lo - b * B] *= (old / new).double().cuda()[:, None, None]
                big[1][p, :, at // B] = new
                codes[p, :, at + lo - b * B:at + hi - b * B] = y[a + lo - first[i]:a + hi - first[i]].transpose(0, 1) / new.double().cuda()[:, None, None]
                b += 1
        out.append((codes, big[1].double()))
    lengths = torch.tensor([first[i] + cu[i + 1] - cu[i] for i in range(len(slots))], dtype=torch.int32)
    (kc, ks), (vc, vs) = out
    return [kc, vc, ks, vs, lengths] + ([q, turned] if s["outputs"] else [])


def exact(case, seed):
    if case["op"] == "plan":
        return None                                                     # whole numbers alone
    s = prepare(case, seed)
    if s["op"] == "append":
        return _exact_append(s) if s["tokens"] / s["block"] + s["seqs"] < 8000 else None
    slots, table, page = s["slots"].tolist(), s["table"], s["page"]
    if s["op"] == "gather":
        out = []
        for pages, scales in ((s["k_pages"], s["k_scales"]), (s["v_pages"], s["v_scales"])):
            x = torch.zeros(s["tokens"], s["hkv"], s["d"], dtype=torch.float64, device="cuda")
            for i, (slot, f, a, b) in enumerate(zip(slots, s["first"].tolist(), s["cu"].tolist(), s["cu"].tolist()[1:])):
                at = torch.arange(f, f + b - a, device="cuda")
                pg = table[slot].long()[at // page]
                for h in range(s["hkv"]):
                    x[a:b, h] = pages.view(torch.uint8)[pg, h, at % page].view(CODE).double() * scales[pg, h, at % page // s["block"]].double()[:, None]
            out.append(x)
        return out
    out = torch.zeros(s["seqs"], s["q_len"], s["hq"], s["d"], dtype=torch.float64, device="cuda")
    group, lengths = s["hq"] // s["hkv"], s["seq_len"].tolist()
    for i, slot in enumerate(slots):
        at = table[slot, :-(-lengths[slot] // page)].long()
        for h in range(s["hkv"]):
            k, v = (x.view(torch.uint8)[at, h].view(CODE).double().mul(f[at, h].double().repeat_interleave(s["block"], dim=1)[..., None]).reshape(-1, s["d"])
                    for x, f in ((s["k_pages"], s["k_scales"]), (s["v_pages"], s["v_scales"])))
            for u in range(s["q_len"]):
                n = lengths[slot] - s["q_len"] + 1 + u
                if n <= 0:
                    continue
                heads = slice(h * group, (h + 1) * group)
                p = torch.softmax(k[:n] @ s["q"][i, u, heads].double().t() / math.sqrt(s["d"]), dim=0)
                out[i, u, heads] = (v[:n].t() @ p).t()
    return out
