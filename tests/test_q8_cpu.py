"""The page plan and the 8-bit cache without a GPU: the definitions' codes and scales, workspace sizes, and the refusals of
every entry point (nothing is launched, no pointer is read)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import q8_oracle as orc
from paper_2511_03092_b200 import binding as B
from paper_2511_03092_b200 import build as snap_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    snap_build.build()


def _cfg(**kw):
    base = dict(n_q_heads=32, n_kv_heads=8, d_qk=128, d_v=128, dtype=B.SNAP_BF16, l_sink=4, l_recent=1024, topk=4096, l_obs=64,
                pool_kernel=7, softmax_scale=0.088, max_seqs=3)
    base.update(kw)
    return B.make_config(**base)


def _q8(block=16, **kw):
    base = dict(page_tokens=64, n_pages=100, max_pages=50, reserved=0, k_page_stride=64 * 1024, k_head_stride=64 * 128, k_row_stride=128,
                v_page_stride=64 * 1024, v_head_stride=64 * 128, v_row_stride=128)
    base.update(kw)
    return B.SnapPagedQ8(B.SnapPaged(**base), block, 0)


# ---------------------------------------------------------------------------------------------------------------
# the definitions
# ---------------------------------------------------------------------------------------------------------------
def test_codes_are_those_of_e4m3():
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(orc.VALUES, t)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.normal(size=2000) * 10.0 ** rng.integers(-4, 3, 2000), (t[:126] + t[1:127]) / 2, t, [0.0, -0.0, 448, 464, 2.0 ** -10, 3e-4]])
    x = x[~(np.abs(x) > 448)]
    want = torch.from_numpy(x).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    nan = np.isnan(x)
    np.testing.assert_array_equal(orc.encode(x)[~nan], want[~nan])
    assert (orc.encode(np.array([math.nan])) & 0x7f == 0x7f).all()
    assert orc.VALUES[orc.encode(np.array([1e9, -math.inf]))].tolist() == [448.0, -448.0]


@pytest.mark.parametrize("largest,scale", [(448.0, 1.0), (448.0001, 2.0), (224.0, 0.5), (1.0, 2.0 ** -8), (0.0, 2.0 ** -126), (1e-45, 2.0 ** -126),
                                           (3.4e38, 2.0 ** 120), (math.inf, 2.0 ** 120)])
def test_the_scale_is_the_smallest_power_that_reaches(largest, scale):
    assert orc.scale_for(largest) == scale


def test_a_plan_by_hand():
    table = np.full((3, 4), -1, dtype=np.int64)
    table[0, :2], table[1, 0] = (5, 6), 7
    got, said = orc.plan([1, 0, 2, -1], [-1, 3, 9, 4], table, np.array([4, 2, 0]), np.array([1, 2, 3, -9, -9, -9, -9, -9]), 3, 4, 8, 20)
    # the pages of slot 1 go onto the stack; slot 0 has rows 0-3 on page 5 and 4-6 on the page that it holds; slot 2 takes three
    assert got["stack"][:4].tolist() == [1, 2, 3, 7] and got["n_free"] == 1 and not said
    assert got["table"].tolist() == [[5, 6, -1, -1], [-1, -1, -1, -1], [7, 3, 2, -1]]
    assert got["granted"] == [0, 3, 9, 0] and got["first"] == [0, 4, 0, 0] and got["cu"] == [0, 0, 3, 12, 12]
    assert got["token_slots"] == [0] * 3 + [2] * 9 + [-1] * 8 and got["token_rows"] == [4, 5, 6, *range(9)] + [0] * 8


# ---------------------------------------------------------------------------------------------------------------
# refusals
# ---------------------------------------------------------------------------------------------------------------
ONE, ODD, BIG = C.c_void_p(256), C.c_void_p(264), 1 << 40


def _append(cfg=None, paged=None, **kw):
    a = dict(slots=ONE, cu=ONE, first=ONE, n=4, t=9, rope=None, freqs=None, pos=None, q=None, qs=(4096, 128), qo=None, k=ONE, ks=(1024, 128),
             ko=None, v=ONE, vs=(1024, 128), kp=ONE, vp=ONE, ksc=ONE, vsc=ONE, table=ONE, seq_len=C.c_void_p(512))
    a.update(kw)
    cfg, paged = cfg or _cfg(), _q8() if paged is None else paged
    return B.lib().snap_paged_q8_append(C.byref(cfg), C.byref(paged) if paged else None, a["slots"], a["cu"], a["first"], a["n"], a["t"],
                                        C.byref(a["rope"]) if a["rope"] else None, a["freqs"], a["pos"], a["q"], *a["qs"], a["qo"], a["k"],
                                        *a["ks"], a["ko"], a["v"], *a["vs"], a["kp"], a["vp"], a["ksc"], a["vsc"], a["table"], a["seq_len"],
                                        None, None)


def _decode(cfg=None, paged=None, **kw):
    a = dict(q=ONE, slots=ONE, n=4, ql=1, kp=ONE, vp=ONE, ksc=ONE, vsc=ONE, table=ONE, seq_len=ONE, out=ONE, ws=ONE, size=BIG)
    a.update(kw)
    cfg, paged = cfg or _cfg(), _q8() if paged is None else paged
    return B.lib().snap_paged_q8_decode_attn(C.byref(cfg), C.byref(paged) if paged else None, a["q"], a["slots"], a["n"], a["ql"], a["kp"], a["vp"],
                                             a["ksc"], a["vsc"], a["table"], a["seq_len"], a["out"], a["ws"], a["size"], None, None)


def _gather(cfg=None, paged=None, **kw):
    a = dict(slots=ONE, cu=ONE, first=ONE, n=4, t=9, kp=ONE, vp=ONE, ksc=ONE, vsc=ONE, table=ONE, k=ONE, ks=(1024, 128), v=ONE, vs=(1024, 128))
    a.update(kw)
    cfg, paged = cfg or _cfg(), _q8() if paged is None else paged
    return B.lib().snap_paged_q8_gather(C.byref(cfg), C.byref(paged) if paged else None, a["slots"], a["cu"], a["first"], a["n"], a["t"], a["kp"],
                                        a["vp"], a["ksc"], a["vsc"], a["table"], a["k"], *a["ks"], a["v"], *a["vs"], None, None)


def _plan(cfg=None, paged=None, **kw):
    a = dict(slots=ONE, new=ONE, n=4, tin=ONE, tout=ONE, seq_len=ONE, free=ONE, nin=ONE, nout=ONE, most=100, granted=None, first=ONE, cu=ONE,
             ts=ONE, tr=ONE, ws=ONE, size=BIG)
    a.update(kw)
    cfg, paged = cfg or _cfg(), _q8().pages if paged is None else paged
    return B.lib().snap_paged_plan(C.byref(cfg), C.byref(paged) if paged else None, a["slots"], a["new"], a["n"], a["tin"], a["tout"], a["seq_len"],
                                   a["free"], a["nin"], a["nout"], a["most"], a["granted"], a["first"], a["cu"], a["ts"], a["tr"], a["ws"],
                                   a["size"], None, None)


@pytest.mark.parametrize("call", [_append, _decode, _gather])
def test_calls_on_the_cache_refuse_bad_arguments(call):
    assert call(n=0) == 0 and call(n=-1) == -1 and call(paged=False) == -4
    for missing in ("kp", "vp", "ksc", "vsc", "table", "slots"):
        assert call(**{missing: None}) == -4, missing
    assert call(kp=ODD) == -1 and call(vp=ODD) == -1
    for bad in (dict(page_tokens=0), dict(n_pages=0), dict(max_pages=0), dict(reserved=1), dict(k_page_stride=-1024), dict(k_row_stride=136),
                dict(v_head_stride=24), dict(k_row_stride=64), dict(v_page_stride=0), dict(page_tokens=1 << 20, max_pages=1 << 20)):
        assert call(paged=_q8(**bad)) == -1, bad
    assert call(paged=_q8(block=0)) == -1 and call(paged=_q8(block=24)) == -1 and call(paged=_q8(block=128)) == -1
    assert call(paged=B.SnapPagedQ8(_q8().pages, 16, 1)) == -1
    wide = dict(k_row_stride=640, v_row_stride=640, k_head_stride=40960, v_head_stride=40960)
    assert call(cfg=_cfg(n_q_heads=128, n_kv_heads=1, d_qk=576, d_v=512, v_aliases_k=True), paged=_q8(**wide)) == -2
    assert call(cfg=_cfg(d_v=272), paged=_q8(**wide)) == -2 and call(cfg=_cfg(topk=-1)) == -1


def test_the_append_refuses_bad_arguments():
    assert _append(t=0) == 0 and _append(t=-1) == -1 and _append(n=65537) == -1 and _append(t=2 ** 31 - 65535) == -1
    for missing in ("cu", "first", "k", "v", "seq_len"):
        assert _append(**{missing: None}) == -4, missing
    assert _append(q=ONE) == -4 and _append(qo=ONE) == -4
    assert _append(rope=B.make_rope(rot_dim=128)) == -4                 # no frequencies
    assert _append(rope=B.make_rope(rot_dim=256), freqs=ONE) == -1 and _append(rope=B.make_rope(rot_dim=64, rot_offset=80), freqs=ONE) == -1
    assert _append(ks=(1024, 100)) == -1 and _append(vs=(-1024, 128)) == -1 and _append(k=ODD) == -1 and _append(q=ONE, qo=ODD) == -1
    assert _append(ko=ONE, ks=(6144, 128)) == -1                        # in place, but not dense like the output
    assert _append(first=ONE, seq_len=ONE) == -1                        # the lengths change while the first rows are read


def test_attention_and_gather_refuse_bad_arguments():
    assert _decode(q=None) == -4 and _decode(out=None) == -4 and _decode(ws=None) == -4 and _decode(seq_len=None) == -4
    assert _decode(q=ODD) == -1 and _decode(out=ODD) == -1 and _decode(ws=ODD) == -1
    assert _decode(ql=0) == -1 and _decode(ql=1025) == -1 and _decode(ql=-3) == -1
    for ql in (1, 5):
        need = B.snap_paged_q8_decode_workspace_bytes(_cfg(), _q8(), 4, ql)
        assert _decode(ql=ql, size=need - 1) == -3
    for bad in (dict(n_active=-1), dict(q_len=0), dict(q_len=1025)):
        with pytest.raises(B.SnapError):
            B.snap_paged_q8_decode_workspace_bytes(_cfg(), _q8(), **{**dict(n_active=4, q_len=1), **bad})
    with pytest.raises(B.SnapError):                                    # more queries than can be counted
        B.snap_paged_q8_decode_workspace_bytes(_cfg(), _q8(), 2 ** 30, 1024)
    assert _gather(t=0) == 0 and _gather(t=-1) == -1 and _gather(n=65537) == -1
    for missing in ("cu", "first", "k", "v"):
        assert _gather(**{missing: None}) == -4, missing
    assert _gather(k=ODD) == -1 and _gather(ks=(1024, 100)) == -1
    assert _gather(vs=(512, 128)) == -1 and _gather(ks=(1024, 64)) == -1    # tokens, heads of an output overlap


def test_the_plan_refuses_bad_arguments():
    for missing in ("slots", "new", "tin", "tout", "seq_len", "free", "nin", "nout", "first", "cu", "ts", "tr", "ws"):
        assert _plan(**{missing: None}) == -4, missing
    assert _plan(paged=False) == -4 and _plan(n=-1) == -1 and _plan(n=65537) == -1 and _plan(most=-1) == -1
    assert _plan(ts=ODD) == -1 and _plan(tr=ODD) == -1 and _plan(ws=ODD) == -1
    for bad in (dict(page_tokens=0), dict(n_pages=0), dict(max_pages=0), dict(reserved=1), dict(page_tokens=1 << 20, max_pages=1 << 20)):
        assert _plan(paged=_q8(**bad).pages) == -1, bad
    pages = B.make_page_map(64, 100, torch.zeros(3, 50, dtype=torch.int32))
    need = B.snap_paged_plan_workspace_bytes(_cfg(), pages, 4)
    assert _plan(paged=pages, size=need - 1) == -3
    assert B.snap_paged_plan_workspace_bytes(_cfg(), _q8(), 4) == need   # either description
    for n in (-1, 65537):
        with pytest.raises(B.SnapError):
            B.snap_paged_plan_workspace_bytes(_cfg(), pages, n)


def test_the_binding_checks_what_tensors_are():
    cfg, e4m3 = _cfg(), torch.float8_e4m3fn
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    k, sc, table = torch.zeros(100, 8, 64, 128, dtype=torch.uint8).view(e4m3), torch.zeros(100, 8, 4), i32(3, 50)
    paged = B.make_paged_q8(k, k, table, 16)
    assert (paged.pages.page_tokens, paged.pages.n_pages, paged.pages.max_pages, paged.pages.k_row_stride, paged.block_tokens) == (64, 100, 50, 128, 16)
    cache = dict(k_pages=k, v_pages=k, k_scales=sc, v_scales=sc, page_table=table)
    q = torch.zeros(2, 3, 32, 128, dtype=torch.bfloat16)
    x = torch.zeros(7, 8, 128, dtype=torch.bfloat16)
    dec = dict(cache, q=q, slot_ids_dev=i32(2), seq_len=i32(3), out=q.clone(), workspace=i32(4))
    app = dict(cache, slot_ids_dev=i32(2), cu_tokens=i32(3), first_rows=i32(2), k=x, v=x, seq_len=i32(3))
    gat = dict(cache, slot_ids_dev=i32(2), cu_tokens=i32(3), first_rows=i32(2), k=x, v=x)
    for call, ok, more in (
            (B.snap_paged_q8_decode_attn, dec, [(dict(q=q.float()), "expected"), (dict(out=q[:, :2]), "shape"), (dict(q=q.transpose(1, 2)), "shape"),
                                                (dict(q=q[0, 0]), "sequences"), (dict(seq_len=i32(4)), "shape")]),
            (B.snap_paged_q8_append, app, [(dict(k=x.float()), "expected"), (dict(v=x[:6]), "shape"), (dict(cu_tokens=i32(2)), "shape"),
                                           (dict(k=x[0]), "tokens"), (dict(first_rows=i32(3)), "shape"), (dict(q=q[0]), "shape")]),
            (B.snap_paged_q8_gather, gat, [(dict(k=x.float()), "expected"), (dict(v=x[:6]), "shape"), (dict(cu_tokens=i32(2)), "shape")])):
        for bad, word in more + [(dict(), "CUDA"), (dict(k_pages=k.view(torch.uint8)), "expected"), (dict(k_scales=sc[:, :, :2]), "shape"),
                                 (dict(v_scales=sc.double()), "expected"), (dict(page_table=i32(3, 49)), "shape"),
                                 (dict(slot_ids_dev=torch.zeros(2, dtype=torch.int64)), "int64")]:
            with pytest.raises(ValueError, match=word):
                call(cfg, paged, **{**ok, **bad})
    plan = dict(slot_ids_dev=i32(2), new_tokens_dev=i32(2), page_table=table, seq_len=i32(3), free_pages=i32(100), n_free=i32(1), first_rows=i32(2),
                cu_tokens=i32(3), token_slots=i32(9), token_rows=i32(9), workspace=i32(4))
    for bad, word in ((dict(), "CUDA"), (dict(new_tokens_dev=i32(3)), "shape"), (dict(page_table_out=i32(3, 49)), "shape"),
                      (dict(free_pages=i32(99)), "shape"), (dict(n_free=i32(2)), "shape"), (dict(token_rows=i32(8)), "shape"),
                      (dict(granted=i32(3)), "shape"), (dict(cu_tokens=i32(2)), "shape")):
        with pytest.raises(ValueError, match=word):
            B.snap_paged_plan(cfg, paged, **{**plan, **bad})
    with pytest.raises(TypeError):                                      # the description of another cache
        B.snap_paged_q8_gather(cfg, paged.pages, **gat)
    with pytest.raises(ValueError):
        B.make_page_map(16, 10, i32(3))


def test_a_plan_refuses_tables_that_overlap():
    size = 4 * 3 * 50                                       # of a table: 3 sequences, 50 pages each
    pages = B.make_page_map(64, 100, torch.zeros(3, 50, dtype=torch.int32))
    base = 1 << 20
    for off in (4, 200, size - 4, -4, 4 - size):
        assert _plan(paged=pages, tin=base, tout=base + off) == -1, off
    for off in (0, size, -size):                            # in place, or apart: the call goes on (to scratch that is too small)
        assert _plan(paged=pages, tin=base, tout=base + off, size=0) == -3, off
