"""Rotary positions and the paged cache without a GPU: the frequency tables against their definition, workspace sizes,
and the refusals of every entry point (nothing is launched, no pointer is read)."""
import ctypes as C
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as orc
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


def _paged(**kw):
    base = dict(page_tokens=16, n_pages=100, max_pages=50, reserved=0, k_page_stride=16 * 1024, k_head_stride=16 * 128, k_row_stride=128,
                v_page_stride=16 * 1024, v_head_stride=16 * 128, v_row_stride=128)
    base.update(kw)
    return B.SnapPaged(**base)


TABLES = [dict(), dict(scaling="linear", factor=4.0), dict(scaling="llama3", factor=8.0, original_len=8192.0),
          dict(scaling="llama3", factor=32.0, original_len=8192.0, low_freq=1.0, high_freq=4.0),
          dict(scaling="yarn", factor=40.0, original_len=4096.0), dict(scaling="yarn", factor=2.0, original_len=1.0),
          dict(scaling="yarn", factor=8.0, original_len=8192.0, beta_fast=16.0, beta_slow=2.0)]


@pytest.mark.parametrize("kw", TABLES, ids=lambda kw: kw.get("scaling", "plain") + str(kw.get("factor", "")))
@pytest.mark.parametrize("rot,base", [(2, 10000.0), (64, 10000.0), (128, 500000.0), (40, 1e6)])
def test_rope_tables_match_their_definition(rot, base, kw):
    freqs, magnitude = B.snap_rope_table(B.make_rope(rot_dim=rot, base=base, **kw))
    # a handful of double-precision operations per entry, powers and logarithms among them
    np.testing.assert_allclose(freqs.numpy(), orc.rope_table(rot, base, **kw), rtol=1e-13)
    want = 0.1 * math.log(kw["factor"]) + 1.0 if kw.get("scaling") == "yarn" else 1.0
    assert magnitude == pytest.approx(want, rel=1e-15)
    assert B.snap_rope_table(B.make_rope(rot_dim=rot, base=base, magnitude=1.25, **kw))[1] == 1.25


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=-2), dict(rot_offset=-1), dict(base=1.0), dict(base=math.nan),
                                dict(base=math.inf), dict(scaling=4), dict(scaling=-1), dict(interleaved=2), dict(magnitude=-1.0),
                                dict(magnitude=math.inf), dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=math.nan),
                                dict(scaling="llama3", factor=8.0), dict(scaling="llama3", factor=8.0, original_len=8192, high_freq=1.0),
                                dict(scaling="yarn", factor=8.0), dict(scaling="yarn", factor=8.0, original_len=4096, beta_fast=1.0),
                                dict(scaling="yarn", factor=8.0, original_len=4096, beta_slow=0.0)])
def test_rope_tables_refuse_what_has_no_meaning(kw):
    rope = B.make_rope(**{**dict(rot_dim=64, base=10000.0), **{k: v for k, v in kw.items() if k != "interleaved"}})
    rope.interleaved = kw.get("interleaved", 0)
    with pytest.raises(B.SnapError) as e:
        B.snap_rope_table(rope)
    assert e.value.code == -1
    assert B.lib().snap_rope_table(None, None, None) == -4


def test_rope_refuses_bad_calls():
    cfg, lib, one, odd = _cfg(), B.lib(), C.c_void_p(256), C.c_void_p(264)
    rope = B.make_rope(rot_dim=128)

    def call(cfg=cfg, rope=rope, freqs=one, pos=one, n=5, q=one, qs=(4096, 128), qo=one, qos=(4096, 128), k=one, ks=(1024, 128), ko=one,
             kos=(1024, 128), inverse=0):
        return lib.snap_rope(C.byref(cfg) if cfg else None, C.byref(rope) if rope else None, freqs, pos, n, q, *qs, qo, *qos, k, *ks, ko,
                             *kos, inverse, None)

    assert call(n=0) == 0                                               # nothing to do
    assert call(cfg=None) == -4 and call(rope=None) == -4 and call(freqs=None) == -4 and call(pos=None) == -4
    assert call(q=None) == -4 and call(ko=None) == -4                   # an input without its output, and the reverse
    assert call(q=None, qo=None, k=None, ko=None) == -4
    assert call(n=-1) == -1 and call(inverse=2) == -1
    assert call(q=odd) == -1 and call(ko=odd) == -1
    assert call(qs=(4097, 128)) == -1 and call(qos=(4096, 127)) == -1   # strides that are no multiple of 16 bytes
    assert call(qs=(8192, 128)) == -1                                   # in place with other strides
    two = C.c_void_p(1 << 20)
    assert call(qo=two, qos=(4096, 64)) == -1                           # heads of the output overlap
    assert call(ko=two, kos=(512, 128)) == -1                           # tokens of the output overlap
    assert call(rope=B.make_rope(rot_dim=130)) == -1                    # wider than the head
    assert call(rope=B.make_rope(rot_dim=64, rot_offset=80)) == -1
    assert call(rope=B.make_rope(rot_dim=63)) == -1
    assert call(cfg=_cfg(n_q_heads=30)) == -1


def _append(lib, cfg, paged, one, **kw):
    a = dict(slots=one, rows=one, n=4, rope=None, freqs=None, pos=None, q=None, qs=(4096, 128), qo=None, k=one, ks=(1024, 128), ko=None,
             v=one, vs=(1024, 128), kp=one, vp=one, table=one, seq_len=one, weights=None)
    a.update(kw)
    return lib.snap_paged_append(C.byref(cfg), C.byref(paged) if paged else None, a["slots"], a["rows"], a["n"],
                                 C.byref(a["rope"]) if a["rope"] else None, a["freqs"], a["pos"], a["q"], *a["qs"], a["qo"], a["k"],
                                 *a["ks"], a["ko"], a["v"], *a["vs"], a["kp"], a["vp"], a["table"], a["seq_len"], a["weights"], None, None)


def test_paged_calls_refuse_bad_arguments():
    cfg, paged, lib, one, odd = _cfg(), _paged(), B.lib(), C.c_void_p(256), C.c_void_p(264)
    ap = lambda cfg=cfg, paged=paged, **kw: _append(lib, cfg, paged, one, **kw)  # noqa: E731
    big = 1 << 40
    dec = lambda cfg=cfg, paged=paged, q=one, slots=one, n=4, kp=one, vp=one, table=one, seq_len=one, wi=None, wo=None, out=one, ws=one, size=big: (  # noqa: E731
        lib.snap_paged_decode_attn(C.byref(cfg), C.byref(paged) if paged else None, q, slots, n, kp, vp, table, seq_len, wi, wo, out, ws,
                                   size, None, None))
    ev = lambda cfg=cfg, paged=paged, src=one, dst=one, n=4, kp=one, vp=one, table=one, seq_len=one, w=one, ws=one, size=big: (  # noqa: E731
        lib.snap_paged_evict(C.byref(cfg), C.byref(paged) if paged else None, src, dst, n, kp, vp, table, seq_len, w, None, None, ws, size,
                             None, None))
    for call in (ap, dec, ev):
        assert call(n=0) == 0 and call(n=-1) == -1 and call(paged=None) == -4
        for missing in ("kp", "vp", "table", "seq_len"):
            assert call(**{missing: None}) == -4, missing
        assert call(kp=odd) == -1 and call(vp=odd) == -1
        for bad in (dict(page_tokens=0), dict(n_pages=0), dict(max_pages=0), dict(reserved=1), dict(k_page_stride=-1024),
                    dict(k_row_stride=100), dict(v_head_stride=12), dict(k_row_stride=64), dict(v_page_stride=0),
                    dict(page_tokens=1 << 20, max_pages=1 << 20)):
            assert call(paged=_paged(**bad)) == -1, bad
        latent = dict(n_q_heads=128, n_kv_heads=1, d_qk=576, d_v=512, v_aliases_k=True)
        wide_rows = dict(k_row_stride=640, v_row_stride=640, k_head_stride=10240, v_head_stride=10240)
        assert call(cfg=_cfg(**latent), paged=_paged(**wide_rows)) == -2
        assert call(cfg=_cfg(d_qk=272), paged=_paged(**wide_rows)) == -2
        assert call(cfg=_cfg(topk=-1)) == -1
    assert ap(slots=None) == -4 and ap(k=None) == -4 and ap(v=None) == -4 and ap(q=one) == -4 and ap(qo=one) == -4
    assert ap(rope=B.make_rope(rot_dim=128)) == -4                      # no frequencies
    assert ap(rope=B.make_rope(rot_dim=256), freqs=one) == -1
    assert ap(ks=(1024, 100)) == -1 and ap(vs=(-1024, 128)) == -1 and ap(k=odd) == -1 and ap(q=one, qo=odd) == -1
    assert ap(rows=None, n=65537) == -1                                 # every token the next one of its sequence: a batch, not a prompt
    assert ap(ko=one, ks=(6144, 128)) == -1                             # in place, but not dense like the output
    assert dec(slots=None) == -4 and dec(q=None) == -4 and dec(out=None) == -4 and dec(ws=None) == -4 and dec(wi=one) == -4
    assert dec(q=odd) == -1 and dec(out=odd) == -1 and dec(ws=odd) == -1
    need = B.snap_paged_decode_workspace_bytes(cfg, paged, 4)
    assert dec(size=need - 1) == -3 and dec(wo=one, size=need) == -3
    assert B.snap_paged_decode_workspace_bytes(cfg, paged, 4, True) >= need + 4 * 32 * 800 * 4
    assert ev(src=None) == -4 and ev(dst=None) == -4 and ev(w=None) == -4 and ev(ws=None) == -4 and ev(ws=odd) == -1
    need = B.snap_paged_evict_workspace_bytes(cfg, paged, 4)
    assert need >= 4 * 8 * 4096 * 4 and ev(size=need - 1) == -3
    assert ev(n=70000) == -1
    for f in (lambda: B.snap_paged_decode_workspace_bytes(cfg, paged, -1), lambda: B.snap_paged_evict_workspace_bytes(cfg, paged, -1)):
        with pytest.raises(B.SnapError):
            f()
    # one page or one KV head: the stride that is never applied may be anything
    assert ap(cfg=_cfg(n_q_heads=4, n_kv_heads=1), paged=_paged(k_head_stride=0, v_head_stride=0), n=0) == 0


def test_paged_weights_of_very_large_groups_are_refused():
    for dtype, d in ((B.SNAP_BF16, 128), (B.SNAP_F32, 128), (B.SNAP_F32, 256)):
        cfg = _cfg(n_q_heads=2048, n_kv_heads=1, d_qk=d, d_v=d, dtype=dtype)
        paged = _paged(k_row_stride=1024, v_row_stride=1024)
        assert B.snap_paged_decode_workspace_bytes(cfg, paged, 1, True) > 800 * 2048 * 4
        cfg.n_q_heads = 2049
        assert B.snap_paged_decode_workspace_bytes(cfg, paged, 1) > 0
        with pytest.raises(B.SnapError):
            B.snap_paged_decode_workspace_bytes(cfg, paged, 1, True)


def test_binding_checks_what_tensors_are():
    """The Python calls refuse tensors of another type, shape or place before the library sees their addresses."""
    cfg = _cfg()
    k = torch.zeros(100, 8, 16, 128, dtype=torch.bfloat16)
    table = torch.zeros(3, 50, dtype=torch.int32)
    paged = B.make_paged(k, k, table)
    assert (paged.page_tokens, paged.n_pages, paged.max_pages, paged.k_page_stride, paged.k_head_stride, paged.k_row_stride) == (
        16, 100, 50, 16384, 2048, 128)
    nhd = torch.zeros(100, 16, 8, 128, dtype=torch.bfloat16).transpose(1, 2)
    assert B.make_paged(nhd, nhd, table).k_head_stride == 128 and B.make_paged(nhd, nhd, table).k_row_stride == 1024
    q, out = torch.zeros(2, 32, 128, dtype=torch.bfloat16), torch.zeros(2, 32, 128, dtype=torch.bfloat16)
    i32 = lambda *s: torch.zeros(*s, dtype=torch.int32)  # noqa: E731
    ok = dict(q=q, slot_ids_dev=i32(2), n_active=2, k_pages=k, v_pages=k, page_table=table, seq_len=i32(3), out=out, workspace=i32(4))
    for bad, word in ((dict(), "CUDA"), (dict(q=q.float()), "expected"), (dict(slot_ids_dev=torch.zeros(2, dtype=torch.int64)), "int64"),
                      (dict(page_table=i32(3, 49)), "shape"), (dict(out=out[:1]), "shape"), (dict(q=q.transpose(0, 1)), "shape"),
                      (dict(weights_out=torch.zeros(3, 8, 799)), "shape"), (dict(k_pages=k.float()), "expected")):
        with pytest.raises(ValueError, match=word):
            B.snap_paged_decode_attn(cfg, paged, **{**ok, **bad})
    with pytest.raises(ValueError):
        B.make_paged(k, k[:, :4], table)
    with pytest.raises(ValueError, match="shape"):
        B.snap_rope(cfg, B.make_rope(rot_dim=128), torch.zeros(32, dtype=torch.float64), i32(2), q=q, q_out=out)
