"""Rotary and paged-cache calls without a GPU: what the Python calls say of arguments that are not what they should be."""
import ctypes as C
import os

import pytest
import torch

from paper_2511_03092_b200 import binding as B
from paper_2511_03092_b200 import build as snap_build


@pytest.fixture(scope="module", autouse=True)
def _built():
    snap_build.build()


def _layer():
    cfg = B.make_config(n_q_heads=4, n_kv_heads=2, d_qk=64, d_v=64, dtype=B.SNAP_BF16, l_sink=1, l_recent=4, topk=8, l_obs=1, pool_kernel=1,
                        softmax_scale=0.125, max_seqs=3)
    k = torch.zeros(10, 2, 16, 64, dtype=torch.bfloat16)
    table = torch.zeros(3, 5, dtype=torch.int32)
    return cfg, k, table, B.make_paged(k, k, table)


def i32(*shape, device="cpu"):
    return torch.zeros(*shape, dtype=torch.int32, device=device)


@pytest.mark.parametrize("bad,error,word", [(None, TypeError, "NoneType"), ([0, 1], TypeError, "list"), (i32(()), ValueError, "one dim"),
                                            (i32(2, 1), ValueError, "one dim"), (i32(2 ** 31, device="meta"), ValueError, "at most"),
                                            (i32(2 ** 32, device="meta"), ValueError, "at most")])
def test_what_counts_the_tokens_is_named_when_it_is_not_a_list_of_them(bad, error, word):
    cfg, k, table, paged = _layer()
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(error, match=f"snap_rope: positions .*{word}"):
        B.snap_rope(cfg, B.make_rope(rot_dim=64), torch.zeros(32, dtype=torch.float64), bad, q=q, q_out=q)
    with pytest.raises(error, match=f"snap_paged_append: slot_ids .*{word}"):
        B.snap_paged_append(cfg, paged, bad, None, k[0], k[0], k, k, table, i32(3))


@pytest.mark.parametrize("n", [2 ** 31, 2 ** 32 + 2, -1])
def test_counts_that_the_library_cannot_take_are_refused(n):
    cfg, k, table, paged = _layer()
    q, ws = torch.zeros(2, 4, 64, dtype=torch.bfloat16), i32(4)
    word = "at most" if n > 0 else "shape"
    with pytest.raises(ValueError, match=word):
        B.snap_paged_decode_attn(cfg, paged, q, i32(2), n, k, k, table, i32(3), q, ws)
    with pytest.raises(ValueError, match=word):
        B.snap_paged_evict(cfg, paged, i32(2), i32(2), n, k, k, table, i32(3), torch.zeros(3, 2, 80), None, ws)


def test_the_library_s_own_answer_comes_first():
    """A status that the call itself returned is raised as such, whatever else is wrong with the arguments."""
    cfg, k, table, paged = _layer()
    for call in (lambda: B.snap_rope(None, B.make_rope(rot_dim=64), None, None), lambda: B.snap_rope(cfg, None, None, None),
                 lambda: B.snap_paged_append(None, paged, None, None, None, None, k, k, table, None),
                 lambda: B.snap_paged_decode_attn(cfg, None, None, None, 2, k, k, table, None, None, None),
                 lambda: B.snap_paged_evict(None, paged, None, None, 2, k, k, table, None, None, None, None)):
        with pytest.raises(B.SnapError) as e:
            call()
        assert e.value.code == -4


def test_more_tokens_than_a_grid_can_number_are_refused():
    """The last block's spare threads number tokens past the last one: in 32 bits, up to 255 of them."""
    cfg, _, _, paged = _layer()
    lib, one, rope = B.lib(), C.c_void_p(256), B.make_rope(rot_dim=64)
    for n in (2 ** 31 - 1, 2 ** 31 - 255):
        assert lib.snap_rope(C.byref(cfg), C.byref(rope), one, one, n, one, 256, 64, one, 256, 64, None, 0, 0, None, 0, 0, 0, None) == -1
        assert lib.snap_paged_append(C.byref(cfg), C.byref(paged), one, one, n, None, None, None, None, 0, 0, None, one, 128, 64, None, one,
                                     128, 64, one, one, one, one, None, None, None) == -1


def test_the_module_belongs_to_its_interpreter_and_torch(monkeypatch, tmp_path):
    """_marshal is rebuilt for another torch even when the file is newer, and a stale one is refused, not used."""
    import sysconfig
    assert os.path.basename(snap_build.MARSHAL) == "_marshal" + sysconfig.get_config_var("EXT_SUFFIX")
    from paper_2511_03092_b200 import _marshal
    assert os.path.samefile(_marshal.__file__, snap_build.MARSHAL) and _marshal.torch_version == torch.__version__
    ran = []

    class Done:
        returncode, stdout, stderr = 0, "", ""
    monkeypatch.setattr(snap_build.subprocess, "run", lambda cmd, **kw: ran.append(cmd) or Done)
    snap_build.build_marshal()
    assert not ran                                          # up to date
    monkeypatch.setattr(torch, "__version__", "0.0.1")
    snap_build.build_marshal()
    assert len(ran) == 1 and '-DBUILT_FOR_TORCH="0.0.1"' in ran[0]
    monkeypatch.setattr(B, "_native", None)
    cfg, *_ = _layer()
    with pytest.raises(RuntimeError, match="not built for torch 0.0.1"):
        B.snap_rope(cfg, B.make_rope(rot_dim=64), torch.zeros(32, dtype=torch.float64), i32(2))


def test_the_library_builds_without_torch(monkeypatch, capsys):
    monkeypatch.setattr(snap_build.importlib.util, "find_spec", lambda name: None)
    monkeypatch.setattr(snap_build, "build_marshal", lambda *a: pytest.fail("the module needs torch"))
    assert snap_build.build() == snap_build.LIB
    assert "torch is not installed" in capsys.readouterr().err
