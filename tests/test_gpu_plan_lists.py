"""What the page plan writes, as its readers take it: lists of tokens and rows for the full-precision append, two tables used in turn; and
plans in place of all sizes."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as porc
from paper_2511_03092_b200 import binding as B
from tests.test_gpu_plan import Step, a_server

pytestmark = pytest.mark.gpu


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("in_turn", [False, True])
@pytest.mark.parametrize("most", [300, 9000])
def test_full_precision_pages_by_the_plans_lists(most, in_turn):
    """Prompts, steps, drafts taken back and sequences that end, appended by the lists of slots and rows (their padding too) and attended; with one
    table, or with two in turn, every live slot being listed.  The longer list takes the plan of two launches."""
    hq, hkv, d, page, seqs, pool, width = 4, 2, 64, 16, 5, 60, 30 if most == 300 else 2000
    cfg = B.make_config(n_q_heads=hq, n_kv_heads=hkv, d_qk=d, d_v=d, dtype=torch.bfloat16, l_sink=2, l_recent=8, topk=16, l_obs=1, pool_kernel=1,
                        softmax_scale=d ** -0.5, max_seqs=seqs)
    k_pages, v_pages = (torch.full((pool, hkv, page, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    tables = [torch.full((seqs, width), -1, dtype=torch.int32, device="cuda") for _ in range(2)]
    seq_len, status = i32([0] * seqs), i32([0])
    rng = np.random.default_rng(0)
    free, n_free = i32(rng.permutation(pool)), i32([pool])
    paged = B.make_paged(k_pages, v_pages, tables[0])
    g = torch.Generator(device="cuda").manual_seed(0)
    truth = [[np.zeros((0, hkv, d))] * 2 for _ in range(seqs)]
    at = 0

    def step(requests):
        nonlocal at
        n = len(requests)
        slots, new = i32([s for s, _ in requests]), i32([x for _, x in requests])
        first, cu, ts, tr = i32([0] * n), i32([0] * (n + 1)), i32([0] * most), i32([0] * most)
        ws = torch.empty(B.snap_paged_plan_workspace_bytes(cfg, paged, n), dtype=torch.uint8, device="cuda")
        before, after = tables[at], tables[1 - at if in_turn else at]
        kept = before.clone()
        B.snap_paged_plan(cfg, paged, slots, new, before, seq_len, free, n_free, first, cu, ts, tr, ws, page_table_out=after if in_turn else None,
                          status=status)
        if in_turn:
            assert torch.equal(before, kept)                # (a step that still runs reads it)
            at = 1 - at
        k, v = (torch.randn(most, hkv, d, device="cuda", generator=g).to(torch.bfloat16) for _ in range(2))
        B.snap_paged_append(cfg, paged, ts, tr, k, v, k_pages, v_pages, after, seq_len, status=status)
        lists = [x.tolist() for x in (first, cu)]
        for i, (s, x) in enumerate(requests):
            a, b, f = lists[1][i], lists[1][i + 1], lists[0][i]
            assert b - a == max(x, 0)
            truth[s] = [np.concatenate([t[:f], z[a:b].double().cpu().numpy()]) for t, z in zip(truth[s], (k, v))]
        assert seq_len.tolist() == [len(t[0]) for t in truth]
        q = torch.randn(seqs, hq, d, device="cuda", generator=g).to(torch.bfloat16)
        out = torch.empty_like(q)
        w = torch.empty(B.snap_paged_decode_workspace_bytes(cfg, paged, seqs), dtype=torch.uint8, device="cuda")
        B.snap_paged_decode_attn(cfg, paged, q, i32(range(seqs)), seqs, k_pages, v_pages, after, seq_len, out, w, status=status)
        for s in range(seqs):
            want, _, mass, _ = porc.decode(q[s].double().cpu().numpy(), *truth[s], cfg.softmax_scale)
            # logits to 2^-18 or so; weights to 8 bits and outputs to 8 bits, half a step each, and a few additions
            assert (np.abs(out[s].double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + (2.0 ** -8 + 2.0 ** -10) * mass).all()

    step([(0, 130), (2, 77), (1, 40), (4, 0)])
    for _ in range(3):
        step([(4, 1), (0, 1), (1, 1), (2, 0)])              # (2 idles, and is listed)
    seq_len.sub_(i32([2, 0, 3, 0, 1]))                      # drafts taken back
    truth = [[t[:n] for t in x] for x, n in zip(truth, seq_len.tolist())]
    step([(0, 1), (1, 3), (2, 20), (4, 1)])
    step([(0, -1), (3, 200), (1, 1), (2, 0), (4, 2)])
    step([(1, 0), (2, 17), (3, 1), (4, 0), (0, 5)])
    assert int(status.item()) == 0
    held = tables[at][tables[at] >= 0].tolist()
    assert len(set(held)) == len(held) and len(held) + int(n_free.item()) == pool


@pytest.mark.parametrize("n,width,page", [(16, 512, 4), (64, 2048, 4), (128, 512, 4), (128, 8192, 1), (200, 160, 4), (250, 512, 4), (250, 8192, 1), (256, 40, 4), (257, 40, 4)])
@pytest.mark.parametrize("ended", [0.0, 0.3, 1.0])
def test_plans_in_place_of_all_sizes(n, width, page, ended):
    """Steps of a token each in place, in one launch and in two by how many requests there are and how wide their rows."""
    rng = np.random.default_rng(n + width)
    slots, grow, table, length, stack, free = a_server(rng, n, width, page, n, width * page // 2, 1, ended=ended, spare=0.8)
    s = Step(slots, grow, table, length, stack, free, page, n, False)
    s.call()
    s.check()
