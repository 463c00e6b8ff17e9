"""The page plan on the GPU against its definition, which serves the requests one after the other."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as orc
from paper_2511_03092_b200 import binding as B

pytestmark = pytest.mark.gpu
BITS = {"slot": B.SNAP_DEV_BAD_SLOT, "page": B.SNAP_DEV_BAD_PAGE, "room": B.SNAP_DEV_NO_ROOM}


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def config(max_seqs):
    return B.make_config(n_q_heads=1, n_kv_heads=1, d_qk=16, d_v=16, dtype=torch.bfloat16, l_sink=4, l_recent=8, topk=4, l_obs=1, pool_kernel=1,
                         softmax_scale=1.0, max_seqs=max_seqs)


class Step:
    """One call's arrays; what is not written stays recognisable."""

    def __init__(self, slots, new, table, seq_len, stack, n_free, page, most, apart=True):
        self.host = (list(slots), list(new), np.asarray(table), np.asarray(seq_len), np.asarray(stack), int(n_free), page, len(stack), most)
        n = len(slots)
        self.cfg = config(len(table))
        self.table, self.seq_len, self.stack, self.n_free = i32(table), i32(seq_len), i32(stack), i32([n_free])
        self.slots, self.new, self.apart = i32(slots).reshape(n), i32(new).reshape(n), apart
        self.out = torch.full_like(self.table, -77) if apart else self.table
        self.n_out = i32([-77]) if apart else self.n_free
        full = lambda *s: torch.full(s, -77, dtype=torch.int32, device="cuda")  # noqa: E731
        self.granted, self.first, self.cu, self.ts, self.tr, self.status = full(n), full(n), full(n + 1), full(most), full(most), i32([0])
        self.paged = B.make_page_map(page, len(stack), self.table)
        self.ws = full(B.snap_paged_plan_workspace_bytes(self.cfg, self.paged, n) // 4)

    def call(self, stream=None):
        B.snap_paged_plan(self.cfg, self.paged, self.slots, self.new, self.table, self.seq_len, self.stack, self.n_free, self.first, self.cu,
                          self.ts, self.tr, self.ws, page_table_out=self.out if self.apart else None,
                          n_free_out=self.n_out if self.apart else None, granted=self.granted, status=self.status, stream=stream)

    def check(self):
        torch.cuda.synchronize()
        want, said = orc.plan(*self.host)
        listed = sorted({s for s in self.host[0] if 0 <= s < len(want["table"])})
        rows = np.full_like(want["table"], -77) if self.apart else self.host[2].copy()
        rows[listed] = want["table"][listed]
        np.testing.assert_array_equal(self.out.cpu().numpy(), rows)
        for got, name in ((self.seq_len, "seq_len"), (self.stack, "stack"), (self.granted, "granted"), (self.first, "first"), (self.cu, "cu"),
                          (self.ts, "token_slots"), (self.tr, "token_rows")):
            np.testing.assert_array_equal(got.cpu().numpy(), np.asarray(want[name]), err_msg=name)
        assert int(self.n_out.item()) == want["n_free"]
        assert int(self.status.item()) == sum(BITS[x] for x in said)
        return want


def a_server(rng, max_seqs, width, page, n, longest, new, ended=0.3, spare=1.0, holes=False, junk=False):
    """A consistent server's state: lengths, their pages anywhere in the pool, a stack of others; and a step's requests."""
    length = rng.integers(0, min(longest, width * page) + 1, max_seqs)
    need = -(-length // page)
    order = rng.permutation(int(need.sum()) + int(spare * n * (new // page + 1)) + 5)
    table, at = np.full((max_seqs, width), -1), 0
    for s in range(max_seqs):
        table[s, :need[s]] = order[at:at + need[s]]
        at += need[s]
    free = order[at:]
    if holes:                                               # pages set aside behind the last row, in no order; numbers that are no page
        for s in rng.permutation(max_seqs)[:max_seqs // 2 + 1]:
            for j in rng.permutation(np.arange(need[s], width))[:rng.integers(0, 4)]:
                if len(free) > 3:
                    table[s, j], free = free[-1], free[:-1]
        table[rng.random(table.shape) < 0.02] = -5
    stack = np.full(len(order), -3)
    stack[:len(free)] = free
    slots = rng.permutation(max_seqs)[:n]
    grow = np.where(rng.random(n) < ended, -1 - rng.integers(0, 3, n), rng.integers(0, new + 1, n))
    if junk:
        slots = np.where(rng.random(n) < 0.15, -1, slots)
        slots = np.where(rng.random(n) < 0.1, slots[rng.integers(0, n, n)], slots)          # listed again
        slots = np.where(rng.random(n) < 0.05, max_seqs + rng.integers(0, 5, n), slots)
        slots = np.where(rng.random(n) < 0.05, -2 - rng.integers(0, 5, n), slots)
        grow = np.where(rng.random(n) < 0.05, width * page + 1, grow)
    return slots.tolist(), grow.tolist(), table, length, stack, len(free)


@pytest.mark.parametrize("apart", [True, False])
@pytest.mark.parametrize("seed", range(24))
def test_plans_match_their_definition(seed, apart):
    rng = np.random.default_rng(seed)
    page = int(rng.choice([1, 5, 16, 64]))
    max_seqs = int(rng.choice([1, 3, 33, 200, 1500]))
    n, width = int(rng.integers(1, max_seqs + 1)), int(rng.choice([1, 7, 40, 300]))
    new = int(rng.choice([1, 3, 50, 400]))
    slots, grow, table, length, stack, free = a_server(rng, max_seqs, width, page, n, width * page, new, spare=float(rng.choice([0.2, 2.0])),
                                                       holes=seed % 3 == 1, junk=seed % 4 >= 2)
    wanted = sum(max(x, 0) for x in grow if x <= new)
    most = int(rng.choice([wanted + 7, wanted // 2, 0]))
    s = Step(slots, grow, table, length, stack, free, page, most, apart)
    s.call()
    s.check()


@pytest.mark.parametrize("n", [2047, 2048, 2049, 9000])
def test_many_requests(n):
    """More requests than a block has threads, or keeps in shared memory."""
    rng = np.random.default_rng(n)
    slots, grow, table, length, stack, free = a_server(rng, n + 3, 6, 16, n, 80, 12, spare=1.5, junk=True)
    s = Step(slots, grow, table, length, stack, free, 16, sum(max(x, 0) for x in grow if x <= 12) - 5)
    s.call()
    s.check()


def test_one_long_prompt_and_a_full_row():
    """A row whose last entry is taken; a request that ends a sequence of every page; the whole list from one request."""
    rng = np.random.default_rng(2)
    width, page = 9000, 4
    order = rng.permutation(3 * width)
    table = np.full((3, width), -1)
    table[1] = order[:width]
    stack = np.full(3 * width, -3)
    stack[:width] = order[width:2 * width]
    s = Step([0, 1, 2], [width * page, -1, width * page - 1], table, [0, width * page, 0], stack, width, page, 2 * width * page - 1)
    s.call()
    want = s.check()
    assert want["granted"] == [width * page, 0, width * page - 1] and want["n_free"] == 0


@pytest.mark.parametrize("apart", [True, False])
def test_what_is_out_of_range(apart):
    table = np.array([[0, 1, -1], [2, -1, -1], [3, 99, -1]])
    stack = np.array([4, 5, 6, 7, 0, 0, 0, 0])
    for n_free, slots, new, length in ((12, [0], [1], [8, 4, 4]),        # more free pages than there are
                                       (-4, [0, 1], [1, 4], [8, 4, 4]),  # fewer than none
                                       (7, [0, 1], [-1, -1], [8, 4, 4]),  # more given back than the stack takes
                                       (4, [2, 0], [-1, 4], [8, 4, 8]),  # a number that is no page is not given back
                                       (4, [0, 1], [2, 2 ** 30], [-6, 4, 4]),            # a length below zero; a request past the table
                                       (4, [0, 1], [2 ** 31 - 1, 2 ** 31 - 1], [8, 4, 4]),
                                       (4, [0, 2 ** 31 - 1, -2 ** 31], [0, 1, 1], [8, 4, 4])):
        s = Step(slots, new, table, length, stack, n_free, 4, 20, apart)
        s.call()
        s.check()


def test_tokens_wanted_past_32_bits_are_refused():
    n = 9
    s = Step(list(range(n)), [2 ** 29] * n, np.full((n, 2 ** 12), -1), [0] * n, np.arange(50), 50, 2 ** 18, 40)
    s.call()
    assert s.check()["granted"] == [0] * n


def test_no_requests_and_no_list():
    s = Step([], [], np.full((2, 3), -1), [5, 6], np.arange(8), 5, 4, 11)
    s.call()
    s.check()
    s = Step([1, 0], [0, -1], np.array([[2, -1], [1, -1]]), [3, 4], np.array([0, 0, 0]), 1, 4, 0)
    s.call()
    s.check()


def test_a_plan_made_again_takes_no_second_page():
    """Tokens that were given up leave their pages to the row: the next plan of the sequence finds them held."""
    rng = np.random.default_rng(4)
    slots, grow, table, length, stack, free = a_server(rng, 20, 40, 8, 20, 200, 60, ended=0.0, spare=3.0)
    s = Step(slots, grow, table, length, stack, free, 8, sum(grow), apart=False)
    s.call()
    once = (s.table.clone(), s.n_free.clone())
    s.check()
    s.call()
    assert torch.equal(s.table, once[0]) and torch.equal(s.n_free, once[1])


def test_captured_replayed_and_on_another_stream():
    rng = np.random.default_rng(6)
    side = torch.cuda.Stream()
    steps = []
    for k in range(2):
        slots, grow, table, length, stack, free = a_server(rng, 60, 50, 16, 40, 500, 90)
        s = Step(slots, grow, table, length, stack, free, 16, 5000)
        steps.append(s)
    a, b = steps
    side.wait_stream(torch.cuda.current_stream())
    a.call(stream=side)                                     # two calls that may overlap, each with scratch of its own
    b.call()
    torch.cuda.synchronize()
    a.check(), b.check()
    # a graph of one call, replayed with other requests
    c = Step(*a.host[:6], 16, 5000)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call()
    graph.replay()
    c.check()
    c.slots.copy_(b.slots), c.new.copy_(b.new), c.table.copy_(b.table), c.seq_len.copy_(i32(b.host[3]))
    stack = np.full(len(c.host[4]), -3)
    keep = min(len(stack), len(b.host[4]))
    stack[:keep] = np.minimum(b.host[4][:keep], len(stack) - 1)
    c.stack.copy_(i32(stack)), c.n_free.fill_(3), c.out.fill_(-77), c.status.zero_()
    c.host = (*b.host[:4], stack, 3, 16, len(stack), 5000)
    graph.replay()
    c.check()
