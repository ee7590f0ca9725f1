"""tkv_table_append against the token-by-token model: everything is whole numbers and has to be equal."""
import numpy as np
import pytest
import torch

from paper_2605_17170_amd import harness, tkv
import gpu_common as gc
from table_model import Table

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


class Device:
    """A table on the GPU beside the model of it."""

    def __init__(self, n_seqs, max_pages, p2, p4, key_axis=0, seed=None):
        self.desc = tkv.tkv_desc.make(1, p2, p4, int2_key_axis=key_axis)
        i32 = lambda *s: torch.full(s, -7, dtype=torch.int32, device=DEV)  # noqa: E731
        self.t = [i32(n_seqs, max_pages), i32(n_seqs), i32(n_seqs), i32(p2 + p4), i32(2)]
        self.table = tkv.tkv_table.make(*self.t)
        tkv.tkv_table_reset(self.desc, self.table)
        free = [None, None]
        if seed is not None:
            rng = np.random.default_rng(seed)
            free = [rng.permutation(p2), p2 + rng.permutation(p4)]
            self.t[3].copy_(torch.from_numpy(np.concatenate(free).astype(np.int32)))
        self.model = Table(n_seqs, max_pages, p2, p4, *free)
        self.kc = key_axis == 1

    def append(self, keep, lens, tags, max_work=None, tag_offset=0, stream=None):
        """Calls both; returns the device's outputs and status, and the model's answer."""
        n, tags = len(self.model.pages), np.asarray(tags, np.uint8)
        max_work = tkv.tkv_table_max_work(n, tags.size) if max_work is None else max_work
        d = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)  # noqa: E731
        held = torch.from_numpy(np.concatenate([np.zeros(tag_offset, np.uint8), tags])).to(DEV)[tag_offset:]
        i32 = lambda *s: torch.full(s, -9, dtype=torch.int32, device=DEV)  # noqa: E731
        out = {"indptr": i32(n + 1), "positions": i32(tags.size), "slots": i32(tags.size), "work_pages": i32(max_work), "work_src": i32(max_work, 64),
               "n_work": i32(1)}
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        ws = torch.full((tkv.tkv_table_workspace_bytes(n, tags.size),), 0xA5, dtype=torch.uint8, device=DEV)
        k = np.asarray(keep, np.int64).reshape(-1, 2) if keep is not None else None
        tkv.tkv_table_append(self.desc, self.table, d(k[:, 0]) if keep is not None else None, d(k[:, 1]) if keep is not None else None, d(lens), held,
                             *[out[x] for x in ("indptr", "positions", "slots", "work_pages", "work_src", "n_work")], ws, status, stream)
        torch.cuda.synchronize()
        return {x: v.cpu().numpy() for x, v in out.items()}, int(status.item()), self.model.append(keep, lens, tags, self.kc, max_work)

    def check_state(self):
        rows, n2, n4, free, n_free = (x.cpu().numpy() for x in self.t)
        m = self.model
        assert np.array_equal(rows, m.rows())
        assert np.array_equal(np.stack([n2, n4], 1), np.array(m.count, np.int32).reshape(-1, 2))
        assert n_free.tolist() == [len(f) for f in m.free]
        for w in range(2):
            assert free[m.lead[w]:m.lead[w] + n_free[w]].tolist() == [int(x) for x in m.free[w]]

    def check(self, got, status, want):
        assert not isinstance(want, str) and status == 0, (status, want)
        n = want["work_pages"].size
        for x in ("indptr", "positions", "slots"):
            assert np.array_equal(got[x], want[x]), x
        assert got["n_work"].tolist() == [n]
        assert np.array_equal(got["work_pages"][:n], want["work_pages"]) and np.all(got["work_pages"][n:] == 0)
        assert np.array_equal(got["work_src"][:n], want["work_src"]) and np.all(got["work_src"][n:] == -1)
        self.check_state()

    def check_refused(self, got, status, bits):
        assert status == bits
        assert np.all(got["positions"] == -1) and np.all(got["slots"] == -1) and np.all(got["work_src"] == -1)
        assert np.all(got["work_pages"] == 0) and got["n_work"].tolist() == [0] and np.all(got["indptr"] == 0)
        self.check_state()


def trace(rng, n, share4=0.4):
    """Runs of either width."""
    return np.repeat(rng.choice([2, 4], n // 9 + 1, p=[1 - share4, share4]), 9)[:n].astype(np.uint8)


@pytest.mark.parametrize("n_seqs,longest,steps", [(1, 1, 3), (1, 700, 4), (3, 64, 4), (17, 129, 3), (300, 5, 4), (1024, 7, 2),   # one workgroup
                                                  (5, 4000, 3), (1, 20000, 2), (64, 900, 3), (1000, 60, 2),      # sums in one
                                                  (1025, 3, 3), (2500, 9, 3), (64, 2500, 2), (2, 70000, 2)])                     # four launches
def test_lengths_cuts_and_widths(n_seqs, longest, steps):
    rng = np.random.default_rng(n_seqs * 31 + longest)
    pages = n_seqs * (longest * steps // 64 + 2) + 3
    dev = Device(n_seqs, 2 * (longest * steps // 64 + 2), pages, pages, seed=1)
    for step in range(steps):
        lens = rng.integers(0, longest + 1, n_seqs)
        lens[rng.random(n_seqs) < 0.1] = 0
        if step == 0:
            lens[-1] = longest
        keep = None
        if step:
            count = np.array(dev.model.count)
            keep = np.maximum(count - rng.integers(0, longest // 2 + 2, (n_seqs, 2)), 0)
            keep[rng.random(n_seqs) < 0.3] = 1 << 30       # everything
            keep[rng.random(n_seqs) < 0.1] = 0             # a request that has ended
        dev.check(*dev.append(keep, lens, trace(rng, int(lens.sum())), tag_offset=step))


@pytest.mark.parametrize("n_seqs,max_pages", [(128, 64), (128, 65), (1024, 64), (41, 2000)])
def test_pages_given_back_by_many_rows(n_seqs, max_pages):
    """Rows of 8192 entries together and of more: their pages go back in the launch of the sums or in one of their own."""
    rng = np.random.default_rng(max_pages)
    dev = Device(n_seqs, max_pages, 50 * n_seqs, 50 * n_seqs, seed=7)
    for step in range(4):
        count = np.array(dev.model.count)
        keep = np.maximum(0, count - rng.integers(0, 64 * 7, (n_seqs, 2)))
        lens = rng.integers(0, 120000 // n_seqs, n_seqs) if step < 3 else np.full(n_seqs, 9)
        while lens.sum() > 65536:
            lens //= 2
        keep[(count + lens[:, None]).sum(1) > 40 * 64] = 0
        dev.check(*dev.append(keep, lens, np.concatenate([trace(rng, int(lens.sum())), np.full(65536 - int(lens.sum()), 1, np.uint8)])))


def test_refusals_with_many_tokens():
    n_seqs, n = 7, 20000
    dev = Device(n_seqs, 60, 300, 40)
    dev.check(*dev.append(None, [100] * n_seqs, np.full(n, 2, np.uint8)))
    refused, exhausted, capacity = tkv.TKV_STATUS_TABLE_REFUSED, tkv.TKV_STATUS_POOL_EXHAUSTED, tkv.TKV_STATUS_CAPACITY
    lens, tags = np.full(n_seqs, 2500), np.full(n, 2, np.uint8)
    full = [(tags, lens + 1000, None, refused), (tags, np.array([5, -1] + [0] * 5), None, refused), (tags, np.array([1 << 29] * n_seqs), None, refused),
            (np.where(np.arange(n) == 17499, 3, tags), lens, None, refused), (np.where(np.arange(n) < 2561, 4, tags), lens, None, exhausted),   # 41 pages
            (tags, np.array([60 * 64] + [0] * 6), None, capacity), (tags, lens, 100, capacity)]
    for tags_, lens_, max_work, bits in full:
        got, status, want = dev.append(None, lens_, tags_.astype(np.uint8), max_work=max_work)
        assert isinstance(want, str)
        dev.check_refused(got, status, bits)
    dev.check(*dev.append([[64, 64]] * n_seqs, lens, np.where(np.arange(n) == 17500, 3, tags).astype(np.uint8)))
    dev.check(*dev.append([[64, 64]] * n_seqs, lens, np.where(np.arange(n) < 2500, 4, tags).astype(np.uint8)))             # all 40 pages


@pytest.mark.parametrize("n_seqs", [6, 1100])
def test_per_channel_keys(n_seqs):
    rng = np.random.default_rng(5)
    dev = Device(n_seqs, 40, n_seqs * 20, n_seqs * 20, key_axis=1, seed=2)
    for _ in range(2):
        chunks = [tkv.tkv_route_residual(trace(rng, int(rng.integers(0, 200)), 0.2)) for _ in range(n_seqs)]
        dev.check(*dev.append(None, [c.size for c in chunks], np.concatenate(chunks)))
    keep = np.array(dev.model.count)
    keep[::2] = 0, 0
    keep[1::2, 0] = np.maximum(0, keep[1::2, 0] - 32)
    dev.check(*dev.append(keep, [0] * n_seqs, np.zeros(0, np.uint8)))


@pytest.mark.parametrize("n_seqs", [4, 1030])
def test_padded_batch_and_tags_behind_it(n_seqs):
    rng = np.random.default_rng(9)
    dev = Device(n_seqs, 8, 4 * n_seqs, 4 * n_seqs)
    lens = rng.integers(0, 30, n_seqs)
    tags = np.concatenate([trace(rng, int(lens.sum())), np.full(77, 9, np.uint8)])     # what lies behind is not looked at
    dev.check(*dev.append(None, lens, tags))


def test_rows_that_move_far():
    """INT2 pages arrive in front of, and are cut from before, thousands of INT4 pages."""
    rng = np.random.default_rng(11)
    for n_seqs in (3, 1040):
        dev = Device(n_seqs, 2500, 600, 2400 + 4 * n_seqs)
        lens = [70] * n_seqs
        lens[1] = 64 * 2100 + 5
        dev.check(*dev.append(None, lens, np.full(sum(lens), 4, np.uint8)))
        lens = [1] * n_seqs
        lens[1] = 64 * 300 + 1
        dev.check(*dev.append(None, lens, np.full(sum(lens), 2, np.uint8) if n_seqs < 10 else np.concatenate(
            [np.full(x, 2 if b == 1 else 4, np.uint8) for b, x in enumerate(lens)])))
        keep = np.array(dev.model.count)
        keep[1, 0] = 64 * 40
        dev.check(*dev.append(keep, [3] * n_seqs, np.full(3 * n_seqs, 4, np.uint8)))
        keep = np.array(dev.model.count)
        keep[1, 0] = 0
        dev.check(*dev.append(keep, [0] * n_seqs, np.zeros(0, np.uint8)))


@pytest.mark.parametrize("n_seqs", [5, 1100])
def test_refusals_leave_everything(n_seqs):
    rng = np.random.default_rng(13)
    spare = 3
    dev = Device(n_seqs, 6, n_seqs + spare, 2 * n_seqs, seed=4)
    lens = np.full(n_seqs, 10)
    dev.check(*dev.append(None, lens, np.full(10 * n_seqs, 2, np.uint8)))
    refused, exhausted, capacity = tkv.TKV_STATUS_TABLE_REFUSED, tkv.TKV_STATUS_POOL_EXHAUSTED, tkv.TKV_STATUS_CAPACITY

    def refuse(bits, *args, **kw):
        got, status, want = dev.append(*args, **kw)
        assert isinstance(want, str)
        dev.check_refused(got, status, bits)

    two = np.full(2 * n_seqs, 4, np.uint8)
    bad = lens * 0 + 2
    bad[n_seqs // 2] = -1
    refuse(refused, None, bad, two)
    bad[n_seqs // 2] = 3
    refuse(refused, None, bad, two)                                         # more than there are
    bad[:] = 1 << 30
    refuse(refused, None, bad, two)
    odd = two.copy()
    odd[-1] = 3
    refuse(refused, None, lens * 0 + 2, odd)
    odd[-1], odd[0] = 4, 0
    refuse(refused, None, lens * 0 + 2, odd)
    keep = np.full((n_seqs, 2), 1 << 30)
    keep[-1, 1] = -1
    refuse(refused, keep, lens * 0 + 2, two)
    # one more page of INT2 for every sequence, and only `spare` are free
    refuse(exhausted, None, lens * 0 + 64, np.full(64 * n_seqs, 2, np.uint8))
    # a row takes six pages
    big = lens * 0
    big[0] = 64 * 5 + 1
    refuse(capacity, None, big, np.full(int(big[0]), 4, np.uint8))
    refuse(capacity, None, lens * 0 + 2, two, max_work=n_seqs - 1)
    # what is given back in the same call counts as free
    keep = np.full((n_seqs, 2), 1 << 30)
    keep[1:5, 0] = 0
    big[0] = 64 * (spare + 2)
    dev.check(*dev.append(keep, big, np.full(int(big[0]), 2, np.uint8)))


def test_a_table_that_contradicts_itself_is_refused():
    for n_seqs in (2, 1030):
        dev = Device(n_seqs, 4, 8, 8)
        tags = np.full(n_seqs, 4, np.uint8)
        for which, at, value in ((1, 0, -1), (2, 1, 64 * 4 + 1), (1, 1, 2 ** 31 - 1), (4, 0, -1), (4, 1, 9), (4, 0, 2 ** 30)):
            old = int(dev.t[which][at])
            dev.t[which][at] = value
            before = [x.clone() for x in dev.t]
            _, status, _ = dev.append(None, [0] * n_seqs, tags)
            assert status & tkv.TKV_STATUS_TABLE_REFUSED and all(torch.equal(a, b) for a, b in zip(before, dev.t))
            dev.t[which][at] = old
        # more pages given back than the pool has
        dev.t[4].zero_()
        dev.t[4] += 8
        dev.t[1][0] = 64
        before = [x.clone() for x in dev.t]
        _, status, _ = dev.append([[0, 0]] * n_seqs, [0] * n_seqs, tags)
        assert status == tkv.TKV_STATUS_TABLE_REFUSED and all(torch.equal(a, b) for a, b in zip(before, dev.t))


def test_outputs_that_are_not_asked_for():
    dev = Device(3, 4, 8, 8)
    n_work, ws = torch.zeros(1, dtype=torch.int32, device=DEV), torch.empty(tkv.tkv_table_workspace_bytes(3, 6), dtype=torch.uint8, device=DEV)
    pages, src = torch.empty(6, dtype=torch.int32, device=DEV), torch.empty((6, 64), dtype=torch.int32, device=DEV)
    lens = torch.tensor([1, 2, 3], dtype=torch.int32, device=DEV)
    tags = torch.full((6,), 4, dtype=torch.uint8, device=DEV)
    tkv.tkv_table_append(dev.desc, dev.table, None, None, lens, tags, None, None, None, pages, src, n_work, ws)
    dev.model.append(None, [1, 2, 3], [4] * 6)
    tkv.tkv_table_append(dev.desc, dev.table, None, None, None, None, None, None, None, None, None, n_work, ws)
    torch.cuda.synchronize()
    assert n_work.item() == 0
    dev.check_state()


@pytest.mark.parametrize("n_seqs", [8, 1200])
def test_captured_drafting_and_rejecting(n_seqs):
    """A graph of one cut and one append, replayed with other lengths in its buffers, against the model."""
    rng = np.random.default_rng(17)
    dev = Device(n_seqs, 12, 8, 8 * n_seqs, seed=6)
    dev.check(*dev.append(None, rng.integers(1, 200, n_seqs), np.full(200 * n_seqs, 4, np.uint8)))
    t, most = 5 * n_seqs, tkv.tkv_table_max_work(n_seqs, 5 * n_seqs)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device=DEV)  # noqa: E731
    keep2, keep4, lens, tags = i32(n_seqs), i32(n_seqs), i32(n_seqs), torch.full((t,), 4, dtype=torch.uint8, device=DEV)
    out = {"indptr": i32(n_seqs + 1), "positions": i32(t), "slots": i32(t), "work_pages": i32(most), "work_src": i32(most, 64), "n_work": i32(1)}
    ws = torch.empty(tkv.tkv_table_workspace_bytes(n_seqs, t), dtype=torch.uint8, device=DEV)
    status = i32(1)
    call = lambda: tkv.tkv_table_append(dev.desc, dev.table, keep2, keep4, lens, tags, *out.values(), ws, status)  # noqa: E731
    state = [x.clone() for x in dev.t]
    keep4.fill_(1 << 30)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for x, y in zip(dev.t, state):
        x.copy_(y)
    for step in range(5):
        keep = np.array(dev.model.count)
        keep[:, 1] = np.maximum(0, keep[:, 1] - rng.integers(0, 6, n_seqs))
        new = rng.integers(0, 6, n_seqs)
        keep4.copy_(torch.from_numpy(keep[:, 1].astype(np.int32)))
        lens.copy_(torch.from_numpy(new.astype(np.int32)))
        graph.replay()
        torch.cuda.synchronize()
        dev.check({k: v.cpu().numpy() for k, v in out.items()}, int(status.item()), dev.model.append(keep, new, np.full(t, 4, np.uint8), max_work=most))


def test_the_work_list_padded_to_its_bound_goes_through_append():
    """tkv_quantize_append with n_work = max_work writes what it writes with the host's list."""
    q, K, V, bits = gc.random_case(23, [150, 1, 333], 4, 1)
    tags = np.concatenate(bits)
    dK, dV = harness.bf16_tensor(K, DEV), harness.bf16_tensor(V, DEV)
    dev = Device(3, 20, 12, 12)
    got, status, want = dev.append(None, [b.size for b in bits], tags)
    dev.check(got, status, want)
    d = lambda a: torch.from_numpy(a).to(DEV)  # noqa: E731
    pools = []
    for n in (got["work_pages"].size, want["work_pages"].size):
        pool = torch.full((tkv.tkv_pool_bytes(dev.desc),), 0xA5, dtype=torch.uint8, device=DEV)
        bmap, st = torch.zeros(24, dtype=torch.uint8, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        tkv.tkv_quantize_append(dev.desc, pool, bmap, dK, dV, d(tags), d(got["work_pages"][:n].copy()), d(got["work_src"][:n].copy()), st)
        torch.cuda.synchronize()
        assert st.item() == 0
        pools.append((pool, bmap))
    assert got["work_pages"].size > want["work_pages"].size
    assert torch.equal(pools[0][0], pools[1][0]) and torch.equal(pools[0][1], pools[1][1])
