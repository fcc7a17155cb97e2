"""cronus_build_tables against its plain form: every output, and what must stay as it was."""
import numpy as np
import pytest
import torch

from paper_2509_17357_amd import binding as B

import draft_util as D

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
FILL = -77


class State:
    def __init__(self, kv, new, held, width, count, capacity, most, seed=1):
        rng = np.random.default_rng(seed)
        self.kv, self.new, self.held = (np.array(x, np.int32) for x in (kv, new, held))
        self.n, self.width, self.count, self.capacity, self.most = len(kv), width, count, capacity, most
        used = int(np.clip(self.held, 0, width).sum())
        ids = rng.permutation(max(used + max(count, 0), 1)).astype(np.int32)
        self.table = np.full((self.n, width), FILL, np.int32)
        at = 0
        for s in range(self.n):
            h = int(np.clip(self.held[s], 0, width))
            self.table[s, :h] = ids[at:at + h]
            at += h
        self.free = np.full(capacity, FILL, np.int32)
        k = min(max(count, 0), capacity)
        self.free[:k] = ids[at:at + k]
        i32 = lambda a: torch.from_numpy(np.array(a, np.int32)).to(DEV)  # noqa: E731
        fill = lambda n, dt=torch.int32: torch.full((n,), FILL, dtype=dt, device=DEV)  # noqa: E731
        self.t = {"table": i32(self.table), "held": i32(self.held), "held_out": fill(self.n), "free": i32(self.free), "count": i32([count]),
                  "count_out": fill(1), "kv": i32(self.kv), "new": i32(self.new), "cu": fill(self.n + 1), "start": fill(self.n),
                  "cub": fill(self.n + 1), "slots": fill(most + 5, torch.int64), "report": fill(4)}

    def call(self, in_place=False, slots=True):
        t = self.t
        B.cronus_build_tables((t["table"], self.width, t["held"], t["held"] if in_place else t["held_out"], t["free"], self.capacity, t["count"],
                               t["count"] if in_place else t["count_out"]), t["kv"], t["new"], self.n, t["cu"], t["start"], t["cub"],
                              t["slots"] if slots else None, self.most, t["report"], torch.cuda.current_stream().cuda_stream)

    def check(self, in_place=False, slots=True):
        want = D.tables(self.kv, self.new, self.held, self.table, self.free, self.count, self.capacity, self.most)
        g = {k: v.cpu().numpy() for k, v in self.t.items()}
        report = g["report"].tolist()
        assert report[0] == want["status"]
        if want["status"] == B.CRONUS_TABLES_BAD_LENGTHS:
            assert report[3] == want["bad"]
        else:
            assert report == [want["status"], *want["asked"], -1]
        assert np.array_equal(g["held" if in_place else "held_out"], want["held"])
        assert g["count" if in_place else "count_out"].tolist() == [want["count"]]
        assert np.array_equal(g["cu"], want["cu_tokens"]) and np.array_equal(g["cub"], want["cu_blocks"])
        assert np.array_equal(g["start"], want["start"])
        table, free, tokens = want.get("table", self.table), self.free.copy(), np.zeros(0, int)
        if want["status"] == 0:
            free[:len(want["pushed"])] = want["pushed"]
            tokens = want["slots"]
        assert np.array_equal(g["table"], table) and np.array_equal(g["free"], free)
        assert np.array_equal(g["slots"][:len(tokens)], tokens) if slots else (g["slots"] == FILL).all()
        assert (g["slots"][len(tokens):] == FILL).all()
        assert np.array_equal(g["kv"], self.kv) and np.array_equal(g["new"], self.new)
        return want

    def run(self, **kw):
        self.call(**kw)
        torch.cuda.synchronize()
        return self.check(**kw)


def random_state(n, seed, ctx=200, new=40, ended=0.2, spare=200, most=None):
    rng = np.random.default_rng(seed)
    kv, add = rng.integers(0, ctx, n, endpoint=True), rng.integers(0, new, n, endpoint=True)
    add[rng.random(n) < ended] = -1
    held = -(-kv // 16) + rng.integers(0, 3, n)
    width = int(max(held.max(), (-(-(kv + np.maximum(add, 0)) // 16)).max()))
    need = int(np.maximum(0, -(-(kv + np.maximum(add, 0)) // 16) - held).sum())
    count = need + spare
    return State(kv, add, held, width, count, count + int(held.sum()), int(np.maximum(add, 0).sum()) if most is None else most, seed)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 300, 1023, 1024, 1025, 2500, 5000])
@pytest.mark.parametrize("in_place", [False, True])
def test_random_batches(n, in_place):
    assert random_state(n, n).run(in_place=in_place)["status"] == 0
    assert random_state(n, n + 1, ctx=3000, new=1, ended=0.5).run(in_place=in_place)["status"] == 0
    assert random_state(n, n + 2, spare=0, most=100_000).run(in_place=in_place, slots=False)["status"] in (0, 2)


@pytest.mark.parametrize("kv,new,held", [
    ([0], [0], [0]), ([0], [1], [0]), ([0], [16], [0]), ([0], [17], [0]), ([15], [1], [1]), ([16], [1], [1]), ([16], [1], [2]), ([16], [16], [1]),
    ([16], [0], [1]), ([31], [2], [2]), ([0, 0, 0], [0, 0, 0], [0, 1, 2]), ([5], [-1], [1]), ([0], [-1], [0]), ([0, 9], [-1, 40], [4, 1]),
    ([30, 0, 0, 7], [0, 3, 0, 12], [2, 0, 5, 1]), ([100, 100], [-1, -1], [7, 9])])
def test_edges(kv, new, held):
    for count in (0, 1, 3, 10):
        State(kv, new, held, 12, count, count + sum(held), 100).run()
        State(kv, new, held, 12, count, count + sum(held), int(np.maximum(new, 0).sum())).run(in_place=True)


def test_granted_blocks_are_the_ones_just_returned():
    w = State([100, 0], [-1, 100], [7, 0], 7, 0, 7, 100).run()
    assert w["status"] == 0 and w["count"] == 0


def test_refused_by_the_device():
    base = dict(width=8, count=10, capacity=40, most=200)
    for kv, new, held in (([5, -1], [1, 1], [1, 1]), ([5, 9], [1, -2], [1, 1]), ([5, 33], [1, 1], [1, 2]), ([5, 9], [1, 1], [1, -1]),
                          ([5, 9], [1, 1], [1, 9]), ([5, 100], [1, 29], [1, 7]), ([5, 9], [1, 2 ** 31 - 1], [1, 1]), ([5, 2 ** 31 - 1], [1, 2 ** 31 - 1], [1, 8]),
                          ([5, -2 ** 31], [1, -2 ** 31], [1, -2 ** 31]), ([5, 17], [1, -1], [1, 1]), ([5, -1], [1, -1], [1, 0])):
        for in_place in (False, True):
            w = State(kv, new, held, **base).run(in_place=in_place)
            assert (w["status"], w["bad"]) == (1, 1), (kv, new, held)
    many = State([5] * 3000, [1] * 3000, [1] * 2999 + [0], 8, 10, 5000, 5000).run()
    assert (many["status"], many["bad"]) == (1, 2999)
    for count, capacity in ((-1, 40), (41, 40), (39, 40)):  # the last: two blocks return to 39 of 40
        assert State([5, 17], [1, -1], [1, 2], 8, count, capacity, 200).run()["bad"] == -1
    assert State([5, 17], [1, -1], [1, 2], 8, 38, 40, 200).run()["status"] == 0
    assert State([5, 0], [1, 33], [1, 0], 8, 2, 40, 200).run()["status"] == 2
    assert State([5, 0], [1, 33], [1, 0], 8, 3, 40, 200).run()["status"] == 0
    assert State([5, 0], [1, 33], [1, 0], 8, 3, 40, 33).run()["status"] == 3
    assert State([5, 0], [1, 33], [1, 0], 8, 3, 40, 34).run()["status"] == 0
    # sums beyond 32 bits: of tokens (2^27 blocks of rows that are never reached), reported as the largest int
    s = State([0] * 40, [2 ** 27] * 40, [0] * 40, 1, 0, 0, 10)
    s.width = 2 ** 23
    s.call()
    torch.cuda.synchronize()
    assert s.t["report"].tolist() == [2, 2 ** 31 - 1, 40 * 2 ** 23, -1] and (s.t["cu"] == 0).all() and (s.t["slots"] == FILL).all()


def test_no_sequences_and_no_tokens():
    s = State([], [], [], 4, 3, 5, 0)
    s.call()
    torch.cuda.synchronize()
    s.check()
    State([5, 20], [0, 0], [1, 2], 4, 3, 5, 0).run()


def test_replays_grow_the_sequences():
    s = random_state(50, 9, ctx=30, new=9, ended=0.0, spare=600)
    s.width = 40
    table = np.full((50, 40), FILL, np.int32)
    table[:, :s.table.shape[1]] = s.table
    s.table, s.t["table"] = table, torch.from_numpy(table).to(DEV)
    s.most = 50 * 20
    s.t["slots"] = torch.full((s.most + 5,), FILL, dtype=torch.int64, device=DEV)
    before = {k: v.clone() for k, v in s.t.items()}
    s.call(in_place=True)  # compiled and loaded before the capture
    torch.cuda.synchronize()
    for k, v in before.items():
        s.t[k].copy_(v)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call(in_place=True)
    rng = np.random.default_rng(3)
    for _ in range(6):
        graph.replay()
        torch.cuda.synchronize()
        want = s.check(in_place=True)
        assert want["status"] == 0
        # the next iteration: some of the new tokens stay, other lengths, a few sequences end
        s.table, s.held, s.count = want["table"], want["held"].astype(np.int32), want["count"]
        s.free = s.t["free"].cpu().numpy()
        s.kv = (want["start"] + rng.integers(0, np.maximum(s.new, 0) + 1)).astype(np.int32)
        s.new = rng.integers(-1, 20, 50).astype(np.int32)
        s.t["kv"].copy_(torch.from_numpy(s.kv))
        s.t["new"].copy_(torch.from_numpy(s.new))
        s.t["slots"].fill_(FILL)


@pytest.mark.parametrize("most", [1, 63, 64, 1023, 1025, 2047, 2048, 2049, 4095, 4096, 4097])
@pytest.mark.parametrize("n", [1, 40, 1024])
def test_batches_on_both_sides_of_a_second_launch(n, most):
    """As many tokens as the call allows, in the sequences that have not ended; the blocks of the others are what these get."""
    new = np.full(n, -1)
    lives = np.arange(0, n, 2)
    new[lives] = most // len(lives) + (np.arange(len(lives)) < most % len(lives))
    kv = np.arange(n) % 37
    held = -(-kv // 16)
    need = int(np.maximum(0, -(-(kv + np.maximum(new, 0)) // 16) - held).sum())
    back = int(held[new == -1].sum())
    count = max(0, need - back)
    want = State(kv, new, held, int((kv.max() + new.max()) // 16 + 1), count, count + back, most, seed=most).run()
    assert want["status"] == 0 and want["asked"][0] == most
