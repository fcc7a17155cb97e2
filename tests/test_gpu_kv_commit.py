"""cronus_kv_commit against its plain form, whole pools bit for bit."""
import numpy as np
import pytest
import torch

from paper_2509_17357_amd import binding as B

import draft_util as D

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


class State:
    def __init__(self, start, count, paths, path_lens=None, hkv=2, d=64, dt="bf16", layers=1, seed=0, first_row=0, max_path=None):
        rng = np.random.default_rng(seed)
        self.hkv, self.d, self.dt, self.n = hkv, d, dt, len(start)
        self.start, self.count = np.array(start, np.int32), np.array(count, np.int32)
        self.cu = (first_row + np.concatenate([[0], np.cumsum(self.count)])).astype(np.int32)
        self.max_path = max(len(p) for p in paths) if max_path is None else max_path
        self.paths = rng.integers(-5, 200, (self.n, self.max_path)).astype(np.int32)  # entries behind a path may be anything
        for s, p in enumerate(paths):
            self.paths[s, :len(p)] = p
        self.path_lens = np.array([len(p) for p in paths] if path_lens is None else path_lens, np.int32)
        need = -(-(np.maximum(self.start.astype(np.int64), 0) + np.maximum(self.count, 0)) // 16)
        self.width = max(1, int(need.max()))
        self.blocks = int(need.sum()) + 2
        self.table, ids, at = np.full((self.n, self.width), -1, np.int32), rng.permutation(self.blocks), 0
        for s in range(self.n):
            self.table[s, :need[s]] = ids[at:at + need[s]]
            at += need[s]
        dtype = np.uint8 if dt == "fp8" else np.uint16
        size = self.blocks * hkv * 16 * d
        self.pools = [[rng.integers(0, 256 ** dtype().itemsize, size).astype(dtype) for _ in range(2)] for _ in range(layers)]
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)  # noqa: E731
        view = lambda a: dev(a if dt == "fp8" else a.view(np.int16))  # noqa: E731
        scale = torch.ones(hkv, device=DEV) if dt == "fp8" else None
        self.t = {"start": dev(self.start), "cu": dev(self.cu), "paths": dev(self.paths), "lens": dev(self.path_lens), "table": dev(self.table),
                  "out": torch.full((self.n,), -7, dtype=torch.int32, device=DEV)}
        self.dev_pools = [[view(x) for x in layer] for layer in self.pools]
        self.scale = scale
        self.caches = [B.make_cache(k, v, self.blocks, 2 * hkv, hkv, d, B.CRONUS_KV_FP8_E4M3 if dt == "fp8" else B.CRONUS_KV_BF16, scale, scale)
                       for k, v in self.dev_pools]

    def call(self, out=True):
        t = self.t
        B.cronus_kv_commit(self.caches, t["start"], t["cu"], t["paths"], self.max_path, t["lens"], t["table"], self.width, self.n,
                           t["out"] if out else None, torch.cuda.current_stream().cuda_stream)

    def check(self, out=True):
        for (k, v), (dk, dv) in zip(self.pools, self.dev_pools):
            lens = D.commit(k, v, self.hkv, self.d, self.start, self.cu, self.paths, self.path_lens, self.table)
            assert np.array_equal(dk.cpu().numpy().view(k.dtype), k) and np.array_equal(dv.cpu().numpy().view(v.dtype), v)
        assert self.t["out"].tolist() == (lens.tolist() if out else [-7] * self.n)
        return lens

    def run(self, out=True):
        self.call(out)
        torch.cuda.synchronize()
        return self.check(out)


def random_path(rng, n, most):
    m = int(rng.integers(0, min(n, most), endpoint=True))
    return sorted(rng.choice(n, m, replace=False).tolist())


SHAPES = [(2, 64, "bf16"), (8, 128, "bf16"), (4, 128, "fp8"), (3, 64, "fp8"), (1, 128, "bf16")]


@pytest.mark.parametrize("hkv,d,dt", SHAPES)
@pytest.mark.parametrize("n,most", [(1, 1), (7, 7), (26, 6), (64, 17), (150, 90), (300, 300)])
def test_random_paths(hkv, d, dt, n, most):
    rng = np.random.default_rng(n)
    count = rng.integers(1, n, 9, endpoint=True)
    start = [0, 1, 15, 16, 17, 100, 255, 7, 31]
    State(start, count, [random_path(rng, c, most) for c in count], hkv=hkv, d=d, dt=dt, seed=n, first_row=3, max_path=most).run()


@pytest.mark.parametrize("hkv,d,dt", SHAPES)
def test_paths_whose_places_are_sources_too(hkv, d, dt):
    n = 80
    paths = [list(range(1, n)), list(range(n)), [0] + list(range(2, n)), list(range(40, n)), list(range(16, n)), list(range(0, n, 2)), [n - 1], []]
    State([5, 0, 16, 31, 48, 100, 3, 9], [n] * 8, paths, hkv=hkv, d=d, dt=dt, seed=1).run()


def test_paths_end_at_the_first_entry_that_does_not_count():
    paths = [[0, 2, 2, 5], [0, 3, 1], [4, 10], [-1, 2], [2, -3, 5], [0, 1, 9, 9], [1, 2, 3, 4], [2 ** 31 - 1, 1], [3, 5, 7, 9]]
    lens = [4, 3, 2, 2, 3, 4, 2, 2, 9]
    s = State([20 + i for i in range(9)], [10] * 9, paths, path_lens=lens, seed=2, max_path=4)
    assert (s.run() - s.start).tolist() == [2, 2, 1, 0, 1, 3, 2, 0, 4]
    long = [list(range(0, 130)) + [7] + list(range(140, 150)), list(range(1, 65)) + [64] + list(range(66, 80)), list(range(3, 131))]
    s = State([5, 6, 7], [160] * 3, long, seed=3)
    assert (s.run() - s.start).tolist() == [130, 64, 128]
    s = State([5, 6], [10] * 2, [[1, 2]] * 2, path_lens=[-4, 2 ** 31 - 1], seed=4, max_path=2)
    assert (s.run() - s.start).tolist() == [0, 2]
    State([5, 6], [10] * 2, [[], []], seed=5, max_path=0).run()


def test_sequences_whose_tokens_lie_nowhere():
    for change in ({0: -1}, {1: 10 ** 9}, {2: -2 ** 31}, {1: 2 ** 31 - 1}):
        s = State([20, 40, 60, 33], [9, 9, 9, 9], [[2, 4, 8]] * 4, seed=6)
        for k, x in change.items():
            s.start[k] = x
        s.t["start"].copy_(torch.from_numpy(s.start))
        s.run()
    s = State([20, 40, 60], [9, 0, 9], [[2, 4, 8]] * 3, seed=7)
    assert (s.run() - s.start).tolist() == [3, 0, 3]
    s = State([20, 40, 60], [9, 5, 9], [[2, 4]] * 3, seed=8)
    s.cu[2] = s.cu[1] - 3  # offsets that fall
    s.t["cu"].copy_(torch.from_numpy(s.cu))
    s.run()


@pytest.mark.parametrize("layers", [2, 63, 64, 65, 130])
def test_layers(layers):
    rng = np.random.default_rng(layers)
    s = State([3, 30, 16], [20, 33, 9], [random_path(rng, c, 8) for c in (20, 33, 9)], hkv=2, d=64, layers=layers, seed=layers)
    s.run()
    State([3, 30], [20, 33], [[1, 5], [0, 1, 9]], dt="fp8", layers=layers, seed=layers).run(out=False)


def test_replays_and_another_stream():
    rng = np.random.default_rng(11)
    s = State([30, 5, 100], [26, 12, 40], [[1], [1], [1]], hkv=8, d=128, layers=3, seed=11, max_path=9)
    s.call()  # loaded before the capture
    torch.cuda.synchronize()
    s.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.call()
    side = torch.cuda.Stream()
    for k in range(6):
        for i in range(s.n):
            p = random_path(rng, int(s.count[i]), 9)
            s.paths[i, :len(p)], s.path_lens[i] = p, len(p)
        s.t["paths"].copy_(torch.from_numpy(s.paths))
        s.t["lens"].copy_(torch.from_numpy(s.path_lens))
        s.t["out"].fill_(-7)
        if k % 2:
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                s.call()
            torch.cuda.current_stream().wait_stream(side)
        else:
            graph.replay()
        torch.cuda.synchronize()
        s.check()


def test_blocks_beyond_4_gib():
    hkv, d = 8, 128
    s = State([30, 5], [26, 12], [[2, 5, 9], [1, 11]], hkv=hkv, d=d, seed=12)
    per, blocks = hkv * 16 * d, (5 << 30) // (hkv * 16 * d * 2)
    big = [torch.empty(blocks * per, dtype=torch.int16, device=DEV) for _ in range(2)]
    for i in range(s.blocks):
        for to, src in zip(big, s.dev_pools[0]):
            to[(blocks - 1 - i) * per:(blocks - i) * per] = src[i * per:(i + 1) * per]
    s.caches = [B.make_cache(big[0], big[1], blocks, 2 * hkv, hkv, d)]
    s.t["table"] = torch.from_numpy(np.where(s.table >= 0, blocks - 1 - s.table, -1).astype(np.int32)).to(DEV)
    s.call()
    torch.cuda.synchronize()
    for i in range(s.blocks):
        for src, to in zip(big, s.dev_pools[0]):
            to[i * per:(i + 1) * per] = src[(blocks - 1 - i) * per:(blocks - i) * per]
    s.check()


def test_positions_end_with_32_bits():
    """Tables with room for 2^31 positions and more: tokens that pass them lie nowhere, those just before them move."""
    width = 2 ** 27 + 8
    b = State([2, 2], [6, 6], [[1, 3, 5], [0, 2]])
    table = torch.empty(2, width, dtype=torch.int32, device=DEV)
    table[:, :] = b.t["table"][:, :1]
    start = np.array([2 ** 31 - 16 + 2, 2 ** 31 - 16 + 12], np.int32)
    b.t["table"], b.t["start"], b.width = table, torch.from_numpy(start).to(DEV), width
    b.call()
    torch.cuda.synchronize()
    for (k, v), (dk, dv) in zip(b.pools, b.dev_pools):  # the first as if at position 2 of its block, the second not at all
        D.commit(k, v, b.hkv, b.d, np.array([2, -1], np.int32), b.cu, b.paths, b.path_lens, b.table)
        assert np.array_equal(dk.cpu().numpy().view(k.dtype), k) and np.array_equal(dv.cpu().numpy().view(v.dtype), v)
    assert b.t["out"].tolist() == [int(start[0]) + 3, int(start[1])]
