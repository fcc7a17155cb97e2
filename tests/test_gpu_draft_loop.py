"""A loop that drafts, verifies and keeps tokens, as it would be used (runtime.DraftLoop): every iteration's tables, attention and
cache against a host model that holds each sequence's K/V rows in order; eagerly, and as replays of one captured iteration."""
import numpy as np
import pytest
import torch

from oracle import cronus_oracle as orc
from paper_2509_17357_amd import binding as B
from paper_2509_17357_amd import workloads as W
from paper_2509_17357_amd.runtime import DraftLoop, bf16_tensor_from_bits, bits_from_bf16_tensor

import draft_util as D

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


class Model:
    """What the loop should hold."""

    def __init__(self, shape, layers, n, seed, scales):
        self.shape, self.layers, self.n, self.rng, self.scales = shape, layers, n, np.random.default_rng(seed), scales
        empty = np.zeros((0, shape.n_kv_heads, shape.head_dim), np.uint8 if shape.kv_dtype == "fp8" else np.uint16)
        self.rows = [[[empty, empty] for _ in range(n)] for _ in range(layers)]

    def codes(self, bits, scale):
        if scale is None:
            return bits
        x = orc.bf16_bits_to_f64(bits).astype(np.float32)
        return np.stack([orc.fp8_e4m3_encode(x[:, g], scale[g]) for g in range(x.shape[1])], axis=1)


def run(loop, model, iterations, chain, captured):
    rng, sh, n, most = model.rng, model.shape, model.n, loop.max_rows
    rows = n * most
    words = (most + 63) // 64
    buf = {"new": torch.zeros(n, dtype=torch.int32, device=DEV), "paths": torch.zeros((n, loop.max_path), dtype=torch.int32, device=DEV),
           "lens": torch.zeros(n, dtype=torch.int32, device=DEV), "mask": torch.zeros((rows, words), dtype=torch.int64, device=DEV)}
    row = lambda h: [torch.zeros((rows, h, sh.head_dim), dtype=torch.bfloat16, device=DEV) for _ in range(model.layers)]  # noqa: E731
    buf |= {"q": row(sh.n_q_heads), "out": row(sh.n_q_heads), "k": row(sh.n_kv_heads), "v": row(sh.n_kv_heads)}

    def iteration():
        loop.begin(buf["new"])
        for layer in range(model.layers):
            loop.append(layer, buf["k"][layer], buf["v"][layer])
            loop.attend(layer, buf["q"][layer], buf["out"][layer], None if chain else buf["mask"])
        loop.commit(buf["paths"], buf["lens"])

    iteration()  # no new tokens: leaves everything as it is, and everything is loaded before the capture
    graph = None
    if captured:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            iteration()
    for it in range(iterations):
        new = rng.integers(0, most, n, endpoint=True)
        if it % 3 == 2:
            new[int(rng.integers(0, n))] = -1  # a sequence ends, and begins anew in the next iteration
        add = np.maximum(new, 0)
        cu = np.concatenate([[0], np.cumsum(add)])
        total = int(cu[-1])
        paths, lens, masks = np.zeros((n, loop.max_path), np.int32), np.zeros(n, np.int32), np.zeros((rows, words), np.int64)
        seen = []
        for s in range(n):
            visible, packed = D.random_tree_mask(rng, int(add[s]), words)
            seen.append(np.tril(np.ones_like(visible)) if chain else visible)
            masks[cu[s]:cu[s + 1]] = packed
            p = sorted(rng.choice(int(add[s]), int(rng.integers(0, min(int(add[s]), loop.max_path), endpoint=True)), replace=False).tolist())
            paths[s, :len(p)], lens[s] = p, len(p)
        q, k, v = ([W.normal_bf16(rng, (rows, h, sh.head_dim), scale) for _ in range(model.layers)]
                   for h, scale in ((sh.n_q_heads, 2.0), (sh.n_kv_heads, 1.0), (sh.n_kv_heads, 1.0)))
        for name, bits in (("q", q), ("k", k), ("v", v)):
            for layer in range(model.layers):
                buf[name][layer].copy_(bf16_tensor_from_bits(bits[layer], DEV))
        for name, a in (("new", new), ("paths", paths), ("lens", lens), ("mask", masks)):
            buf[name].copy_(torch.from_numpy(np.ascontiguousarray(a)))
        for out in buf["out"]:
            out.fill_(7.25)
        graph.replay() if captured else iteration()
        torch.cuda.synchronize()

        assert loop.report.tolist()[:2] == [0, total], it
        assert loop.cu_rows.tolist() == cu.tolist()
        table, held = loop.block_tables.cpu().numpy(), loop.held.cpu().numpy()
        used = [table[s, :held[s]] for s in range(n)] + [loop.free_blocks.cpu().numpy()[:int(loop.free_count)]]
        assert sorted(np.concatenate(used).tolist()) == list(range(loop.num_blocks)), it  # every block has one owner
        for layer in range(model.layers):
            got = orc.bf16_bits_to_f64(bits_from_bf16_tensor(buf["out"][layer]))
            assert (got[total:] == 7.25).all()
            pools = [p[layer].cpu().numpy() for p in (loop.k_pools, loop.v_pools)]
            pools = [p if sh.kv_dtype == "fp8" else p.view(np.uint16) for p in pools]
            for s in range(n):
                if new[s] == -1:
                    model.rows[layer][s] = [x[:0] for x in model.rows[layer][s]]
                old, at = model.rows[layer][s], slice(cu[s], cu[s + 1])
                fresh = [model.codes(x[layer][at], scale) for x, scale in zip((k, v), model.scales)]
                all_rows = [np.concatenate([a, b]) for a, b in zip(old, fresh)]
                if add[s]:
                    ref, bound = D.attention(orc.bf16_bits_to_f64(q[layer][at]), *(D.values(x, scale) for x, scale in zip(all_rows, model.scales)),
                                             D.seen_of(len(old[0]), int(add[s]), seen[s]), loop.sm_scale)
                    assert (np.abs(got[at] - ref) <= bound).all(), (it, layer, s)
                model.rows[layer][s] = [np.concatenate([a, b[paths[s, :lens[s]]]]) for a, b in zip(old, fresh)]
                kept = model.rows[layer][s]
                cached = D.read_rows(*pools, sh.n_kv_heads, sh.head_dim, table[s], np.arange(len(kept[0])))
                assert np.array_equal(cached[0], kept[0]) and np.array_equal(cached[1], kept[1]), (it, layer, s)
        assert loop.kv_lens.tolist() == [len(model.rows[0][s][0]) for s in range(n)]


@pytest.mark.parametrize("captured", [False, True])
@pytest.mark.parametrize("shape,layers,n,most,chain", [
    (W.HeadShape(8, 2, 64), 2, 5, 9, False), (W.HeadShape(32, 8, 128), 1, 4, 33, False), (W.HeadShape(28, 4, 128), 2, 3, 5, True),
    (W.HeadShape(16, 2, 128, "fp8"), 2, 4, 20, False), (W.HeadShape(4, 4, 64, "fp8"), 1, 70, 3, False)])
def test_loop(shape, layers, n, most, chain, captured):
    scales = (None, None)
    if shape.kv_dtype == "fp8":
        scales = tuple(np.linspace(0.008, 0.012, shape.n_kv_heads).astype(np.float32) for _ in range(2))
    loop = DraftLoop(shape, layers, n, num_blocks=n * 14, max_blocks=13, max_rows=most, max_path=min(most, 6), scales=scales,
                     pool_fill=0x7F if shape.kv_dtype == "fp8" else 0x7FC1)
    run(loop, Model(shape, layers, n, most, scales), 10, chain, captured)


def test_an_iteration_without_blocks_leaves_everything_as_it_was():
    shape = W.HeadShape(8, 2, 64)
    loop = DraftLoop(shape, 1, 2, num_blocks=3, max_blocks=4, max_rows=30, max_path=30, pool_fill=0x1234)
    i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)  # noqa: E731
    k = torch.randn((60, 2, 64), device=DEV).to(torch.bfloat16)
    q, out = torch.randn((60, 8, 64), device=DEV).to(torch.bfloat16), torch.full((60, 8, 64), 7.25, device=DEV, dtype=torch.bfloat16)
    paths = i32([list(range(30))] * 2)
    for new, status, lens in (([20, 10], 0, [20, 10]), ([13, 7], 2, [20, 10]), ([3, 6], 0, [23, 16]), ([1, 1], 2, [23, 16]),
                              ([-1, 18], 0, [0, 34]), ([1, 2], 2, [0, 34])):  # 34 tokens: the held block and the two that return
        before = [t.clone() for t in (loop.k_pools[0], loop.v_pools[0], loop.block_tables, loop.held, loop.free_blocks, loop.free_count, loop.kv_lens)]
        out.fill_(7.25)
        loop.begin(i32(new))
        loop.append(0, k, k)
        loop.attend(0, q, out)
        loop.commit(paths, i32([30, 30]))
        torch.cuda.synchronize()
        assert loop.report[0] == status and loop.kv_lens.tolist() == lens, new
        after = (loop.k_pools[0], loop.v_pools[0], loop.block_tables, loop.held, loop.free_blocks, loop.free_count, loop.kv_lens)
        same = [torch.equal(a, b) for a, b in zip(before, after)]
        assert all(same) if status else not any(same[:1]), (new, same)
        assert bool((out == 7.25).all()) == (status != 0)
