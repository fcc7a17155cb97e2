"""What the entry points for drafted tokens refuse on the host, with made-up device addresses (nothing may touch them); on a
machine without a GPU a valid call ends in CRONUS_ERR_HIP, so the other codes also show that nothing was launched.  And the plain
forms that the GPU tests compare with, on cases worked by hand."""
import numpy as np
import pytest

from paper_2509_17357_amd import binding as B

import draft_util as D

FAKE = 0x7F0000001000
BAD, UNSUPPORTED, WORKSPACE = B.CRONUS_ERR_INVALID_ARG, B.CRONUS_ERR_UNSUPPORTED, B.CRONUS_ERR_WORKSPACE


def cache(**kw):
    return B.make_cache(kw.pop("k", FAKE), kw.pop("v", FAKE), kw.pop("blocks", 100), kw.pop("hq", 8), kw.pop("hkv", 2), kw.pop("d", 64), **kw)


BAD_CACHES = [(dict(k=None), BAD), (dict(blocks=0), BAD), (dict(k_scale=FAKE, v_scale=FAKE), BAD),
              (dict(kv_dtype=B.CRONUS_KV_FP8_E4M3), BAD), (dict(d=96), UNSUPPORTED), (dict(hkv=3), UNSUPPORTED),
              (dict(block_size=32), UNSUPPORTED), (dict(kv_dtype=7), UNSUPPORTED)]


def no_gpu():
    import torch
    return not torch.cuda.is_available()


def tree(**kw):
    a = dict(cache=cache(), q=FAKE, out=FAKE, prefix=FAKE, cu=FAKE, mask=FAKE, words=1, bt=FAKE, width=4, n=3, rows=8, scale=0.125,
             ws=FAKE & ~255, ws_bytes=1 << 30)
    a.update(kw)
    return B.cronus_attn_tree(a["cache"], a["q"], a["out"], a["prefix"], a["cu"], a["mask"], a["words"], a["bt"], a["width"], a["n"], a["rows"],
                              a["scale"], a["ws"], a["ws_bytes"], check=False)


def test_attn_tree_refusals():
    for name in ("q", "out", "prefix", "cu", "bt"):
        assert tree(**{name: None}) == BAD, name
    for kw in (dict(n=-1), dict(rows=-1), dict(width=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
               dict(words=0), dict(rows=65), dict(rows=129, words=2), dict(mask=FAKE + 4), dict(rows=0x7FFFFFFF, mask=None)):
        assert tree(**kw) == BAD, kw
    for kw, code in BAD_CACHES:
        assert tree(cache=cache(**kw)) == code, kw
        if code == UNSUPPORTED:
            assert B.cronus_attn_tree_workspace_bytes(cache(**kw), 8) == 0, kw
    need = B.cronus_attn_tree_workspace_bytes(cache(), 8)
    assert need > 0 and need % 256 == 0 and B.cronus_attn_tree_workspace_bytes(cache(), -1) == 0
    sizes = [B.cronus_attn_tree_workspace_bytes(cache(), r) for r in range(0, 300)]
    assert sizes == sorted(sizes)
    for kw in (dict(ws=None), dict(ws=FAKE + 8), dict(ws_bytes=need - 1), dict(ws_bytes=0)):
        assert tree(**kw) == WORKSPACE, kw
    for kw in (dict(n=0x7FFFFFFF), dict(n=0x7FFFFFFF, rows=0x0FFFFFF, mask=None), dict(n=0x7FFFFFFF, rows=1, cache=cache(hq=0x7FFFFFFF, hkv=0x7FFFFFFF))):
        assert tree(ws_bytes=1 << 40, **kw) == BAD, kw  # more row tiles than shares are counted in
    assert tree(n=0, q=None, ws=None) == B.CRONUS_OK and tree(rows=0, q=None, ws=None) == B.CRONUS_OK
    if no_gpu():
        assert tree(ws_bytes=need) == B.CRONUS_ERR_HIP
        assert tree(mask=None, words=0) == B.CRONUS_ERR_HIP and tree(rows=128, words=2) == B.CRONUS_ERR_HIP


def build(**kw):
    a = dict(bt=FAKE, width=4, held=FAKE, held_out=FAKE, free=FAKE, capacity=100, count=FAKE, count_out=FAKE, kv=FAKE, new=FAKE, n=3, cu=FAKE,
             start=FAKE, cub=FAKE, slots=FAKE, most=40, report=FAKE)
    a.update(kw)
    return B.cronus_build_tables((a["bt"], a["width"], a["held"], a["held_out"], a["free"], a["capacity"], a["count"], a["count_out"]), a["kv"],
                                 a["new"], a["n"], a["cu"], a["start"], a["cub"], a["slots"], a["most"], a["report"], check=False)


def test_build_tables_refusals():
    for name in ("bt", "held", "held_out", "free", "count", "count_out", "kv", "new", "cu", "start", "cub", "report"):
        assert build(**{name: None}) == BAD, name
    for kw in (dict(n=-1), dict(n=(1 << 30) + 1), dict(width=0), dict(capacity=-1), dict(most=-1)):
        assert build(**kw) == BAD, kw
    assert B.lib().cronus_build_tables(None, FAKE, FAKE, 1, FAKE, FAKE, FAKE, None, 1, FAKE, None) == BAD
    if no_gpu():
        assert build() == B.CRONUS_ERR_HIP and build(slots=None) == B.CRONUS_ERR_HIP and build(free=None, capacity=0) == B.CRONUS_ERR_HIP
        assert build(n=0, bt=None, held=None, held_out=None, kv=None, new=None, start=None) == B.CRONUS_ERR_HIP  # still reports


def commit(**kw):
    a = dict(caches=[cache(), cache(k=FAKE + 64, v=FAKE + 64)], start=FAKE, cu=FAKE + 0x1000, paths=FAKE + 0x2000, most=4, lens=FAKE + 0x3000, bt=FAKE, width=4, n=3,
             out=FAKE + 0x4000)
    a.update(kw)
    return B.cronus_kv_commit(a["caches"], a["start"], a["cu"], a["paths"], a["most"], a["lens"], a["bt"], a["width"], a["n"], a["out"], check=False)


def test_kv_commit_refusals():
    for name in ("start", "cu", "paths", "lens", "bt"):
        assert commit(**{name: None}) == BAD, name
    for kw in (dict(n=-1), dict(most=-1), dict(width=0), dict(caches=[]), dict(out=FAKE), dict(out=FAKE + 8), dict(out=FAKE - 8),
               dict(out=FAKE + 0x100C), dict(out=FAKE + 0x1000 - 8), dict(out=FAKE + 0x2000 + 44), dict(out=FAKE + 0x3008)):
        assert commit(**kw) == BAD, kw
    assert B.lib().cronus_kv_commit(None, 1, FAKE, FAKE, FAKE, 1, FAKE, FAKE, 1, 1, None, None) == BAD
    for kw, code in BAD_CACHES:
        assert commit(caches=[cache(), cache(**kw)]) == code, kw
    for other in (dict(hkv=4), dict(d=128), dict(kv_dtype=B.CRONUS_KV_FP8_E4M3, k_scale=FAKE, v_scale=FAKE)):
        assert commit(caches=[cache(), cache(**other)]) == BAD, other
    assert commit(caches=[cache(hq=131072, hkv=65536)]) == BAD
    for twice in (cache(), cache(k=FAKE + 64), cache(v=FAKE + 64)):
        assert commit(caches=[cache(), cache(k=FAKE + 128, v=FAKE + 128), twice]) == BAD
    assert commit(n=0, start=None) == B.CRONUS_OK
    if no_gpu():
        assert commit() == B.CRONUS_ERR_HIP and commit(out=None) == B.CRONUS_ERR_HIP
        assert commit(most=0, paths=None) == B.CRONUS_ERR_HIP and commit(out=FAKE + 12) == commit(out=FAKE + 0x1010) == commit(out=FAKE + 0x2030) == B.CRONUS_ERR_HIP


def test_errors_are_raised_by_name():
    with pytest.raises(B.CronusError, match="cronus_attn_tree"):
        B.cronus_attn_tree(cache(), None, FAKE, FAKE, FAKE, None, 0, FAKE, 4, 1, 1, 0.125, FAKE & ~255, 1 << 30)
    with pytest.raises(B.CronusError, match="cronus_kv_commit"):
        B.cronus_kv_commit([cache()], FAKE, FAKE, FAKE, 1, FAKE, FAKE, 4, 1, FAKE)
    with pytest.raises(B.CronusError, match="cronus_build_tables"):
        B.cronus_build_tables((FAKE, 0, FAKE, FAKE, FAKE, 1, FAKE, FAKE), FAKE, FAKE, 1, FAKE, FAKE, FAKE, FAKE, 1, FAKE)


def test_plain_tables_by_hand():
    # 17 cached + 15 new fill two blocks, the second already held; 0 + 33 need three; the third sequence has ended
    table = np.array([[7, 8, -1], [-1, -1, -1], [4, 5, -1]])
    r = D.tables([17, 0, 20], [15, 33, -1], [2, 0, 2], table, [0, 1, 2], 3, 10, 48)
    assert r["status"] == 0 and r["asked"] == (48, 3) and r["pushed"] == [0, 1, 2, 4, 5] and r["count"] == 2
    assert r["table"].tolist() == [[7, 8, -1], [5, 4, 2], [4, 5, -1]] and r["held"].tolist() == [2, 3, 0]
    assert r["start"].tolist() == [17, 0, 0] and r["cu_tokens"].tolist() == [0, 15, 48, 48] and r["cu_blocks"].tolist() == [0, 0, 3, 3]
    assert r["slots"][:2].tolist() == [129, 130] and r["slots"][15:17].tolist() == [80, 81] and r["slots"][-1] == 32
    assert D.tables([17, 0, 20], [15, 33, 0], [2, 0, 2], table, [0, 1], 2, 10, 48)["status"] == 2
    assert D.tables([17, 0, 20], [15, 33, 0], [2, 0, 2], table, [0, 1, 2], 3, 10, 47)["status"] == 3
    assert D.tables([17, 33], [1, 0], [2, 2], table[:2], [0], 1, 10, 47)["bad"] == 1
    assert D.tables([17, 20], [1, -1], [2, 2], table[[0, 2]], [0] * 9, 9, 10, 47)["bad"] == -1


def test_plain_attention_by_hand():
    # two keys with scores 0 and ln 2: weights 1/3 and 2/3; a row that sees one key takes its value; one that sees none gives 0
    q, k = np.ones((3, 1, 1)), np.array([0.0, np.log(2.0)]).reshape(2, 1, 1)
    v = np.array([3.0, 6.0]).reshape(2, 1, 1)
    seen = np.array([[True, True], [False, True], [False, False]])
    out, bound = D.attention(q, k, v, seen, 1.0)
    assert np.allclose(out.ravel(), [5.0, 6.0, 0.0]) and (bound >= 0).all() and bound[0, 0, 0] < 0.1
    v[0] = np.inf
    assert D.attention(q, k, v, seen, 1.0)[0].ravel().tolist() == [np.inf, 6.0, 0.0]
    rows, packed = D.random_tree_mask(np.random.default_rng(1), 70, 2)
    assert all(bool(int(packed[i].view(np.uint64)[j // 64]) >> (j % 64) & 1) == rows[i, j] for i in (0, 63, 64, 69) for j in range(70))
    assert D.path_in_effect([0, 2, 2, 5], 4, 9) == 2 and D.path_in_effect([0, 9], 2, 9) == 1 and D.path_in_effect([3, 4], 7, 9) == 2
