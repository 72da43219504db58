"""Cross attention's plan against a plain one, its rules, and what its entry points refuse; no GPU."""
import ctypes

import numpy as np
import pytest

import paper_2503_07680_amd as H

FAKE = 0x10000  # never dereferenced


def desc(**kw):
    base = dict(total_queries=300, total_keys=500, n_samples=2, n_q_heads=8, n_kv_heads=2, d_qk=128, d_v=128)
    base.update(kw)
    return H.CrossDesc(**base)


def plain_plan(ql, kl, rows, kind):
    tiles, at = [], 0
    for i, (a, b) in enumerate(zip(ql, kl)):
        n, cost = (a, b) if kind == H.HBP_TILES_QUERY else (b, a)
        tiles += [(-cost, i, t, at + t * rows, at + min(n, (t + 1) * rows)) for t in range(-(-n // rows))]
        at += n
    return [t[1:] for t in sorted(tiles)]


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("rows", [1, 64, 128, 256])
def test_plan(seed, rows):
    r = np.random.default_rng(seed)
    n = int(r.integers(0, 40))
    ql, kl = (r.integers(0, 600, n) * (r.random(n) > 0.2) for _ in range(2))
    for kind in (H.HBP_TILES_QUERY, H.HBP_TILES_KEY):
        cu_q, cu_kv, tiles, pairs = H.hbp_cross_plan(ql, kl, rows, kind)
        assert cu_q.tolist() == [0] + np.cumsum(ql).tolist() and cu_kv.tolist() == [0] + np.cumsum(kl).tolist()
        assert [tuple(t) for t in tiles.tolist()] == plain_plan(ql.tolist(), kl.tolist(), rows, kind)
        assert pairs == int(np.dot(ql.astype(np.int64), kl.astype(np.int64)))


def test_plan_refusals():
    for ql, kl, rows, kind in (([-1], [4], 64, 0), ([4], [-1], 64, 0), ([1, 2], [1], 64, 0), ([4], [4], 0, 0), ([4], [4], 64, 2),
                               ([2 ** 31 - 1, 1], [1, 1], 1 << 30, 0), ([1, 1], [2 ** 31 - 1, 1], 64, 0)):
        with pytest.raises(H.HbpError) as e:
            H.hbp_cross_plan(ql, kl, rows, kind)
        assert e.value.status == 1
    lib, n, pairs = H.load_library(), ctypes.c_int32(), ctypes.c_int64()
    q = np.array([300, 5], dtype=np.int32)
    k = np.array([30, 5], dtype=np.int32)
    cu, tiles = np.zeros(3, dtype=np.int32), np.zeros((8, 4), dtype=np.int32)
    at = [x.ctypes.data for x in (q, k, cu, tiles)]
    out = (ctypes.byref(n), ctypes.byref(pairs))
    assert lib.hbp_cross_plan(at[0], at[1], 2, 128, 0, at[2], None, 3, None, 0, *out) == 1      # both bounds or neither
    assert lib.hbp_cross_plan(at[0], at[1], 2, 128, 0, at[2], at[2], 2, None, 0, *out) == 4
    assert lib.hbp_cross_plan(at[0], at[1], 2, 128, 0, None, None, 0, at[3], 3, *out) == 4 and n.value == 4
    assert lib.hbp_cross_plan(at[0], at[1], 2, 128, 0, None, None, 0, at[3], 4, *out) == 0 and n.value == 4
    assert lib.hbp_cross_plan(None, at[1], 2, 128, 0, None, None, 0, None, 0, *out) == 1
    assert lib.hbp_cross_plan(at[0], at[1], 2, 128, 0, None, None, 0, None, 0, None, out[1]) == 1
    assert lib.hbp_cross_plan(None, None, 0, 128, 0, None, None, 0, None, 0, *out) == 0 and n.value == 0


@pytest.mark.parametrize("hq,hkv,fold", [(1, 1, 1), (3, 1, 1), (6, 2, 1), (2, 1, 2), (12, 3, 4), (32, 8, 4), (64, 8, 8), (24, 1, 8),
                                         (32, 1, 32), (64, 1, 32), (128, 1, 32), (7, 7, 1)])
def test_rows_of_a_query_tile(hq, hkv, fold):
    for d, e in ((64, 64), (128, 128), (192, 128)):
        x = desc(n_q_heads=hq, n_kv_heads=hkv, d_qk=d, d_v=e)
        assert H.hbp_cross_tile_rows(x, H.HBP_FWD) == 256 // fold
        assert H.hbp_cross_tile_rows(x, H.HBP_BWD) == 128
        for n in ("q", "o"):     # a head outside its token's stride: not folded
            far = desc(n_q_heads=hq, n_kv_heads=hkv, d_qk=d, d_v=e, **{n + "_stride_t": d, n + "_stride_h": 300 * d})
            assert H.hbp_cross_tile_rows(far, H.HBP_FWD) == 256


@pytest.mark.parametrize("kw,status", [
    (dict(n_q_heads=7), 2), (dict(d_qk=96), 3), (dict(d_v=64), 3), (dict(total_queries=-1), 1), (dict(total_keys=-1), 1),
    (dict(n_samples=-1), 1), (dict(n_kv_heads=0), 1), (dict(softmax_scale=float("nan")), 1), (dict(q_stride_h=64), 2),
    (dict(k_stride_t=100), 2), (dict(v_stride_t=-256), 2), (dict(o_stride_t=(1 << 22) + 8), 2),
    (dict(total_queries=1 << 30, n_q_heads=64), 3), (dict(total_keys=2 ** 31 - 1), 3),
])
def test_descriptors(kw, status):
    lib, d = H.load_library(), desc(**kw)
    for f in (lambda: H.hbp_cross_tile_rows(d, 0), lambda: H.hbp_cross_workspace_bytes(d, 1)):
        with pytest.raises(H.HbpError) as e:
            f()
        assert e.value.status == status
    assert lib.hbp_cross_attn_fwd(ctypes.byref(d), *[FAKE] * 6, 1, FAKE, FAKE, FAKE, 1 << 40, None) == status
    assert lib.hbp_cross_attn_bwd(ctypes.byref(d), *[FAKE] * 9, 1, FAKE, 1, *[FAKE] * 4, 1 << 40, None) == status


def test_calls():
    lib, d = H.load_library(), desc()
    p = ctypes.byref(d)
    assert lib.hbp_cross_attn_fwd(None, *[FAKE] * 6, 1, FAKE, FAKE, FAKE, 1 << 30, None) == 1
    assert lib.hbp_cross_attn_fwd(p, *[FAKE] * 6, -1, FAKE, FAKE, FAKE, 1 << 30, None) == 1
    assert lib.hbp_cross_attn_fwd(p, *[None] * 6, 0, None, None, None, 0, None) == 0
    fwd = [FAKE] * 9
    for i in range(9):
        for bad in (None, FAKE + 8 if i in (0, 1, 2, 6) else None):
            a = list(fwd)
            a[i] = bad
            if i == 8:   # the workspace: none is needed
                continue
            q, k, v, cu_q, cu_kv, tiles, o, lse, ws = a
            assert lib.hbp_cross_attn_fwd(p, q, k, v, cu_q, cu_kv, tiles, 1, o, lse, ws, 1 << 30, None) == 1, i
    need = H.hbp_cross_workspace_bytes(d, H.HBP_BWD)
    assert need >= 2 * 300 * 8 * 4
    bwd = lambda q_tiles=1, kv_tiles=1, ws=FAKE, size=need, **kw: lib.hbp_cross_attn_bwd(  # noqa: E731
        p, *[kw.get(n, FAKE) for n in ("q", "k", "v", "o", "lse", "d_o", "cu_q", "cu_kv", "qt")], q_tiles, kw.get("kt", FAKE), kv_tiles,
        *[kw.get(n, FAKE) for n in ("dq", "dk", "dv")], ws, size, None)
    assert bwd(q_tiles=-1) == 1 and bwd(kv_tiles=-1) == 1
    assert bwd(ws=None) == 5 and bwd(ws=FAKE + 16) == 5 and bwd(size=need - 1) == 5
    for n in ("q", "k", "v", "o", "lse", "d_o", "cu_q", "cu_kv", "qt", "kt", "dq", "dk", "dv"):
        assert bwd(**{n: None}) == 1, n
    for n in ("q", "k", "v", "o", "d_o", "dq", "dk", "dv"):
        assert bwd(**{n: FAKE + 8}) == 1, n
    assert bwd(q_tiles=0, kv_tiles=0, cu_q=None) == 0


def test_the_forwards_workspace():
    lib, few, many = H.load_library(), desc(total_queries=2, total_keys=6000), desc(total_queries=60000, total_keys=6000)
    assert H.hbp_cross_workspace_bytes(many, H.HBP_FWD) == 0          # tiles enough: the keys in one part
    need = H.hbp_cross_workspace_bytes(few, H.HBP_FWD)
    assert need > 2 * 8 * 128 * 4
    for ws, size in ((None, need), (FAKE + 16, need), (FAKE, need - 1)):
        assert lib.hbp_cross_attn_fwd(ctypes.byref(few), *[FAKE] * 6, 1, FAKE, FAKE, ws, size, None) == 5


def test_nothing_to_attend_or_to_ask():
    for kw in (dict(total_queries=0), dict(total_keys=0), dict(total_queries=0, total_keys=0, n_samples=0)):
        d = desc(**kw)
        assert H.hbp_cross_workspace_bytes(d, H.HBP_BWD) >= 0


def test_the_longest_sample_goes_into_the_workspace():
    """One sample of 50000 keys among short ones has parts of its own; a mild spread, an unknown one and a refused one do not."""
    kw = dict(total_queries=32, total_keys=56200, n_samples=32, n_q_heads=24, n_kv_heads=24, d_qk=128, d_v=128)
    need = {k: H.hbp_cross_workspace_bytes(H.CrossDesc(longest_keys=k, **kw), H.HBP_FWD) for k in (0, 1756, 3000, 50000)}
    assert need[0] == need[1756] == need[3000] == 0 and need[50000] > 0
    all_keys, more = (H.hbp_cross_workspace_bytes(H.CrossDesc(longest_keys=k, **kw), H.HBP_FWD) for k in (56200, 2 ** 31 - 1))
    assert all_keys == more >= need[50000]
    for field in ("longest_keys", "longest_queries", "pairs"):
        with pytest.raises(H.HbpError):
            H.hbp_cross_workspace_bytes(H.CrossDesc(**{field: -1}, **kw), H.HBP_FWD)


def test_long_samples_go_into_the_backwards_workspace():
    """Long query runs on few keys, and long keys under few queries, have parts of their own; samples long on both sides do not."""
    kw = dict(total_queries=11000, total_keys=11000, n_samples=31, n_q_heads=32, n_kv_heads=8, d_qk=128, d_v=128)

    def need(**more):
        return H.hbp_cross_workspace_bytes(H.CrossDesc(**kw, **more), H.HBP_BWD)

    assert need(longest_queries=8000, longest_keys=200, pairs=8000 * 100 + 30 * 100 * 360) > need() < need(longest_keys=10000, pairs=2000000)
    assert need(longest_queries=8000, longest_keys=8000, pairs=8000 * 8000 + 30 * 100 * 100) == need() == need(longest_queries=500, longest_keys=500)
