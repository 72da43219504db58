"""What the embedding's and the gradients' entry points refuse, on the host, before anything is launched."""
import ctypes

import numpy as np
import pytest

import paper_2503_07680_amd as H

FAKE = 0x10000  # never dereferenced


def embed(**kw):
    base = dict(total_tokens=10, vocab=100, dim=64, table_type=H.HBP_BF16, row_type=H.HBP_BF16, scale=1.0)
    base.update(kw)
    return H.EmbedDesc(**base)


@pytest.mark.parametrize("kw,status", [
    (dict(total_tokens=-1), 1), (dict(vocab=0), 1), (dict(dim=0), 1), (dict(scale=float("nan")), 1),
    (dict(scale=float("inf")), 1), (dict(table_type=2), 1), (dict(row_type=-1), 1),
    (dict(dim=(1 << 24) + 1), 3), (dict(total_tokens=(1 << 24) + 1), 3), (dict(vocab=2 ** 31 - 1), 3),
    (dict(table_stride=63), 2), (dict(row_stride=-64), 2),
])
def test_embedding_descriptors(kw, status):
    lib, d = H.load_library(), embed(**kw)
    with pytest.raises(H.HbpError) as e:
        H.hbp_embed_bwd_workspace_bytes(d)
    assert e.value.status == status
    assert lib.hbp_embed_fwd(ctypes.byref(d), FAKE, FAKE, FAKE, None) == status
    assert lib.hbp_embed_bwd(ctypes.byref(d), FAKE, FAKE, 0, FAKE, FAKE, 1 << 40, None) == status


def test_embedding_calls():
    lib, d = H.load_library(), embed()
    p, need = ctypes.byref(d), H.hbp_embed_bwd_workspace_bytes(embed())
    f32 = ctypes.byref(embed(table_type=H.HBP_F32))
    assert lib.hbp_embed_fwd(None, FAKE, FAKE, FAKE, None) == 1
    for args in ((None, FAKE, FAKE), (FAKE, None, FAKE), (FAKE, FAKE, None), (FAKE + 1, FAKE, FAKE), (FAKE, FAKE + 2, FAKE), (FAKE, FAKE, FAKE + 1)):
        assert lib.hbp_embed_fwd(p, *args, None) == 1
    assert lib.hbp_embed_fwd(f32, FAKE + 2, FAKE, FAKE, None) == 1
    assert lib.hbp_embed_bwd(p, FAKE, FAKE, 2, FAKE, FAKE, need, None) == 1
    for ws, size in ((None, need), (FAKE + 128, need), (FAKE, need - 1)):
        assert lib.hbp_embed_bwd(p, FAKE, FAKE, 0, FAKE, ws, size, None) == 5
    for args in ((None, FAKE, 0, FAKE), (FAKE, None, 0, FAKE), (FAKE, FAKE, 0, None), (FAKE, FAKE, 1, FAKE + 1), (FAKE + 1, FAKE, 0, FAKE)):
        assert lib.hbp_embed_bwd(p, *args, FAKE, need, None) == 1
    empty = ctypes.byref(embed(total_tokens=0))
    assert lib.hbp_embed_fwd(empty, None, None, None, None) == 0
    assert lib.hbp_embed_bwd(empty, None, None, 1, None, None, 0, None) == 0     # nothing to add
    assert lib.hbp_embed_bwd(empty, None, None, 0, None, None, 0, None) == 1     # would have to be zeroed


def test_workspaces_grow_with_the_tokens():
    sizes = [H.hbp_embed_bwd_workspace_bytes(embed(total_tokens=T)) for T in (0, 1, 1000, 16384, 16385, 100000, 1 << 24)]
    assert all(b >= a for a, b in zip(sizes, sizes[1:])) and sizes[1] > 0


def grads(n=3, **kw):
    base = dict(addresses=[FAKE * (i + 1) for i in range(n)], sizes=[100] * n, types=[H.HBP_F32] * n)
    base.update(kw)
    return H.GradList(**base)


def sumsq(g, ws=FAKE, size=1 << 20, out=FAKE, accumulate=0):
    t, s, y, _ = g.args
    return H.load_library().hbp_grad_sumsq(t, s, y, g.n, accumulate, out, ws, size, None)


def clip(g, max_norm=1.0, q=FAKE):
    t, s, y, o = g.args
    return H.load_library().hbp_grad_clip(t, o, s, y, g.n, q, max_norm, None, None)


def both(g, max_norm=1.0, q=FAKE, ws=FAKE, size=1 << 20):
    t, s, y, o = g.args
    return H.load_library().hbp_grad_clip_norm(t, o, s, y, g.n, max_norm, q, None, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(sizes=[100, -1, 100]), 1), (dict(types=[0, 1, 2]), 1), (dict(addresses=[FAKE, 0, 3 * FAKE]), 1),
    (dict(addresses=[FAKE, 2 * FAKE + 2, 3 * FAKE]), 1), (dict(sizes=[100, (1 << 40) + 1, 100]), 3),
])
def test_gradient_lists(kw, status):
    assert sumsq(grads(**kw)) == status and clip(grads(**kw)) == status and both(grads(**kw)) == status


def test_gradient_calls():
    lib, g = H.load_library(), grads()
    assert sumsq(g, out=None) == 1 and sumsq(g, out=FAKE + 4) == 1 and sumsq(g, accumulate=2) == 1
    assert sumsq(g, ws=None) == 5 and sumsq(g, ws=FAKE + 8) == 5 and sumsq(g, size=8) == 5
    for bad in (-1.0, float("nan"), float("-inf")):
        assert clip(g, max_norm=bad) == 1 and both(g, max_norm=bad) == 1
    assert both(g, q=None) == 1 and both(g, q=FAKE + 4) == 1
    assert both(g, ws=None) == 5 and both(g, ws=FAKE + 8) == 5 and both(g, size=8) == 5
    assert clip(g, q=None) == 1 and clip(g, q=FAKE + 4) == 1
    assert lib.hbp_grad_sumsq(None, None, None, 2, 0, FAKE, FAKE, 1 << 20, None) == 1
    assert lib.hbp_grad_clip(None, None, None, None, -1, FAKE, 1.0, None, None) == 1
    with pytest.raises(H.HbpError):
        H.hbp_grad_workspace_bytes(-1)
    with pytest.raises(H.HbpError):
        H.GradList([FAKE], [1, 2], [0])


def test_overlapping_gradients_are_not_clipped():
    assert clip(grads(addresses=[FAKE, FAKE, 3 * FAKE])) == 1                            # the same tensor twice
    assert both(grads(addresses=[FAKE, FAKE, 3 * FAKE])) == 1
    assert clip(grads(addresses=[FAKE, FAKE + 396, 3 * FAKE])) == 1                      # its last element
    far = [FAKE * (i + 10) for i in range(3)]
    assert clip(grads(outs=[far[0], far[0] + 4, far[2]])) == 1                           # two outputs
    assert clip(grads(outs=[far[0], FAKE + 4, far[2]])) == 1                             # an output on another's input
    assert clip(grads(outs=[FAKE + 4, far[1], far[2]])) == 1                             # an output shifted over its own input
    assert clip(grads(outs=[2 * FAKE, FAKE, far[2]])) == 1                               # inputs and outputs swapped


def test_every_batch_of_a_long_list_has_its_place_in_the_workspace():
    for n in (0, 1, 119, 120, 121, 240, 1000):
        assert H.hbp_grad_workspace_bytes(n) >= -(-n // 120) * 2048 * 8


def test_lists_are_plain_arrays():
    g = grads()
    assert g.addresses.dtype == np.uint64 and g.sizes.dtype == np.int64 and g.types.dtype == np.int32
