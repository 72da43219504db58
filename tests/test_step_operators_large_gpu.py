"""Cross attention, the embedding and gradient clipping beyond 32-bit offsets, and at work on two streams at once."""
import pytest
import torch

from cross_util import check, exact, inputs

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32
STRIDE = 65536   # elements of a token, 128 KiB: offsets pass 2^31 elements at row 32768, 2^32 bytes too


def spread_out(t):
    """The same values with rows STRIDE elements apart."""
    view = torch.empty((t.shape[0], STRIDE), dtype=t.dtype, device="cuda")[:, :t[0].numel()].unflatten(1, t.shape[1:])
    return view.copy_(t)


def test_cross_attention_of_rows_far_apart():
    import paper_2503_07680_amd as H
    from paper_2503_07680_amd.runner import PackedCrossAttention
    ql, kl, hq, hkv, d = [3, 38000, 300], [39000, 5, 500], 2, 1, 64
    x = inputs(ql, kl, hq, hkv, d, d, 23)
    a = PackedCrossAttention(ql, kl, hq, hkv, d, d)
    o, lse = a.forward(*x[:3])
    dense = {n: t.clone() for n, t in zip(("o", "lse", "dq", "dk", "dv"), (o, lse) + tuple(a.backward(*x)))}
    check(dense, exact(ql, kl, *x), dense)
    q, k, v, d_o = (spread_out(t) for t in x)
    out = {n: spread_out(torch.full_like(t, float("nan"))) for n, t in (("o", x[3]), ("dq", x[0]), ("dk", x[1]), ("dv", x[2]))}
    s = {n + "_stride_t": STRIDE for n in "qkvo"}
    s.update({n + "_stride_h": d for n in "qkvo"})
    desc = H.CrossDesc(total_queries=sum(ql), total_keys=sum(kl), n_samples=3, n_q_heads=hq, n_kv_heads=hkv, d_qk=d, d_v=d, **s)
    assert H.hbp_cross_tile_rows(desc, H.HBP_FWD) == H.hbp_cross_tile_rows(a.desc, H.HBP_FWD)   # folded alike: the same plan
    lse = torch.full((hq, sum(ql)), 3.0, device="cuda")
    ws = [torch.empty(H.hbp_cross_workspace_bytes(desc, w), dtype=torch.uint8, device="cuda") for w in (H.HBP_FWD, H.HBP_BWD)]
    stream = torch.cuda.current_stream().cuda_stream
    H.hbp_cross_attn_fwd(desc, q, k, v, a.cu_q_dev, a.cu_kv_dev, a.q_tiles_dev, a.n_q_tiles, out["o"], lse, ws[0], stream)
    H.hbp_cross_attn_bwd(desc, q, k, v, out["o"], lse, d_o, a.cu_q_dev, a.cu_kv_dev, a.q_tiles_dev, a.n_q_tiles, a.kv_tiles_dev,
                         a.n_kv_tiles, out["dq"], out["dk"], out["dv"], ws[1], stream)
    out["lse"] = lse
    for n, t in dense.items():
        assert torch.equal(out[n], t), n


@pytest.mark.parametrize("table_type", [BF, F32])
def test_embedding_of_rows_far_apart(table_type):
    from paper_2503_07680_amd.runner import PackedEmbedding
    T, vocab, dim = 33000, 36000, 72
    e = PackedEmbedding(T, vocab, dim, 1.5, table_type, BF)
    g = torch.Generator(device="cuda").manual_seed(9)
    t = torch.randint(0, vocab, (T,), generator=g, device="cuda").to(torch.int32)
    t[-1] = vocab - 1
    w, d = (torch.randn(n, dim, generator=g, device="cuda").to(x) for n, x in ((vocab, table_type), (T, BF)))
    rows = spread_out(torch.full_like(d, float("nan")))
    assert torch.equal(e.forward(spread_out(w), t, rows), e.forward(w, t))
    for accumulate in (False, True):
        assert torch.equal(e.backward(spread_out(d), t, spread_out(w), accumulate), e.backward(d, t, w.clone(), accumulate))


def test_clipping_of_a_tensor_of_more_than_31_bits():
    from paper_2503_07680_amd.runner import GradientClip
    n = 2 ** 31 + 4097 * 8 + 5
    x = torch.full((n,), 2.0 ** -10, dtype=BF, device="cuda")
    x[-1], x[2 ** 31 - 1] = 16.0, -8.0
    q = (n - 2) * 2.0 ** -20 + 256.0 + 64.0     # exact: every partial sum is a multiple of 2^-20 below 2^53 of them
    clip = GradientClip([x])
    norm = clip.clip(q ** 0.5 / 4)
    assert abs(float(norm) - q ** 0.5) <= 2.0 ** -23 * q ** 0.5
    # a quarter up to two roundings of 2^-24 and the root's; the products are far from half a step of bf16
    assert float(x[-1]) == 4.0 and float(x[2 ** 31 - 1]) == -2.0
    x[-1] = x[2 ** 31 - 1] = 2.0 ** -12
    assert bool((x == 2.0 ** -12).all())


def test_two_streams_at_once():
    from paper_2503_07680_amd.runner import GradientClip, PackedCrossAttention, PackedEmbedding
    ql, kl, hq, hkv, d = [700, 40, 1200], [900, 3000, 64], 8, 2, 128
    T, vocab, dim = 20000, 5000, 264

    def program(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        x = inputs(ql, kl, hq, hkv, d, d, seed)
        a, e = PackedCrossAttention(ql, kl, hq, hkv, d, d), PackedEmbedding(T, vocab, dim, 2.0, F32, BF)
        a.alloc_backward()
        t = torch.randint(0, vocab, (T,), generator=g, device="cuda").to(torch.int32)
        d_y = torch.randn(T, dim, generator=g, device="cuda").to(BF)
        dw = torch.empty(vocab, dim, device="cuda")
        outs = [torch.empty_like(dw), torch.empty_like(a.dk)]
        e.backward(d_y, t, dw)   # the workspace
        clip = GradientClip([dw, a.dk], outs)

        def step():
            a.forward(*x[:3])
            a.backward(*x)
            e.backward(d_y, t, dw)
            clip.clip(1.0)
        return step, [a.o, a.lse, a.dq, a.dk, a.dv, dw] + outs

    programs = [program(s) for s in (1, 2)]
    want = []
    for step, held in programs:
        step()
        want.append([t.clone() for t in held])
        for t in held:
            t.zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in programs]
    for _ in range(4):
        for stream, (step, _) in zip(streams, programs):
            with torch.cuda.stream(stream):
                step()
    torch.cuda.synchronize()
    for (_, held), ref in zip(programs, want):
        assert all(torch.equal(t, r) for t, r in zip(held, ref))
