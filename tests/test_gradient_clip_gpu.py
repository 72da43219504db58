"""The global gradient norm and clipping against their definition in 64 bits."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def make(sizes, seed, sigma=1.0, offset=0):
    """Tensors of the sizes, bf16 and fp32 in turn, as views of one bucket a type that starts at `offset` elements."""
    g = torch.Generator().manual_seed(seed)
    total = {BF: offset, F32: offset}
    places = []
    for i, n in enumerate(sizes):
        t = F32 if i % 3 == 1 else BF
        places.append((t, total[t], n))
        total[t] += n
    buckets = {t: (torch.randn(n + 1, generator=g) * sigma).to(t).cuda() for t, n in total.items()}
    return buckets, [buckets[t][a:a + n] for t, a, n in places]


def exact_norm(tensors):
    return math.sqrt(sum(float((t.double() ** 2).sum()) for t in tensors))


def check(tensors, before, norm, max_norm, got_norm):
    assert abs(got_norm - norm) <= 2.0 ** -23 * norm          # 64-bit sums, rounded to fp32 once
    factor = max_norm / norm if norm > max_norm else 1.0
    for t, b in zip(tensors, before):
        want = b.double() * factor
        # the factor in fp32, the product, and the rounding to the type
        tol = want.abs() * (torch.finfo(t.dtype).eps / 2 + 2.0 ** -22) + 1e-38
        if factor == 1.0:
            assert torch.equal(t, b)
        else:
            assert bool(((t.double() - want).abs() <= tol).all())


SIZES = [[1], [7], [16384], [16385, 16383], [5, 0, 3, 100000, 8, 1, 0], [1 << 20, 17, 300001],
         [(i * 37) % 5000 for i in range(250)], [16384 * 3 + 5] * 121, [3 << 20]]


@pytest.mark.parametrize("sizes", SIZES, ids=lambda s: "%dx%d" % (len(s), max(s)))
@pytest.mark.parametrize("offset", [0, 1])
def test_norm_and_clipping(sizes, offset):
    from paper_2503_07680_amd.runner import GradientClip
    print("case", len(sizes), max(sizes), offset, flush=True)
    buckets, grads = make(sizes, len(sizes) + offset, offset=offset)
    before, whole = [g.clone() for g in grads], {t: b.clone() for t, b in buckets.items()}
    norm = exact_norm(grads)
    into, outs = make(sizes, 99, offset=offset)
    beside = {t: (b[:offset].clone(), b[-1:].clone()) for t, b in into.items()}
    clip = GradientClip(grads, outs)
    for limit in (norm * 0.37, norm * 2, float("inf"), 0.0):
        got = float(clip.clip(limit))
        check(outs, before, norm, limit, got)
        assert all(torch.equal(b, whole[t]) for t, b in buckets.items())      # the inputs stay
    for t, b in into.items():                                                   # and what lies beside the outputs
        assert torch.equal(b[:offset], beside[t][0]) and torch.equal(b[-1:], beside[t][1])
    clip.clip(norm * 0.8)
    one, n1, q1 = {t: b.clone() for t, b in into.items()}, clip.norm.clone(), clip.sumsq_buf.clone()
    q2 = clip.sumsq().clone()                                                   # the two calls give the same bits
    n2 = clip.clip_with(q2, norm * 0.8).clone()
    assert torch.equal(q1, q2) and torch.equal(n1, n2) and all(torch.equal(b, one[t]) for t, b in into.items())
    place = GradientClip(grads)
    check(grads, before, norm, norm * 2, float(place.clip(norm * 2)))
    check(grads, before, norm, norm * 0.6, float(place.clip(norm * 0.6)))
    assert torch.equal(place.sumsq(), place.sumsq().clone())


def test_sums_of_ranks_and_of_several_lists():
    from paper_2503_07680_amd.runner import GradientClip
    _, a = make([5000, 70000, 33], 1)
    _, b = make([800, 20001], 2)
    ca, cb = GradientClip(a), GradientClip(b)
    before = [t.clone() for t in a + b]
    q = ca.sumsq().clone()
    cb.sumsq_buf.copy_(q)
    total = cb.sumsq(accumulate=True).clone()
    norm = exact_norm(before)
    assert abs(float(total) - norm ** 2) <= 1e-12 * norm ** 2
    na, nb = float(ca.clip_with(total, norm / 3)), float(cb.clip_with(total, norm / 3))
    assert na == nb
    check(a + b, before, norm, norm / 3, na)


@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_a_norm_that_is_not_finite_scales_nothing(bad):
    from paper_2503_07680_amd.runner import GradientClip
    _, grads = make([400, 9000, 5], 3)
    grads[1][8999] = bad
    before = [g.clone() for g in grads]
    norm = float(GradientClip(grads).clip(0.5))
    assert not math.isfinite(norm)
    assert all(torch.equal(g.view(torch.int16 if g.dtype == BF else torch.int32), b.view(torch.int16 if b.dtype == BF else torch.int32))
               for g, b in zip(grads, before))
    outs = [torch.zeros_like(g) for g in grads]
    GradientClip(grads, outs).clip(0.5)
    assert all(torch.equal(o.nan_to_num(7.0), b.nan_to_num(7.0)) for o, b in zip(outs, before))


def test_large_and_small_values():
    from paper_2503_07680_amd.runner import GradientClip
    huge = torch.full((1000,), 3e38, dtype=F32, device="cuda")       # their squares leave fp32
    tiny = torch.full((1000,), 1e-30, dtype=F32, device="cuda")
    for x in (huge, tiny):
        norm, before = exact_norm([x]), x.clone()
        got = GradientClip([x]).clip(norm / 2 if norm < 3e38 else 1e30)
        want = before.double() * ((norm / 2 if norm < 3e38 else 1e30) / norm)
        if norm < 3.4e38:
            assert abs(float(got) - norm) <= 2.0 ** -23 * norm
        else:
            assert float(got) == float("inf")                         # the norm does not fit fp32; the clipping is right all the same
        assert bool(((x.double() - want).abs() <= want.abs() * 2.0 ** -22).all())


def test_empty_lists():
    from paper_2503_07680_amd.runner import GradientClip
    for grads in ([], [torch.empty(0, device="cuda")]):
        c = GradientClip(grads)
        c.norm.fill_(5.0)
        assert float(c.clip(1.0)) == 0.0 and float(c.sumsq_buf) == 0.0


def test_captured_and_on_another_stream():
    from paper_2503_07680_amd.runner import GradientClip
    sizes = [(i * 311) % 70000 for i in range(150)]
    buckets, grads = make(sizes, 8)
    into, outs = make(sizes, 9)
    clip = GradientClip(grads, outs)
    sets = [make(sizes, 20 + k, sigma=0.5 + k)[0] for k in range(3)]

    def eager(s):
        for t in buckets:
            buckets[t].copy_(s[t])
        n = clip.clip(40.0).clone()
        return n, {t: b.clone() for t, b in into.items()}

    want = [eager(s) for s in sets]
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        clip.clip(40.0)
        side.synchronize()
        with torch.cuda.graph(graph, stream=side):
            norm = clip.clip(40.0)
    torch.cuda.synchronize()
    for k in (0, 1, 2, 1, 0):
        for t in buckets:
            buckets[t].copy_(sets[k][t])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(norm, want[k][0]) and all(torch.equal(into[t], want[k][1][t]) for t in into), k
        eager(sets[(k + 1) % 3])
