"""The embedding's gradient where a few ids have very many of the tokens: runs of the sorted tokens over many chunks."""
import pytest
import torch

from test_embedding_gpu import check_grad, exact_grad, module

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

RUNS = [  # tokens of each id, in order; up to 16384 tokens are cut into chunks of 16, more into chunks of 32
    [1024, 1024, 1040, 8, 1008, 1023, 1],                   # 64 chunks from a boundary to a boundary, one more, one fewer
    [5, 1019, 1, 1030, 2000, 3, 3000],                      # beginning and ending inside chunks
    [16 * 63 + 15, 2, 16 * 64 + 1, 16 * 65, 7000],
    [32 * 64, 32 * 64 + 1, 32 * 63, 32 * 128, 9, 32 * 65 - 9, 6000, 1, 1, 40],
    [31, 32 * 300 + 2, 0, 32 * 64 - 1, 12345],
    [40000], [1, 65535, 1], [60000, 0, 0, 60000, 11072],
]


@pytest.mark.parametrize("runs", RUNS, ids=lambda r: "-".join(map(str, r[:5])))
@pytest.mark.parametrize("dim,spread,table_type,out_type", [(24, 1, F32, BF), (137, 1, BF, F32), (5, 37, F32, F32), (520, 5000, BF, BF)])
def test_runs(runs, dim, spread, table_type, out_type):
    """`spread` ids lie between those with tokens: one workgroup's range has them all, or one of them."""
    T, vocab = sum(runs), (len(runs) - 1) * spread + 2
    print("case", runs[:4], dim, spread, table_type, out_type, flush=True)
    g = torch.Generator().manual_seed(T + dim)
    t = torch.repeat_interleave(torch.arange(len(runs)) * spread + 1, torch.tensor(runs))
    t = t[torch.randperm(T, generator=g)].to(torch.int32)
    t[::97] = -1                                            # some are none, at the end of the order
    scale = 0.75
    d = torch.randn(T, dim, generator=g).to(out_type)
    e = module()(T, vocab, dim, scale, table_type, out_type)
    want, size, count = exact_grad(d, t, vocab, scale)
    dw = torch.full((vocab, dim), float("nan"), dtype=table_type, device="cuda")
    first = e.backward(d.cuda(), t.cuda(), dw).clone()
    check_grad(first, want, size, count)
    assert bool((first.cpu()[count[:, 0] == 0] == 0).all())
    assert torch.equal(e.backward(d.cuda(), t.cuda(), dw), first)       # the same bits
    old = torch.randn(vocab, dim, generator=g).to(table_type)
    want, size, count = exact_grad(d, t, vocab, scale, old)
    got = e.backward(d.cuda(), t.cuda(), old.cuda(), accumulate=True)
    check_grad(got, want, size, count)


@pytest.mark.parametrize("runs", RUNS[:3] + RUNS[4:5], ids=lambda r: "-".join(map(str, r[:5])))
def test_whole_runs(runs):
    """Every token counts, in the order of the ids: runs that begin and end exactly where they are said to."""
    T, vocab, dim = sum(runs), len(runs), 16
    t = torch.repeat_interleave(torch.arange(vocab), torch.tensor(runs)).to(torch.int32)
    d = (torch.arange(T) % 7 + 1).to(F32)[:, None].expand(T, dim).contiguous()
    e = module()(T, vocab, dim, 1.0, F32, F32)
    got = e.backward(d.cuda(), t.cuda(), torch.empty(vocab, dim, device="cuda"))
    want = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, t.long(), d.double())
    assert torch.equal(got.cpu().double(), want)            # whole numbers below 2^24: exact


@pytest.mark.parametrize("dim,table_type", [(1, BF), (3, F32), (8, BF), (9, BF), (100, BF), (255, BF), (256, BF), (257, BF), (300, F32), (2049, BF)])
def test_rows_without_tokens_are_zeroed_and_nothing_else(dim, table_type):
    T, vocab = 300, 1100
    g = torch.Generator().manual_seed(dim)
    t = torch.randint(0, vocab // 3, (T,), generator=g).to(torch.int32)
    d = torch.randn(T, dim, generator=g).to(BF).cuda()
    for stride, offset in ((dim, 0), (dim, 1), (dim + 5, 3)):
        base = torch.full((offset + vocab * stride + 70,), 7.0, dtype=table_type, device="cuda")
        view = base[offset:offset + vocab * stride].view(vocab, stride)[:, :dim]
        e = module()(T, vocab, dim, 1.0, table_type, BF)
        e.backward(d, t.cuda(), view)
        none = torch.ones(vocab, dtype=torch.bool)
        none[t.long()] = False
        assert bool((view[none.cuda()] == 0).all())
        assert bool((view[t.long().cuda()] != 0).any())
        view.fill_(7.0)
        assert bool((base == 7.0).all())


@pytest.mark.parametrize("runs", [[12288, 1, 700], [20000, 30000, 4000, 9], [9000] * 7, [800, 13000, 1, 1, 600, 65, 30000], [65535, 1], [13000]],
                         ids=lambda r: "-".join(map(str, r[:5])))
@pytest.mark.parametrize("ordered", [False, True])
def test_frequent_ids_beside_each_other(runs, ordered):
    """All of them in one workgroup's range of ids, mixed, or each in a stretch of its own."""
    T, vocab, dim = sum(runs), 300000, 16
    g = torch.Generator().manual_seed(T)
    t = torch.repeat_interleave(torch.arange(len(runs)) * 3 + 200000, torch.tensor(runs)).to(torch.int32)
    t = t.flip(0) if ordered else t[torch.randperm(T, generator=g)]
    d = torch.randint(-8, 9, (T, dim), generator=g).to(F32)
    e = module()(T, vocab, dim, 1.0, F32, F32)
    got = e.backward(d.cuda(), t.cuda(), torch.empty(vocab, dim, device="cuda"))
    want = torch.zeros(vocab, dim, dtype=torch.float64).index_add_(0, t.long(), d.double())
    assert torch.equal(got.cpu().double(), want)            # whole numbers below 2^24: exact
