"""Cross attention where one sample has far more keys or query rows than the others: they go to more workgroups than the others'."""
import pytest
import torch

from cross_util import check, exact
from test_cross_attention_gpu import DIMS, inputs, run

pytestmark = pytest.mark.gpu

CASES = [  # queries, keys: the longest first, last and in the middle, samples without keys or queries, one key, whole tiles and a key more
    ([1] * 9, [6000, 200, 64, 65, 0, 1, 128, 129, 40]), ([1, 1, 0, 1, 1], [100, 192, 9000, 5000, 7]), ([1] * 40, [30] * 39 + [4099]),
    ([9, 3, 33], [64, 5000, 100]), ([100] * 6, [200, 300, 4500, 0, 64, 1]), ([2] * 3 + [70], [9, 0, 3333, 6]),
]


@pytest.mark.parametrize("ql,kl", CASES, ids=lambda v: "-".join(map(str, v[:5])))
@pytest.mark.parametrize("d,e", DIMS)
@pytest.mark.parametrize("hq,hkv", [(3, 3), (8, 2)])
def test_uneven_keys(ql, kl, d, e, hq, hkv):
    print("case", ql[:5], kl[:5], d, hq, hkv, flush=True)
    x = inputs(ql, kl, hq, hkv, d, e, sum(kl) + d)
    a, got = run(ql, kl, hq, hkv, d, e, x)
    want = exact(ql, kl, *x)
    check(got, want, got)
    first = {n: got[n].clone() for n in ("o", "lse")}
    a.ws_fwd.fill_(255)      # NaN wherever a part that a sample does not have would be read
    o, lse = a.forward(*x[:3])
    assert torch.equal(o, first["o"]) and torch.equal(lse, first["lse"])


BACKWARD = [
    ([8000] + [30] * 20, [100] + [40] * 20), ([20, 0, 300, 7000, 1], [500, 64, 0, 260, 1]), ([10] + [30] * 20, [20000] + [60] * 20),
    ([0, 64, 1, 500], [300, 12000, 63, 0]), ([6000, 40, 3], [130, 9000, 64]), ([4097] + [1] * 30, [1] * 31), ([1] * 31, [1] * 30 + [6401]),
]


@pytest.mark.parametrize("ql,kl", BACKWARD, ids=lambda v: "-".join(map(str, v[:5])))
@pytest.mark.parametrize("d,e", DIMS)
@pytest.mark.parametrize("hq,hkv", [(3, 3), (8, 2), (8, 1)])
def test_uneven_backward(ql, kl, d, e, hq, hkv):
    print("case", ql[:5], kl[:5], d, hq, hkv, flush=True)
    x = inputs(ql, kl, hq, hkv, d, e, sum(ql) + d)
    a, got = run(ql, kl, hq, hkv, d, e, x)
    check(got, exact(ql, kl, *x), got)
    first = {n: got[n].clone() for n in ("dq", "dk", "dv")}
    a.ws_bwd.fill_(255)
    again = dict(zip(("dq", "dk", "dv"), a.backward(*x)))
    assert all(torch.equal(first[n], again[n]) for n in first)


@pytest.mark.parametrize("longest", [0, 1, 700, 2 ** 31 - 1])
def test_a_longest_sample_that_is_not(longest):
    """What the descriptor says of the longest sample decides how the keys are dealt out, not what comes out."""
    import paper_2503_07680_amd as H
    ql, kl = [1] * 8, [4000, 20, 0, 300, 64, 1, 1200, 70]
    x = inputs(ql, kl, 8, 2, 128, 128, 3)
    a, got = run(ql, kl, 8, 2, 128, 128, x)
    a.desc.longest_keys = a.desc.longest_queries = longest
    a.ws_fwd = torch.full((H.hbp_cross_workspace_bytes(a.desc, H.HBP_FWD),), 255, dtype=torch.uint8, device="cuda")
    o, lse = a.forward(*x[:3])
    got.update(o=o, lse=lse)
    a.ws_bwd = torch.full((H.hbp_cross_workspace_bytes(a.desc, H.HBP_BWD),), 255, dtype=torch.uint8, device="cuda")
    got.update(zip(("dq", "dk", "dv"), a.backward(*x)))
    check(got, exact(ql, kl, *x), got)
