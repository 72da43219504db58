"""Cross attention in the race-hunting build (a workgroup fence after every phase, tile and step) against the release build: the
same arithmetic in the same order, so every output has to agree bit for bit."""
import json
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CASES = [  # query lengths, key lengths, Hq, Hkv, d_qk, d_v
    ([300, 0, 64, 1200, 1], [90, 20, 0, 70, 700], 8, 2, 128, 128),
    ([700, 129, 33], [513, 1000, 64], 4, 4, 64, 64), ([700, 129, 33], [513, 1000, 64], 6, 2, 64, 64),
    ([500, 31], [700, 129], 4, 2, 192, 128), ([40], [3000], 4, 4, 192, 128),
    ([1] * 9, [900, 3, 4000, 0, 64, 1000, 129, 2500, 700], 8, 2, 128, 128), ([3000], [100], 8, 1, 128, 128),
    ([2500, 900], [60, 300], 16, 1, 64, 64), ([1500], [90], 8, 1, 192, 128), ([900] * 8, [700] * 8, 32, 8, 128, 128),
    ([64], [5000], 8, 2, 128, 128), ([257, 511, 1023], [255, 513, 1025], 12, 3, 128, 128),
]
RUNNER = r"""
import hashlib, json, sys
sys.path.insert(0, %(root)r)
import torch
from paper_2503_07680_amd.runner import PackedCrossAttention
import paper_2503_07680_amd as H
out = {}
for i, (ql, kl, hq, hkv, d, e) in enumerate(%(cases)r):
    g = torch.Generator(device="cuda").manual_seed(i)
    x = [torch.randn(s, generator=g, device="cuda").to(torch.bfloat16) for s in ((sum(ql), hq, d), (sum(kl), hkv, d), (sum(kl), hkv, e), (sum(ql), hq, e))]
    a = PackedCrossAttention(ql, kl, hq, hkv, d, e)
    a.forward(*x[:3])
    a.backward(*x)
    torch.cuda.synchronize()
    for name in ("o", "lse", "dq", "dk", "dv"):
        out["%%d %%s" %% (i, name)] = hashlib.sha256(getattr(a, name).contiguous().view(torch.uint8).cpu().numpy().tobytes()).hexdigest()
    print("case", i, "done with", H.library_path(), flush=True)
json.dump(out, open(sys.argv[1], "w"))
"""


def run_with(library, path):
    env = dict(os.environ)
    env.pop("HBP_LIBRARY", None)
    if library:
        env["HBP_LIBRARY"] = library
    r = subprocess.run([sys.executable, "-c", RUNNER % {"root": ROOT, "cases": CASES}, path], env=env, stdout=subprocess.PIPE,
                       stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-3000:]
    assert ("libhbp_racehunt.so" in r.stdout) == bool(library), r.stdout[-500:]
    with open(path) as f:
        return json.load(f)


def test_release_and_race_hunting_builds_agree_bit_for_bit(tmp_path):
    release, fenced = run_with(None, str(tmp_path / "release.json")), run_with("libhbp_racehunt.so", str(tmp_path / "fenced.json"))
    assert len(release) == 5 * len(CASES)
    assert release == fenced, [k for k in release if release[k] != fenced.get(k)]
