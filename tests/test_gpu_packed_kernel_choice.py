"""Both kernels behind sparsed_attn_packed: the tests of the call again with each of them forced, and calls that the rule itself
(tests/test_packed_choice.py) gives the CTA-pair kernel."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import paper_2509_24014_b200 as sd
from oracle import packed_and_paged as orc
from tests import serving_util as su

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kernel", ["pair", "single"])
def test_packed_suite_with_one_kernel_forced(kernel):
    env = dict(os.environ, SPARSED_PACKED_KERNEL=kernel)
    cmd = [sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_gpu_attn_packed.py"]
    res = subprocess.run(cmd, cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    tail = (res.stdout + res.stderr)[-3000:]
    assert res.returncode == 0, tail
    assert " passed" in res.stdout and "failed" not in res.stdout, tail


@pytest.mark.parametrize("lens,past,heads_q,heads_kv,causal,dtype", [
    ([9000, 8300], 0, 8, 8, False, "bf16"), ([13001], 0, 8, 8, True, "fp16"), ([6000, 9001, 37], 0, 14, 2, True, "bf16"),
    ([2111, 1900, 2047, 3001], 9000, 16, 4, True, "bf16"), ([5000, 4600, 5003], 0, 12, 1, False, "fp16")])
def test_long_sequences(lens, past, heads_q, heads_kv, causal, dtype):
    gen, dtype = su.generator(len(lens)), su.DTYPES[dtype]
    total = [n + past for n in lens]
    q = su.rows(sum(lens) + 5, heads_q, dtype, gen)
    k, v = (su.rows(sum(total) + 5, heads_kv, dtype, gen) for _ in "kv")
    for t in (k, v):
        t[sum(total):] = float("nan")
    cu_q, cu_k = su.offsets(lens), su.offsets(total)
    o, lse = torch.full_like(q, 7.0), torch.full((heads_q, q.shape[0]), 7.0, device="cuda")
    ws = sd.new_workspace(256, "cuda")
    sd.sparsed_attn_packed(q, k, v, o, cu_q, cu_k, ws, causal=causal, lse=lse)
    torch.cuda.synchronize()
    assert su.status(ws) == (0, 0)
    assert (o[sum(lens):] == 7.0).all() and (lse[:, sum(lens):] == 7.0).all()
    cq, ck = cu_q.tolist(), cu_k.tolist()
    for b, n in enumerate(lens):
        for h in (0, heads_q - 1):
            kb, vb = (su.to_f64(t[ck[b]:ck[b + 1], h * heads_kv // heads_q]) for t in (k, v))
            rows = sorted({0, 1, 63, 64, 127, 128, 255, 256, 511, 512, n // 2, n - 2, n - 1} & set(range(n)))
            last = np.array(rows) + past if causal else np.full(len(rows), total[b])
            seen = np.arange(total[b])[None] <= last[:, None]
            qb = su.to_f64(q[cq[b]:cq[b + 1], h])[rows]
            w, l, a, _, s = orc.attend(qb, kb, vb, seen)
            su.assert_within(su.to_f64(o[cq[b]:cq[b + 1], h])[rows], w, su.output_bound(w, a, s, dtype, np.abs(vb).sum(axis=0).max()), f"{b} {h} O")
            su.assert_within(su.to_f64(lse[h, cq[b]:cq[b + 1]])[rows], l, su.lse_bound(l, s), f"{b} {h} LSE")


def test_a_later_nan_in_a_long_sequence():
    """An infinity in V: rows before it are what they were, bit for bit, rows from it on have it."""
    gen, n, at = su.generator(2), 13000, 9000
    q, k, v = (su.rows(n, 8, torch.bfloat16, gen) for _ in "qkv")
    cu, ws = su.offsets([n]), sd.new_workspace(256, "cuda")
    want, got = torch.empty_like(q), torch.empty_like(q)
    sd.sparsed_attn_packed(q, k, v, want, cu, cu, ws, causal=True)
    for column in (5, 120):
        for bad in (float("inf"), float("nan")):
            v2 = v.clone()
            v2[at, 3, column] = bad
            sd.sparsed_attn_packed(q, k, v2, got, cu, cu, ws, causal=True)
            torch.cuda.synchronize()
            assert torch.equal(got[:at], want[:at])
            tail = got[at:, 3, column]
            assert (tail.isnan() if bad != bad else tail == bad).all()
            other = torch.ones(8, 128, dtype=torch.bool, device="cuda")
            other[3, column] = False
            assert torch.equal(got[at:][:, other], want[at:][:, other])
    assert su.status(ws) == (0, 0)
