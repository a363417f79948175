"""The packed kernel whose MMAs span CTA pairs: infinities and NaN in V's masked places, which two streams of warps take out of
one tile, must not reach a row that does not see them, and must reach every row that does."""
import pytest
import torch

import paper_2509_24014_b200 as sd
from tests import host_rules
from tests import serving_util as su

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens,heads_q,heads_kv,causal,dtype", [
    ([9000, 8999, 9001, 9037], 8, 8, False, "bf16"), ([30001], 8, 8, True, "bf16"), ([16000, 16300], 14, 2, True, "fp16"),
    ([4700, 4811, 5003, 4999], 28, 4, False, "fp16")])
def test_rows_behind_a_sequence(lens, heads_q, heads_kv, causal, dtype):
    """Behind every sequence lie 64 rows of keys that no query has (a sequence of no queries), which its last tiles hold: finite
    ones first, then infinities and NaN everywhere, in one column, and in one row. The outputs are the same bits, call after call."""
    gen, dtype = su.generator(sum(lens)), su.DTYPES[dtype]
    lens_q, lens_k = [], []
    for n in lens:
        lens_q += [n, 0]
        lens_k += [n, 64]
    assert host_rules.packed_is_pair(len(lens_q), sum(lens_q), sum(lens_k), heads_q, heads_kv, causal)
    q = su.rows(sum(lens_q), heads_q, dtype, gen)
    k, v = (su.rows(sum(lens_k), heads_kv, dtype, gen) for _ in "kv")
    cu_q, cu_k = su.offsets(lens_q), su.offsets(lens_k)
    ws = sd.new_workspace(256, "cuda")
    want, got = torch.empty_like(q), torch.empty_like(q)
    want_lse, lse = torch.empty(heads_q, q.shape[0], device="cuda"), torch.empty(heads_q, q.shape[0], device="cuda")
    sd.sparsed_attn_packed(q, k, v, want, cu_q, cu_k, ws, causal=causal, lse=want_lse)
    gaps = torch.cat([torch.arange(cu_k[2 * i + 1], cu_k[2 * i + 2], device="cuda") for i in range(len(lens))])
    for bad in (float("nan"), float("inf"), -float("inf")):
        for columns, some in ((slice(None), gaps), (slice(5, 6), gaps), (slice(127, 128), gaps), (slice(None), gaps[::64])):
            k2, v2 = k.clone(), v.clone()
            v2[some, :, columns] = bad
            k2[some, :, columns] = bad
            for _ in range(4):
                got.fill_(7.0)
                sd.sparsed_attn_packed(q, k2, v2, got, cu_q, cu_k, ws, causal=causal, lse=lse)
                assert torch.equal(got, want) and torch.equal(lse, want_lse), (bad, columns)
    assert su.status(ws) == (0, 0)


@pytest.mark.parametrize("at", [0, 63, 64, 511, 12288, 12800, 15990, 15999])
def test_a_row_on_the_diagonal(at):
    """With a causal mask: every number of V's row `at` infinite. Rows before it keep their bits, rows from it on are infinite."""
    gen, n = su.generator(at), 16000
    assert host_rules.packed_is_pair(1, n, n, 8, 8, True)
    q, k, v = (su.rows(n, 8, torch.bfloat16, gen) for _ in "qkv")
    cu, ws = su.offsets([n]), sd.new_workspace(256, "cuda")
    want, got = torch.empty_like(q), torch.empty_like(q)
    sd.sparsed_attn_packed(q, k, v, want, cu, cu, ws, causal=True)
    v[at] = float("inf")
    for _ in range(4):
        sd.sparsed_attn_packed(q, k, v, got, cu, cu, ws, causal=True)
        assert torch.equal(got[:at], want[:at]) and (got[at:] == float("inf")).all()
    assert su.status(ws) == (0, 0)
