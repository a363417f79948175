"""fp16: keys whose weights are far below a row's largest one, in the packed and the one-token call. One key takes most of the
weight and has a V of zero, so that the output is what the many others give."""
import numpy as np
import pytest
import torch

import paper_2509_24014_b200 as sd
from oracle import packed_and_paged as orc
from tests import serving_util as su

pytestmark = pytest.mark.gpu
# How far below the one key's logit the others' are, in powers of two. 12 to 22: probabilities that fp16 holds in full against a
# reference 2^8 below the largest, but as few bits (or, from 25 on, not at all) against the largest itself.
GAPS = np.array([10.0, 12.3, 14.7, 16.6, 18.45, 19.55, 20.6, 21.45, 22.6, 24.6, 25.4, 26.3])


def inputs(n, rows, heads_q, heads_kv, sink, gen):
    """q [rows, heads_q, 128], k, v [n, heads_kv, 128]: logits (at a scale of 1) of gap * ln 2 for key `sink`, 0 for the others."""
    gap = torch.from_numpy(GAPS[(np.arange(rows)[:, None] + 5 * np.arange(heads_q)) % len(GAPS)]).to(gen.device)
    q = torch.zeros(rows, heads_q, 128, dtype=torch.float16, device=gen.device)
    q[:, :, 0] = (gap * np.log(2) / 8).half()
    k = torch.zeros(n, heads_kv, 128, dtype=torch.float16, device=gen.device)
    k[sink, :, 0] = 8.0
    v = (64 * (0.5 + torch.rand(n, heads_kv, 128, generator=gen, device=gen.device))).half()
    v[sink] = 0.0
    return q, k, v


def bound(o, absolute, spread, v_abs_sum):
    """As su.output_bound, but what a probability loses below 2^-14 of the reference, 2^-25 of that, is 2^-33 of the row's sum at
    most: the reference lies 2^8 below a row's largest logit or lower."""
    return su.output_bound(o, absolute, spread, torch.float16, 2.0 ** -8 * v_abs_sum)


# the single-CTA kernel (few queries), and enough long ones that the rule takes CTA pairs
@pytest.mark.parametrize("rows,n,heads_q,heads_kv", [(40, 9000, 4, 2), (8192, 8192, 5, 5)])
@pytest.mark.parametrize("sink", [0, 4003])
def test_packed(rows, n, heads_q, heads_kv, sink):
    q, k, v = inputs(n, rows, heads_q, heads_kv, sink, su.generator(sink))
    o, lse, ws = torch.empty_like(q), torch.empty(heads_q, rows, device="cuda"), sd.new_workspace(256, "cuda")
    sd.sparsed_attn_packed(q, k, v, o, su.offsets([rows]), su.offsets([n]), ws, lse=lse, softmax_scale=1.0)
    torch.cuda.synchronize()
    assert su.status(ws) == (0, 0)
    some = list(range(0, rows, max(rows // 37, 1)))
    for h in range(heads_q):
        vb = su.to_f64(v[:, h * heads_kv // heads_q])
        w, l, a, _, s = orc.attend(su.to_f64(q[some, h]), su.to_f64(k[:, h * heads_kv // heads_q]), vb, np.ones((len(some), n), bool), 1.0)
        su.assert_within(su.to_f64(o[some, h]), w, bound(w, a, s, np.abs(vb).sum(axis=0).max()), f"{h} O")
        su.assert_within(su.to_f64(lse[h, some]), l, su.lse_bound(l, s), f"{h} LSE")


# (batches large enough that a CTA has whole sequences: parts have references of their own)
@pytest.mark.parametrize("batch,n,heads_q,heads_kv", [(40, 4000, 32, 32), (150, 2500, 60, 4), (1, 131072, 24, 2), (1, 3001, 12, 12)])
@pytest.mark.parametrize("sink", [0, 1000])
def test_paged(batch, n, heads_q, heads_kv, sink):
    """Eight and sixteen heads at once; four keys with much weight, one for each of a CTA's warps, that have references of their
    own too."""
    q, k, v = inputs(n, batch, heads_q, heads_kv, [sink + 16 * w for w in range(4)], su.generator(sink + n))
    pages = -(-n // 64)
    order = torch.randperm(pages, generator=su.generator(1), device="cuda")
    pools = []
    for t in (k, v):
        pool = torch.zeros(pages * 64, heads_kv, 128, dtype=torch.float16, device="cuda")
        pool[:n] = t
        pools.append(torch.empty_like(pool.view(pages, 64, heads_kv, 128)))
        pools[-1][order] = pool.view(pages, 64, heads_kv, 128)
    table = order.int().expand(batch, pages).contiguous()   # (all sequences share their pages)
    cache = sd.make_cache(*pools, table, torch.full((batch,), n, dtype=torch.int32, device="cuda"))
    o, lse = torch.empty_like(q), torch.empty(batch, heads_q, device="cuda")
    ws = sd.new_workspace(sd.sparsed_paged_workspace_bytes(cache, heads_q), "cuda")
    sd.sparsed_attn_paged(q, cache, o, ws, lse=lse, softmax_scale=1.0)
    torch.cuda.synchronize()
    assert su.status(ws) == (0, 0)
    for h in range(heads_q):
        kb, vb = (su.to_f64(t[:, h * heads_kv // heads_q]) for t in (k, v))
        some = list(range(h % 4, batch, 7)) or [0]
        w, l, a, _, s = orc.attend(su.to_f64(q[some, h]), kb, vb, np.ones((len(some), n), bool), 1.0)
        su.assert_within(su.to_f64(o[some, h]), w, bound(w, a, s, np.abs(vb).sum(axis=0).max()), f"{h} O")
        su.assert_within(su.to_f64(lse[some, h]), l, su.lse_bound(l, s), f"{h} LSE")
