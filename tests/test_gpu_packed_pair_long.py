"""Long packed sequences on the CTA-pair kernel, which the rule itself chooses for every case here: tiles of one head, of several
grouped heads, and sequences whose last cluster has rows for some of its two CTAs and two streams only."""
import numpy as np
import pytest
import torch

import paper_2509_24014_b200 as sd
from oracle import packed_and_paged as orc
from tests import host_rules
from tests import serving_util as su

pytestmark = pytest.mark.gpu


def ends(per_cta, base):
    """Lengths whose last cluster, four tiles of `per_cta` tokens, ends with a tile's first or last token or between."""
    rest = [1, per_cta, per_cta + 1, 2 * per_cta + 1, 3 * per_cta, 3 * per_cta + 1, 4 * per_cta]
    return [(base + 611 * i) // (4 * per_cta) * 4 * per_cta + r for i, r in enumerate(rest)]


CASES = [  # lengths, cached tokens before them, heads, mask, type
    ([5000, 9000, 3000], 0, 28, 4, True, "bf16"), ([5000, 9000, 3000], 2500, 28, 4, True, "fp16"),
    (ends(18, 5000), 0, 14, 2, True, "bf16"), (ends(18, 4300), 0, 7, 1, False, "fp16"),
    (ends(128, 5000), 0, 8, 8, False, "bf16"), (ends(128, 5000), 8000, 4, 4, True, "bf16"),
    (ends(42, 5000), 0, 6, 2, False, "bf16"), (ends(25, 5000), 4000, 10, 2, True, "fp16"),
    (ends(32, 5000), 4000, 8, 2, True, "bf16"),
]


@pytest.mark.parametrize("lens,past,heads_q,heads_kv,causal,dtype", CASES)
def test_against_the_definition(lens, past, heads_q, heads_kv, causal, dtype):
    gen, dtype = su.generator(sum(lens)), su.DTYPES[dtype]
    total = [n + past for n in lens]
    q = su.rows(sum(lens) + 5, heads_q, dtype, gen)
    k, v = (su.rows(sum(total) + 5, heads_kv, dtype, gen) for _ in "kv")
    # (the tensors' rows behind the last sequence go into the rule as well)
    assert host_rules.packed_is_pair(len(lens), q.shape[0], k.shape[0], heads_q, heads_kv, causal)
    for t in (k, v):
        t[sum(total):] = float("nan")
    cu_q, cu_k = su.offsets(lens), su.offsets(total)
    o, lse = torch.full_like(q, 7.0), torch.full((heads_q, q.shape[0]), 7.0, device="cuda")
    ws = sd.new_workspace(256, "cuda")
    sd.sparsed_attn_packed(q, k, v, o, cu_q, cu_k, ws, causal=causal, lse=lse)
    torch.cuda.synchronize()
    assert su.status(ws) == (0, 0)
    assert (o[sum(lens):] == 7.0).all() and (lse[:, sum(lens):] == 7.0).all()
    assert torch.isfinite(o[:sum(lens)]).all() and torch.isfinite(lse[:, :sum(lens)]).all()
    cq, ck = cu_q.tolist(), cu_k.tolist()
    for b, n in enumerate(lens):
        for h in sorted({0, heads_q // 2, heads_q - 1}):
            kb, vb = (su.to_f64(t[ck[b]:ck[b + 1], h * heads_kv // heads_q]) for t in (k, v))
            rows = sorted({0, 1, 17, 18, 71, 72, 127, 128, 511, 512, n // 2, n - 130, n - 73, n - 19, n - 2, n - 1})
            last = np.array(rows) + past if causal else np.full(len(rows), total[b] - 1)
            seen = np.arange(total[b])[None] <= last[:, None]
            w, l, a, _, s = orc.attend(su.to_f64(q[cq[b]:cq[b + 1], h])[rows], kb, vb, seen)
            su.assert_within(su.to_f64(o[cq[b]:cq[b + 1], h])[rows], w,
                             su.output_bound(w, a, s, dtype, np.abs(vb).sum(axis=0).max()), f"{b} {h} O")
            su.assert_within(su.to_f64(lse[h, cq[b]:cq[b + 1]])[rows], l, su.lse_bound(l, s), f"{b} {h} LSE")
