"""bf16: values as large as the calls allow, 2^103 / n for n keys, with logits that keep the softmax reference as far below them as
it ever lies: the fp32 sums of probabilities times values must not overflow."""
import numpy as np
import pytest
import torch

import paper_2509_24014_b200 as sd
from tests import host_rules
from tests import serving_util as su

pytestmark = pytest.mark.gpu
# P and the output are rounded by half a step each, and all values are alike; beside that the fp32 sums: up to 1024 additions of 16
# keys each, off by 2^-23 each where the hardware cuts off, and the exponentials (2^-22)
BOUND = 2 * 2.0 ** -8 + 2.0 ** -12


def keys_and_values(n, first, heads, logit):
    """Logits of 0 for the first keys and `logit` (base 2, for a query of one at a scale of 1) for the others."""
    k = torch.zeros(n, heads, 128, dtype=torch.bfloat16, device="cuda")
    k[first:, :, 0] = logit * np.log(2.0)
    v = torch.full((n, heads, 128), 2.0 ** 103 / n, dtype=torch.bfloat16, device="cuda")
    v[:, :, 1::2] *= -1
    return k, v


def check(o, n):
    want = torch.full((128,), 2.0 ** 103 / n, dtype=torch.float64, device="cuda")
    want[1::2] *= -1
    assert ((o.double() - want).abs() <= BOUND * want.abs()).all()


@pytest.mark.parametrize("rows,n,heads,pair", [(3, 16384, 2, False), (8192, 8192, 5, True)])
def test_packed(rows, n, heads, pair):
    """A tile of 64 keys adds up to just under 2^24 of the first tile's largest."""
    assert host_rules.packed_is_pair(1, rows, n, heads, heads, False) == pair
    k, v = keys_and_values(n, 64, heads, 17.95)
    q = torch.zeros(rows, heads, 128, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 1.0
    o, ws = torch.empty_like(q), sd.new_workspace(256, "cuda")
    sd.sparsed_attn_packed(q, k, v, o, su.offsets([rows]), su.offsets([n]), ws, softmax_scale=1.0)
    check(o, n)
    assert su.status(ws) == (0, 0)


@pytest.mark.parametrize("batch,heads_q,heads_kv", [(40, 32, 32), (150, 60, 4)])
def test_paged(batch, heads_q, heads_kv):
    """A key just under 2^24 of the first ones, in sequences that one CTA has from start to end."""
    n = 4096
    k, v = keys_and_values(n, 64, heads_kv, 23.9)
    table = torch.arange(n // 64, dtype=torch.int32, device="cuda").expand(batch, n // 64).contiguous()
    cache = sd.make_cache(k.view(-1, 64, heads_kv, 128), v.view(-1, 64, heads_kv, 128), table,
                          torch.full((batch,), n, dtype=torch.int32, device="cuda"))
    q = torch.zeros(batch, heads_q, 128, dtype=torch.bfloat16, device="cuda")
    q[:, :, 0] = 1.0
    o, ws = torch.empty_like(q), sd.new_workspace(sd.sparsed_paged_workspace_bytes(cache, heads_q), "cuda")
    sd.sparsed_attn_paged(q, cache, o, ws, softmax_scale=1.0)
    check(o, n)
    assert su.status(ws) == (0, 0)
