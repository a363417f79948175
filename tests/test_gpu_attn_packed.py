"""sparsed_attn_packed against its fp64 definition, at the lengths, masks and layouts where it can go wrong."""
import numpy as np
import pytest
import torch

import paper_2509_24014_b200 as sd
from oracle import packed_and_paged as orc
from tests import serving_util as su

pytestmark = pytest.mark.gpu


def run(q, k, v, cu_q, cu_k, causal, scale=0.0, o=None, lse=None):
    o = torch.full_like(q, 7.0) if o is None else o
    lse = torch.full((q.shape[1], q.shape[0]), 7.0, device=q.device) if lse is None else lse
    ws = sd.new_workspace(sd.sparsed_workspace_bytes(sd.OP_ATTN_PACKED), q.device)
    sd.sparsed_attn_packed(q, k, v, o, cu_q, cu_k, ws, causal=causal, lse=lse, softmax_scale=scale)
    torch.cuda.synchronize()
    assert su.status(ws) == (0, 0)
    return o, lse


def check(q, k, v, lens_q, lens_k, causal, scale=0.0, what=""):
    cu_q, cu_k = su.offsets(lens_q), su.offsets(lens_k)
    o, lse = run(q, k, v, cu_q, cu_k, causal, scale)
    n = int(cu_q[-1])
    want_o, want_lse, absolute, spread = orc.attn_packed(su.to_f64(q), su.to_f64(k), su.to_f64(v), cu_q.tolist(), cu_k.tolist(),
                                                         causal, scale=float(np.float32(scale)) if scale else None)
    v64 = np.abs(np.where(np.isfinite(su.to_f64(v)), su.to_f64(v), 0.0))
    v_sum = v64.sum(axis=0).max() if v64.size else 0.0
    su.assert_within(su.to_f64(o)[:n], want_o[:n],
                     su.output_bound(want_o[:n], absolute[:n], spread.T[:n], q.dtype, v_sum), what + " O")
    su.assert_within(su.to_f64(lse)[:, :n], want_lse[:, :n], su.lse_bound(want_lse[:, :n], spread[:, :n]), what + " LSE")
    assert (o[n:] == 7.0).all() and (lse[:, n:] == 7.0).all()      # rows behind the last sequence
    return o, lse


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("lens", [[1], [2, 1, 3], [63, 64, 65], [127, 1, 128, 129], [300, 5], [0, 17, 0, 0, 200, 0], [1] * 40])
def test_lengths(lens, dtype, causal):
    gen = su.generator(sum(lens))
    q, k, v = (su.rows(sum(lens) + 3, 2, su.DTYPES[dtype], gen) for _ in "qkv")
    check(q, k, v, lens, lens, causal, what=str(lens))


@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("lens_q,lens_k", [([1], [300]), ([5, 70], [64, 500]), ([130, 1, 64], [200, 1, 129]),
                                           ([200], [70]), ([140, 3], [0, 9]), ([256], [1]), ([1, 1], [0, 0])])
def test_queries_and_keys_of_different_lengths(lens_q, lens_k, causal):
    """More keys than queries (cached text), fewer (the first rows see none), and none at all."""
    gen = su.generator(3)
    q = su.rows(sum(lens_q) + 2, 4, torch.bfloat16, gen)
    k, v = (su.rows(sum(lens_k) + 1, 2, torch.bfloat16, gen) for _ in "kv")
    check(q, k, v, lens_q, lens_k, causal)


def test_no_keys_at_all():
    gen = su.generator(3)
    q = su.rows(5, 2, torch.bfloat16, gen)
    k = torch.empty(0, 2, 128, dtype=torch.bfloat16, device="cuda")
    check(q, k, k, [2, 3], [0, 0], False)


@pytest.mark.parametrize("heads_q,heads_kv", [(1, 1), (7, 1), (6, 2), (28, 4), (5, 5)])
@pytest.mark.parametrize("layouts", [("token", "token", "token"), ("head", "fused", "head"), ("fused", "head", "fused")])
def test_heads_and_layouts(heads_q, heads_kv, layouts):
    lens, gen = [100, 161], su.generator(heads_q)
    q = su.rows(sum(lens), heads_q, torch.bfloat16, gen, layouts[0])
    k, v = (su.rows(sum(lens), heads_kv, torch.bfloat16, gen, x) for x in layouts[1:])
    check(q, k, v, lens, lens, True, scale=0.05)


def test_output_layout():
    lens, gen = [150, 20], su.generator(1)
    q, k, v = (su.rows(170, 3, torch.bfloat16, gen) for _ in "qkv")
    cu = su.offsets(lens)
    a, _ = run(q, k, v, cu, cu, True)
    o = torch.zeros(3, 170, 128, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    b, _ = run(q, k, v, cu, cu, True, o=o)
    assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("causal", [False, True])
def test_logits_that_keep_outgrowing_the_reference(causal, dtype):
    """Keys ordered so that every row's logits grow with the key index: the running reference moves in every tile."""
    gen = su.generator(5)
    q, k, v = (su.rows(400, 1, su.DTYPES[dtype], gen, scale=2.0) for _ in "qkv")
    order = torch.argsort(k[:, 0].float() @ q[0, 0].float())
    k = k[order].contiguous()
    q = (q[:1] + 0.05 * q).contiguous()
    check(q, k, v, [400], [400], causal)


def test_masked_places_of_nan_and_infinity():
    """What a row does not see does not reach it: rows behind the sequences, other sequences, later keys."""
    lens, gen = [70, 130, 200], su.generator(7)
    total = sum(lens)
    q, k, v = (su.rows(total + 100, 2, torch.bfloat16, gen) for _ in "qkv")
    for t in (q, k, v):
        t[total:] = float("nan")
    clean = [t.clone() for t in (q, k, v)]
    cu = su.offsets(lens)
    want, want_lse = run(*clean, cu, cu, True)
    check(q, k, v, lens, lens, True)
    # the second sequence's V and K from its row 90 on: only its rows from 90 on may change
    for bad in (float("nan"), float("inf"), -float("inf")):
        k2, v2 = k.clone(), v.clone()
        v2[70 + 90, 0, 3] = bad
        v2[70 + 129, 1, 127] = bad
        k2[70 + 100, 0, 5] = bad
        o, lse = run(q, k2, v2, cu, cu, True)
        same = torch.ones(total, 2, dtype=torch.bool, device="cuda")
        same[70 + 90:200, 0] = False      # head 0: from the first bad V on
        same[199, 1] = False
        assert torch.equal(o[:total][same], want[:total][same])
        # head 0, rows 90..99: element 3 is what V holds there, the others are as they were
        mid = o[70 + 90:70 + 100, 0]
        assert (mid[:, 3].isnan() if bad != bad else mid[:, 3] == bad).all()
        keep = [i for i in range(128) if i != 3]
        assert torch.equal(mid[:, keep], want[70 + 90:70 + 100, 0][:, keep])
        last = o[199, 1]
        assert last[127].isnan() if bad != bad else last[127] == bad
        assert torch.equal(last[:127], want[199, 1][:127])
        lse_same = torch.ones(2, total, dtype=torch.bool, device="cuda")
        lse_same[0, 70 + 100:200] = False
        assert torch.equal(lse[:, :total][lse_same], want_lse[:, :total][lse_same])


@pytest.mark.parametrize("causal", [False, True])
def test_visible_infinities(causal):
    """A V of infinity that every row sees, far from the diagonal: it comes out; a later sequence is not touched."""
    gen = su.generator(8)
    q, k, v = (su.rows(500, 1, torch.bfloat16, gen) for _ in "qkv")
    v[3, 0, 9] = float("inf")
    lens = [300, 200]
    cu = su.offsets(lens)
    o, _ = run(q, k, v, cu, cu, causal)
    first = 3 if causal else 0
    assert (o[first:300, 0, 9] == float("inf")).all() and torch.isfinite(o[:first]).all() and torch.isfinite(o[300:]).all()
    keep = [i for i in range(128) if i != 9]
    assert torch.isfinite(o[:, 0][:, keep]).all()


def test_a_long_sequence_and_many_short_ones():
    """Several passes over the heads' keys and values (beyond what L2 is given), 1100 sequences; sampled rows."""
    lens, gen = [1] * 600 + [20000] + [3] * 500, su.generator(9)
    q, k, v = (su.rows(sum(lens), 8, torch.bfloat16, gen) for _ in "qkv")
    cu = su.offsets(lens)
    o, lse = run(q, k, v, cu, cu, True)
    c = cu.tolist()
    picks = [(0, 0), (599, 0), (600, 0), (600, 1), (600, 127), (600, 128), (600, 9999), (600, 19999), (601, 0), (1100, 2)]
    for b, i in picks:
        kb, vb, qb = (su.to_f64(t[c[b]:c[b + 1]]) for t in (k, v, q))
        for h in (0, 7):
            seen = (np.arange(lens[b]) <= i)[None]
            w, l, a, _, s = orc.attend(qb[i:i + 1, h], kb[:, h], vb[:, h], seen)
            su.assert_within(su.to_f64(o[c[b] + i, h])[None], w, su.output_bound(w, a, s, torch.bfloat16, 0.0), f"{b} {i} {h}")
            su.assert_within(su.to_f64(lse[h, c[b] + i])[None], l, su.lse_bound(l, s), f"{b} {i} {h} LSE")


def test_one_sequence_equals_the_rectangular_call():
    """A single packed sequence without a mask is sparsed_attn_full's problem."""
    gen = su.generator(10)
    q, k, v = (su.rows(777, 4, torch.bfloat16, gen) for _ in "qkv")
    cu = su.offsets([777])
    o, lse = run(q, k, v, cu, cu, False)
    full = torch.empty(1, 4, 777, 128, dtype=torch.bfloat16, device="cuda")
    full_lse = torch.empty(1, 4, 777, device="cuda")
    ws = sd.new_workspace(256, "cuda")
    sd.sparsed_attn_full(*(t.transpose(0, 1)[None] for t in (q, k, v)), full, full_lse, ws)
    d = (o.transpose(0, 1).double() - full[0].double()).abs()
    assert (d <= 2 * 2.0 ** -8 * full[0].double().abs() + 2 * 2.0 ** -8 * 4.0 / 27).all()   # two roundings of P each, |V| < 4 in a mean of 777
    assert (lse - full_lse[0]).abs().max() <= 1e-5


def test_results_are_the_same_bits_again_and_in_a_graph():
    lens, gen = [5, 300, 64], su.generator(11)
    q, k, v = (su.rows(sum(lens), 4, torch.bfloat16, gen) for _ in "qkv")
    cu = su.offsets(lens)
    want, want_lse = run(q, k, v, cu, cu, True)
    o, lse = torch.zeros_like(q), torch.zeros_like(want_lse)
    ws = sd.new_workspace(256, "cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        sd.sparsed_attn_packed(q, k, v, o, cu, cu, ws, causal=True, lse=lse)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.sparsed_attn_packed(q, k, v, o, cu, cu, ws, causal=True, lse=lse)
    o.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(o, want) and torch.equal(lse, want_lse)
    # other lengths in the same buffers: the graph reads them when it runs
    cu.copy_(su.offsets([100, 9, 260]))
    graph.replay()
    again, again_lse = run(q, k, v, cu, cu, True)
    assert torch.equal(o, again) and torch.equal(lse, again_lse)


@pytest.mark.parametrize("cu_q,cu_k", [([0, 50, 40, 100], [0, 30, 60, 90]), ([0, 50, 60, 1000], [0, 30, 60, 90]),
                                       ([0, 50, 60, 100], [0, -30, 2000, 90]), ([-5, 50, 60, 100], [0, 30, 60, 90])])
def test_offsets_that_point_nowhere_are_reported_and_not_followed(cu_q, cu_k):
    gen = su.generator(12)
    q, k, v = (su.rows(100, 2, torch.bfloat16, gen) for _ in "qkv")
    o = torch.zeros_like(q)
    ws = sd.new_workspace(256, "cuda")
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    sd.sparsed_attn_packed(q, k, v, o, i32(cu_q), i32(cu_k), ws, causal=True)
    torch.cuda.synchronize()
    assert su.status(ws)[0] == 6
    sd.sparsed_workspace_init(ws)
    cu = su.offsets([100])
    sd.sparsed_attn_packed(q, k, v, o, cu, cu, ws, causal=True)
    torch.cuda.synchronize()
    assert su.status(ws) == (0, 0)


@pytest.mark.parametrize("causal", [False, True])
def test_offsets_beyond_32_bits(causal):
    """Rows of q, k, v and o more than 2^32 elements from the start; what lies before belongs to sequences of no keys or queries."""
    total, heads, n = 1_060_000, 32, 300
    assert (total - n) * heads * 128 > 1 << 32
    gen = su.generator(16)
    q, k, v, o = (torch.empty(total, heads, 128, dtype=torch.bfloat16, device="cuda") for _ in "qkvo")
    for t in (q, k, v):
        t[total - n:] = su.rows(n, heads, torch.bfloat16, gen)
    v[total - 5, 3, 7] = float("inf")
    cu_q, cu_k = su.offsets([total - n, 0, n]), su.offsets([0, total - n, n])
    o[:8] = 7.0
    lse = torch.zeros(heads, total, device="cuda")
    run(q, k, v, cu_q, cu_k, causal, o=o, lse=lse)
    want, want_lse = run(*(t[total - n:].clone() for t in (q, k, v)), su.offsets([n]), su.offsets([n]), causal)
    assert torch.equal(o[total - n:].view(torch.int16), want.view(torch.int16)) and torch.equal(lse[:, total - n:], want_lse)
    assert (o[:total - n] == 0).all() and (lse[:, :total - n] == -float("inf")).all()
