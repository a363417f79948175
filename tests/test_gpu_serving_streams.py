"""The packed and paged calls as a server makes them: captured and replayed together, several at once on streams of their own,
batches with room to spare, many sequences, tables that name a page twice."""
import numpy as np
import pytest
import torch

import paper_2509_24014_b200 as sd
from tests import serving_util as su
from tests.test_gpu_attn_packed import check
from tests.test_gpu_paged_cache import attend, check_evict, check_paged, i32

pytestmark = pytest.mark.gpu


def step(state):
    """New tokens written, attention with the weights added up, the cache brought down to `keep` keys a head."""
    s = state
    sd.sparsed_cache_write(s["cache"], s["k_new"], s["v_new"], s["cu"], s["ws"][0])
    sd.sparsed_attn_paged(s["q"], s["cache"], s["o"], s["ws"][1], lse=s["lse"], mass_in=s["mass"], mass_out=s["mass"])
    sd.sparsed_cache_evict(s["cache"], s["mass"], s["keep"], 4, s["small"], s["small_mass"], s["kept"], s["ws"][2])
    sd.sparsed_attn_paged(s["q"], s["small"], s["o2"], s["ws"][3])


def make_state(seed, batch=3, heads_q=8, heads_kv=2, room=512, keep=70, page=32):
    gen, s = su.generator(seed), dict(keep=keep)
    s["k"], s["v"], s["table"] = su.paged_pool([room] * batch, page, heads_kv, torch.bfloat16, gen)
    s["lens"] = i32([1] * batch)
    s["q"] = su.rows(batch, heads_q, torch.bfloat16, gen)
    s["k_new"], s["v_new"] = (su.rows(batch + 2, heads_kv, torch.bfloat16, gen) for _ in "kv")
    s["cu"] = su.offsets([1] * batch)
    s["o"], s["o2"] = torch.zeros_like(s["q"]), torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(batch, heads_q, device="cuda")
    s["mass"] = torch.zeros(batch, heads_kv, room, device="cuda")
    s["cache"] = sd.make_cache(s["k"], s["v"], s["table"], s["lens"])
    s["small_k"], s["small_v"], s["small_table"] = su.paged_pool([keep] * batch, 16, heads_kv, torch.bfloat16, gen)
    s["small_lens"] = i32([0] * batch)
    s["small"] = sd.make_cache(s["small_k"], s["small_v"], s["small_table"], s["small_lens"])
    s["small_mass"] = torch.zeros(batch, heads_kv, keep, device="cuda")
    s["kept"] = torch.zeros(batch, heads_kv, keep, dtype=torch.int32, device="cuda")
    s["ws"] = [sd.new_workspace(n, "cuda") for n in (sd.sparsed_workspace_bytes(sd.OP_CACHE_WRITE), sd.sparsed_paged_workspace_bytes(s["cache"], heads_q, True),
                                                     sd.sparsed_evict_workspace_bytes(s["cache"]), sd.sparsed_paged_workspace_bytes(s["small"], heads_q, False))]
    return s


WRITTEN = ("k", "v", "o", "o2", "lse", "mass", "small_k", "small_v", "small_lens", "small_mass", "kept")


def set_inputs(s, lens, seed):
    """The tensors' contents for a step, whatever they held before."""
    gen = su.generator(seed)
    s["lens"].copy_(i32(lens))
    for name in ("k", "v", "q", "k_new", "v_new"):
        s[name].copy_(torch.randn(s[name].shape, generator=gen, device="cuda"))
    s["mass"].copy_(torch.rand(s["mass"].shape, generator=gen, device="cuda"))
    for name in ("o", "o2", "lse", "small_k", "small_v", "small_lens", "small_mass", "kept"):
        s[name].zero_()


def outcome(s):
    return {name: s[name].clone() for name in WRITTEN}


def same(a, b):
    return all(torch.equal(a[name], b[name]) for name in WRITTEN)


LENGTHS = ([1, 300, 70], [512, 71, 69], [17, 1, 512], [100, 100, 100])


def test_a_serving_step_captured_and_replayed():
    s = make_state(1)
    want = []
    for i, lens in enumerate(LENGTHS):
        set_inputs(s, lens, i)
        step(s)
        torch.cuda.synchronize()
        want.append(outcome(s))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(s)
    for i, lens in enumerate(LENGTHS):
        set_inputs(s, lens, i)
        graph.replay()
        torch.cuda.synchronize()
        assert same(outcome(s), want[i]), lens
    assert all(su.status(ws) == (0, 0) for ws in s["ws"])


def test_steps_at_once_on_streams_and_graphs_of_their_own():
    states = [make_state(seed, batch=b, room=r) for seed, b, r in ((1, 3, 512), (2, 5, 4096), (3, 1, 16384), (4, 40, 160))]
    streams = [torch.cuda.Stream() for _ in states]
    lens = [[1 + (37 * i * i) % s["mass"].shape[2] for i in range(s["q"].shape[0])] for s in states]
    want = []
    for s, n in zip(states, lens):
        set_inputs(s, n, 9)
        step(s)
        torch.cuda.synchronize()
        want.append(outcome(s))
    graphs = []
    for s in states:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            step(s)
    for replay in (False, True, False, True):
        for s, n in zip(states, lens):
            set_inputs(s, n, 9)
        torch.cuda.synchronize()
        for s, stream, graph in zip(states, streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay() if replay else step(s)
        torch.cuda.synchronize()
        assert all(same(outcome(s), w) for s, w in zip(states, want)), replay
    assert all(su.status(ws) == (0, 0) for s in states for ws in s["ws"])


def test_packed_calls_at_once():
    """Calls of both kernels side by side, on one workspace (it holds their status only), alone and as graphs."""
    gen = su.generator(5)
    calls = []
    for lens, heads, causal in (([9000, 8300], 8, False), ([300, 5, 0, 129] * 6, 4, True), ([13001], 8, True), ([1] * 500, 2, True)):
        q, k, v = (su.rows(sum(lens), heads, torch.bfloat16, gen) for _ in "qkv")
        calls.append(dict(q=q, k=k, v=v, cu=su.offsets(lens), causal=causal, o=torch.zeros_like(q), lse=torch.zeros(heads, q.shape[0], device="cuda")))
    ws = sd.new_workspace(256, "cuda")

    def call(c):
        sd.sparsed_attn_packed(c["q"], c["k"], c["v"], c["o"], c["cu"], c["cu"], ws, causal=c["causal"], lse=c["lse"])

    want = []
    for c in calls:
        call(c)
        torch.cuda.synchronize()
        want.append((c["o"].clone(), c["lse"].clone()))
    graphs = []
    for c in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(c)
    streams = [torch.cuda.Stream() for _ in calls]
    for replay in (False, True):
        for c in calls:
            c["o"].zero_()
            c["lse"].zero_()
        torch.cuda.synchronize()
        for c, stream, graph in zip(calls, streams, graphs):
            with torch.cuda.stream(stream):
                graph.replay() if replay else call(c)
        torch.cuda.synchronize()
        for c, (o, lse) in zip(calls, want):
            assert torch.equal(c["o"], o) and torch.equal(c["lse"], lse)
    assert su.status(ws) == (0, 0)


@pytest.mark.parametrize("causal", [False, True])
def test_packed_batch_with_room_to_spare(causal):
    """Offsets that repeat behind the last real sequence, tensors longer than the batch."""
    lens, gen = [40, 200, 1] + [0] * 29, su.generator(6)
    q, k, v = (su.rows(sum(lens) + 300, 4, torch.bfloat16, gen) for _ in "qkv")
    for t in (q, k, v):
        t[sum(lens):] = float("nan")
    check(q, k, v, lens, lens, causal)


def test_packed_many_sequences():
    lens = [(7 * i) % 4 for i in range(5000)]
    gen = su.generator(7)
    q, k, v = (su.rows(sum(lens), 2, torch.float16, gen) for _ in "qkv")
    check(q, k, v, lens, lens, True)


@pytest.mark.parametrize("causal", [False, True])
def test_a_sequences_bits_do_not_depend_on_the_batch(causal):
    lens, gen = [70, 1, 300, 128, 41], su.generator(15)
    q, k, v = (su.rows(sum(lens), h, torch.bfloat16, gen) for h in (14, 2, 2))
    at, ws = 0, sd.new_workspace(256, "cuda")

    def call(q, k, v, lens):
        o = torch.zeros_like(q)
        sd.sparsed_attn_packed(q, k, v, o, su.offsets(lens), su.offsets(lens), ws, causal=causal)
        return o

    batch = call(q, k, v, lens)
    for n in lens:
        assert torch.equal(call(q[at:at + n], k[at:at + n], v[at:at + n], [n]), batch[at:at + n])
        at += n
    assert su.status(ws) == (0, 0)


def test_packed_keys_that_are_the_values():
    lens, gen = [70, 300], su.generator(8)
    q, kv = su.rows(370, 8, torch.bfloat16, gen), su.rows(370, 2, torch.bfloat16, gen)
    check(q, kv, kv, lens, lens, True)


def test_paged_many_sequences():
    lens = [(13 * i) % 41 for i in range(3001)]
    gen = su.generator(9)
    k, v, table = su.paged_pool(lens, 16, 1, torch.bfloat16, gen)
    check_paged(su.rows(len(lens), 2, torch.bfloat16, gen), k, v, table, lens, with_mass=True)


def test_paged_many_query_heads_to_one_head():
    """More query heads to a key-value head than a CTA takes at once, several times over, and weights of all of them."""
    lens, gen = [1000, 0, 33], su.generator(10)
    k, v, table = su.paged_pool(lens, 64, 1, torch.float16, gen)
    check_paged(su.rows(3, 71, torch.float16, gen), k, v, table, lens, with_mass=True)


@pytest.mark.parametrize("lens,heads_q,heads_kv,page,dtype", [
    ([117, 250, 318, 337, 404, 233, 122, 149, 95], 32, 32, 256, "bf16"), ([104, 98, 128, 112, 132, 91, 111] * 5, 32, 32, 16, "bf16"),
    ([1060, 975, 1253, 1157, 869, 1047] * 9, 2, 2, 32, "fp16"), ([700, 33, 5000, 64], 28, 4, 64, "bf16"), ([300] * 30, 40, 2, 128, "fp16")])
def test_paged_keys_that_are_in_l2(lens, heads_q, heads_kv, page, dtype):
    """Keys and values that have just been written come back much sooner than ones from memory: the same bits, and no trace of the
    unused places (NaN) around them."""
    gen = su.generator(18)
    k, v, table = su.paged_pool(lens, page, heads_kv, su.DTYPES[dtype], gen)
    su.poison_unused(k, v, table, lens)
    k0, v0 = k.clone(), v.clone()
    q = su.rows(len(lens), heads_q, su.DTYPES[dtype], gen, scale=2.0)
    cache = sd.make_cache(k, v, table, i32(lens))
    ws = sd.new_workspace(sd.sparsed_paged_workspace_bytes(cache, heads_q, True), "cuda")
    mass, o = torch.zeros(len(lens), heads_kv, table.shape[1] * page, device="cuda"), torch.empty_like(q)
    flush = torch.empty(300 << 20, dtype=torch.uint8, device="cuda")

    def call(warm):
        mass.zero_()
        if warm:
            k.copy_(k0)
            v.copy_(v0)
        else:
            flush.fill_(1)
        sd.sparsed_attn_paged(q, cache, o, ws, mass_out=mass)
        return o.clone(), mass.clone()

    check_paged(q, k, v, table, lens, with_mass=True)
    want_o, want_mass = call(False)
    assert want_o.isfinite().all() and want_mass.isfinite().all()
    for i in range(20):
        got_o, got_mass = call(i % 4 != 3)
        assert torch.equal(got_o, want_o) and torch.equal(got_mass, want_mass), i
    assert su.status(ws) == (0, 0)


def test_the_same_page_twice():
    lens, gen = [200, 130], su.generator(11)
    k, v, table = su.paged_pool(lens, 16, 2, torch.bfloat16, gen)
    table[0, 3], table[0, 9] = table[0, 1], table[0, 1]
    table[1, :4] = table[0, 2]
    check_paged(su.rows(2, 6, torch.bfloat16, gen), k, v, table, lens, with_mass=True)
    check_evict(k, v, table, lens, torch.rand(2, 2, table.shape[1] * 16, generator=gen, device="cuda"), 60, 5)


def test_rows_of_the_padded_batch_stay_empty():
    """A fixed batch of which the last sequences have ended: zeros, -inf, nothing of the cache touched."""
    lens, gen = [90, 5, 0, 0, 0], su.generator(12)
    k, v, table = su.paged_pool(lens, 16, 2, torch.bfloat16, gen)
    before = k.clone(), v.clone()
    k_new = su.rows(6, 2, torch.bfloat16, gen)
    ws = sd.new_workspace(256, "cuda")
    cache = sd.make_cache(k, v, table, i32(lens))
    sd.sparsed_cache_write(cache, k_new, k_new, i32([0, 1, 2, 2, 2, 2]), ws)
    assert su.status(ws) == (0, 0)
    for pool, was in zip((k, v), before):
        was[int(table[0, 5]), 9] = k_new[0]
        was[int(table[1, 0]), 4] = k_new[1]
        assert torch.equal(pool, was)
    o, lse, _ = attend(su.rows(5, 4, torch.bfloat16, gen), k, v, table, i32(lens))
    assert (o[2:] == 0).all() and (lse[2:] == -float("inf")).all() and o[:2].isfinite().all()


@pytest.mark.parametrize("heads_kv", [1, 2, 3, 4, 5, 8, 9, 16])
@pytest.mark.parametrize("lens", [[9000, 0, 1, 700], [3] * 400 + [0] * 3 + [1] * 50, [1], [7, 0, 0, 0, 9]])
def test_write_tokens_per_warp(heads_kv, lens):
    """One, two and several tokens to a warp, over sequences' ends and empty sequences, rows behind the last one left out."""
    gen = su.generator(17)
    lens_all = [n + (5 * i) % 40 for i, n in enumerate(lens)]
    k, v, table = su.paged_pool(lens_all, 16, heads_kv, torch.bfloat16, gen)
    want_k, want_v = k.clone(), v.clone()
    n = sum(lens)
    k_new, v_new = su.rows(n + 3, heads_kv, torch.bfloat16, gen, "fused"), su.rows(n + 3, heads_kv, torch.bfloat16, gen, "head")
    ws = sd.new_workspace(256, "cuda")
    sd.sparsed_cache_write(sd.make_cache(k, v, table, i32(lens_all)), k_new, v_new, su.offsets(lens), ws)
    seq = np.repeat(np.arange(len(lens)), lens)
    first = np.cumsum([0] + lens[:-1])
    place = torch.from_numpy(np.array(lens_all)[seq] - np.array(lens)[seq] + np.arange(n) - first[seq]).cuda()
    page = table[torch.from_numpy(seq).cuda(), place // 16].long()
    want_k[page, place % 16], want_v[page, place % 16] = k_new[:n], v_new[:n]
    assert torch.equal(k, want_k) and torch.equal(v, want_v) and su.status(ws) == (0, 0)


def test_write_wide_rows_and_slices():
    """Heads enough that a warp takes a token's row in several turns; K and V as slices of one projection, a head-major pool."""
    heads, gen = 21, su.generator(13)
    fused = torch.randn(50, 3 * heads, 128, generator=gen, device="cuda").half()
    k_new, v_new = fused[:, heads:2 * heads], fused[:, 2 * heads:]
    k, v, table = su.paged_pool([64, 64], 32, heads, torch.float16, gen, layout="head")
    want_k, want_v = k.clone(), v.clone()
    lens, new = [60, 33], [30, 20]
    sd.sparsed_cache_write(sd.make_cache(k, v, table, i32(lens)), k_new, v_new, su.offsets(new), sd.new_workspace(256, "cuda"))
    at = 0
    for b in range(2):
        for i in range(new[b]):
            j = lens[b] - new[b] + i
            want_k[int(table[b, j // 32]), j % 32], want_v[int(table[b, j // 32]), j % 32] = k_new[at], v_new[at]
            at += 1
    assert torch.equal(k, want_k) and torch.equal(v, want_v)


@pytest.mark.parametrize("batch,heads_kv,length", [(1, 1, 100001), (3, 7, 20000), (70, 1, 2100), (70, 1, 2040), (64, 1, 2040), (2, 1, 1000)])
def test_evict_is_the_same_again(batch, heads_kv, length):
    """Rows over one, four and eight CTAs of a cluster, and over CTAs of 1024 and 256 threads: the places by the definition."""
    gen = su.generator(14)
    k, v, table = su.paged_pool([length] * batch, 256, heads_kv, torch.bfloat16, gen)
    mass = torch.rand(batch, heads_kv, table.shape[1] * 256, generator=gen, device="cuda").round(decimals=3)
    check_evict(k, v, table, [length - i for i in range(batch)], mass, length // 3, 100)
