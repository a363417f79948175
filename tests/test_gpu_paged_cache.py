"""The paged key-value cache: writing, attention of one token per sequence, eviction, and a run of them together."""
import numpy as np
import pytest
import torch

import paper_2509_24014_b200 as sd
from oracle import packed_and_paged as orc
from tests import serving_util as su

pytestmark = pytest.mark.gpu
F32 = torch.float32


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ writing
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("page_size", [16, 64, 256])
@pytest.mark.parametrize("new,past,heads_kv,layout", [([1], [0], 1, "place"), ([1, 1, 1], [15, 16, 17], 2, "place"),
                                                      ([0, 5, 0, 70, 0], [3, 9, 0, 100, 1], 3, "head"),
                                                      ([300, 2], [0, 500], 9, "place"), ([1] * 70, [7] * 70, 4, "head")])
def test_write(new, past, heads_kv, layout, page_size, dtype):
    gen, total = su.generator(len(new)), [n + p for n, p in zip(new, past)]
    k, v, table = su.paged_pool(total, page_size, heads_kv, su.DTYPES[dtype], gen, layout)
    lens, cu = i32(total), su.offsets(new)
    k_new = su.rows(sum(new) + 2, heads_kv, su.DTYPES[dtype], gen, "fused")
    v_new = su.rows(sum(new) + 2, heads_kv, su.DTYPES[dtype], gen, "head")
    want_k, want_v = k.clone(), v.clone()
    for b in range(len(new)):
        for i in range(new[b]):
            j = past[b] + i
            want_k[int(table[b, j // page_size]), j % page_size] = k_new[int(cu[b]) + i]
            want_v[int(table[b, j // page_size]), j % page_size] = v_new[int(cu[b]) + i]
    ws = sd.new_workspace(sd.sparsed_workspace_bytes(sd.OP_CACHE_WRITE), "cuda")
    sd.sparsed_cache_write(sd.make_cache(k, v, table, lens), k_new, v_new, cu, ws)
    torch.cuda.synchronize()
    assert su.status(ws) == (0, 0)
    assert torch.equal(k, want_k) and torch.equal(v, want_v)


def test_write_where_there_is_no_place():
    """Positions below zero, beyond the table, or of a page that does not exist are skipped and reported."""
    gen = su.generator(1)
    k, v, table = su.paged_pool([40, 40, 40], 16, 2, torch.bfloat16, gen)
    table[1, 2] = 1000
    before_k, before_v = k.clone(), v.clone()
    k_new, v_new = (su.rows(9, 2, torch.bfloat16, gen) for _ in "kv")
    for lens in ([2, 40, 40], [40, 40, 50], [-7, 40, 40]):
        ws = sd.new_workspace(256, "cuda")
        k.copy_(before_k)
        sd.sparsed_cache_write(sd.make_cache(k, v, table, i32(lens)), k_new, v_new, su.offsets([3, 3, 3]), ws)
        torch.cuda.synchronize()
        assert su.status(ws)[0] == 5
        want = before_k.clone()
        for b in range(3):
            for i in range(3):
                j = max(lens[b], 0) - 3 + i
                if 0 <= j < 48 and 0 <= int(table[b, j // 16]) < k.shape[0]:
                    want[int(table[b, j // 16]), j % 16] = k_new[3 * b + i]
        assert torch.equal(k, want)


# ------------------------------------------------------------------ attention
def attend(q, k, v, table, lens, mass_in=None, with_mass=False, scale=0.0, code=0, in_place=False):
    cache = sd.make_cache(k, v, table, lens)
    o = torch.full_like(q, 7.0)
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    mass_out = None
    if with_mass:
        capacity = table.shape[1] * k.shape[1] + 5 if mass_in is None else mass_in.shape[2]
        mass_out = mass_in.clone() if in_place else torch.full((q.shape[0], k.shape[2], capacity), 7.0, device="cuda")
    ws = sd.new_workspace(sd.sparsed_paged_workspace_bytes(cache, q.shape[1], with_mass), "cuda")
    sd.sparsed_attn_paged(q, cache, o, ws, lse=lse, mass_in=mass_out if in_place else mass_in, mass_out=mass_out, softmax_scale=scale)
    torch.cuda.synchronize()
    assert su.status(ws)[0] == code
    return o, lse, mass_out


def check_paged(q, k, v, table, lens, mass_in=None, with_mass=False, scale=0.0, code=0):
    o, lse, mass = attend(q, k, v, table, i32(lens), mass_in, with_mass, scale, code)
    want_o, want_lse, absolute, spread, want_mass = orc.attn_paged(
        su.to_f64(q), su.to_f64(k), su.to_f64(v), table.cpu().numpy(), lens, None if mass_in is None else su.to_f64(mass_in),
        float(np.float32(scale)) if scale else None)
    v64 = np.where(np.isfinite(su.to_f64(v)), np.abs(su.to_f64(v)), 0.0)
    su.assert_within(su.to_f64(o), want_o, su.output_bound(want_o, absolute, spread, q.dtype, v64.sum(axis=(0, 1)).max()), "O")
    su.assert_within(su.to_f64(lse), want_lse, su.lse_bound(want_lse, spread), "LSE")
    if with_mass:
        heads_kv, group, room = k.shape[2], q.shape[1] // k.shape[2], want_mass.shape[2]
        got = su.to_f64(mass)
        e = su.logit_error(spread).reshape(len(lens), heads_kv, group).max(axis=2)[..., None]
        had = 0.0 if mass_in is None else su.to_f64(mass_in)[:, :, :room]
        for b, n in enumerate(lens):
            n = min(max(n, 0), room)
            assert (got[b, :, n:] == 7.0).all()
            w = want_mass[b, :, :n]
            h = had if mass_in is None else had[b, :, :n]
            # weights: the logit's error and the LSE's (at most as large), 2^-21 of log2, sum and addition rounded
            su.assert_within(got[b, :, :n], w, (2 * e[b] + 2.0 ** -20 * (1 + np.abs(want_lse[b]).max(initial=0.0, where=np.isfinite(want_lse[b])))) * np.abs(w - h)
                             + 2.0 ** -23 * np.abs(w) + 1e-37, "mass")
    return o, lse, mass


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("page_size", [16, 128])
@pytest.mark.parametrize("lens", [[1], [0], [15, 16, 17], [63, 64, 65, 0, 2], [700], [1, 0, 0, 333, 128], [40] * 150])
def test_lengths(lens, page_size, dtype):
    gen = su.generator(sum(lens))
    k, v, table = su.paged_pool(lens, page_size, 2, su.DTYPES[dtype], gen)
    su.poison_unused(k, v, table, lens)
    q = su.rows(len(lens), 4, su.DTYPES[dtype], gen)
    check_paged(q, k, v, table, lens, with_mass=True)


@pytest.mark.parametrize("heads_q,heads_kv", [(1, 1), (3, 3), (7, 1), (28, 4), (8, 1), (9, 1), (32, 2), (40, 2), (17, 1)])
@pytest.mark.parametrize("layout", ["place", "head"])
def test_heads_and_layouts(heads_q, heads_kv, layout):
    lens, gen = [200, 3, 130], su.generator(heads_q)
    k, v, table = su.paged_pool(lens, 32, heads_kv, torch.bfloat16, gen, layout)
    v = v.clone(memory_format=torch.contiguous_format)      # (K and V of different strides)
    q = su.rows(3, heads_q, torch.bfloat16, gen, "fused")
    mass_in = torch.rand(3, heads_kv, table.shape[1] * 32 + 5, generator=gen, device="cuda")
    check_paged(q, k, v, table, lens, mass_in=mass_in, with_mass=True, scale=0.06)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_long_sequences_beside_short_ones(dtype):
    """Sequences that many CTAs share beside ones that share a CTA."""
    lens, gen = [9000, 1, 20, 0, 5000, 64, 64, 129], su.generator(4)
    k, v, table = su.paged_pool(lens, 64, 2, su.DTYPES[dtype], gen)
    su.poison_unused(k, v, table, lens)
    q = su.rows(len(lens), 14, su.DTYPES[dtype], gen, scale=2.0)
    check_paged(q, k, v, table, lens, with_mass=True)


def test_logits_that_keep_outgrowing_the_reference():
    lens, gen = [1500], su.generator(6)
    k, v, table = su.paged_pool(lens, 16, 1, torch.bfloat16, gen, scale=2.0)
    q = su.rows(1, 2, torch.bfloat16, gen, scale=2.0)
    pages = table[0].long()
    flat = k[pages].view(-1, 128)[:1500]
    flat = flat[torch.argsort(flat.float() @ q[0, 0].float())]
    dense = k[pages].view(-1, 128)
    dense[:1500] = flat
    k[pages] = dense.view(len(pages), 16, 1, 128)
    check_paged(q, k, v, table, lens, with_mass=True)


def test_infinities_and_nan_in_cached_places():
    """A cached NaN reaches the heads that read it and no other sequence or head."""
    lens, gen = [100, 100], su.generator(7)
    k, v, table = su.paged_pool(lens, 16, 2, torch.bfloat16, gen)
    q = su.rows(2, 4, torch.bfloat16, gen)
    want, _, _ = attend(q, k, v, table, i32(lens))
    v[int(table[0, 3]), 5, 1, 7] = float("inf")
    k[int(table[1, 2]), 1, 0, 7] = float("nan")
    o, lse, _ = attend(q, k, v, table, i32(lens))
    assert torch.equal(o[0, :2], want[0, :2]) and torch.equal(o[1, 2:], want[1, 2:])
    assert (o[0, 2:, 7] == float("inf")).all() and o[1, :2].isnan().all() and lse[1, :2].isnan().all()
    keep = [i for i in range(128) if i != 7]
    assert torch.equal(o[0, 2:][:, keep], want[0, 2:][:, keep])


def test_keys_of_minus_infinity():
    """Keys whose logits are all -inf beside others, and the type's lowest value."""
    lens, gen = [130], su.generator(8)
    k, v, table = su.paged_pool(lens, 16, 1, torch.bfloat16, gen)
    q = su.rows(1, 2, torch.bfloat16, gen).abs()
    q[..., 0] = 1.0
    for j in range(20):
        k[int(table[0, j // 16]), j % 16, 0, 0] = -float("inf")
    for j in range(20, 40):
        k[int(table[0, j // 16]), j % 16, 0] = 0
        k[int(table[0, j // 16]), j % 16, 0, 0] = torch.finfo(torch.bfloat16).min / 8
    o, lse, mass = attend(q, k, v, table, i32(lens), with_mass=True)
    k2 = su.to_f64(k)
    at = orc.positions(table[0].cpu().numpy(), 130, 16, k.shape[0])[40:]
    kk, vv = (np.stack([x[p, s, 0] for _, p, s in at]) for x in (k2, su.to_f64(v)))
    for h in range(2):
        w, l, a, p, s = orc.attend(su.to_f64(q)[0, h][None], kk, vv, np.ones((1, 90), bool))
        su.assert_within(su.to_f64(o)[0, h][None], w, su.output_bound(w, a, s, torch.bfloat16, 0.0), "O")
        su.assert_within(su.to_f64(lse)[0, h][None], l, su.lse_bound(l, s), "LSE")
    assert (mass[0, 0, :40] == 0).all()


def test_pages_that_do_not_exist():
    """Their positions are absent, and reported; so is a length beyond the table."""
    lens, gen = [100, 50, 16], su.generator(9)
    k, v, table = su.paged_pool(lens, 16, 2, torch.bfloat16, gen)
    q = su.rows(3, 4, torch.bfloat16, gen)
    table[0, 2], table[0, 5], table[2, 0] = -1, 10000, k.shape[0]
    check_paged(q, k, v, table, lens, with_mass=True, code=5)     # (sequence 2 has no key left: zeros, -inf)
    table[0, 2], table[0, 5], table[2, 0] = 0, 1, 2
    check_paged(q, k, v, table, [100, 1000, -3], with_mass=True, code=5)


def test_sequences_that_share_pages():
    lens, gen = [200, 200, 90], su.generator(10)
    k, v, table = su.paged_pool(lens, 32, 2, torch.bfloat16, gen)
    table[1, :4] = table[0, :4]
    table[2, :2] = table[0, :2]
    q = su.rows(3, 4, torch.bfloat16, gen)
    check_paged(q, k, v, table, lens, with_mass=True)


def test_mass_in_place_and_table_rows_apart():
    lens, gen = [300, 77], su.generator(11)
    k, v, table = su.paged_pool(lens, 16, 2, torch.bfloat16, gen)
    q = su.rows(2, 14, torch.bfloat16, gen)
    mass_in = torch.rand(2, 2, table.shape[1] * 16, generator=gen, device="cuda")
    wide = torch.full((2, table.shape[1] + 9), -7, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    a = attend(q, k, v, table, i32(lens), mass_in, True)
    b = attend(q, k, v, wide[:, :table.shape[1]], i32(lens), mass_in, True, in_place=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    for s, n in enumerate(lens):
        assert torch.equal(a[2][s, :, :n], b[2][s, :, :n]) and torch.equal(b[2][s, :, n:], mass_in[s, :, n:])


def test_offsets_beyond_32_bits():
    """A pool of more than 2^32 elements: pages at its far end."""
    pages, page_size, heads_kv = 16500, 256, 8
    k = torch.zeros(pages, page_size, heads_kv, 128, dtype=torch.bfloat16, device="cuda")
    assert k.numel() > 1 << 32
    gen = su.generator(12)
    lens, table = [700], i32([[pages - 1, 0, pages - 2]])
    for p in table[0].tolist():
        k[p] = su.rows(page_size, heads_kv, torch.bfloat16, gen)
    q = su.rows(1, heads_kv, torch.bfloat16, gen)
    small = k[table[0].long()].clone()
    a = attend(q, k, k, table, i32(lens))
    b = attend(q, small, small, i32([[0, 1, 2]]), i32(lens))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_written_and_moved_beyond_32_bits():
    """New tokens into pages at the far end of a pool, and an eviction from there to the far end."""
    pages, page_size, heads_kv = 16500, 256, 8
    k = torch.zeros(pages, page_size, heads_kv, 128, dtype=torch.bfloat16, device="cuda")
    v = torch.zeros_like(k)
    gen, ws = su.generator(15), sd.new_workspace(256, "cuda")
    table, new_table = i32([[pages - 1, pages - 4, 2]]), i32([[pages - 2]])
    n = i32([600])
    cache = sd.make_cache(k, v, table, n)
    k_new, v_new = (su.rows(600, heads_kv, torch.bfloat16, gen) for _ in "kv")
    sd.sparsed_cache_write(cache, k_new, v_new, i32([0, 600]), ws)
    for j in (0, 255, 256, 511, 512, 599):
        assert torch.equal(k[table[0, j // 256], j % 256], k_new[j]) and torch.equal(v[table[0, j // 256], j % 256], v_new[j])
    assert int((k != 0).any(-1).any(-1).sum()) == 600
    mass = torch.rand(1, heads_kv, 768, generator=gen, device="cuda")
    new_lens, new_mass = i32([0]), torch.zeros(1, heads_kv, 256, device="cuda")
    kept = torch.zeros(1, heads_kv, 100, dtype=torch.int32, device="cuda")
    sd.sparsed_cache_evict(cache, mass, 100, 10, sd.make_cache(k, v, new_table, new_lens), new_mass, kept, ws)
    assert su.status(ws) == (0, 0) and new_lens.tolist() == [100]
    for h in range(heads_kv):
        stay = orc.kept_positions(mass[0, h].cpu().numpy(), 600, 100, 10)
        assert kept[0, h].tolist() == list(stay)
        assert torch.equal(k[pages - 2, :100, h], k_new[stay, h]) and torch.equal(v[pages - 2, :100, h], v_new[stay, h])


def test_graph_replays_read_the_lengths_of_the_moment():
    lens, gen = [200, 900], su.generator(13)
    k, v, table = su.paged_pool([1000, 1000], 64, 2, torch.bfloat16, gen)
    q = su.rows(2, 14, torch.bfloat16, gen)
    n = i32(lens)
    cache = sd.make_cache(k, v, table, n)
    mass = torch.zeros(2, 2, table.shape[1] * 64, device="cuda")
    o = torch.zeros_like(q)
    ws = sd.new_workspace(sd.sparsed_paged_workspace_bytes(cache, 14, True), "cuda")
    sd.sparsed_attn_paged(q, cache, o, ws, mass_out=mass)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        sd.sparsed_attn_paged(q, cache, o, ws, mass_out=mass)
    for lens in ([200, 900], [1000, 3], [0, 640], [65, 1000]):
        n.copy_(i32(lens))
        mass.zero_()
        o.zero_()
        graph.replay()
        want = attend(q, k, v, table, i32(lens), with_mass=True)
        assert torch.equal(o, want[0])
        for s in range(2):
            assert torch.equal(mass[s, :, :lens[s]], want[2][s, :, :lens[s]]) and (mass[s, :, lens[s]:] == 0).all()


# ------------------------------------------------------------------ eviction
def evict(k, v, table, lens, mass, keep, recent, new_page_size=None, layout="place", gen=None):
    gen = gen or su.generator(99)
    new_page_size = new_page_size or k.shape[1]
    new_k, new_v, new_table = su.paged_pool([min(keep, max(n, 0)) for n in lens], new_page_size, k.shape[2], k.dtype, gen, layout)
    if new_table.shape[1] * new_page_size < keep:
        more = -(-keep // new_page_size) - new_table.shape[1]
        new_table = torch.nn.functional.pad(new_table, (0, more), value=-1)
    before = (new_k.clone(), new_v.clone())
    n = i32(lens)
    new_lens = torch.full_like(n, 7)
    cache, to = sd.make_cache(k, v, table, n), sd.make_cache(new_k, new_v, new_table, new_lens)
    new_mass = torch.full((len(lens), k.shape[2], new_table.shape[1] * new_page_size), 7.0, device="cuda")
    kept = torch.full((len(lens), k.shape[2], keep), 7, dtype=torch.int32, device="cuda")
    ws = sd.new_workspace(sd.sparsed_evict_workspace_bytes(cache), "cuda")
    sd.sparsed_cache_evict(cache, mass, keep, recent, to, new_mass, kept, ws)
    torch.cuda.synchronize()
    assert su.status(ws) == (0, 0)
    return new_k, new_v, new_table, new_lens, new_mass, kept, before


def check_evict(k, v, table, lens, mass, keep, recent, **kw):
    new_k, new_v, new_table, new_lens, new_mass, kept, before = evict(k, v, table, lens, mass, keep, recent, **kw)
    page, new_page = k.shape[1], new_k.shape[1]
    m, tab, new_tab = mass.cpu().numpy(), table.cpu().numpy(), new_table.cpu().numpy()
    want_k, want_v = before[0].cpu(), before[1].cpu()
    k, v = k.cpu(), v.cpu()
    want_kept = np.full(tuple(kept.shape), -1, np.int32)
    want_mass = np.zeros(tuple(new_mass.shape), np.float32)
    for b, n in enumerate(lens):
        for h in range(k.shape[2]):
            stay = orc.kept_positions(m[b, h], max(n, 0), keep, recent)
            want_kept[b, h, :len(stay)] = stay
            want_mass[b, h, :len(stay)] = m[b, h, stay]
            j, to = np.array(stay, dtype=np.int64), np.arange(len(stay))
            want_k[new_tab[b, to // new_page], to % new_page, h] = k[tab[b, j // page], j % page, h]
            want_v[new_tab[b, to // new_page], to % new_page, h] = v[tab[b, j // page], j % page, h]
    np.testing.assert_array_equal(kept.cpu().numpy(), want_kept)
    np.testing.assert_array_equal(new_mass.cpu().numpy(), want_mass)
    assert new_lens.tolist() == [min(max(n, 0), keep) for n in lens]
    assert torch.equal(new_k.cpu(), want_k) and torch.equal(new_v.cpu(), want_v)


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("lens,keep,recent,page,new_page", [
    ([1, 0, 2], 1, 0, 16, 16), ([100], 100, 10, 16, 16), ([101, 99, 5], 100, 10, 16, 64), ([300, 64, 65, 0], 64, 64, 32, 16),
    ([300, 301], 64, 0, 16, 16), ([1000, 40, 777], 333, 100, 64, 128), ([5000, 4999], 5, 4, 256, 16), ([2100], 2099, 1, 16, 256)])
def test_evict(lens, keep, recent, page, new_page, ties):
    gen = su.generator(keep)
    k, v, table = su.paged_pool(lens, page, 3, torch.bfloat16, gen)
    mass = torch.rand(len(lens), 3, table.shape[1] * page + 3, generator=gen, device="cuda")
    if ties:
        mass = (mass * 4).floor() / 4
        mass[:, 0] = 0.25                                   # all alike: the first ones stay
        mass[:, 1, ::3] = float("nan")
        mass[:, 1, 1::3] = float("-0.0")
        mass[:, 1, 2::6] = 0.0
        mass[:, 2, ::7] = float("inf")
        mass[:, 2, 1::7] = -1.5
    check_evict(k, v, table, lens, mass, keep, recent, new_page_size=new_page)


@pytest.mark.parametrize("batch,length,keep,recent", [(1, 70000, 20000, 500), (2, 40000, 39000, 0), (40, 3000, 700, 32), (1, 260000, 100, 10)])
def test_evict_long_rows_and_many(batch, length, keep, recent):
    """Rows that several CTAs share, rows beyond what a CTA holds in shared memory, more rows than CTAs."""
    gen, heads = su.generator(length), 2 if length > 200000 else 4
    lens = [length - 13 * b for b in range(batch)]
    k, v, table = su.paged_pool(lens, 128, heads, torch.float16, gen)
    mass = torch.rand(batch, heads, table.shape[1] * 128, generator=gen, device="cuda") ** 12
    mass[mass < 1e-3] = 0.0
    check_evict(k, v, table, lens, mass, keep, recent, layout="head")


def test_evict_within_one_pool():
    """Old and new pages of the same pool."""
    lens, gen = [200], su.generator(3)
    k, v, table = su.paged_pool(lens, 16, 2, torch.bfloat16, gen, extra=10)
    used = set(table[0].tolist())
    free = [p for p in range(k.shape[0]) if p not in used][:5]
    mass = torch.rand(1, 2, table.shape[1] * 16, generator=gen, device="cuda")
    k0 = k.clone()
    new_lens, kept = i32([0]), torch.zeros(1, 2, 70, dtype=torch.int32, device="cuda")
    new_mass = torch.zeros(1, 2, 80, device="cuda")
    cache, to = sd.make_cache(k, v, table, i32(lens)), sd.make_cache(k, v, i32([free]), new_lens)
    sd.sparsed_cache_evict(cache, mass, 70, 7, to, new_mass, kept, sd.new_workspace(256, "cuda"))
    for h in range(2):
        stay = orc.kept_positions(mass[0, h].cpu().numpy(), 200, 70, 7)
        assert kept[0, h].tolist() == stay
        for at, j in enumerate(stay):
            assert torch.equal(k[free[at // 16], at % 16, h], k0[int(table[0, j // 16]), j % 16, h])
    assert new_lens.tolist() == [70]


@pytest.mark.parametrize("keep,recent", [(33, 0), (40, 40), (5000, 1), (100000, 99999)])
def test_evict_with_nothing_to_evict(keep, recent):
    """More may stay than there is room for: all keys move, to as many places as the cache itself has."""
    lens, gen = [5, 32, 0, 17], su.generator(keep)
    k, v, table = su.paged_pool(lens, 16, 2, torch.bfloat16, gen)
    assert table.shape[1] * 16 == 32
    mass = torch.rand(4, 2, 32, generator=gen, device="cuda")
    new_k, new_v = torch.zeros_like(k), torch.zeros_like(v)
    new_lens, kept = i32([-1] * 4), torch.zeros(4, 2, keep, dtype=torch.int32, device="cuda")
    new_mass = torch.full((4, 2, 32), -1.0, device="cuda")
    new_table = i32([[2 * b, 2 * b + 1] for b in range(4)])
    if new_k.shape[0] < 8:
        new_k, new_v = (torch.zeros(8, *k.shape[1:], dtype=k.dtype, device="cuda") for _ in "kv")
    ws = sd.new_workspace(256, "cuda")
    sd.sparsed_cache_evict(sd.make_cache(k, v, table, i32(lens)), mass, keep, recent, sd.make_cache(new_k, new_v, new_table, new_lens),
                           new_mass, kept, ws)
    assert su.status(ws)[0] == 0 and new_lens.tolist() == lens
    for b, n in enumerate(lens):
        for h in range(2):
            assert kept[b, h, :n].tolist() == list(range(n)) and (kept[b, h, n:] == -1).all()
            assert torch.equal(new_mass[b, h, :n], mass[b, h, :n]) and (new_mass[b, h, n:] == 0).all()
        for j in range(n):
            assert torch.equal(new_k[2 * b + j // 16, j % 16], k[int(table[b, j // 16]), j % 16])
            assert torch.equal(new_v[2 * b + j // 16, j % 16], v[int(table[b, j // 16]), j % 16])


def test_evict_pages_that_do_not_exist():
    lens, gen = [100], su.generator(4)
    k, v, table = su.paged_pool(lens, 16, 1, torch.bfloat16, gen)
    table[0, 1] = 999
    new_k, new_v = torch.full((4, 16, 1, 128), 3.0, dtype=torch.bfloat16, device="cuda"), torch.zeros(4, 16, 1, 128, dtype=torch.bfloat16, device="cuda")
    mass = torch.zeros(1, 1, table.shape[1] * 16, device="cuda")
    mass[0, 0, 16:32] = 1.0
    kept, new_mass, ws = torch.zeros(1, 1, 32, dtype=torch.int32, device="cuda"), torch.zeros(1, 1, 32, device="cuda"), sd.new_workspace(256, "cuda")
    to = sd.make_cache(new_k, new_v, i32([[2, -1]]), i32([0]))
    sd.sparsed_cache_evict(sd.make_cache(k, v, table, i32(lens)), mass, 32, 0, to, new_mass, kept, ws)
    torch.cuda.synchronize()
    assert su.status(ws)[0] == 5
    assert kept[0, 0].tolist() == list(range(32))
    assert torch.equal(new_k[2], k[int(table[0, 0])]) and (new_k[[0, 1, 3]] == 3.0).all()


# ------------------------------------------------------------------ together
def test_prompts_then_tokens_then_an_eviction():
    """What a server does: prompts of different lengths through the packed call and into the cache, some tokens with the keys'
    weights added up, an eviction, more tokens. Every step against the definition on a plain copy of the cache."""
    gen, heads_q, heads_kv, page = su.generator(20), 8, 2, 16
    lens, room, keep = [45, 130, 1], 160, 64
    pages = room // page
    k_pool, v_pool = (torch.full((3 * pages, page, heads_kv, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    table = torch.randperm(3 * pages, generator=gen, device="cuda").int().view(3, pages)
    n = i32(lens)
    cache = sd.make_cache(k_pool, v_pool, table, n)
    ws = sd.new_workspace(sd.sparsed_paged_workspace_bytes(cache, heads_q, True), "cuda")
    q, = (su.rows(sum(lens), heads_q, torch.bfloat16, gen) for _ in "q")
    k, v = (su.rows(sum(lens), heads_kv, torch.bfloat16, gen) for _ in "kv")
    cu, o = su.offsets(lens), torch.zeros_like(q)
    sd.sparsed_attn_packed(q, k, v, o, cu, cu, ws, causal=True)
    sd.sparsed_cache_write(cache, k, v, cu, ws)
    want, _, absolute, spread = orc.attn_packed(su.to_f64(q), su.to_f64(k), su.to_f64(v), cu.tolist(), cu.tolist(), True)
    su.assert_within(su.to_f64(o), want, su.output_bound(want, absolute, spread.T, torch.bfloat16, 0.0), "prompts")
    # plain copies: per sequence and head, lists of keys, values, weights
    ref = [[[su.to_f64(t)[c0:c1, h] for t in (k, v)] + [np.zeros(c1 - c0)] for h in range(heads_kv)]
           for c0, c1 in zip(cu.tolist(), cu.tolist()[1:])]
    mass = torch.zeros(3, heads_kv, room, device="cuda")
    ones = su.offsets([1, 1, 1])

    def token(cache, n, mass):
        q1 = su.rows(3, heads_q, torch.bfloat16, gen)
        k1, v1 = (su.rows(3, heads_kv, torch.bfloat16, gen) for _ in "kv")
        o1 = torch.zeros_like(q1)
        n += 1
        sd.sparsed_cache_write(cache, k1, v1, ones, ws)
        sd.sparsed_attn_paged(q1, cache, o1, ws, mass_in=mass, mass_out=mass)
        torch.cuda.synchronize()
        assert su.status(ws) == (0, 0)
        for b in range(3):
            for h in range(heads_kv):
                r = ref[b][h]
                r[0], r[1] = np.vstack([r[0], su.to_f64(k1)[b, h][None]]), np.vstack([r[1], su.to_f64(v1)[b, h][None]])
                r[2] = np.append(r[2], 0.0)
                rows = slice(h * 4, h * 4 + 4)
                w, _, a, p, s = orc.attend(su.to_f64(q1)[b, rows], r[0], r[1], np.ones((4, len(r[0])), bool))
                su.assert_within(su.to_f64(o1)[b, rows], w, su.output_bound(w, a, s, torch.bfloat16, 0.0), f"token {b} {h}")
                r[2] = r[2] + p.sum(axis=0)
                np.testing.assert_allclose(su.to_f64(mass)[b, h, :len(r[2])], r[2], rtol=1e-4, atol=1e-7)

    for _ in range(6):
        token(cache, n, mass)
    new_pages = 6
    nk, nv = (torch.full((3 * new_pages, page, heads_kv, 128), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in "kv")
    new_n, new_mass = i32([0, 0, 0]), torch.full((3, heads_kv, new_pages * page), 5.0, device="cuda")
    to = sd.make_cache(nk, nv, torch.randperm(3 * new_pages, generator=gen, device="cuda").int().view(3, new_pages), new_n)
    kept = torch.zeros(3, heads_kv, keep, dtype=torch.int32, device="cuda")
    sd.sparsed_cache_evict(cache, mass, keep, 8, to, new_mass, kept, ws)
    assert new_n.tolist() == [51, 64, 7]
    for b in range(3):
        for h in range(heads_kv):
            stay = orc.kept_positions(mass[b, h].cpu().numpy(), int(n[b]), keep, 8)
            assert kept[b, h].tolist() == stay + [-1] * (keep - len(stay))
            ref[b][h] = [x[stay] for x in ref[b][h]]
    for _ in range(5):
        token(to, new_n, new_mass)
    assert new_n.tolist() == [56, 69, 12]
