"""Refusals of the packed and the paged calls, the workspace they ask for and the binding's checks, all before any launch
(there is no GPU here to launch on); the fp64 definitions against torch and hand-worked cases."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2509_24014_b200 as sd
from oracle import packed_and_paged as orc
from paper_2509_24014_b200 import binding

OK, OFF = 4096, 4096 + 4


@pytest.fixture(scope="module")
def lib():
    return sd.load_library()


def packed(**kw):
    f = dict(num_seqs=2, total_q=100, total_k=100, heads_q=4, heads_kv=2, head_dim=128, dtype=0, causal=1)
    f.update(kw)
    return binding.Packed(**f)


def call_packed(lib, shape, cu_q=OK, cu_k=OK, q=OK, k=OK, v=OK, o=OK, lse=None, ws=OK, nbytes=256):
    return lib.sparsed_attn_packed(ctypes.byref(shape), cu_q, cu_k, q, k, v, o, lse, ws, nbytes, None)


def test_packed_refusals(lib):
    bad = [(dict(heads_q=3), 1), (dict(heads_kv=0), 1), (dict(total_q=-1), 1), (dict(num_seqs=-1), 1), (dict(causal=2), 1),
           (dict(head_dim=64), 2), (dict(dtype=2), 2), (dict(softmax_scale=-1.0), 1), (dict(softmax_scale=float("nan")), 1),
           (dict(softmax_scale=float("inf")), 1), (dict(total_q=2 ** 31 - 1, heads_q=2000, heads_kv=2), 2)]
    for kw, status in bad:
        assert call_packed(lib, packed(**kw)) == status, kw
    for name in ("q_strides", "k_strides", "v_strides", "o_strides"):
        for strides, status in (((516, 128), 3), ((512, 132), 3), ((64, 128), 1), ((512, 0), 1), ((512, -128), 1)):
            s = packed()
            getattr(s, name)[0], getattr(s, name)[1] = strides
            assert call_packed(lib, s) == status, (name, strides)
    assert lib.sparsed_attn_packed(None, OK, OK, OK, OK, OK, OK, None, OK, 256, None) == 1
    for name in ("cu_q", "cu_k", "q", "k", "v", "o"):
        assert call_packed(lib, packed(), **{name: None}) == 1, name
    for name in ("q", "k", "v", "o", "ws"):
        assert call_packed(lib, packed(), **{name: OFF}) == 3, name
    for name in ("cu_q", "cu_k", "lse"):
        assert call_packed(lib, packed(), **{name: OK + 2}) == 3, name
    assert call_packed(lib, packed(), nbytes=255) == 4 and call_packed(lib, packed(), ws=None) == 4
    # nothing to do is done without a GPU
    assert call_packed(lib, packed(num_seqs=0)) == 0
    assert call_packed(lib, packed(total_q=0), q=None, o=None) == 0


def cache(**kw):
    f = dict(k=OK, v=OK, page_table=OK, seq_lens=OK, num_pages=10, page_size=16, heads_kv=2, head_dim=128, batch=3, max_pages=4,
             dtype=0)
    f.update(kw)
    return binding.Cache(**f)


BAD_CACHES = [(dict(num_pages=0), 1), (dict(batch=0), 1), (dict(max_pages=0), 1), (dict(heads_kv=0), 1), (dict(head_dim=64), 2),
              (dict(dtype=5), 2), (dict(page_size=8), 2), (dict(page_size=48), 2), (dict(page_size=512), 2),
              (dict(max_pages=2 ** 27), 2), (dict(batch=2 ** 26, heads_kv=2), 2)]
BAD_POINTERS = [(dict(k=None), 1), (dict(page_table=None), 1), (dict(seq_lens=None), 1), (dict(k=OFF), 3), (dict(v=OK + 8), 3),
                (dict(page_table=OK + 1), 3), (dict(seq_lens=OK + 2), 3), (dict(table_stride=-4), 1)]


def bad_stride_caches():
    for name in ("k_strides", "v_strides"):
        for strides, status in (((4096, 256, 100), 1), ((4096, 260, 128), 3), ((0, 256, 128), 1), ((4100, 256, 128), 3)):
            c = cache()
            for i in range(3):
                getattr(c, name)[i] = strides[i]
            yield c, status


def all_bad_caches():
    for kw, status in BAD_CACHES + BAD_POINTERS:
        yield cache(**kw), status
    yield from bad_stride_caches()


def call_write(lib, c, k=OK, v=OK, cu=OK, total=5, ws=OK, nbytes=256, ks=None, vs=None):
    two = ctypes.c_int64 * 2
    return lib.sparsed_cache_write(ctypes.byref(c), k, two(*ks) if ks else None, v, two(*vs) if vs else None, cu, total, ws, nbytes, None)


def test_write_refusals(lib):
    for c, status in all_bad_caches():
        assert call_write(lib, c) == status
    assert call_write(lib, cache(), k=None) == 1 and call_write(lib, cache(), v=None) == 1 and call_write(lib, cache(), cu=None) == 1
    assert call_write(lib, cache(), total=-1) == 1
    assert call_write(lib, cache(), k=OFF) == 3 and call_write(lib, cache(), v=OK + 2) == 3 and call_write(lib, cache(), cu=OK + 2) == 3
    assert call_write(lib, cache(), ks=(100, 128)) == 3 and call_write(lib, cache(), vs=(256, 64)) == 1
    assert call_write(lib, cache(), nbytes=8) == 4 and call_write(lib, cache(), ws=None) == 4 and call_write(lib, cache(), ws=OFF) == 3
    assert call_write(lib, cache(), total=0, k=None, v=None) == 0


def call_paged(lib, c, heads_q=4, q=OK, o=OK, scale=0.0, lse=None, mass_in=None, mass_out=None, capacity=0, ws=OK, nbytes=1 << 30,
               qs=None, os=None):
    two = ctypes.c_int64 * 2
    return lib.sparsed_attn_paged(ctypes.byref(c), heads_q, q, two(*qs) if qs else None, o, two(*os) if os else None, scale, lse,
                                  mass_in, mass_out, capacity, ws, nbytes, None)


def test_paged_refusals(lib):
    for c, status in all_bad_caches():
        assert call_paged(lib, c) == status
    assert call_paged(lib, cache(), heads_q=3) == 1 and call_paged(lib, cache(), heads_q=0) == 1
    assert call_paged(lib, cache(), q=None) == 1 and call_paged(lib, cache(), o=None) == 1
    assert call_paged(lib, cache(), scale=-0.5) == 1 and call_paged(lib, cache(), scale=float("inf")) == 1
    assert call_paged(lib, cache(), qs=(516, 128)) == 3 and call_paged(lib, cache(), os=(512, 8)) == 1
    assert call_paged(lib, cache(), mass_in=OK) == 1                                  # weights in, but none out
    assert call_paged(lib, cache(), mass_out=OK, capacity=63) == 1                    # max_pages * page_size is 64
    for name in ("q", "o"):
        assert call_paged(lib, cache(), **{name: OFF}) == 3
    assert call_paged(lib, cache(), lse=OK + 2) == 3 and call_paged(lib, cache(), mass_out=OK + 1, capacity=64) == 3
    assert call_paged(lib, cache(batch=1 << 20, max_pages=1 << 17), heads_q=64) == 2  # units beyond 32 bits
    need, more = ctypes.c_size_t(), ctypes.c_size_t()
    assert lib.sparsed_paged_workspace_bytes(ctypes.byref(cache()), 4, 0, ctypes.byref(need)) == 0
    assert lib.sparsed_paged_workspace_bytes(ctypes.byref(cache()), 4, 1, ctypes.byref(more)) == 0
    assert more.value == need.value + 3 * 4 * 64 * 4                                  # one logit per query head and place
    for with_mass, bytes_ in ((False, need.value), (True, more.value)):
        kw = dict(mass_out=OK, capacity=64) if with_mass else {}
        assert call_paged(lib, cache(), nbytes=bytes_ - 1, **kw) == 4
        assert call_paged(lib, cache(), nbytes=bytes_, ws=OFF, **kw) == 3             # large enough: refused for its alignment
    assert lib.sparsed_paged_workspace_bytes(ctypes.byref(cache()), 4, 0, None) == 1
    assert lib.sparsed_paged_workspace_bytes(ctypes.byref(cache()), 5, 0, ctypes.byref(need)) == 1
    assert lib.sparsed_paged_workspace_bytes(None, 4, 0, ctypes.byref(need)) == 1


def call_evict(lib, c=None, to=None, mass=OK, capacity=64, keep=20, recent=5, mass_out=OK + 64, out_capacity=20, kept=OK, ws=OK,
               nbytes=256):
    c, to = c or cache(), to or cache(seq_lens=OK + 64)
    return lib.sparsed_cache_evict(ctypes.byref(c), mass, capacity, keep, recent, ctypes.byref(to), mass_out, out_capacity, kept, ws,
                                   nbytes, None)


def test_evict_refusals(lib):
    for c, status in all_bad_caches():
        assert call_evict(lib, c=c) == status
        if c.seq_lens == OK:
            c.seq_lens = OK + 64
        assert call_evict(lib, to=c) == status
    assert call_evict(lib, to=cache()) == 1                                           # writes the lengths it reads
    for kw in (dict(batch=2), dict(heads_kv=1), dict(dtype=1)):
        assert call_evict(lib, to=cache(seq_lens=OK + 64, **kw)) == 1, kw
    for kw in (dict(keep=0), dict(recent=-1), dict(recent=21), dict(keep=65, out_capacity=63), dict(capacity=63),
               dict(out_capacity=19), dict(mass=None), dict(mass_out=None), dict(kept=None), dict(mass_out=OK)):
        assert call_evict(lib, **kw) == 1, kw
    small = cache(seq_lens=OK + 64, page_size=16, max_pages=2)                        # 32 places, of `from` 64
    assert call_evict(lib, to=small, keep=33, out_capacity=100) == 1 and call_evict(lib, to=small, keep=100, out_capacity=100) == 1
    # as many as `from` has places, however many may stay: the next check, of the masses' alignment, refuses these
    assert call_evict(lib, keep=65, out_capacity=64, mass=OK + 2) == 3 and call_evict(lib, to=small, keep=32, out_capacity=32, mass=OK + 2) == 3
    assert call_evict(lib, keep=(1 << 30) + 5, out_capacity=64) == 2
    # arrays that the call writes while others of its CTAs read them: lengths (3 of them), masses (3 x 2 rows)
    for off in (-8, -4, 4, 8):
        assert call_evict(lib, to=cache(seq_lens=OK + off)) == 1, off
    for off in (-6 * 20 * 4 + 4, 4, 6 * 64 * 4 - 4):
        assert call_evict(lib, mass_out=OK + off) == 1, off
    for kw in (dict(mass=OK + 2), dict(mass_out=OK + 1), dict(kept=OK + 2), dict(ws=OFF)):
        assert call_evict(lib, **kw) == 3, kw
    assert call_evict(lib, nbytes=100) == 4 and call_evict(lib, ws=None) == 4
    assert sd.sparsed_evict_workspace_bytes(cache()) == 256


def test_binding_checks():
    cu = torch.zeros(2, dtype=torch.int32)
    ws = torch.zeros(256, dtype=torch.uint8)
    q = torch.zeros(4, 2, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="CUDA"):
        sd.sparsed_attn_packed(q, q, q, q, cu, cu, ws)
    for args in ((q.float(), q, q, q, cu, cu), (q, q.half(), q, q, cu, cu), (q, q, q, q[:2], cu, cu), (q, q, q[:2], q, cu, cu),
                 (q, q, q, q, cu.long(), cu), (q, q, q, q, cu, torch.zeros(3, dtype=torch.int32)),
                 (q.transpose(1, 2).contiguous().transpose(1, 2), q, q, q, cu, cu)):
        with pytest.raises(ValueError):
            sd.sparsed_attn_packed(*args, ws)
    with pytest.raises(ValueError):
        sd.sparsed_attn_packed(q, q, q, q, cu, cu, ws, lse=torch.zeros(4, 2))
    pool, table, lens = torch.zeros(5, 16, 2, 128, dtype=torch.bfloat16), torch.zeros(3, 2, dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    for args in ((pool, pool.half(), table, lens), (pool.float(), pool.float(), table, lens), (pool, pool[:2], table, lens),
                 (pool, pool, table.long(), lens), (pool, pool, table, lens[:2]), (pool[0], pool[0], table, lens),
                 (pool.transpose(2, 3), pool.transpose(2, 3), table, lens), (pool, pool, table.t().contiguous().t(), lens)):
        with pytest.raises(ValueError):
            sd.make_cache(*args)
    c = sd.make_cache(pool, pool, table, lens)
    assert (c.num_pages, c.page_size, c.heads_kv, c.batch, c.max_pages, c.dtype) == (5, 16, 2, 3, 2, 0)
    assert list(c.k_strides) == [4096, 256, 128]
    qb = torch.zeros(3, 4, 128, dtype=torch.bfloat16)
    mass = torch.zeros(3, 2, 32)
    for kw in (dict(q=qb[:2], o=qb[:2]), dict(q=qb.half(), o=qb.half()), dict(mass_in=mass), dict(mass_out=mass.double()),
               dict(mass_out=mass[:, :1]), dict(mass_in=mass[..., :5], mass_out=mass), dict(lse=torch.zeros(4, 3))):
        args = dict(q=qb, o=qb)
        args.update(kw)
        with pytest.raises(ValueError):
            sd.sparsed_attn_paged(args.pop("q"), c, args.pop("o"), ws, **args)
    for kn, cu_ in ((torch.zeros(3, 2, 128), su_cu(3)), (pool[0][:3], su_cu(2)), (pool[0][:3, :1], su_cu(3))):
        with pytest.raises(ValueError):
            sd.sparsed_cache_write(c, kn, kn, cu_, ws)
    to = sd.make_cache(pool, pool, table, lens.clone())
    for kept in (torch.zeros(3, 2, 7, dtype=torch.int32), torch.zeros(3, 2, 8)):
        with pytest.raises(ValueError):
            sd.sparsed_cache_evict(c, mass, 8, 2, to, mass.clone(), kept, ws)


def su_cu(n):
    return torch.zeros(n + 1, dtype=torch.int32)


def test_broadcast_tensors_are_refused():
    """Strides of zero mean contiguous to the library: a tensor that has them would be read beyond its end."""
    cu, ws = torch.tensor([0, 4], dtype=torch.int32), torch.zeros(256, dtype=torch.uint8)
    q, one = torch.zeros(4, 2, 128, dtype=torch.bfloat16), torch.zeros(1, 1, 128, dtype=torch.bfloat16)
    for wide in (one.expand(4, 2, 128), torch.zeros(4, 1, 128, dtype=torch.bfloat16).expand(4, 2, 128),
                 torch.zeros(1, 2, 128, dtype=torch.bfloat16).expand(4, 2, 128)):
        for args in ((wide, q, q, q), (q, wide, q, q), (q, q, wide, q), (q, q, q, wide)):
            with pytest.raises(ValueError, match="broadcast"):
                sd.sparsed_attn_packed(*args, cu, cu, ws)
    pool, lens = torch.zeros(5, 16, 2, 128, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    table = torch.zeros(3, 4, dtype=torch.int32)
    for args in ((torch.zeros(1, 1, 1, 128, dtype=torch.bfloat16).expand(5, 16, 2, 128), pool, table, lens),
                 (pool, pool[:1].expand(5, 16, 2, 128), table, lens), (pool, pool[:, :, :1].expand(5, 16, 2, 128), table, lens),
                 (pool, pool, table[:1].expand(3, 4), lens)):
        with pytest.raises(ValueError, match="broadcast"):
            sd.make_cache(*args)
    cache = sd.make_cache(pool, pool, table, lens)
    q3 = torch.zeros(3, 2, 128, dtype=torch.bfloat16)
    for args in ((one.expand(3, 2, 128), q3), (q3, one.expand(3, 2, 128))):
        with pytest.raises(ValueError, match="broadcast"):
            sd.sparsed_attn_paged(args[0], cache, args[1], ws)
        with pytest.raises(ValueError, match="broadcast"):
            sd.sparsed_cache_write(cache, *args, torch.zeros(4, dtype=torch.int32), ws)
    # one row of everything may have any stride
    c = sd.make_cache(pool[:1].expand(1, 16, 2, 128), pool[:1], table[:1].expand(1, 4), lens[:1])
    assert (c.table_stride, tuple(c.k_strides)) == (0, (16 * 2 * 128, 256, 128))


def test_the_current_device_is_the_tensors(monkeypatch):
    """A call whose tensors are on another device than the current one runs with theirs current, on their stream."""
    entered, called = [], []

    class FakeDevice:
        def __init__(self, device):
            self.device = device

        def __enter__(self):
            entered.append(self.device)

        def __exit__(self, *error):
            entered.append("left")

    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 0, raising=False)
    monkeypatch.setattr(torch.cuda, "device", FakeDevice)

    def function(*args):
        called.append((args, list(entered)))
        return 0

    binding._call(1, "call", function, "a")
    assert called == [(("a", 1001), [1])] and entered == [1, "left"]
    binding._call(0, "call", function, "b")
    assert called[1] == (("b", 1000), [1, "left"]) and len(entered) == 2
    with pytest.raises(sd.SparsedError):
        binding._call(1, "call", lambda *a: 1)
    assert entered[-1] == "left"
    with pytest.raises(ValueError, match="CUDA"):
        binding._call(-1, "call", function)


def test_struct_layouts_match_header():
    assert ctypes.sizeof(binding.Packed) == 8 * 4 + 8 * 8 + 8
    assert ctypes.sizeof(binding.Cache) == 4 * 8 + 8 + 6 * 8 + 7 * 4 + 4


# ------------------------------------------------------------------ the definitions themselves
def test_attend_against_library_attention():
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(9, 128, generator=g, dtype=torch.float64) for _ in "qkv")
    seen = np.tril(np.ones((9, 9), bool))
    o, lse, absolute, w, _ = orc.attend(q.numpy(), k.numpy(), v.numpy(), seen)
    want = torch.nn.functional.scaled_dot_product_attention(q, k, v, attn_mask=torch.from_numpy(seen))
    np.testing.assert_allclose(o, want.numpy(), atol=1e-12)
    np.testing.assert_allclose(w.sum(axis=1), 1.0, atol=1e-12)
    np.testing.assert_allclose(np.exp(lse), (np.exp((q @ k.T).numpy() / np.sqrt(128)) * seen).sum(axis=1), rtol=1e-12)
    k[8], v[8] = float("nan"), float("inf")      # seen by the last row only
    o2, *_ = orc.attend(q.numpy(), k.numpy(), v.numpy(), seen)
    np.testing.assert_array_equal(o2[:8], o[:8])
    assert np.isnan(o2[8]).all()
    none, l0, *_ = orc.attend(q.numpy()[:1], k.numpy(), v.numpy(), np.zeros((1, 9), bool))
    assert (none == 0).all() and l0[0] == -np.inf


def test_causal_rows_are_the_last_tokens():
    """Two queries on four keys: the first sees three of them. Equal logits: means of V."""
    q, k = np.zeros((2, 1, 4)), np.zeros((4, 1, 4))
    v = np.arange(16, dtype=np.float64).reshape(4, 1, 4)
    o, lse, _, _ = orc.attn_packed(q, k, v, [0, 2], [0, 4], True)
    np.testing.assert_allclose(o[0, 0], v[:3, 0].mean(axis=0))
    np.testing.assert_allclose(o[1, 0], v[:, 0].mean(axis=0))
    np.testing.assert_allclose(lse[0], np.log([3.0, 4.0]))


def test_paged_equals_dense_and_weights_sum_to_one():
    rng = np.random.default_rng(0)
    k, v = rng.normal(size=(6, 4, 2, 8)), rng.normal(size=(6, 4, 2, 8))
    q, table = rng.normal(size=(2, 4, 8)), np.array([[3, 0, 5], [1, -1, 2]])
    o, lse, _, _, mass = orc.attn_paged(q, k, v, table, [9, 10])
    flat = k[[3, 0, 5]].reshape(12, 2, 8)[:9], v[[3, 0, 5]].reshape(12, 2, 8)[:9]
    want, *_ = orc.attend(q[0, 2:3], flat[0][:, 1], flat[1][:, 1], np.ones((1, 9), bool))
    np.testing.assert_allclose(o[0, 2], want[0])
    np.testing.assert_allclose(np.nansum(mass[0], axis=1), 2.0)
    np.testing.assert_allclose(np.nansum(mass[1], axis=1), 2.0)
    assert (mass[1, :, 4:8] == 0).all()            # positions of the page that does not exist


def test_kept_positions_by_hand():
    nan = float("nan")
    assert orc.kept_positions([1, 2, 3], 3, 5, 1) == [0, 1, 2]
    assert orc.kept_positions([5, 1, 4, 1, 3], 5, 3, 1) == [0, 2, 4]
    assert orc.kept_positions([1, 1, 1, 1], 4, 2, 0) == [0, 1]
    assert orc.kept_positions([nan, 0.0, -0.0, nan, 2], 5, 3, 0) == [1, 2, 4]
    assert orc.kept_positions([nan, nan, -1, 7], 4, 3, 1) == [0, 2, 3]
    assert orc.kept_positions([9, 8, 7], 3, 2, 2) == [1, 2]
