"""Arrays of a one-token call that share memory: refused before any launch where results would depend on the order of threads."""
import ctypes

import pytest

import paper_2509_24014_b200 as sd
from paper_2509_24014_b200 import binding

OK, BYTES = 4096, 3 * 2 * 64 * 4   # the weights of three sequences of two heads with 64 places each


@pytest.mark.parametrize("offset,refused", [(0, False), (4, True), (-4, True), (64 * 4, True), (BYTES - 4, True), (4 - BYTES, True),
                                            (BYTES, False), (-BYTES, False), (3 * BYTES, False)])
def test_weights_in_and_out(offset, refused):
    """The same array and arrays side by side are fine; these fail later, for a workspace that is too small."""
    lib = sd.load_library()
    cache = binding.Cache(k=OK, v=OK, page_table=OK, seq_lens=OK, num_pages=10, page_size=16, heads_kv=2, head_dim=128, batch=3,
                          max_pages=4, dtype=0)
    out = 1 << 20
    got = lib.sparsed_attn_paged(ctypes.byref(cache), 4, OK, None, OK, None, 0.0, None, out + offset, out, 64, OK, 256, None)
    assert got == (1 if refused else 4)
