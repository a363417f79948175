"""Inputs and error bounds for the tests of packed sequences and the paged cache (no method arithmetic here)."""
import numpy as np
import torch

import paper_2509_24014_b200 as sd

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}


def to_f64(t: torch.Tensor) -> np.ndarray:
    return t.detach().to("cpu").to(torch.float64).numpy()


def rounded(dtype):
    """Half a step of the type, relative to the value."""
    return torch.finfo(dtype).eps / 2


def logit_error(spread):
    """Relative error of a probability before it is rounded to 16 bits, against one of exact logits: a logit is an fp32 sum of
    128 products (each addition errs by 2^-24 of at most the sum of magnitudes, `spread`; twice that where the hardware cuts
    off instead of rounding), scaled in one more fp32 operation, less its reference in another (magnitudes up to spread, in
    base 2: a factor 1.45), and the exponential errs by 2^-22."""
    return (2 * 128 + 4) * 2.0 ** -24 * 1.45 * spread + 2.0 ** -21


def output_bound(o, absolute, spread, dtype, v_abs_sum):
    """Largest |error| of an output: every probability is rounded to 16 bits (relative half a step; fp16: below 2^-14 an
    absolute 2^-25 of the row's reference, which the sum of the row is at least) and off by logit_error, the row's sum by
    logit_error, the output itself is rounded once (below the smallest normal number: an absolute half step of it)."""
    u, e = rounded(dtype), logit_error(spread)[..., None]
    tiny = torch.finfo(dtype).tiny * torch.finfo(dtype).eps
    small_p = 2.0 ** -25 * v_abs_sum if dtype == torch.float16 else 0.0
    return 1.01 * ((u + 2 * e) * absolute + u * np.abs(o) + small_p) + tiny


def lse_bound(lse, spread):
    return 2 * logit_error(spread) + 2.0 ** -21 * (1 + np.abs(np.where(np.isfinite(lse), lse, 0.0)))


def assert_within(got, want, bound, what):
    assert got.shape == want.shape, what
    same = (np.isnan(got) & np.isnan(want)) | (got == want)
    with np.errstate(invalid="ignore"):
        off = np.where(same, 0.0, np.abs(got - want))
    bad = ~(off <= bound) & ~same
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} off, first at {tuple(np.argwhere(bad)[0])}: " \
                          f"{got[tuple(np.argwhere(bad)[0])]} for {want[tuple(np.argwhere(bad)[0])]}"


def generator(seed, device="cuda"):
    g = torch.Generator(device=device)
    g.manual_seed(seed)
    return g


def rows(total, heads, dtype, gen, layout="token", scale=1.0):
    """[total, heads, 128] of N(0, scale^2): token-major, head-major (a transposed view), or a slice of a fused projection."""
    dev = gen.device
    if layout == "head":
        return (torch.randn(heads, total, 128, generator=gen, device=dev) * scale).to(dtype).transpose(0, 1)
    if layout == "fused":
        return (torch.randn(total, 3 * heads + 2, 128, generator=gen, device=dev) * scale).to(dtype)[:, 1:1 + heads]
    return (torch.randn(total, heads, 128, generator=gen, device=dev) * scale).to(dtype)


def offsets(lens, device="cuda"):
    return torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device=device)


def paged_pool(lens, page_size, heads_kv, dtype, gen, layout="place", extra=2, scale=1.0):
    """k, v, table of a cache whose pages lie in no order; -1 behind a sequence's last page."""
    dev = gen.device
    count = [-(-max(n, 0) // page_size) for n in lens]
    pool = sum(count) + extra
    order = torch.randperm(pool, generator=gen, device=dev).int()
    table = torch.full((len(lens), max(max(count), 1)), -1, dtype=torch.int32, device=dev)
    at = 0
    for b, c in enumerate(count):
        table[b, :c] = order[at:at + c]
        at += c
    def one():
        if layout == "head":   # [pages, heads, places, 128], as seen place by place
            return (torch.randn(pool, heads_kv, page_size, 128, generator=gen, device=dev) * scale).to(dtype).transpose(1, 2)
        return (torch.randn(pool, page_size, heads_kv, 128, generator=gen, device=dev) * scale).to(dtype)
    return one(), one(), table


def poison_unused(cache_k, cache_v, table, lens):
    """NaN in every place of the pools that no sequence has."""
    page_size = cache_k.shape[1]
    used = torch.zeros(cache_k.shape[:2], dtype=torch.bool)
    t = table.cpu()
    for b, n in enumerate(lens):
        for j in range(n):
            used[t[b, j // page_size], j % page_size] = True
    for pool in (cache_k, cache_v):
        pool[~used.to(pool.device)] = float("nan")


def status(ws):
    return sd.sparsed_last_device_status(ws)
