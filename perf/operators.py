"""What a program that serves prompts of different lengths out of a paged key-value cache asks of this library, as timed
cases with plain forms of the operators beside the calls.

A case's ``op`` names the operator:

* ``packed``  attention of prompts of different lengths packed into one call, causal or bidirectional, grouped heads; with
              ``past`` > 0 the keys of a sequence begin before its queries do (a prompt that continues cached text)
* ``write``   keys and values of new tokens go to their places in the pages of the cache
* ``paged``   attention of one new token per sequence over its cached keys, with or without adding each key's attention
              weight to an accumulated one (``mass``)
* ``evict``   of each sequence and key-value head the keys with the most accumulated weight, and the latest ones, move to
              fewer pages

Lengths of a case's sequences are spread by their logarithm between ``shortest`` and ``longest`` (``mix`` says which spread).
``own`` is False where the operators run in their plain form, and set to True where the library's entry points are called.
"""
from __future__ import annotations

import math
import random

import torch

own = False

HEAD_DIM = 128
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}

# Bounds of a drawn case: what the largest listed one of its operator needs.
MOST_PAIRS = 32 * 32768 * 32768 // 2       # packed: seen (head, row, key) triples
MOST_PACKED_TOKENS = 32768                 # ... and rows
MOST_CACHED = 24 * 32 * 8192               # paged: (kv head, key) pairs
MOST_WRITTEN = 32 * 24576                  # write: (kv head, token) pairs
MOST_KEPT = 2 * 8 * 65536                  # evict: (kv head, key) pairs in the cache


def _case(name, op, dtype, seqs, shortest, longest, heads_q, heads_kv, mix=1, causal=True, past=0, page=64, mass=False,
          keep=0, recent=0):
    return {"name": name, "op": op, "dtype": dtype, "seqs": seqs, "shortest": shortest, "longest": longest,
            "heads_q": heads_q, "heads_kv": heads_kv, "mix": mix, "causal": causal, "past": past, "page": page,
            "mass": mass, "keep": keep, "recent": recent}


def listed():
    return [
        # The last turns of a few short conversations, a single token among them: the smallest call, where latency counts.
        _case("packed_short_turns", "packed", "bf16", 6, 1, 160, 8, 8, mix=2),
        # A batch of Dream-shaped prompts (28 heads on 4) of which some continue cached text.
        _case("packed_dream_prompts", "packed", "bf16", 12, 150, 4000, 28, 4, mix=5, past=4096),
        # A denoising batch of LLaDA-shaped requests of different lengths: no mask but the sequences' ends.
        _case("packed_denoise_batch", "packed", "fp16", 8, 500, 4096, 32, 32, mix=15, causal=False),
        # One long document, prefilled in one call: the heaviest one.
        _case("packed_32k_prompt", "packed", "bf16", 1, 32768, 32768, 32, 32, past=0),
        # A generation step of a batch: one new token each ...
        _case("write_one_token_each", "write", "bf16", 64, 1, 1, 4, 4, past=6000, page=64),
        # ... and the keys and values of a batch of prompts.
        _case("write_prompts", "write", "fp16", 12, 100, 4000, 32, 32, mix=5, past=100, page=32),
        # A single conversation's next token: latency again.
        _case("paged_one_chat", "paged", "bf16", 1, 1500, 1500, 28, 4, page=16),
        # A batch of conversations of different lengths whose keys are ranked by their accumulated weight.
        _case("paged_batch_mass", "paged", "bf16", 48, 300, 8000, 28, 4, mix=11, page=64, mass=True),
        # One very long conversation: all the work is along one axis.
        _case("paged_128k", "paged", "fp16", 1, 131072, 131072, 32, 8, page=256),
        # A LLaDA-shaped batch with a head of keys for every query head: the most bytes.
        _case("paged_batch_32_heads", "paged", "bf16", 24, 6000, 8192, 32, 32, mix=2, page=128),
        # Conversations that outgrew their share of the cache are cut back to it ...
        _case("evict_batch", "evict", "bf16", 8, 1500, 4608, 28, 4, mix=13, page=64, keep=2048, recent=256),
        # ... and a long document's cache to a quarter.
        _case("evict_long", "evict", "fp16", 2, 50000, 65536, 32, 8, mix=4, page=128, keep=16384, recent=1024),
    ]


def _spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    while True:
        op = rng.choice(["packed", "packed", "write", "paged", "paged", "evict"])
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        heads_q, heads_kv = rng.choice([(2, 2), (8, 8), (12, 1), (16, 4), (28, 4), (32, 8), (32, 32), (40, 2)])
        longest = _spread(rng, 16, {"packed": 16384, "write": 8192, "paged": 65536, "evict": 32768}[op])
        shortest = max(1, _spread(rng, max(1, longest // 16), longest))
        seqs = _spread(rng, 1, 64)
        past = _spread(rng, 1, 8192) if op == "write" or op == "packed" and rng.random() < 0.4 else 0
        case = _case("", op, dtype, seqs, shortest, longest, heads_q, heads_kv, mix=rng.randrange(1000),
                     causal=rng.random() < 0.6, past=past, page=rng.choice([16, 32, 64, 128, 256]),
                     mass=op == "paged" and rng.random() < 0.4)
        if op == "evict":
            case["keep"] = max(2, int(longest * rng.uniform(0.1, 0.9)))
            case["recent"] = int(case["keep"] * rng.uniform(0.0, 0.5))
        new, total = _lengths(case)
        if op == "packed":
            fits = (sum(new) <= MOST_PACKED_TOKENS and sum(total) <= 4 * MOST_PACKED_TOKENS
                    and heads_q * _pairs(case) <= MOST_PAIRS)
        elif op == "write":
            fits = sum(new) * heads_kv <= MOST_WRITTEN and seqs * (past + longest) * heads_kv <= 4 * MOST_WRITTEN
        else:
            fits = seqs * longest * heads_kv <= (MOST_CACHED if op == "paged" else MOST_KEPT)
        if fits:
            del case["name"]
            return case


def _lengths(case):
    """New tokens of each sequence, and the tokens it has in all."""
    rng = random.Random(case["mix"])
    new = [_spread(rng, case["shortest"], case["longest"]) for _ in range(case["seqs"])]
    # a call's past: none for every third sequence, up to all of it for the others
    past = [0 if i % 3 == 2 else int(case["past"] * rng.random()) for i in range(case["seqs"])]
    return new, [n + p for n, p in zip(new, past)]


def _pairs(case):
    """Seen (row, key) pairs of a packed call, one head's."""
    new, total = _lengths(case)
    if not case["causal"]:
        return sum(n * t for n, t in zip(new, total))
    return sum(n * t - n * (n - 1) // 2 for n, t in zip(new, total))


def _offsets(lengths, device):
    at = [0]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=device)


def _pages(lengths, page, gen, extra=0):
    """A table of pages in no order, -1 behind a sequence's last page, and how many pages the pool has."""
    count = [-(-n // page) for n in lengths]
    pool = sum(count) + extra
    order = torch.randperm(pool, generator=gen, device=gen.device).int()
    table = torch.full((len(lengths), max(count)), -1, dtype=torch.int32, device=gen.device)
    owner = torch.repeat_interleave(torch.arange(len(lengths), device=gen.device),
                                    torch.tensor(count, device=gen.device))
    nth = torch.cat([torch.arange(c, device=gen.device) for c in count])
    table[owner, nth] = order[:len(owner)]
    return table, pool


def _queries_keys(rows_q, rows_k, heads_q, heads_kv, dtype, gen):
    """Queries and keys of unit scale; every head has a direction that all its queries share and that one key in 64 has
    too, so that a few keys get much of the weight, as sinks and anchors do."""
    dev = gen.device
    q = torch.randn(rows_q, heads_q, HEAD_DIM, generator=gen, device=dev)
    k = torch.randn(rows_k, heads_kv, HEAD_DIM, generator=gen, device=dev)
    u = torch.randn(heads_kv, HEAD_DIM, generator=gen, device=dev)
    u = u / u.norm(dim=-1, keepdim=True)
    q += 5.0 * u.repeat_interleave(heads_q // heads_kv, dim=0)
    strong = torch.rand(rows_k, heads_kv, 1, generator=gen, device=dev) < 1 / 64
    k += strong * (9.0 * u)
    return q.to(dtype), k.to(dtype)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 7919 + 17)
    dev, dtype = gen.device, TYPES[case["dtype"]]
    hq, hkv, op = case["heads_q"], case["heads_kv"], case["op"]
    new, total = _lengths(case)
    s = {"op": op, "new": new, "total": total, "causal": case["causal"], "heads_kv": hkv}
    if op == "packed":
        # room for more rows than the batch has, as a program's fixed buffers have
        rows_q, rows_k = sum(new) + 7, sum(total) + 7
        s["q"], s["k"] = _queries_keys(rows_q, rows_k, hq, hkv, dtype, gen)
        s["v"] = torch.randn(rows_k, hkv, HEAD_DIM, generator=gen, device=dev).to(dtype)
        for t, used in ((s["q"], sum(new)), (s["k"], sum(total)), (s["v"], sum(total))):
            t[used:] = float("nan")     # nothing has been written there yet
        s["cu_q"], s["cu_k"] = _offsets(new, dev), _offsets(total, dev)
        s["o"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(hq, rows_q, dtype=torch.float32, device=dev)
    elif op == "write":
        s["table"], pool = _pages(total, case["page"], gen, extra=3)
        s["lens"] = torch.tensor(total, dtype=torch.int32, device=dev)
        s["cu"] = _offsets(new, dev)
        s["k_new"], s["v_new"] = (torch.randn(sum(new), hkv, HEAD_DIM, generator=gen, device=dev).to(dtype) for _ in "kv")
        s["k"], s["v"] = (torch.randn(pool, case["page"], hkv, HEAD_DIM, generator=gen, device=dev, dtype=dtype)
                          for _ in "kv")
    elif op == "paged":
        n, page = case["seqs"], case["page"]
        s["table"], pool = _pages(total, page, gen, extra=2)
        s["lens"] = torch.tensor(total, dtype=torch.int32, device=dev)
        s["q"], k = _queries_keys(n, pool * page, hq, hkv, dtype, gen)
        s["k"] = k.view(pool, page, hkv, HEAD_DIM)
        s["v"] = torch.randn(pool, page, hkv, HEAD_DIM, generator=gen, device=dev, dtype=dtype)
        used = torch.zeros(pool, page, dtype=torch.bool, device=dev)
        at = torch.arange(s["table"].shape[1] * page, device=dev)
        b, j = torch.nonzero(at < s["lens"][:, None], as_tuple=True)
        used[s["table"][b, j // page].long(), j % page] = True
        s["k"][~used] = float("nan")    # pages that nobody has and the ends of last pages: nothing written yet
        s["v"][~used] = float("nan")
        s["o"] = torch.zeros_like(s["q"])
        s["mass_in"] = s["mass_out"] = None
        if case["mass"]:
            s["mass_in"] = torch.rand(n, hkv, s["table"].shape[1] * page, generator=gen, device=dev) ** 4
            s["mass_out"] = torch.zeros_like(s["mass_in"])
    else:
        n, page, keep = case["seqs"], case["page"], case["keep"]
        s["keep"], s["recent"] = keep, case["recent"]
        s["table"], pool = _pages(total, page, gen, extra=2)
        s["lens"] = torch.tensor(total, dtype=torch.int32, device=dev)
        s["k"], s["v"] = (torch.randn(pool, page, hkv, HEAD_DIM, generator=gen, device=dev, dtype=dtype) for _ in "kv")
        # accumulated weights: a few large, most small, and many equal (a key that no query ever looked at has none)
        s["mass"] = torch.rand(n, hkv, s["table"].shape[1] * page, generator=gen, device=dev) ** 12
        s["mass"][s["mass"] < 1e-4] = 0.0
        s["new_table"], new_pool = _pages([min(keep, t) for t in total], page, gen, extra=1)
        s["new_k"], s["new_v"] = (torch.zeros(new_pool, page, hkv, HEAD_DIM, dtype=dtype, device=dev) for _ in "kv")
        s["new_lens"] = torch.zeros(n, dtype=torch.int32, device=dev)
        s["new_mass"] = torch.zeros(n, hkv, s["new_table"].shape[1] * page, device=dev)
        s["kept"] = torch.zeros(n, hkv, keep, dtype=torch.int32, device=dev)
    if own:
        import paper_2509_24014_b200 as sd
        s["sd"] = sd
        if op == "packed":
            s["ws"] = sd.new_workspace(sd.sparsed_workspace_bytes(sd.OP_ATTN_PACKED), dev)
        else:
            s["cache"] = sd.make_cache(s["k"], s["v"], s["table"], s["lens"])
            if op == "write":
                s["ws"] = sd.new_workspace(sd.sparsed_workspace_bytes(sd.OP_CACHE_WRITE), dev)
            elif op == "paged":
                s["ws"] = sd.new_workspace(sd.sparsed_paged_workspace_bytes(s["cache"], hq, with_mass=case["mass"]), dev)
            else:
                s["new_cache"] = sd.make_cache(s["new_k"], s["new_v"], s["new_table"], s["new_lens"])
                s["ws"] = sd.new_workspace(sd.sparsed_evict_workspace_bytes(s["cache"]), dev)
    return s


# ---------------------------------------------------------------------------------------------- the library's calls
def _own_packed(s):
    s["sd"].sparsed_attn_packed(s["q"], s["k"], s["v"], s["o"], s["cu_q"], s["cu_k"], s["ws"], causal=s["causal"],
                                lse=s["lse"])
    return {"o": s["o"], "lse": s["lse"]}


def _own_write(s):
    s["sd"].sparsed_cache_write(s["cache"], s["k_new"], s["v_new"], s["cu"], s["ws"])
    return {"k": s["k"], "v": s["v"]}


def _own_paged(s):
    s["sd"].sparsed_attn_paged(s["q"], s["cache"], s["o"], s["ws"], mass_in=s["mass_in"], mass_out=s["mass_out"])
    return {"o": s["o"]} if s["mass_out"] is None else {"o": s["o"], "mass": s["mass_out"]}


def _own_evict(s):
    s["sd"].sparsed_cache_evict(s["cache"], s["mass"], s["keep"], s["recent"], s["new_cache"], s["new_mass"], s["kept"],
                                s["ws"])
    return {"kept": s["kept"], "lens": s["new_lens"], "k": s["new_k"], "v": s["new_v"], "mass": s["new_mass"]}


# ---------------------------------------------------------------------------------------------- plain forms
def _plain_packed(s):
    q, k, v, o, lse, hkv = s["q"], s["k"], s["v"], s["o"], s["lse"], s["heads_kv"]
    group, first_q, first_k = q.shape[1] // hkv, 0, 0
    for n, t in zip(s["new"], s["total"]):
        keys = k[first_k:first_k + t].float().permute(1, 2, 0)                                   # [hkv, d, t]
        values = v[first_k:first_k + t].float().transpose(0, 1)                                  # [hkv, t, d]
        seen_of = torch.arange(t - n, t, device=q.device)                                        # last key a row sees
        step = max(1, (1 << 30) // (q.shape[1] * t))
        for a in range(0, n, step):                                                              # (as memory allows)
            b = min(n, a + step)
            rows = q[first_q + a:first_q + b].float().transpose(0, 1).reshape(hkv, group * (b - a), HEAD_DIM)
            x = torch.matmul(rows, keys).div_(math.sqrt(HEAD_DIM)).view(hkv, group, b - a, t)
            if s["causal"]:
                x.masked_fill_(torch.arange(t, device=q.device) > seen_of[a:b, None], -math.inf)
            top = x.amax(dim=-1, keepdim=True)
            p = x.sub_(top).exp_()
            total = p.sum(dim=-1, keepdim=True)
            out = torch.matmul(p.view(hkv, group * (b - a), t), values).view(hkv * group, b - a, HEAD_DIM)
            out = out / total.view(hkv * group, b - a, 1)
            o[first_q + a:first_q + b] = out.transpose(0, 1).to(o.dtype)
            lse[:, first_q + a:first_q + b] = (top + total.log()).view(hkv * group, b - a)
        first_q, first_k = first_q + n, first_k + t
    return {"o": o, "lse": lse}


def _plain_write(s):
    page, cu, lens = s["k"].shape[1], s["cu"].long(), s["lens"].long()
    token = torch.arange(s["k_new"].shape[0], device=cu.device)
    seq = torch.searchsorted(cu, token, right=True) - 1
    place = lens[seq] - cu[seq + 1] + token
    at = (s["table"][seq, place // page].long(), place % page)
    s["k"][at] = s["k_new"]
    s["v"][at] = s["v_new"]
    return {"k": s["k"], "v": s["v"]}


def _plain_paged(s):
    n, hkv, page = s["q"].shape[0], s["heads_kv"], s["k"].shape[1]
    table = s["table"].long().clamp(min=0)
    length = table.shape[1] * page
    seen = torch.arange(length, device=table.device) < s["lens"][:, None]                        # [n, length]
    keys = s["k"][table].view(n, length, hkv, HEAD_DIM).permute(0, 2, 3, 1).float()              # [n, hkv, d, length]
    x = torch.matmul(s["q"].float().view(n, hkv, -1, HEAD_DIM), keys) / math.sqrt(HEAD_DIM)
    del keys
    x = torch.where(seen[:, None, None], x, -math.inf)
    p = (x - x.amax(dim=-1, keepdim=True)).exp()
    p = p / p.sum(dim=-1, keepdim=True)
    values = s["v"][table].view(n, length, hkv, HEAD_DIM).permute(0, 2, 1, 3).float()
    values = torch.where(seen[:, None, :, None], values, 0.0)
    s["o"].copy_(torch.matmul(p, values).view(n, -1, HEAD_DIM))
    if s["mass_out"] is None:
        return {"o": s["o"]}
    s["mass_out"].copy_(torch.where(seen[:, None], s["mass_in"] + p.sum(dim=2), s["mass_out"]))
    return {"o": s["o"], "mass": s["mass_out"]}


def _plain_evict(s):
    keep, page, new_page = s["keep"], s["k"].shape[1], s["new_k"].shape[1]
    n, hkv, length = s["mass"].shape
    at, lens = torch.arange(length, device=s["mass"].device), s["lens"].long()[:, None, None]
    rank = torch.where(at >= lens - s["recent"], math.inf, s["mass"])
    rank = torch.where(at < lens, rank, -math.inf)
    first = torch.sort(rank, dim=-1, descending=True, stable=True).indices[..., :keep]
    if first.shape[-1] < keep:                                                                   # a cache shorter than that
        first = torch.nn.functional.pad(first, (0, keep - first.shape[-1]), value=length)
    kept = torch.where(first < lens, first, length).sort(dim=-1).values                          # the others go last
    b, h, j = torch.nonzero(kept < length, as_tuple=True)
    src = kept[b, h, j]
    read = (s["table"][b, src // page].long(), src % page, h)
    write = (s["new_table"][b, j // new_page].long(), j % new_page, h)
    s["new_k"][write] = s["k"][read]
    s["new_v"][write] = s["v"][read]
    s["new_mass"].zero_()
    s["new_mass"][b, h, j] = s["mass"][b, h, src]
    s["kept"].copy_(torch.where(kept < length, kept, -1))
    s["new_lens"].copy_(s["lens"].clamp(max=keep))
    return {"kept": s["kept"], "lens": s["new_lens"], "k": s["new_k"], "v": s["new_v"], "mass": s["new_mass"]}


def run(state):
    calls = {"packed": (_plain_packed, _own_packed), "write": (_plain_write, _own_write),
             "paged": (_plain_paged, _own_paged), "evict": (_plain_evict, _own_evict)}
    return calls[state["op"]][1 if own else 0](state)


# ---------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """What run() returns, in 64 bits from the definitions, one head of one sequence after the other. The write and the
    eviction compute no numbers: what they give are copies and places."""
    if case["op"] in ("write", "evict"):
        return None
    s = prepare(case, seed)
    new, total = _lengths(case)
    hq, hkv = case["heads_q"], case["heads_kv"]
    q, group, scale = s["q"], hq // hkv, HEAD_DIM ** -0.5
    o = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    if case["op"] == "packed":
        lse = torch.zeros(hq, q.shape[0], dtype=torch.float64, device=q.device)
        cu_q, cu_k = s["cu_q"].tolist(), s["cu_k"].tolist()
        for b in range(case["seqs"]):
            for h in range(hq):
                kh = s["k"][cu_k[b]:cu_k[b + 1], h // group].double()
                vh = s["v"][cu_k[b]:cu_k[b + 1], h // group].double()
                step = max(1, (1 << 26) // total[b])
                for lo in range(cu_q[b], cu_q[b + 1], step):
                    hi = min(lo + step, cu_q[b + 1])
                    x = (q[lo:hi, h].double() * scale) @ kh.t()
                    if case["causal"]:
                        last = torch.arange(lo, hi, device=q.device) - cu_q[b + 1] + total[b]
                        x = x.where(torch.arange(total[b], device=q.device) <= last[:, None], -math.inf)
                    lse[h, lo:hi] = torch.logsumexp(x, dim=-1)
                    o[lo:hi, h] = torch.exp(x - lse[h, lo:hi, None]) @ vh
        return {"o": o, "lse": lse}
    mass = s["mass_out"].double() if case["mass"] else None
    for b in range(case["seqs"]):
        pages = s["table"][b, :-(-total[b] // case["page"])].long()
        kb = s["k"][pages].flatten(0, 1)[:total[b]].double()
        vb = s["v"][pages].flatten(0, 1)[:total[b]].double()
        for g in range(hkv):
            w = torch.softmax((q[b, g * group:(g + 1) * group].double() * scale) @ kb[:, g].t(), dim=-1)
            o[b, g * group:(g + 1) * group] = w @ vb[:, g]
            if mass is not None:
                mass[b, g, :total[b]] = s["mass_in"][b, g, :total[b]].double() + w.sum(dim=0)
    return {"o": o} if mass is None else {"o": o, "mass": mass}


def work(case):
    hq, hkv, op = case["heads_q"], case["heads_kv"], case["op"]
    new, total = _lengths(case)
    row = 2 * HEAD_DIM
    if op == "packed":
        return {"bytes": 2 * row * hq * sum(new) + 2 * row * hkv * sum(total) + 4 * hq * sum(new),
                "flops": 4 * HEAD_DIM * hq * _pairs(case)}
    if op == "write":
        return {"bytes": 4 * row * hkv * sum(new), "flops": 0}
    if op == "paged":
        return {"bytes": 2 * row * hkv * sum(total) + 2 * row * hq * case["seqs"]
                + (8 * hkv * sum(total) if case["mass"] else 0), "flops": 4 * HEAD_DIM * hq * sum(total)}
    kept = sum(min(case["keep"], t) for t in total)
    return {"bytes": 4 * hkv * sum(total) + hkv * kept * (4 * row + 4 + 4), "flops": 0}
