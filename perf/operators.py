"""What a program does around the hooked attention call in one step of generation, as timed cases: rotating
queries and keys (into the paged cache), sharing, extending and compacting the cache's pages, and penalties,
biases and grammar masks on the logits.

    listed()          the named cases
    draw(rng)         one more case of the same ranges
    prepare(case, s)  inputs and output buffers, from the seed `s` (lengths: from the case's own `lens`)
    run(state)        one pass: elementary torch operations, or with `own` the library's entry points
    work(case)        bytes and operations the pass cannot do without
    exact(case, s)    the same outputs from the definitions, in 64 bits
"""
import math
import random

import torch

own = False

BLOCK = 16
E4M3_MAX = 448.0
E4M3_SIGMAS = 5.0      # an 8-bit cache's scale maps this many standard deviations to the format's largest number
HALVES, PAIRS = 0, 1   # which elements of a head turn together
BLOCKED, CYCLIC = 0, 1  # how the pairs are dealt out to the axes
FULL = 1


def _case(name, op, base, more):
    c = {"name": name, "op": op, "lens": 1}
    c.update(base)
    c.update(more)
    return c


def rope(name, **more):
    return _case(name, "rope", {"tokens": 8, "seqs": 8, "hq": 32, "hkv": 8, "d": 128, "r": 128, "axes": 1, "order": BLOCKED,
                                "pairs": HALVES, "inverse": False, "dtype": "bf16", "cache": True, "kv8": False, "far": 8192}, more)


def fork(name, **more):
    return _case(name, "fork", {"parents": 4, "rows": 16, "lo": 500, "hi": 2000, "table": 512, "prefix": False}, more)


def append(name, **more):
    return _case(name, "append", {"rows": 64, "share": 1, "lo": 500, "hi": 2000, "new_lo": 1, "new_hi": 1, "table": 512,
                                  "caches": 8, "hkv": 8, "d": 128, "dtype": "bf16"}, more)


def compact(name, **more):
    return _case(name, "compact", {"blocks": 512, "live": 0.5, "rows": 16, "caches": 8, "hkv": 8, "d": 128, "dtype": "bf16"}, more)


def logits(name, **more):
    return _case(name, "logits", {"rows": 4, "vocab": 32000, "dtype": "bf16", "lo": 200, "hi": 1000, "bias": 16, "masked": 0.5}, more)


def listed():
    return [
        # a lightly loaded server's decode step: the eight new tokens' heads turned, keys and values stored. Latency only
        rope("rope_few_rows"),
        # a full server's decode step over an 8-bit cache
        rope("rope_many_rows_kv8", tokens=256, seqs=256, kv8=True),
        # prompts with images on a wide model: three axes (time, height, width) dealt out in turn
        rope("rope_image_prompts", tokens=16384, seqs=5, hq=64, axes=3, order=CYCLIC, far=32768),
        # captured queries and keys of a small model turned back before they are compared; half of each head turns
        rope("rope_turned_back", tokens=2048, seqs=1, hq=8, hkv=8, d=64, r=32, pairs=PAIRS, inverse=True, dtype="f32", cache=False),
        # four samples for each of four prompts, and all but one of them dropped again
        fork("fork_few"),
        # a full table: 64 prompts, some of them only shared up to a prefix
        fork("fork_many", parents=64, rows=512, lo=4000, hi=32000, table=2048, prefix=True),
        # a decode step: one token each
        append("append_step"),
        # the first step after a fork: nearly every row copies the page that it shared
        append("append_forked", rows=512, share=8, lo=512, hi=4096, new_hi=4),
        # a small cache tidied up
        compact("compact_few"),
        # a large one after many requests ended
        compact("compact_many", blocks=8192, rows=128),
        # a few samples: latency; full precision and a vocabulary of odd size
        logits("logits_few", vocab=50021, dtype="f32"),
        # a full server's step
        logits("logits_many", rows=256, vocab=131072, lo=500, hi=8000),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "rope", "fork", "append", "compact", "logits", "logits"])
    lens = rng.randrange(1 << 20)
    if op == "rope":
        d = rng.choice([64, 128, 128, 80])
        r = rng.choice([d, d, d // 2, 2 * rng.randint(1, d // 2)])
        hq, hkv = rng.choice([(32, 8), (64, 8), (8, 8), (8, 1), (14, 2), (1, 1)])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        cache = rng.random() < 0.7
        kv8 = cache and dtype == "bf16" and rng.random() < 0.4
        tokens = _log(rng, 1, 12000 if dtype == "bf16" else 6000)
        c = rope("", tokens=tokens, seqs=tokens if tokens < 300 and rng.random() < 0.6 else rng.randint(1, min(tokens, 9)), hq=hq, hkv=hkv, d=d,
                 r=r, axes=rng.choice([1, 1, 2, 3, 4]) if r >= 16 else 1, order=rng.choice([BLOCKED, CYCLIC]), pairs=rng.choice([HALVES, PAIRS]),
                 inverse=not cache and rng.random() < 0.5, dtype=dtype, cache=cache, kv8=kv8, far=_log(rng, 20000, 1000000))
    elif op == "fork":
        parents, hi = _log(rng, 1, 64), _log(rng, 40, 30000)
        c = fork("", parents=parents, rows=parents + _log(rng, 1, 400), lo=_log(rng, 1, hi), hi=hi, table=2000, prefix=rng.random() < 0.5)
    elif op == "append":
        share, hi = rng.choice([1, 1, 2, 3, 8]), _log(rng, 20, 3000)
        new = _log(rng, 1, 300)
        c = append("", rows=share * _log(rng, 1, 512 // share // 2), share=share, lo=_log(rng, 1, hi), hi=hi, new_lo=rng.choice([0, 1, new]), new_hi=new,
                   table=256, caches=rng.choice([2, 4, 8]), hkv=rng.choice([8, 8, 1, 3]), d=rng.choice([128, 64]))
    elif op == "compact":
        c = compact("", blocks=_log(rng, 40, 7000), live=round(rng.uniform(0.05, 0.98), 3), rows=_log(rng, 1, 128), caches=rng.choice([2, 4, 8]),
                    hkv=rng.choice([8, 8, 1, 3]), d=rng.choice([128, 64]), dtype=rng.choice(["bf16", "bf16", "f32"]) )
        if c["dtype"] == "f32":
            c["caches"] = 2
    else:
        rows, vocab = _log(rng, 1, 200), _log(rng, 500, 150000)
        dtype = rng.choice(["bf16", "bf16", "f32"])
        rows = max(1, min(rows, (28000000 if dtype == "bf16" else 14000000) // vocab))
        hi = _log(rng, 2, 8000)
        c = logits("", rows=rows, vocab=vocab, dtype=dtype, lo=rng.randint(0, hi), hi=hi, bias=rng.choice([0, 1, 16, 300]),
                   masked=rng.choice([0.0, 0.5, 1.0]))
    c["lens"] = lens
    del c["name"]
    return c


# ---- shapes, from the case alone ----------------------------------------------------------------------------

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


def _size(case):
    return 4 if case["dtype"] == "f32" else 2


def _axis_pairs(case):
    """Pairs of each axis: about equal shares, the first one takes the rest."""
    n = case["r"] // 2
    share = n // case["axes"]
    return [n - share * (case["axes"] - 1)] + [share] * (case["axes"] - 1)


def _new_rows(case):
    """New tokens of each sequence of a rope case."""
    T, n = case["tokens"], case["seqs"]
    if n == T:
        return [1] * n
    r = random.Random(case["lens"])
    cuts = sorted(r.sample(range(1, T), n - 1)) if n > 1 else []
    return [b - a for a, b in zip([0] + cuts, cuts + [T])]


def _contexts(case, n):
    r = random.Random(case["lens"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(n)]


def _pages(tokens):
    return (tokens + BLOCK - 1) // BLOCK


def _fork_plan(case):
    """(contexts of the parents, parent of each row, tokens that each row takes over)."""
    P, N = case["parents"], case["rows"]
    L = _contexts(case, P)
    r = random.Random(case["lens"] + 1)
    first = list(range(P))
    r.shuffle(first)
    src = first + [r.randrange(P) for _ in range(N - P)]
    keep = [L[p] for p in src]
    if case["prefix"]:
        keep[P:] = [k if r.random() < 0.5 else r.randint(1, k) for k in keep[P:]]
    return L, src, keep


def _append_plan(case):
    """(contexts, new tokens, holders of each row's pages beside the rows)."""
    groups = case["rows"] // case["share"]
    per = _contexts(case, groups)
    r = random.Random(case["lens"] + 1)
    L, new, more = [], [], []
    for c in per:
        kept = 1 if case["share"] > 1 and r.random() < 0.25 else 0      # a prefix that the program itself keeps
        for _ in range(case["share"]):
            L.append(c)
            new.append(r.randint(case["new_lo"], case["new_hi"]))
            more.append(kept)
    return L, new, more


def _copies(case):
    """Rows of the shared last pages that have to be copied, one entry per copy."""
    L, new, more = _append_plan(case)
    out = []
    for g in range(0, len(L), case["share"]):
        holders = case["share"] + more[g]
        for i in range(g, g + case["share"]):
            if new[i] > 0 and L[i] % BLOCK and holders > 1:
                holders -= 1
                out.append(L[i] % BLOCK)
    return out


def _live_pages(case):
    """Live pages of a compact case, in the order in which its rows hold them."""
    r = random.Random(case["lens"])
    n = max(1, int(case["blocks"] * case["live"]))
    return r.sample(range(case["blocks"]), n)


def _moves(case):
    live = _live_pages(case)
    return sum(p >= len(live) for p in live)


# ---- inputs -------------------------------------------------------------------------------------------------

def _ints(values, **kw):
    return torch.tensor(values, dtype=torch.int32, **kw).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return _PREPARE[case["op"]](case, seed, gen)


def _randn(shape, dtype, gen):
    return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)


def _prepare_rope(case, seed, gen):
    T, hq, hkv, d, n = case["tokens"], case["hq"], case["hkv"], case["d"], case["seqs"]
    dt = _DTYPE[case["dtype"]]
    r, lens = random.Random(seed), random.Random(case["lens"] + 1)
    new = _new_rows(case)
    # queries, keys and values lie side by side, as one projection leaves them
    qkv = _randn((T, (hq + 2 * hkv) * d), dt, gen)
    q, k, v = (x.unflatten(1, (-1, d)) for x in qkv.split([hq * d, hkv * d, hkv * d], dim=1))
    pos, prior = [], []
    for m in new:
        p0 = r.randrange(0, max(1, case["far"] - m))
        prior.append(lens.randint(0, 300))
        pos += range(p0, p0 + m)
    positions = torch.tensor(pos, dtype=torch.int32)[None].repeat(case["axes"], 1)
    if case["axes"] > 1:       # rows and columns of images
        positions[1:] -= torch.randint(0, 64, (case["axes"] - 1, T), generator=torch.Generator().manual_seed(seed)).int()
        positions.clamp_(min=0)
    freq = (10000.0 ** (-torch.arange(case["r"] // 2, dtype=torch.float64) * 2 / case["r"])).float()
    s = {"op": "rope", "q": q, "k": k, "v": v, "positions": positions.cuda(), "inv_freq": freq.cuda(), "axis_pairs": _axis_pairs(case),
         "order": case["order"], "pairs": case["pairs"], "inverse": case["inverse"], "cache": case["cache"], "kv8": case["kv8"],
         "q_out": torch.empty((T, hq, d), dtype=dt, device="cuda"), "k_out": torch.empty((T, hkv, d), dtype=dt, device="cuda")}
    # the pair's axis, for the plain form
    A, sec = case["axes"], s["axis_pairs"]
    if case["order"] == BLOCKED:
        axis = [a for a in range(A) for _ in range(sec[a])]
    else:
        axis = [c % A if c // A < sec[c % A] else 0 for c in range(case["r"] // 2)]
    s["axis"] = torch.tensor(axis).cuda()
    if case["cache"]:
        L = [p + m for p, m in zip(prior, new)]
        need = [_pages(x) for x in L]
        blocks = sum(need) + 5
        ids = r.sample(range(blocks), sum(need))
        table = torch.zeros((n, max(need) + 1), dtype=torch.int32)
        at = 0
        for i, m in enumerate(need):
            table[i, :m] = torch.tensor(ids[at:at + m], dtype=torch.int32)
            at += m
        cu = [0]
        for m in new:
            cu.append(cu[-1] + m)
        s["table"], s["seq_lens"], s["cu"] = table.cuda(), _ints(L), _ints(cu)
        shape = (2, blocks, hkv, BLOCK, d)
        cache = _randn(shape, torch.bfloat16 if case["kv8"] else dt, gen)
        if case["kv8"]:
            cache = (cache.float() * (E4M3_MAX / E4M3_SIGMAS)).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
            s["scale"] = torch.linspace(1.0, 1.25, hkv, device="cuda") * (E4M3_SIGMAS / E4M3_MAX)
        s["k_cache"], s["v_cache"] = cache[0], cache[1]
    return s


def _prepare_fork(case, seed, gen):
    r = random.Random(seed)
    L, src, keep = _fork_plan(case)
    P, N, mb = case["parents"], case["rows"], case["table"]
    need = [_pages(x) for x in L]
    blocks = sum(need) + 64
    ids = r.sample(range(blocks), sum(need))
    table = torch.zeros((P, mb), dtype=torch.int32)
    refs = torch.zeros(blocks, dtype=torch.int32)
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = torch.tensor(ids[at:at + m], dtype=torch.int32)
        at += m
    refs[torch.tensor(ids)] = 1
    back = [src.index(p) for p in range(P)]        # the row that holds all of parent p
    return {"op": "fork", "table": table.cuda(), "seq_lens": _ints(L), "refs": refs.cuda(), "src": _ints(src), "keep": _ints(keep),
            "table_b": torch.zeros((N, mb), dtype=torch.int32, device="cuda"), "lens_b": torch.zeros(N, dtype=torch.int32, device="cuda"),
            "back": _ints(back), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def _prepare_append(case, seed, gen):
    r = random.Random(seed)
    L, new, more = _append_plan(case)
    n, share, mb = len(L), case["share"], case["table"]
    held = sum(_pages(L[g]) for g in range(0, n, share))
    room = sum(_pages(a + b) - _pages(a) for a, b in zip(L, new)) + len(_copies(case)) + 7
    blocks = held + room
    ids = r.sample(range(blocks), held)
    table = torch.zeros((n, mb), dtype=torch.int32)
    refs = torch.zeros(blocks, dtype=torch.int32)
    at = 0
    for g in range(0, n, share):
        m = _pages(L[g])
        own_ids = torch.tensor(ids[at:at + m], dtype=torch.int32)
        table[g:g + share, :m] = own_ids
        refs[own_ids.long()] = share + more[g]
        at += m
    cu = [0]
    for m in new:
        cu.append(cu[-1] + m)
    dt = _DTYPE[case["dtype"]]
    return {"op": "append", "cu": _ints(cu), "table": table.cuda(), "seq_lens": _ints(L), "refs": refs.cuda(),
            "caches": _randn((case["caches"], blocks, case["hkv"], BLOCK, case["d"]), dt, gen),
            "table_out": torch.zeros((n, mb), dtype=torch.int32, device="cuda"), "lens_out": torch.zeros(n, dtype=torch.int32, device="cuda"),
            "refs_out": torch.zeros(blocks, dtype=torch.int32, device="cuda"), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}


def _prepare_compact(case, seed, gen):
    live = _live_pages(case)
    r = random.Random(seed)
    r.shuffle(live)
    n = min(case["rows"], len(live))
    cuts = [0] + sorted(random.Random(case["lens"] + 1).sample(range(1, len(live)), n - 1)) + [len(live)]
    need = [b - a for a, b in zip(cuts, cuts[1:])]
    table = torch.zeros((n, max(need)), dtype=torch.int32)
    for i in range(n):
        table[i, :need[i]] = torch.tensor(live[cuts[i]:cuts[i + 1]], dtype=torch.int32)
    refs = torch.zeros(case["blocks"], dtype=torch.int32)
    refs[torch.tensor(live)] = 1
    L = [BLOCK * m - r.randrange(BLOCK) for m in need]
    z = lambda *shape: torch.zeros(shape, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"op": "compact", "table": table.cuda(), "seq_lens": _ints(L), "refs": refs.cuda(),
            "caches": _randn((case["caches"], case["blocks"], case["hkv"], BLOCK, case["d"]), _DTYPE[case["dtype"]], gen),
            "table_out": z(*table.shape), "refs_out": z(case["blocks"]), "page_map": z(case["blocks"]), "num_live": z(1), "status": z(1)}


def _prepare_logits(case, seed, gen):
    R, V = case["rows"], case["vocab"]
    r = random.Random(seed)
    hist = _contexts(case, R)
    cu = [0]
    for h in hist:
        cu.append(cu[-1] + h)
    # frequent tokens are frequent: a cube of uniform numbers
    ids = (torch.rand(max(1, cu[-1]), generator=gen, device="cuda") ** 3 * V).long().clamp_(max=V - 1)
    ids = (ids * 7919 % V).int()
    nb = case["bias"]
    words = (V + 31) // 32
    masks = max(1, R // 2)
    bits = torch.randint(-(1 << 31), 1 << 31, (2, masks, words), generator=gen, device="cuda", dtype=torch.int64).int()
    rows = [r.randrange(masks) if r.random() < case["masked"] else -1 for _ in range(R)]
    u = torch.rand((3, R), generator=gen, device="cuda")
    return {"op": "logits", "logits": (_randn((R, V), torch.float32, gen) * 4).to(_DTYPE[case["dtype"]]),
            "out": torch.empty((R, V), dtype=_DTYPE[case["dtype"]], device="cuda"),
            "history": ids, "cu_history": _ints(cu), "prompt_lens": _ints([h // 2 for h in hist]),
            "repetition": 1.0 + 0.3 * u[0], "frequency": 0.5 * u[1], "presence": 0.5 * u[2],
            "cu_bias": _ints(list(range(0, nb * R + 1, nb)) if nb else [0] * (R + 1)),
            "bias_ids": torch.randint(0, V, (max(1, nb * R),), generator=gen, device="cuda").int(),
            "bias_values": torch.randn(max(1, nb * R), generator=gen, device="cuda") * 3,
            "biased": nb > 0, "mask": bits[0] & bits[1], "mask_rows": _ints(rows)}


_PREPARE = {"rope": _prepare_rope, "fork": _prepare_fork, "append": _prepare_append, "compact": _prepare_compact, "logits": _prepare_logits}


# ---- one pass -----------------------------------------------------------------------------------------------

def run(s):
    return _RUN[s["op"]](s)


def _run_rope(s):
    if own:
        from paper_2603_06588_amd import binding
        more = {}
        if s["cache"]:
            more = {"v": s["v"], "block_table": s["table"], "seq_lens": s["seq_lens"], "cu_q_lens": s["cu"], "k_cache": s["k_cache"],
                    "v_cache": s["v_cache"]}
            if s["kv8"]:
                more["k_scale"] = more["v_scale"] = s["scale"]
        binding.hook_rope(s["q"], s["k"], s["positions"], s["inv_freq"], axis_pairs=s["axis_pairs"], axis_order=s["order"], layout=s["pairs"],
                          inverse=s["inverse"], q_out=s["q_out"], k_out=s["k_out"], **more)
    else:
        plain_rope(s)
    out = {"q": s["q_out"], "k": s["k_out"]}
    if s["cache"]:
        kind = torch.float8_e4m3fn if s["kv8"] else s["k_cache"].dtype
        out["k_cache"], out["v_cache"] = s["k_cache"].view(kind), s["v_cache"].view(kind)
    return out


def plain_rope(s):
    angle = s["positions"].double()[s["axis"]].T * s["inv_freq"].double()        # [T, r/2], far positions need 64 bits
    if s["inverse"]:
        angle = -angle
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    s["q_out"].copy_(_turn(s["q"], cos, sin, s["pairs"]))
    s["k_out"].copy_(_turn(s["k"], cos, sin, s["pairs"]))
    if s["cache"]:
        t = torch.arange(s["k"].shape[0], device="cuda", dtype=torch.int32)
        i = torch.searchsorted(s["cu"][1:], t, right=True)
        at = s["seq_lens"][i] - s["cu"][1:][i] + t
        page, slot = s["table"][i, (at // BLOCK).long()].long(), (at % BLOCK).long()
        k, v = s["k_out"], s["v"]
        if s["kv8"]:
            k, v = _to_e4m3(k, s["scale"]), _to_e4m3(v, s["scale"])
        s["k_cache"][page, :, slot] = k
        s["v_cache"][page, :, slot] = v


def _turn(x, cos, sin, pairs):
    n = cos.shape[-1]
    y = x.float()
    a, b = (y[..., 0:2 * n:2], y[..., 1:2 * n:2]) if pairs == PAIRS else (y[..., :n], y[..., n:2 * n])
    u, w = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([u, w], dim=-1).flatten(-2) if pairs == PAIRS else torch.cat([u, w], dim=-1)
    return torch.cat([turned, y[..., 2 * n:]], dim=-1).to(x.dtype)


def _to_e4m3(x, scale):
    return (x.float() / scale[:, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn).view(torch.uint8)


def _run_fork(s):
    if own:
        from paper_2603_06588_amd import binding
        binding.hook_pages_fork(s["src"], s["table"], s["seq_lens"], s["refs"], s["table_b"], s["lens_b"], s["status"], src_lens=s["keep"])
        # all rows but one of each parent are dropped again
        binding.hook_pages_fork(s["back"], s["table_b"], s["lens_b"], s["refs"], s["table"], s["seq_lens"], s["status"])
    else:
        plain_fork(s["src"], s["keep"], s["table"], s["seq_lens"], s["refs"], s["table_b"], s["lens_b"])
        plain_fork(s["back"], None, s["table_b"], s["lens_b"], s["refs"], s["table"], s["seq_lens"])
    return {"rows": s["table_b"], "lens": s["lens_b"], "table": s["table"], "seq_lens": s["seq_lens"], "refs": s["refs"], "status": s["status"]}


def _held(table, lens):
    return torch.arange(table.shape[1], device="cuda", dtype=torch.int32) * BLOCK < lens[:, None]


def plain_fork(src, keep, table, lens, refs, table_out, lens_out):
    new_lens = lens[src] if keep is None else torch.minimum(lens[src], keep)
    before, after = _held(table, lens), _held(table_out, new_lens)
    new = torch.where(after, table[src], table_out)
    any_page = torch.arange(table.shape[1], device="cuda") % refs.shape[0]          # gets 0 where a row holds none
    refs.scatter_add_(0, torch.where(before, table.long(), any_page).flatten(), -before.flatten().int())
    refs.scatter_add_(0, torch.where(after, new.long(), any_page).flatten(), after.flatten().int())
    table_out.copy_(new)
    lens_out.copy_(new_lens)


def _run_append(s):
    if own:
        from paper_2603_06588_amd import binding
        binding.hook_pages_append(s["cu"], s["table"], s["seq_lens"], s["refs"], s["caches"], s["status"], block_table_out=s["table_out"],
                                  seq_lens_out=s["lens_out"], ref_counts_out=s["refs_out"])
    else:
        plain_append(s)
    return {"table": s["table_out"], "lens": s["lens_out"], "refs": s["refs_out"], "caches": s["caches"], "status": s["status"]}


def plain_append(s):
    table, lens, refs, caches = s["table"], s["seq_lens"], s["refs"], s["caches"]
    n, mb = table.shape
    new = s["cu"][1:] - s["cu"][:-1]
    part = lens % BLOCK
    row = torch.arange(n, device="cuda")
    last = table[row, (lens // BLOCK).clamp(max=mb - 1).long()].long()
    writes = (new > 0) & (part > 0)
    earlier = ((last[:, None] == last) & writes & (row[:, None] > row)).sum(1)      # rows that leave the page before this one
    copy = writes & (refs[last] - earlier > 1)
    start = (lens + BLOCK - 1) // BLOCK - copy.int()
    end = torch.where(new > 0, (lens + new + BLOCK - 1) // BLOCK, start)
    need = end - start
    first = need.cumsum(0) - need
    free = refs == 0
    fits = (need.sum() <= free.sum()) & (lens + new <= mb * BLOCK).all()
    pages = torch.argsort(free.logical_not().int(), stable=True)                    # free pages first, the lowest first
    j = torch.arange(mb, device="cuda")
    fresh = (j >= start[:, None]) & (j < end[:, None]) & fits
    got = pages[(first[:, None] + j - start[:, None]).clamp(0, refs.shape[0] - 1)]
    kept = _held(table, lens)
    s["table_out"].copy_(torch.where(fresh, got.int(), torch.where(kept, table, s["table_out"])))
    s["lens_out"].copy_(torch.where(fits, lens + new, lens))
    s["refs_out"].copy_(refs)
    s["refs_out"].scatter_add_(0, got.flatten(), fresh.flatten().int())
    s["refs_out"].scatter_add_(0, last, -(copy & fits).int())
    s["status"].bitwise_or_(torch.where(fits, 0, FULL))
    rows = ((copy & fits).nonzero()[:, 0])
    to, slots = pages[first[rows]], torch.arange(BLOCK, device="cuda") < part[rows][:, None]
    caches[:, to] = torch.where(slots[:, None, :, None], caches[:, last[rows]], caches[:, to])


def _run_compact(s):
    if own:
        from paper_2603_06588_amd import binding
        binding.hook_pages_compact(s["table"], s["seq_lens"], s["refs"], s["caches"], s["page_map"], s["num_live"], s["status"],
                                   block_table_out=s["table_out"], ref_counts_out=s["refs_out"])
    else:
        plain_compact(s)
    return {"table": s["table_out"], "refs": s["refs_out"], "map": s["page_map"], "live": s["num_live"], "caches": s["caches"],
            "status": s["status"]}


def plain_compact(s):
    refs, caches = s["refs"], s["caches"]
    live = refs > 0
    count = live.sum()
    at = torch.arange(refs.shape[0], device="cuda")
    movers, holes = (live & (at >= count)).nonzero()[:, 0], (~live & (at < count)).nonzero()[:, 0]
    s["page_map"].copy_(torch.where(live, at, -1))
    s["page_map"][movers] = holes.int()
    s["refs_out"].copy_(refs)
    s["refs_out"][holes] = refs[movers]
    s["refs_out"][movers] = 0
    s["num_live"].copy_(count)
    s["table_out"].copy_(torch.where(_held(s["table"], s["seq_lens"]), s["page_map"][s["table"].long()], s["table_out"]))
    caches[:, holes] = caches[:, movers]


def _run_logits(s):
    if own:
        from paper_2603_06588_amd import binding
        bias = {"cu_bias": s["cu_bias"], "bias_ids": s["bias_ids"], "bias_values": s["bias_values"]} if s["biased"] else {}
        binding.hook_steer_logits(s["logits"], out=s["out"], history=s["history"], cu_history=s["cu_history"], prompt_lens=s["prompt_lens"],
                                  repetition=s["repetition"], frequency=s["frequency"], presence=s["presence"], mask=s["mask"],
                                  mask_rows=s["mask_rows"], **bias)
    else:
        plain_logits(s)
    return s["out"]


def plain_logits(s):
    R, V = s["logits"].shape
    x = s["logits"].float()
    cu = s["cu_history"]
    at = torch.arange(s["history"].shape[0], device="cuda", dtype=torch.int32)
    row = torch.searchsorted(cu[1:], at, right=True).clamp(max=R - 1)
    valid = at < cu[-1]
    cell = row * V + s["history"]
    seen, count = torch.zeros((2, R * V), dtype=torch.int32, device="cuda")
    seen.scatter_add_(0, cell, valid.int())
    count.scatter_add_(0, cell, (valid & (at - cu[row] >= s["prompt_lens"][row])).int())
    seen, count = seen.view(R, V), count.view(R, V)
    x = torch.where(seen > 0, torch.where(x > 0, x / s["repetition"][:, None], x * s["repetition"][:, None]), x)
    x = torch.where(count > 0, x - count * s["frequency"][:, None] - s["presence"][:, None], x)
    if s["biased"]:      # of a token named twice the last entry counts
        at = torch.arange(s["bias_ids"].shape[0], device="cuda", dtype=torch.int32)
        cell = torch.searchsorted(s["cu_bias"][1:], at, right=True) * V + s["bias_ids"]
        last = torch.full((R * V,), -1, dtype=torch.int32, device="cuda").scatter_reduce_(0, cell, at, "amax").view(R, V)
        x = torch.where(last >= 0, x + s["bias_values"][last.clamp(min=0)], x)
    token = torch.arange(V, device="cuda")
    words = s["mask"][:, token // 32]
    allowed = (words >> (token % 32).int()) & 1
    barred = (s["mask_rows"] >= 0)[:, None] & (allowed[s["mask_rows"].clamp(min=0)] == 0)
    s["out"].copy_(torch.where(barred, -math.inf, x))


_RUN = {"rope": _run_rope, "fork": _run_fork, "append": _run_append, "compact": _run_compact, "logits": _run_logits}


# ---- what a pass cannot do without --------------------------------------------------------------------------

def work(case):
    op = case["op"]
    if op == "rope":
        T, hq, hkv, d, e = case["tokens"], case["hq"], case["hkv"], case["d"], _size(case)
        b = T * (2 * hq + 2 * hkv) * d * e + 4 * T * case["axes"]
        if case["cache"]:
            b += T * hkv * d * (e + 2 * (1 if case["kv8"] else e))
        return {"bytes": b, "flops": T * (hq + hkv) * case["r"] * 3}
    if op == "fork":
        L, src, keep = _fork_plan(case)
        before, after = sum(map(_pages, L)), sum(map(_pages, keep))
        return {"bytes": 2 * (4 * (before + after) + 8 * before), "flops": 0}
    if op == "append":
        L, new, more = _append_plan(case)
        held = sum(map(_pages, L[::case["share"]]))
        table = sum(_pages(a) + _pages(a + b) for a, b in zip(L, new))
        blocks = held + sum(_pages(a + b) - _pages(a) for a, b in zip(L, new)) + len(_copies(case)) + 7
        data = 2 * sum(_copies(case)) * case["caches"] * case["hkv"] * case["d"] * _size(case)
        return {"bytes": data + 4 * table + 8 * blocks, "flops": 0}
    if op == "compact":
        page = case["hkv"] * BLOCK * case["d"] * _size(case)
        live = max(1, int(case["blocks"] * case["live"]))
        return {"bytes": 2 * _moves(case) * case["caches"] * page + 12 * case["blocks"] + 8 * live, "flops": 0}
    R, V, hist = case["rows"], case["vocab"], sum(_contexts(case, case["rows"]))
    return {"bytes": 2 * R * V * _size(case) + 4 * hist + 8 * R * case["bias"] + int(R * case["masked"]) * ((V + 31) // 32) * 4, "flops": 0}


# ---- the definitions, in 64 bits ----------------------------------------------------------------------------

def exact(case, seed):
    return _EXACT[case["op"]](case, prepare(case, seed))


def _exact_rope(case, s):
    n, d = case["r"] // 2, case["d"]
    ax = s["axis"].tolist()
    f, pos = s["inv_freq"].double(), s["positions"].double()
    phase = torch.stack([pos[ax[c]] * f[c] for c in range(n)], dim=1) * (-1.0 if case["inverse"] else 1.0)
    spin = torch.polar(torch.ones_like(phase), phase)[:, None, :]
    lo, hi = (list(range(0, 2 * n, 2)), list(range(1, 2 * n, 2))) if case["pairs"] == PAIRS else (list(range(n)), list(range(n, 2 * n)))
    out = {}
    for name in ("q", "k"):
        x = s[name].double().clone()
        z = torch.complex(x[..., lo], x[..., hi]) * spin
        x[..., lo], x[..., hi] = z.real, z.imag
        out[name] = x
    if case["cache"]:
        new, L, table = _new_rows(case), s["seq_lens"].tolist(), s["table"].tolist()
        where, t = [], 0
        for i, m in enumerate(new):
            where += [(table[i][p // BLOCK], p % BLOCK) for p in range(L[i] - m, L[i])]
        page, slot = (torch.tensor(w, device="cuda") for w in zip(*where))
        for name, x in (("k_cache", out["k"]), ("v_cache", s["v"].double())):
            c = s[name].view(torch.float8_e4m3fn).double() if case["kv8"] else s[name].double()
            c[page, :, slot] = x / s["scale"].double()[:, None] if case["kv8"] else x
            out[name] = c
    return out


def _exact_pages(case, s):
    """The rows one after the other, as the definition has it; whole numbers, and the values of moved pages."""
    table, lens, refs, caches = s["table"].tolist(), s["seq_lens"].tolist(), s["refs"].tolist(), s["caches"].double()
    if case["op"] == "compact":
        live = [p for p, n in enumerate(refs) if n > 0]
        top = [p for p in live if p >= len(live)]
        holes = sorted(set(range(len(live))) - set(live))
        if top:
            caches[:, torch.tensor(holes, device="cuda")] = caches[:, torch.tensor(top, device="cuda")]
        return {"caches": caches}
    cu, free = s["cu"].tolist(), [p for p, n in enumerate(refs) if n == 0][::-1]
    for i, L in enumerate(lens):
        m = cu[i + 1] - cu[i]
        if m > 0 and L % BLOCK and refs[table[i][L // BLOCK]] > 1:
            old, new = table[i][L // BLOCK], free.pop()
            refs[old] -= 1
            caches[:, new, :, :L % BLOCK] = caches[:, old, :, :L % BLOCK]
        for _ in range(_pages(L + m) - _pages(L)):
            free.pop()
    return {"caches": caches}


def _exact_logits(case, s):
    R, V = case["rows"], case["vocab"]
    y = s["logits"].double()
    hist, cu, prompt = s["history"].long(), s["cu_history"].tolist(), s["prompt_lens"].tolist()
    rows, cub = s["mask_rows"].tolist(), s["cu_bias"].tolist()
    bit = torch.arange(32, device="cuda")
    for i in range(R):
        mine = hist[cu[i]:cu[i + 1]]
        seen = torch.zeros(V, dtype=torch.bool, device="cuda")
        seen[mine] = True
        c = torch.bincount(mine[prompt[i]:], minlength=V).double()
        rep, fr, pr = (float(s[n][i]) for n in ("repetition", "frequency", "presence"))
        x = y[i]
        x[seen & (x > 0)] /= rep
        x[seen & (x < 0)] *= rep            # (a logit that became smaller than 0 by the division: there is none)
        x -= c * fr + (c > 0).double() * pr
        last = dict(zip(s["bias_ids"][cub[i]:cub[i + 1]].tolist(), s["bias_values"][cub[i]:cub[i + 1]].tolist()))
        if last:
            x[torch.tensor(list(last), device="cuda")] += torch.tensor(list(last.values()), dtype=torch.float64, device="cuda")
        if rows[i] >= 0:
            ok = ((s["mask"][rows[i]][:, None] >> bit) & 1).flatten()[:V].bool()
            x[~ok] = -math.inf
    return y


_EXACT = {"rope": _exact_rope, "fork": lambda case, s: None, "append": _exact_pages, "compact": _exact_pages, "logits": _exact_logits}
