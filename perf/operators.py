"""Operators over the paged cache whose time is measured: each in a plain form, and as the library's calls.

A case is a dict of plain values; its lengths follow from the case alone (so that its bytes are known), all other inputs
from the seed.  Kinds:

  tree     attention of a tree of drafted tokens per sequence over the cache and the drafts
  window   decode attention with a sliding window and a few first tokens that stay visible; pages outside are released
  append   several tokens of every sequence written into their pages, along an accepted path or in order
  fork     copies of a page for the forks of a sequence, and their first tokens written behind the copied ones
  compact  live pages moved to the free places at the pool's start
"""
import math

import numpy as np
import torch

own = False

BLOCK = 256  # tokens of a block of the plain attention
FP8_MAX = 448.0


def listed():
    return [
        # drafts of a small model in a latency-bound loop: a handful of short sequences, four nodes each
        {"name": "tree_tiny", "kind": "tree", "seqs": 8, "q_heads": 8, "kv_heads": 2, "d": 64, "page": 16, "fp8": False, "nodes": 4, "ragged": False,
         "median": 256, "sigma": 1.0, "lo": 1, "hi": 2048},
        # a 7B-class long-tailed batch whose sequences have drafts of up to eight nodes
        {"name": "tree_rollout7b", "kind": "tree", "seqs": 64, "q_heads": 28, "kv_heads": 4, "d": 128, "page": 16, "fp8": False, "nodes": 8, "ragged": True,
         "median": 2048, "sigma": 1.2, "lo": 64, "hi": 32768},
        # a larger model on fp8 pages, sixteen nodes a sequence
        {"name": "tree_moe_fp8", "kind": "tree", "seqs": 256, "q_heads": 64, "kv_heads": 8, "d": 128, "page": 32, "fp8": True, "nodes": 16, "ragged": False,
         "median": 4096, "sigma": 1.0, "lo": 128, "hi": 32768},
        # the last few responses, with the widest trees: as much arithmetic as a short prefill
        {"name": "tree_wide_tail", "kind": "tree", "seqs": 5, "q_heads": 32, "kv_heads": 8, "d": 128, "page": 16, "fp8": False, "nodes": 64, "ragged": True,
         "median": 30000, "sigma": 0.4, "lo": 8192, "hi": 65536},
        # a short window over a few sequences of a small model
        {"name": "window_tiny", "kind": "window", "seqs": 8, "q_heads": 8, "kv_heads": 2, "d": 64, "page": 16, "fp8": False, "window": 128, "sinks": 4,
         "median": 400, "sigma": 1.0, "lo": 1, "hi": 4096},
        # a full long-tailed batch: shorter rows than the window among ones far longer
        {"name": "window_multi", "kind": "window", "seqs": 512, "q_heads": 64, "kv_heads": 8, "d": 128, "page": 16, "fp8": False, "window": 1024, "sinks": 4,
         "median": 1024, "sigma": 1.3, "lo": 16, "hi": 65536},
        # a wide window over fp8 pages, at an odd offset
        {"name": "window_moe_fp8", "kind": "window", "seqs": 500, "q_heads": 64, "kv_heads": 8, "d": 128, "page": 32, "fp8": True, "window": 4090, "sinks": 20,
         "median": 4096, "sigma": 1.2, "lo": 128, "hi": 131072},
        # what a verification has accepted of eight-node trees: one to eight tokens a sequence
        {"name": "append_path7b", "kind": "append", "seqs": 64, "kv_heads": 4, "d": 128, "page": 16, "fp8": False, "nodes": 8, "path": True, "least": 1},
        # the same for the largest batch, fp8 pages
        {"name": "append_path_fp8", "kind": "append", "seqs": 1024, "kv_heads": 8, "d": 128, "page": 32, "fp8": True, "nodes": 16, "path": True, "least": 1},
        # a chunk of new prompts: hundreds of tokens of each sequence in order
        {"name": "append_prompt_fp8", "kind": "append", "seqs": 24, "kv_heads": 8, "d": 128, "page": 32, "fp8": True, "nodes": 700, "path": False, "least": 300},
        # 16 responses for each of 16 prompts begin: a copy of the prompt's last page, and their first token
        {"name": "fork_group_fp8", "kind": "fork", "seqs": 256, "group": 16, "kv_heads": 8, "d": 128, "page": 32, "fp8": True},
        # the pool shrinks after a long tail has ended: its last live pages move down
        {"name": "compact7b", "kind": "compact", "kv_heads": 4, "d": 128, "page": 16, "fp8": False, "moves": 6000},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "window", "window", "append", "append", "fork", "compact"])
    case = {"kind": kind, "d": rng.choice([64, 128, 128]), "page": rng.choice([16, 32]), "fp8": rng.random() < 0.5, "kv_heads": rng.choice([1, 2, 4, 8])}
    token_bytes = case["kv_heads"] * case["d"] * 2 * (1 if case["fp8"] else 2)
    if kind == "compact":
        case["moves"] = _log(rng, 1, max(1, (1 << 28) // (token_bytes * case["page"])))
        return case
    if kind == "fork":
        case["group"] = rng.choice([2, 3, 5, 8, 16])
        case["seqs"] = case["group"] * _log(rng, 1, 32)
        return case
    if kind == "append":
        case["path"] = rng.random() < 0.7
        case["seqs"] = _log(rng, 1, 1024 if case["path"] else 24)
        case["nodes"] = _log(rng, 1, 64) if case["path"] else _log(rng, 1, 1200)
        case["least"] = rng.choice([0, min(1, case["nodes"]), case["nodes"] // 2, case["nodes"]])
        if case["seqs"] * case["nodes"] > 24576:
            case["seqs"] = 24576 // case["nodes"]
        return case
    heads = rng.choice([1, 2, 4, 6, 7, 8, 16])
    case.update(seqs=_log(rng, 1, 256 if kind == "tree" else 512), q_heads=heads * case["kv_heads"], median=_log(rng, 32, 32768), sigma=rng.uniform(0.0, 1.3),
                lo=rng.choice([0, 1]))
    if kind == "window":
        case.update(window=_log(rng, 1, 8192), sinks=rng.choice([0, 1, 4, 16, 40]))
        seen = min(case["window"] + case["sinks"] + 2 * case["page"], 8 * case["median"])
        case["seqs"] = max(1, min(case["seqs"], (3 << 30) // (token_bytes * seen)))
        case["hi"] = min(131072, 16 * case["median"])
        return case
    case.update(nodes=_log(rng, 1, 64), ragged=rng.random() < 0.5)
    # at most 1 GiB of keys and values, and no more products than the largest listed cases have
    most = min((1 << 30) // token_bytes, (1 << 39) // (4 * case["d"] * case["q_heads"] * case["nodes"]))
    case["hi"] = max(32, min(65536, 16 * case["median"], most // case["seqs"]))
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _rng(case):
    return np.random.default_rng(case.get("seqs", 1) * 1000003 + case.get("median", 0) * 31 + case.get("nodes", 0))


def _lengths(case):
    """Tokens in the cache of each sequence: lognormal, clipped, the same for every seed of the case."""
    x = np.exp(_rng(case).normal(math.log(case["median"]), case["sigma"], case["seqs"]))
    return np.clip(np.rint(x), case["lo"], case["hi"]).astype(np.int64)


def _counts(case):
    """Nodes (tree) or tokens (append) of each sequence."""
    if case["kind"] == "tree":
        return _rng(case).integers(1, case["nodes"] + 1, case["seqs"]) if case["ragged"] else np.full(case["seqs"], case["nodes"])
    return _rng(case).integers(case["least"], case["nodes"] + 1, case["seqs"])


def _page_shapes(case):
    x = 16 if case["fp8"] else 8
    return (case["kv_heads"], case["d"] // x, case["page"], x), (case["kv_heads"], case["d"], case["page"])


def _pages(case, n, gen):
    """n K or V pages' worth of N(0, 1) values: (bf16, None), or fp8 codes and one scale a page."""
    size = case["kv_heads"] * case["page"] * case["d"]
    if not case["fp8"]:
        t = torch.empty((n, size), dtype=torch.bfloat16, device="cuda")
        t.normal_(generator=gen)
        return t, None
    t = torch.empty((n, size), dtype=torch.uint8, device="cuda")
    scales = torch.empty(n, dtype=torch.float32, device="cuda")
    step = max(1, (1 << 28) // size)
    for i in range(0, n, step):
        x = torch.empty((min(step, n - i), size), dtype=torch.float32, device="cuda").normal_(generator=gen)
        s = x.abs().amax(dim=1) / FP8_MAX
        scales[i:i + step] = s
        t[i:i + step] = (x / s[:, None]).clamp_(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
    return t, scales


def _pool(case, n, gen):
    ks, vs = _page_shapes(case)
    k, k_scales = _pages(case, n, gen)
    v, v_scales = _pages(case, n, gen)
    return {"k": k.view((n,) + ks), "v": v.view((n,) + vs), "k_scales": k_scales, "v_scales": v_scales}


def _dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=dtype)).cuda()


def _normal(shape, gen):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _trees(rng, counts, nodes):
    """A random tree for each sequence: a node's parent is an earlier node, or none (a root).  The mask of a node has its
    own bit and its ancestors'."""
    b = len(counts)
    mask = np.zeros((b, nodes), np.uint64)
    for i in range(nodes):
        up = rng.integers(0, i + 1, b)  # 0: a root
        above = np.where(up > 0, mask[np.arange(b), np.maximum(up, 1) - 1], np.uint64(0))
        mask[:, i] = np.where(i < counts, above | (np.uint64(1) << np.uint64(i)), np.uint64(0))
    return mask.view(np.int64)


def _scattered(rng, n):
    """A table whose row b has n[b] distinct pages of a pool that they nearly fill, and that pool's pages."""
    total = int(n.sum())
    num_pages = total + total // 8 + 1
    perm = rng.permutation(num_pages)
    table = np.zeros((len(n), max(1, int(n.max()))), np.int32)
    at = np.arange(table.shape[1])[None, :]
    table[at < n[:, None]] = perm[:total]
    return table, num_pages


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    page = case["page"]
    if case["kind"] == "compact":
        live = rng.permutation(2 * case["moves"])  # live pages of the upper half, free places of the lower one
        src = np.sort(live[live >= case["moves"]])
        dst = np.sort(live[live < case["moves"]])
        return {"case": case, "pool": _pool(case, 2 * case["moves"], gen), "src": _dev(src), "dst": _dev(dst)}
    if case["kind"] in ("append", "fork"):
        return _prepare_write(case, gen, rng)
    lens = _lengths(case)
    n = -(-lens // page)
    if case["kind"] == "window":
        _, first, sink = _visible_pages(case, lens)
        table, num_pages = _scattered(rng, sink + n - first)
        full = np.zeros((len(lens), max(1, int(n.max()))), np.int32)
        for b in range(len(lens)):  # a released page's entry is 0 and is never read
            full[b, :sink[b]] = table[b, :sink[b]]
            full[b, first[b]:n[b]] = table[b, sink[b]:sink[b] + n[b] - first[b]]
        table = full
    else:
        table, num_pages = _scattered(rng, n)
    s = {"case": case, "pool": _pool(case, num_pages, gen), "table": _dev(table), "lens": _dev(lens), "host_lens": lens, "versions": _dev(0 * lens)}
    if case["kind"] == "window":
        s["q"] = _normal((len(lens), case["q_heads"], case["d"]), gen)
    else:
        counts = _counts(case)
        s["q"] = _normal((len(lens), case["nodes"], case["q_heads"], case["d"]), gen)
        s["k_draft"], s["v_draft"] = (_normal((len(lens), case["nodes"], case["kv_heads"], case["d"]), gen) for _ in range(2))
        s["mask"] = _dev(_trees(rng, counts, case["nodes"]), np.int64)
        s["counts"] = _dev(counts)
    s["out"] = torch.zeros_like(s["q"])
    return s


def _visible_pages(case, lens):
    """Of each sequence: pages, first page that the window reaches (behind the sinks' pages), pages of the sinks."""
    n = -(-lens // case["page"])
    sink = np.minimum(n, -(-case["sinks"] // case["page"]))
    first = np.maximum(sink, np.maximum(0, lens - case["window"]) // case["page"])
    return n, first, sink


def _prepare_write(case, gen, rng):
    """Sequences somewhere in a page, and the tokens that come next.  The table has random entries where nothing is
    written.  fork: the first member of each group holds the prompt, the others' last page is copied from its."""
    b, page = case["seqs"], case["page"]
    counts = _counts(case) if case["kind"] == "append" else np.ones(b, np.int64)
    nodes = case.get("nodes", 1)
    if case["kind"] == "append":
        base = _rng(case).integers(0, 64 * page, b)  # tokens in the cache before the call
    else:
        prompts = b // case["group"]
        base = np.repeat(_rng(case).integers(0, 8, prompts) * page + _rng(case).integers(1, page, prompts), case["group"])
    lens = base + counts
    first, last = base // page, -(-lens // page)
    written = np.maximum(0, last - first)
    own_pages, num_pages = _scattered(rng, np.maximum(written, 1))
    table = rng.integers(0, num_pages, (b, int(max(last.max(), first.max() + 1)) + 2)).astype(np.int32)
    for i in range(b):
        table[i, first[i]:first[i] + max(1, written[i])] = own_pages[i, :max(1, written[i])]
    s = {"case": case, "pool": _pool(case, num_pages, gen), "table": _dev(table), "lens": _dev(lens), "counts": _dev(counts), "host_base": base,
         "host_counts": counts, "path": None}
    s["k_new"], s["v_new"] = (_normal((b, nodes, case["kv_heads"], case["d"]), gen) for _ in range(2))
    if case.get("path"):  # ascending nodes, as a path through a tree has them
        order = np.argsort(rng.random((b, nodes)), axis=1)
        order[np.arange(nodes)[None, :] >= counts[:, None]] = nodes
        path = np.sort(order, axis=1)
        s["path"] = _dev(np.where(path < nodes, path, 0))
    if case["kind"] == "fork":
        mine = table[np.arange(b), first]
        lead = np.repeat(mine[::case["group"]], case["group"])
        forks = np.arange(b) % case["group"] != 0
        s["src"], s["dst"] = _dev(lead[forks]), _dev(mine[forks])
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if kind == "tree":
        return _own_tree(s) if own else _plain_tree(s)
    if kind == "window":
        return _own_window(s) if own else _plain_window(s)
    if kind == "append":
        return _own_append(s) if own else _plain_append(s)
    if kind == "fork":
        if own:
            _own_copy(s)
            return _own_append(s)
        _plain_copy(s)
        return _plain_append(s)
    return _own_copy(s) if own else _plain_copy(s)


def _kw(s):
    case, pool = s["case"], s["pool"]
    return {"num_kv_heads": case["kv_heads"], "page_size": case["page"], "kv_dtype": int(case["fp8"]), "k_scales": pool["k_scales"],
            "v_scales": pool["v_scales"]}


def _written(s):
    """The pool after a write; fp8 codes as the values they stand for (before the page's scale, which is there too)."""
    if not s["case"]["fp8"]:
        return {"k": s["pool"]["k"], "v": s["pool"]["v"]}
    return {"k": s["pool"]["k"].view(torch.float8_e4m3fn), "v": s["pool"]["v"].view(torch.float8_e4m3fn), "k_scales": s["pool"]["k_scales"],
            "v_scales": s["pool"]["v_scales"]}


def _own_tree(s):
    from paper_2604_26256_amd import dora
    return dora.dora_decode_attn_tree(s["q"], s["k_draft"], s["v_draft"], s["mask"], s["pool"]["k"], s["pool"]["v"], s["table"], s["lens"], s["versions"],
                                      s["out"], node_counts=s["counts"] if s["case"]["ragged"] else None, **_kw(s))


def _own_window(s):
    from paper_2604_26256_amd import dora
    return dora.dora_decode_attn_window(s["q"], s["pool"]["k"], s["pool"]["v"], s["table"], s["lens"], s["versions"], s["out"],
                                        window=s["case"]["window"], sinks=s["case"]["sinks"], **_kw(s))


def _own_append(s):
    from paper_2604_26256_amd import dora
    dora.dora_kv_append_path(s["k_new"], s["v_new"], s["table"], s["lens"], s["pool"]["k"], s["pool"]["v"], path=s["path"], counts=s["counts"], **_kw(s))
    return _written(s)


def _own_copy(s):
    from paper_2604_26256_amd import dora
    dora.dora_kv_page_copy(s["pool"]["k"], s["pool"]["v"], s["src"], s["dst"], head_dim=s["case"]["d"], **_kw(s))
    return _written(s)


def _widened(pages, scales, ids, case, key):
    """Pages ids [n][m] as 32-bit values [n][Hkv][m * P][d]."""
    x = pages[ids]
    if case["fp8"]:
        x = x.view(torch.float8_e4m3fn).float() * scales[ids].view(ids.shape + (1,) * (x.dim() - 2))
    else:
        x = x.float()
    n, m, heads, p, d = ids.shape[0], ids.shape[1], case["kv_heads"], case["page"], case["d"]
    if key:  # [n][m][Hkv][d / X][P][X]
        return x.permute(0, 2, 1, 4, 3, 5).reshape(n, heads, m * p, d)
    return x.permute(0, 2, 1, 4, 3).reshape(n, heads, m * p, d)


def _partial(q, k, v, seen):
    """Maximum, sum and weighted values over the tokens k, v [n][Hkv][t][d] of the rows q [n][Hkv][C][d]; seen:
    [n][1][C or 1][t]."""
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(q.shape[3]))
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(dim=3)
    weights = torch.exp(scores - torch.where(torch.isinf(top), 0.0, top)[..., None])
    return top, weights.sum(dim=3), torch.matmul(weights, v)


def _over_blocks(q, table, lens, seen_of, first, pages, host_pages, case, pool):
    """Attention partials over blocks of the sequences' pages first .. first + pages - 1 (of the list that `table` holds);
    seen_of(b, page, token in page) says which tokens count.  q: [B][Hkv][C][d], 32 bits."""
    per = BLOCK // case["page"]
    blocks = -(-pages // per)
    total = int(np.sum(-(-host_pages // per)))
    dev = q.device
    b = torch.repeat_interleave(torch.arange(len(pages), device=dev), blocks, output_size=total)
    start = torch.cumsum(blocks, 0) - blocks
    block = torch.arange(total, device=dev) - start[b]
    at = block[:, None] * per + torch.arange(per, device=dev)  # [n][per] in the sequence's list
    there = at < pages[b][:, None]
    j = torch.where(there, first[b][:, None] + at, 0)
    j = torch.minimum(j, torch.full_like(j, table.shape[1] - 1))
    ids = table[b[:, None], j].long()
    token = torch.arange(case["page"], device=dev)
    seen = there[:, :, None] & seen_of(b[:, None, None], j[:, :, None], token[None, None, :])
    seen = seen.reshape(total, 1, 1, per * case["page"])
    k = _widened(pool["k"], pool["k_scales"], ids, case, True)
    v = _widened(pool["v"], pool["v_scales"], ids, case, False)
    top, weight, value = _partial(q[b], k, v, seen)
    # join a sequence's blocks
    shape = q.shape[:3]
    m = torch.full(shape, -math.inf, device=dev).index_reduce_(0, b, top, "amax")
    scale = torch.exp(top - torch.where(torch.isinf(m), 0.0, m)[b])
    weight = torch.zeros(shape, device=dev).index_add_(0, b, weight * scale)
    value = torch.zeros(shape + (case["d"],), device=dev).index_add_(0, b, value * scale[..., None])
    return m, weight, value


def _plain_tree(s):
    case, pool, lens = s["case"], s["pool"], s["lens"].long()
    b, t, hq, d = s["q"].shape
    hkv, p = case["kv_heads"], case["page"]
    g = hq // hkv
    q = s["q"].float().view(b, t, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(b, hkv, t * g, d)
    pages = -(-lens // p)
    seen = lambda i, j, u: j * p + u < lens[i]  # noqa: E731
    m, weight, value = _over_blocks(q, s["table"], lens, seen, torch.zeros_like(pages), pages, -(-s["host_lens"] // p), case, pool)
    bits = torch.arange(t, device=q.device)
    live = bits[None, :] < s["counts"][:, None]  # [B][T]
    see = ((s["mask"][:, :, None] >> bits) & 1).bool() & live[:, None, :]  # [B][node][draft]
    see = see[:, None, :, None, :].expand(b, 1, t, g, t).reshape(b, 1, t * g, t)
    kd, vd = (s[x].float().permute(0, 2, 1, 3).contiguous() for x in ("k_draft", "v_draft"))
    # padded nodes hold anything
    kd, vd = (torch.where(live[:, None, :, None], x, 0.0) for x in (kd, vd))
    m2, weight2, value2 = _partial(q, kd, vd, see)
    top = torch.maximum(m, m2)
    base = torch.where(torch.isinf(top), 0.0, top)
    f, f2 = torch.exp(m - base), torch.exp(m2 - base)
    total = weight * f + weight2 * f2
    out = (value * f[..., None] + value2 * f2[..., None]) / torch.where(total > 0, total, 1.0)[..., None]
    out = out.view(b, hkv, t, g, d).permute(0, 2, 1, 3, 4).reshape(b, t, hq, d).to(torch.bfloat16)
    s["out"].copy_(torch.where(live[:, :, None, None], out, s["out"]))
    return s["out"]


def _plain_window(s):
    case, pool, lens = s["case"], s["pool"], s["lens"].long()
    b, hq, d = s["q"].shape
    hkv, p, sinks = case["kv_heads"], case["page"], case["sinks"]
    q = s["q"].float().view(b, hkv, hq // hkv, d)
    pages = -(-lens // p)
    begin = (lens - case["window"]).clamp_min(0)
    sink = torch.minimum(pages, torch.full_like(pages, -(-sinks // p)))
    first = torch.maximum(sink, begin // p)
    # the sinks' pages in front of the window's: one list a sequence
    n, host_first, host_sink = _visible_pages(case, s["host_lens"])
    host_pages = host_sink + n - host_first
    at = torch.arange(max(1, int(host_pages.max())), device=q.device)[None, :]
    page = torch.where(at < sink[:, None], at, first[:, None] + at - sink[:, None])
    listed = s["table"].gather(1, page.clamp_max(s["table"].shape[1] - 1))

    def seen(i, j, u):
        token = page[i, j] * p + u
        return (token < lens[i]) & ((token < sinks) | (token >= begin[i]))

    m, weight, value = _over_blocks(q, listed, lens, seen, torch.zeros_like(pages), sink + pages - first, host_pages, case, pool)
    out = value / torch.where(weight > 0, weight, 1.0)[..., None]
    s["out"].copy_(out.view(b, hq, d).to(torch.bfloat16))
    return s["out"]


def _plain_copy(s):
    pool, src, dst = s["pool"], s["src"].long(), s["dst"].long()
    pool["k"][dst] = pool["k"][src]
    pool["v"][dst] = pool["v"][src]
    if s["case"]["fp8"]:
        pool["k_scales"][dst] = pool["k_scales"][src]
        pool["v_scales"][dst] = pool["v_scales"][src]
    return _written(s)


def _plain_append(s):
    """bf16: one scatter.  fp8: the slots of the pages in turn (a page's scale follows from its tokens in order), for all
    pages at once."""
    case, pool, p = s["case"], s["pool"], s["case"]["page"]
    total = int(s["host_counts"].sum())
    if total == 0:
        return _written(s)
    counts, dev = s["counts"].long(), s["k_new"].device
    base = s["lens"].long() - counts
    if not case["fp8"]:
        b = torch.repeat_interleave(torch.arange(len(counts), device=dev), counts, output_size=total)
        i = torch.arange(total, device=dev) - (torch.cumsum(counts, 0) - counts)[b]
        t = base[b] + i
        ids, slot = s["table"][b, t // p].long(), t % p
        row = i if s["path"] is None else s["path"][b, i].long()
        pool["k"][ids, :, :, slot] = s["k_new"][b, row].view(total, case["kv_heads"], -1, 8)
        pool["v"][ids, :, :, slot] = s["v_new"][b, row]
        return _written(s)
    host_first = s["host_base"] // p
    touched = int((-(-(s["host_base"] + s["host_counts"]) // p) - host_first)[s["host_counts"] > 0].sum())
    first = base // p
    pages = torch.where(counts > 0, -(-(base + counts) // p) - first, 0)
    b = torch.repeat_interleave(torch.arange(len(counts), device=dev), pages, output_size=touched)
    j = first[b] + torch.arange(touched, device=dev) - (torch.cumsum(pages, 0) - pages)[b]
    ids = s["table"][b, j].long()
    for name, new, key in (("k", s["k_new"], True), ("v", s["v_new"], False)):
        scale = pool[name + "_scales"][ids]
        # [page][Hkv * d][slot]
        codes = pool[name][ids].view(torch.float8_e4m3fn)
        codes = (codes.view(touched, -1, p, 16).float().transpose(2, 3) if key else codes.view(touched, -1, p).float()).reshape(touched, -1, p)
        for u in range(p):
            i = j * p + u - base[b]
            here = (i >= 0) & (i < counts[b])
            i = i.clamp(0, new.shape[1] - 1)
            x = new[b, i if s["path"] is None else s["path"][b, i].long()].float().view(touched, -1)
            fresh = (x.abs().amax(dim=1) / FP8_MAX).clamp_min(2.0 ** -126)
            grow = here & ~(fresh <= scale) if u else torch.zeros_like(here)
            s1 = torch.where(here & (fresh > scale if u else here), fresh, scale)
            if u:
                again = _code(codes[:, :, :u] * scale[:, None, None] / s1[:, None, None])
                codes[:, :, :u] = torch.where(grow[:, None, None], again, codes[:, :, :u])
            codes[:, :, u] = torch.where(here[:, None], _code(x / s1[:, None]), codes[:, :, u])
            scale = s1
        codes = codes.view(touched, -1, 16, p).transpose(2, 3) if key else codes
        pool[name].view(torch.uint8)[ids] = codes.to(torch.float8_e4m3fn).reshape((touched,) + pool[name].shape[1:]).view(torch.uint8)
        pool[name + "_scales"][ids] = scale
    return _written(s)


def _code(x):
    """The nearest fp8 value, ties to even, saturating."""
    return x.clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).float()


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it gives in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    e = 1 if case["fp8"] else 2
    row = case["kv_heads"] * case["d"]  # values of one token's K (or V)
    page_bytes = 2 * (case["page"] * row * e + (4 if case["fp8"] else 0))
    if case["kind"] == "compact":
        return {"bytes": 2 * case["moves"] * page_bytes + 8 * case["moves"], "flops": 0}
    if case["kind"] == "fork":  # a group's page read once; a token of each read and stored, its entry, length and count, a page's scales
        copies = case["seqs"] // case["group"] * (case["group"] - 1)
        size = (copies + case["seqs"] // case["group"]) * page_bytes + 8 * copies
        return {"bytes": size + case["seqs"] * (2 * row * 2 + 2 * row * e + 12 + (16 if case["fp8"] else 0)), "flops": 0}
    if case["kind"] == "append":  # each token read and stored, its place in the path, a page's entry and scales, lengths and counts
        tokens = int(_counts(case).sum())
        pages = tokens // case["page"] + int((_counts(case) > 0).sum())
        size = tokens * (2 * row * 2 + 2 * row * e + (4 if case["path"] else 0)) + pages * (4 + (16 if case["fp8"] else 0))
        return {"bytes": size + 8 * case["seqs"], "flops": 0}
    lens = _lengths(case)
    if case["kind"] == "window":
        begin = np.maximum(0, lens - case["window"])
        tokens = int((lens - begin + np.minimum(begin, case["sinks"])).sum())
        n, first, sink = _visible_pages(case, lens)
        pages = int((sink + n - first).sum())
        rows, extra, pairs = case["seqs"], 0, tokens
    else:
        counts = _counts(case)
        tokens, pages = int(lens.sum()), int((-(-lens // case["page"])).sum())
        rows = int(counts.sum())
        extra = rows * (2 * row * 2 + 8) + 4 * case["seqs"]
        pairs = int((lens * counts).sum()) + rows  # and at least itself
    size = tokens * 2 * row * e + pages * ((8 if case["fp8"] else 0) + 4) + 4 * case["seqs"]
    return {"bytes": size + 2 * rows * case["q_heads"] * case["d"] * 2 + extra, "flops": 4 * pairs * case["q_heads"] * case["d"]}


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] in ("tree", "window"):
        return _exact_attention(s)
    pool = {k: None if x is None else x.clone() for k, x in s["pool"].items()}
    if "src" in s:
        for i, j in zip(s["src"].tolist(), s["dst"].tolist()):
            for name in ("k", "v") + (("k_scales", "v_scales") if case["fp8"] else ()):
                pool[name][j] = s["pool"][name][i]
    if case["kind"] != "compact":
        pool = _exact_append(s, pool)
    if not case["fp8"]:
        return {"k": pool["k"], "v": pool["v"]}
    if case["kind"] == "compact":
        return dict(pool, k=pool["k"].view(torch.float8_e4m3fn), v=pool["v"].view(torch.float8_e4m3fn))
    return {"k": None, "v": None, "k_scales": pool["k_scales"].double(), "v_scales": pool["v_scales"].double()}


def _exact_append(s, pool):
    """bf16: token by token.  fp8: a page's scale is its largest token's, or the one it had (the codes, rounded once or
    more, have no 64-bit value of their own)."""
    case, p = s["case"], s["case"]["page"]
    table = s["table"].cpu().numpy()
    if case["fp8"]:
        pool = dict(pool, k_scales=pool["k_scales"].double(), v_scales=pool["v_scales"].double())
    path = None if s["path"] is None else s["path"].cpu().numpy()
    for b in range(len(table)):
        n = int(s["host_counts"][b])
        if n == 0:
            continue
        rows = torch.from_numpy(np.arange(n) if path is None else path[b, :n].astype(np.int64)).cuda()
        t = int(s["host_base"][b]) + np.arange(n)
        for j in range(t[0] // p, t[-1] // p + 1):
            at = np.nonzero(t // p == j)[0]
            page = int(table[b, j])
            for x in "kv":
                tokens = s[x + "_new"][b, rows[at[0]:at[-1] + 1]]
                lo, hi = int(t[at[0]]) - j * p, int(t[at[-1]]) - j * p + 1
                if case["fp8"]:
                    fresh = (tokens.double().abs().max() / FP8_MAX).clamp_min(2.0 ** -126)
                    pool[x + "_scales"][page] = fresh if lo == 0 else torch.maximum(fresh, pool[x + "_scales"][page])
                elif x == "k":
                    pool["k"][page, :, :, lo:hi] = tokens.view(hi - lo, case["kv_heads"], -1, 8).permute(1, 2, 0, 3)
                else:
                    pool["v"][page, :, :, lo:hi] = tokens.permute(1, 2, 0)
    return pool


def _exact_attention(s):
    """Sequence by sequence, in 64 bits: the visible tokens by their numbers, each read from its page and slot."""
    case, pool, p = s["case"], s["pool"], s["case"]["page"]
    hkv, d = case["kv_heads"], case["d"]
    out = s["out"].double()
    for b, length in enumerate(s["host_lens"].tolist()):
        t = torch.arange(length, device="cuda")
        if case["kind"] == "window":
            t = t[(t < case["sinks"]) | (t >= length - case["window"])]
        ids, slot = s["table"][b, t // p].long(), t % p
        k, v = pool["k"][ids, :, :, slot], pool["v"][ids, :, :, slot]
        if case["fp8"]:
            k = k.view(torch.float8_e4m3fn).float().double() * pool["k_scales"][ids].double().view(-1, 1, 1, 1)
            v = v.view(torch.float8_e4m3fn).float().double() * pool["v_scales"][ids].double().view(-1, 1, 1)
        k, v = k.double().reshape(-1, hkv, d), v.double().reshape(-1, hkv, d)
        nodes = 1
        if case["kind"] == "tree":
            nodes = int(s["counts"][b])
            k, v = torch.cat([k, s["k_draft"][b, :nodes].double()]), torch.cat([v, s["v_draft"][b, :nodes].double()])
        q = (s["q"][b, :nodes] if case["kind"] == "tree" else s["q"][b][None]).double().view(nodes, hkv, -1, d)
        for h in range(hkv):
            x = torch.matmul(q[:, h].reshape(-1, d), k[:, h].T.contiguous()).view(nodes, -1, k.shape[0]) * d ** -0.5
            if case["kind"] == "tree":
                bit = (s["mask"][b, :nodes, None] >> torch.arange(nodes, device="cuda")) & 1
                x[:, :, length:] += torch.where(bit.bool(), 0.0, -math.inf)[:, None]
            if x.shape[2]:
                y = torch.matmul(torch.softmax(x, dim=2).view(-1, x.shape[2]), v[:, h].contiguous()).view(nodes, -1, d)
            else:
                y = torch.zeros_like(q[:, h])
            g = y.shape[1]
            if case["kind"] == "tree":
                out[b, :nodes, h * g:(h + 1) * g] = y
            else:
                out[b, h * g:(h + 1) * g] = y[0]
    return out
