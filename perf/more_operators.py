"""Operators that read less of the paged cache, as they are timed: each in a plain form, and as the library's calls.

A case is a dict of plain values; its lengths follow from the case alone (so that its bytes are known), all other inputs
from the seed.  Kinds:

  decode4  decode attention over pages of 4 bits a value
  store4   several tokens of every sequence written into 4-bit pages, and read back as bf16 rows
  bounds   the bounds of the keys of every page that the last tokens of a sequence lie in
  select   for each sequence and KV head the pages whose bounds promise the largest scores
  pages    decode attention over a list of pages for each sequence and KV head

A 4-bit page is a tile of bytes for each KV head.  K: E2M1 codes [d / 32][P][32] (two in a byte, the even one in its low
half), then a power of two for each 32 dims of a token, as its exponent with a bias of 127, [d / 32][P / 16][4][4] (slot
16 a + 4 b + c at [a][c][b]).  V: E2M1 codes [d][P], then a bf16 scale for each 64 dims of a token, [d / 64][P].  A page's
bounds are, for each KV head, int8 [2][d] (the largest and smallest value of each dim), and behind those of all heads a
32-bit scale for each.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 256  # tokens of a block of the plain attention
FP8_MAX = 448.0
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
HALFWAY = (0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)  # between two of them; the even code wins a tie
BF16_MAX = 3.3895313892515355e38
TINY = 2.0 ** -126


def listed():
    return [
        # a small model's latency-bound loop over a handful of short sequences
        {"name": "decode4_tiny", "kind": "decode4", "dtype": "fp4", "seqs": 8, "q_heads": 8, "kv_heads": 2, "d": 64, "page": 16, "median": 256, "sigma": 1.0,
         "lo": 1, "hi": 2048},
        # a 7B-class long-tailed rollout batch
        {"name": "decode4_rollout7b", "kind": "decode4", "dtype": "fp4", "seqs": 64, "q_heads": 28, "kv_heads": 4, "d": 128, "page": 16, "median": 2048, "sigma": 1.2,
         "lo": 64, "hi": 32768},
        # a larger model's full batch, where bytes alone count
        {"name": "decode4_moe", "kind": "decode4", "dtype": "fp4", "seqs": 256, "q_heads": 64, "kv_heads": 8, "d": 128, "page": 32, "median": 4096, "sigma": 1.0,
         "lo": 128, "hi": 32768},
        # one to eight accepted tokens of each sequence of a rollout batch
        {"name": "store4_path7b", "kind": "store4", "dtype": "fp4", "seqs": 64, "kv_heads": 4, "d": 128, "page": 16, "tokens": 8, "least": 1},
        # a chunk of new prompts: hundreds of tokens of each sequence in order
        {"name": "store4_prompt", "kind": "store4", "dtype": "fp4", "seqs": 24, "kv_heads": 8, "d": 128, "page": 32, "tokens": 700, "least": 300},
        # after each step of the largest batch: the page that the newest token lies in
        {"name": "bounds_step", "kind": "bounds", "dtype": "bf16", "seqs": 1024, "kv_heads": 8, "d": 128, "page": 16, "tokens": 1, "least": 1},
        # after a chunk of new prompts over fp8 pages
        {"name": "bounds_prompt_fp8", "kind": "bounds", "dtype": "fp8", "seqs": 24, "kv_heads": 8, "d": 128, "page": 32, "tokens": 1900, "least": 900},
        # a few sequences of a small model
        {"name": "select_tiny", "kind": "select", "seqs": 8, "q_heads": 8, "kv_heads": 2, "d": 64, "page": 16, "budget": 16, "sinks": 1, "recent": 2,
         "median": 1000, "sigma": 1.0, "lo": 1, "hi": 8192},
        # the long tail of a rollout: every sequence far longer than what is read of it
        {"name": "select_tail", "kind": "select", "seqs": 64, "q_heads": 64, "kv_heads": 8, "d": 128, "page": 16, "budget": 128, "sinks": 1, "recent": 4,
         "median": 32768, "sigma": 0.8, "lo": 1024, "hi": 131072},
        # what the tail's selection lists, in bf16: 2,048 tokens of each row
        {"name": "pages_tail", "kind": "pages", "dtype": "bf16", "seqs": 64, "q_heads": 64, "kv_heads": 8, "d": 128, "page": 16, "budget": 128,
         "median": 32768, "sigma": 0.8, "lo": 1024, "hi": 131072},
        # a full fp8 batch, rows shorter than the budget among far longer ones
        {"name": "pages_moe_fp8", "kind": "pages", "dtype": "fp8", "seqs": 500, "q_heads": 64, "kv_heads": 8, "d": 128, "page": 32, "budget": 100,
         "median": 4096, "sigma": 1.2, "lo": 16, "hi": 65536},
        # the same over 4-bit pages, 7 query heads a KV head
        {"name": "pages_fp4", "kind": "pages", "dtype": "fp4", "seqs": 256, "q_heads": 28, "kv_heads": 4, "d": 128, "page": 16, "budget": 160,
         "median": 8192, "sigma": 1.0, "lo": 16, "hi": 65536},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["decode4", "decode4", "pages", "pages", "pages", "select", "select", "store4", "bounds"])
    case = {"kind": kind, "d": rng.choice([64, 128, 128]), "page": rng.choice([16, 32]), "kv_heads": rng.choice([1, 2, 4, 8])}
    if kind != "select":
        case["dtype"] = "fp4" if kind in ("decode4", "store4") else rng.choice(["bf16", "fp8", "fp4"])
    if kind in ("store4", "bounds"):
        case["tokens"] = _log(rng, 1, 1200)
        case["seqs"] = min(_log(rng, 1, 1024), max(1, 24576 // case["tokens"]))
        case["least"] = rng.choice([0, min(1, case["tokens"]), case["tokens"] // 2, case["tokens"]])
        return case
    heads = rng.choice([1, 2, 4, 6, 7, 8, 16])
    case.update(q_heads=heads * case["kv_heads"], median=_log(rng, 32, 32768), sigma=rng.uniform(0.0, 1.3), lo=rng.choice([0, 1]))
    row = case["kv_heads"] * case["d"]
    if kind == "decode4":  # at most 1 Gi values of keys and values
        case["seqs"] = _log(rng, 1, 256)
        case["hi"] = max(32, min(65536, 16 * case["median"], (1 << 30) // (2 * row * case["seqs"])))
        return case
    case["budget"] = _log(rng, 3, 200)
    case["hi"] = max(32, min(131072, 16 * case["median"]))
    if kind == "select":
        case.update(sinks=rng.choice([0, 1, 2]), recent=rng.choice([0, 1, 1]))
        case["seqs"] = min(_log(rng, 1, 256), max(1, (1 << 22) // (case["hi"] // case["page"] * case["kv_heads"])))
    else:
        case["seqs"] = max(1, min(_log(rng, 1, 500), (1 << 29) // (row * min(case["budget"] * case["page"], case["hi"]))))
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _rng(case):
    return np.random.default_rng(case["seqs"] * 1000003 + case.get("median", 0) * 31 + case.get("tokens", 0))


def _lengths(case):
    """Tokens in the cache of each sequence: lognormal, clipped, the same for every seed of the case."""
    x = np.exp(_rng(case).normal(math.log(case["median"]), case["sigma"], case["seqs"]))
    return np.clip(np.rint(x), case["lo"], case["hi"]).astype(np.int64)


def _counts(case):
    """Tokens of each sequence that a write or its bounds take."""
    return _rng(case).integers(case["least"], case["tokens"] + 1, case["seqs"])


def _tile(case):
    return case["page"] * case["d"] * 17 // 32


def _e2m1(y):
    """The code of the nearest value, of an even one at a tie; what is larger than 6 is 6."""
    a = y.abs()
    code = torch.zeros_like(a, dtype=torch.uint8)
    for i, h in enumerate(HALFWAY):
        code += (a > h) if i % 2 == 0 else (a >= h)
    return code | (torch.signbit(y).to(torch.uint8) << 3)


def _pairs(codes):
    return codes[..., 0::2] | (codes[..., 1::2] << 4)


def _key_bytes(x):
    """Exponents (biased by 127) and codes of keys [...][32], 32 bits: the largest value lies below 7 of its power of two."""
    top = x.abs().amax(dim=-1)
    # in bf16's bits: 2 below the exponent, or 1 where the mantissa is 1.75 or more
    power = (((top.to(torch.bfloat16).view(torch.int16).int() + 0x20) >> 7) - 2).clamp(1, 252)
    return power, _e2m1(x / (power << 23).view(torch.float32)[..., None])


def _value_bytes(x):
    """Scales (bf16) and codes of values [...][64], 32 bits: the largest value is 6 steps."""
    top = x.abs().amax(dim=-1).clamp_max(BF16_MAX)
    scale = (top.double() / 6.0).float().to(torch.bfloat16).clamp_min(TINY)
    return scale, _e2m1((x.double() / scale.double()[..., None]).float())


def _key_tiles(x, case):
    """Tiles [n][Hkv][bytes] of keys [n][Hkv][P][d], 32 bits."""
    n, heads, p, d = x.shape
    power, codes = _key_bytes(x.view(n, heads, p, d // 32, 32).transpose(2, 3).contiguous())
    order = power.to(torch.uint8).view(n, heads, d // 32, p // 16, 4, 4).transpose(4, 5)
    return torch.cat([_pairs(codes).reshape(n, heads, -1), order.reshape(n, heads, -1)], dim=2)


def _value_tiles(x, case):
    """Tiles [n][Hkv][bytes] of values [n][Hkv][P][d], 32 bits."""
    n, heads, p, d = x.shape
    scale, codes = _value_bytes(x.view(n, heads, p, d // 64, 64).transpose(2, 3).contiguous())
    codes = codes.permute(0, 1, 2, 4, 3).reshape(n, heads, d, p)
    return torch.cat([_pairs(codes).reshape(n, heads, -1), scale.view(torch.uint8).reshape(n, heads, -1)], dim=2)


def _pages(case, n, key, gen):
    """n pages of N(0, 1) keys or values, and fp8's scales."""
    heads, p, d, dtype = case["kv_heads"], case["page"], case["d"], case["dtype"]
    x = 16 if dtype == "fp8" else 8
    shape = (heads, _tile(case)) if dtype == "fp4" else (heads, d // x, p, x) if key else (heads, d, p)
    if dtype == "bf16":
        return torch.empty((n,) + shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen), None
    t = torch.empty((n,) + shape, dtype=torch.uint8, device="cuda")
    scales = torch.empty(n, dtype=torch.float32, device="cuda") if dtype == "fp8" else None
    step = max(1, (1 << 26) // (heads * p * d))
    for i in range(0, n, step):
        m = min(step, n - i)
        v = torch.empty((m, heads, p, d), dtype=torch.float32, device="cuda").normal_(generator=gen)
        if dtype == "fp4":
            v = v.to(torch.bfloat16).float()
            t[i:i + m] = _key_tiles(v, case) if key else _value_tiles(v, case)
        else:
            s = v.abs().amax(dim=(1, 2, 3)) / FP8_MAX
            scales[i:i + m] = s
            t[i:i + m] = (v / s[:, None, None, None]).clamp_(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8).view((m,) + shape)
    return t, scales


def _pool(case, n, gen, values=True):
    k, k_scales = _pages(case, n, True, gen)
    v, v_scales = _pages(case, n, False, gen) if values else (None, None)
    return {"k": k, "v": v, "k_scales": k_scales, "v_scales": v_scales}


def _dev(x, dtype=np.int32):
    return torch.from_numpy(np.ascontiguousarray(x, dtype=dtype)).cuda()


def _normal(shape, gen):
    return torch.empty(shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


def _scattered(rng, n):
    """A table whose row b has n[b] distinct pages of a pool that they nearly fill, and that pool's pages."""
    total = int(n.sum())
    num_pages = total + total // 8 + 1
    perm = rng.permutation(num_pages)
    table = np.zeros((len(n), max(1, int(n.max()))), np.int32)
    at = np.arange(table.shape[1])[None, :]
    table[at < n[:, None]] = perm[:total]
    return table, num_pages


def _record(case):
    """Bytes of a page's bounds."""
    return -(-case["kv_heads"] * (2 * case["d"] + 4) // 16) * 16


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.default_rng(seed)
    page = case["page"]
    if case["kind"] in ("store4", "bounds"):
        return _prepare_write(case, gen, rng)
    lens = _lengths(case)
    n = -(-lens // page)
    if case["kind"] == "pages":
        return _prepare_pages(case, gen, rng, lens, n)
    table, num_pages = _scattered(rng, n)
    s = {"case": case, "table": _dev(table), "lens": _dev(lens), "host_lens": lens, "versions": _dev(0 * lens)}
    s["q"] = _normal((len(lens), case["q_heads"], case["d"]), gen)
    if case["kind"] == "decode4":
        s["pool"] = _pool(case, num_pages, gen)
        s["out"] = torch.zeros_like(s["q"])
        return s
    # select: keys of a page lie about a mean of their own
    b, heads, d = len(lens), case["kv_heads"], case["d"]
    mean = torch.empty((num_pages, heads, d), device="cuda").normal_(0.0, 0.7, generator=gen)
    reach = torch.empty((2, num_pages, heads, d), device="cuda").uniform_(0.5, 2.5, generator=gen)
    s["bounds"] = torch.zeros((num_pages, _record(case)), dtype=torch.uint8, device="cuda")
    _put_bounds(s["bounds"], torch.arange(num_pages, device="cuda"), mean + reach[0], mean - reach[1], case)
    s["lists"] = torch.full((b, heads, case["budget"]), -1, dtype=torch.int32, device="cuda")
    s["counts"] = torch.zeros((b, heads), dtype=torch.int32, device="cuda")
    s["scores"] = torch.zeros((b, heads, table.shape[1]), dtype=torch.float32, device="cuda")
    return s


def _prepare_pages(case, gen, rng, lens, n):
    """Every head lists min(n, budget) pages of a sequence, its first and its last among them; the table's other entries
    are 0 and are never read."""
    b, heads = len(lens), case["kv_heads"]
    count = np.minimum(n, case["budget"])
    width = max(1, int(n.max()))
    # each sequence's heads pick from a pool of pages that any of them lists
    lists = np.full((b, heads, case["budget"]), -1, np.int64)
    used = np.zeros((b, width), bool)
    for i in range(b):
        if n[i] == 0:
            continue
        inner = max(0, int(count[i]) - 2)
        keys = rng.random((heads, max(0, int(n[i]) - 2)))
        pick = np.sort(np.argsort(keys, axis=1)[:, :inner], axis=1) + 1
        ends = [np.zeros((heads, 1), np.int64)] + ([pick] if inner else []) + ([np.full((heads, 1), n[i] - 1)] if n[i] > 1 else [])
        lists[i, :, :count[i]] = np.concatenate(ends, axis=1)[:, :count[i]] if count[i] > 1 else n[i] - 1
        used[i, lists[i, :, :count[i]].ravel()] = True
    small, num_pages = _scattered(rng, used.sum(axis=1))
    table = np.zeros((b, width), np.int32)
    table[used] = small[np.arange(small.shape[1])[None, :] < used.sum(axis=1)[:, None]]
    s = {"case": case, "pool": _pool(case, num_pages, gen), "table": _dev(table), "lens": _dev(lens), "host_lens": lens, "versions": _dev(0 * lens)}
    s["lists"], s["counts"] = _dev(lists), _dev(np.repeat(count[:, None], heads, axis=1))
    s["q"] = _normal((b, case["q_heads"], case["d"]), gen)
    s["out"] = torch.zeros_like(s["q"])
    return s


def _prepare_write(case, gen, rng):
    """Sequences somewhere in a page, and the tokens that come next (store4) or have just come (bounds).  The table has
    random entries where nothing is looked at."""
    b, page = case["seqs"], case["page"]
    counts = _counts(case)
    base = _rng(case).integers(0, 64 * page, b)  # tokens before them
    lens = base + counts
    first, last = base // page, -(-lens // page)
    touched = np.where(counts > 0, last - first, 0)
    own_pages, num_pages = _scattered(rng, np.maximum(touched, 1))
    table = rng.integers(0, num_pages, (b, int(max(last.max(), first.max() + 1)) + 2)).astype(np.int32)
    for i in range(b):
        table[i, first[i]:first[i] + max(1, touched[i])] = own_pages[i, :max(1, touched[i])]
    s = {"case": case, "pool": _pool(case, num_pages, gen, values=case["kind"] == "store4"), "table": _dev(table), "lens": _dev(lens), "counts": _dev(counts),
         "host_base": base, "host_counts": counts}
    if case["kind"] == "store4":
        s["k_new"], s["v_new"] = (_normal((b, case["tokens"], case["kv_heads"], case["d"]), gen) for _ in range(2))
        s["k_out"], s["v_out"] = (torch.zeros_like(s["k_new"]) for _ in range(2))
    else:
        s["bounds"] = torch.zeros((num_pages, _record(case)), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    kind = s["case"]["kind"]
    if kind == "decode4":
        return _own_decode(s) if own else _plain_decode(s)
    if kind == "store4":
        return _own_store(s) if own else _plain_store(s)
    if kind == "bounds":
        return _own_bounds(s) if own else _plain_bounds(s)
    if kind == "select":
        return _own_select(s) if own else _plain_select(s)
    return _own_pages(s) if own else _plain_pages(s)


def _kw(s):
    case, pool = s["case"], s["pool"]
    return {"num_kv_heads": case["kv_heads"], "page_size": case["page"], "kv_dtype": {"bf16": 0, "fp8": 1, "fp4": 4}[case["dtype"]], "k_scales": pool["k_scales"]}


def _bounds_of(bounds, case):
    """A view of the bounds as they are held: int8 and the scales that are beside them."""
    heads, d = case["kv_heads"], case["d"]
    edge = bounds[:, :heads * 2 * d].view(torch.int8)
    return {"edge": edge, "scale": bounds[:, heads * 2 * d:heads * (2 * d + 4)].view(torch.float32)}


def _own_decode(s):
    from paper_2604_26256_amd import dora
    return dora.dora_decode_attn(s["q"], s["pool"]["k"], s["pool"]["v"], s["table"], s["lens"], s["versions"], s["out"], **_kw(s))


def _own_store(s):
    from paper_2604_26256_amd import dora
    dora.dora_kv_append_path(s["k_new"], s["v_new"], s["table"], s["lens"], s["pool"]["k"], s["pool"]["v"], counts=s["counts"], **_kw(s))
    dora.dora_kv_read(s["pool"]["k"], s["pool"]["v"], s["table"], s["lens"], s["k_out"], s["v_out"], counts=s["counts"], **_kw(s))
    return {"k": s["k_out"], "v": s["v_out"]}


def _own_bounds(s):
    from paper_2604_26256_amd import dora
    dora.dora_kv_page_bounds(s["pool"]["k"], s["table"], s["lens"], s["bounds"], num_tokens=s["case"]["tokens"], head_dim=s["case"]["d"], counts=s["counts"], **_kw(s))
    return _bounds_of(s["bounds"], s["case"])


def _own_select(s):
    from paper_2604_26256_amd import dora
    case = s["case"]
    dora.dora_page_select(s["q"], s["bounds"], s["table"], s["lens"], s["lists"], s["counts"], num_kv_heads=case["kv_heads"], page_size=case["page"],
                          sink_pages=case["sinks"], recent_pages=case["recent"], scores=s["scores"])
    return {"lists": s["lists"], "counts": s["counts"], "scores": s["scores"]}


def _own_pages(s):
    from paper_2604_26256_amd import dora
    return dora.dora_decode_attn_pages(s["q"], s["lists"], s["counts"], s["pool"]["k"], s["pool"]["v"], s["table"], s["lens"], s["versions"], s["out"],
                                       v_scales=s["pool"]["v_scales"], **_kw(s))


def _halves(b):
    """The values of E2M1 codes, two a byte: [...][n] -> [...][2 n]."""
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=b.device)
    return torch.stack([table[(b & 15).long()], table[(b >> 4).long()]], dim=-1).flatten(-2)


def _widened(pages, scales, ids, case, key):
    """Pages ids [...] as 32-bit values [...][Hkv][P][d]; a KV head of its own for each where the ids' last axis is Hkv."""
    heads, p, d = case["kv_heads"], case["page"], case["d"]
    by_head = isinstance(ids, tuple)  # (ids [...][Hkv], heads [Hkv])
    x = pages[ids]
    lead = x.shape[:ids[0].dim() - 1] if by_head else x.shape[:ids.dim()]
    if case["dtype"] == "fp4":
        codes = _halves(x[..., :p * d // 2])
        rest = x[..., p * d // 2:].contiguous()
        if key:
            power = rest.view(lead + (heads, d // 32, p // 16, 4, 4)).transpose(-1, -2).reshape(lead + (heads, d // 32, p))
            x = codes.view(lead + (heads, d // 32, p, 32)) * (power.int() << 23).view(torch.float32)[..., None]
            return x.transpose(-3, -2).reshape(lead + (heads, p, d))
        scale = rest.view(torch.bfloat16).float().view(lead + (heads, d // 64, 1, p))
        return (codes.view(lead + (heads, d // 64, 64, p)) * scale).view(lead + (heads, d, p)).transpose(-1, -2)
    if case["dtype"] == "fp8":
        scale = scales[ids[0]] if by_head else scales[ids][..., None]
        x = x.view(torch.float8_e4m3fn).float() * scale.view(scale.shape + (1,) * (x.dim() - scale.dim()))
    else:
        x = x.float()
    if key:  # [...][Hkv][d / X][P][X]
        return x.transpose(-3, -2).reshape(lead + (heads, p, d))
    return x.transpose(-1, -2)


def _attend(q, k, v, seen):
    """Maximum, sum and weighted values over the tokens k, v [n][Hkv][t][d] of the rows q [n][Hkv][G][d]; seen: [n][Hkv or 1][1][t]."""
    scores = torch.matmul(q, k.transpose(2, 3).contiguous()) * (1.0 / math.sqrt(q.shape[3]))
    scores = torch.where(seen, scores, -math.inf)
    top = scores.amax(dim=3)
    weights = torch.exp(scores - torch.where(torch.isinf(top), 0.0, top)[..., None])
    return top, weights.sum(dim=3), torch.matmul(weights, torch.where(seen.transpose(2, 3), v, 0.0))


def _joined(q, b, top, weight, value, s):
    """The rows' outputs from their blocks' partials, block i of sequence b[i]."""
    m = torch.full(q.shape[:3], -math.inf, device=q.device).index_reduce_(0, b, top, "amax")
    scale = torch.exp(top - torch.where(torch.isinf(m), 0.0, m)[b])
    weight = torch.zeros(q.shape[:3], device=q.device).index_add_(0, b, weight * scale)
    value = torch.zeros(q.shape, device=q.device).index_add_(0, b, value * scale[..., None])
    out = value / torch.where(weight > 0, weight, 1.0)[..., None]
    s["out"].copy_(out.view(s["out"].shape).to(torch.bfloat16))
    return s["out"]


def _blocks(per_row, host_rows, per):
    """Blocks of `per` pages of rows of per_row[b] pages: each block's row and first page in it."""
    blocks = -(-per_row // per)
    total = int(np.sum(-(-host_rows // per)))
    b = torch.repeat_interleave(torch.arange(len(per_row), device=per_row.device), blocks, output_size=total)
    start = torch.cumsum(blocks, 0) - blocks
    return b, (torch.arange(total, device=per_row.device) - start[b]) * per


def _plain_decode(s):
    case, pool, lens, p = s["case"], s["pool"], s["lens"].long(), s["case"]["page"]
    heads, d = case["kv_heads"], case["d"]
    q = s["q"].float().view(len(lens), heads, -1, d)
    per = BLOCK // p
    pages = -(-lens // p)
    b, first = _blocks(pages, -(-s["host_lens"] // p), per)
    j = first[:, None] + torch.arange(per, device=q.device)
    ids = s["table"][b[:, None], torch.where(j < pages[b][:, None], j, 0)].long()
    seen = (j[:, :, None] * p + torch.arange(p, device=q.device)).flatten(1) < lens[b][:, None]
    k = _widened(pool["k"], pool["k_scales"], ids, case, True).transpose(1, 2).reshape(len(b), heads, BLOCK, d)
    v = _widened(pool["v"], pool["v_scales"], ids, case, False).transpose(1, 2).reshape(len(b), heads, BLOCK, d)
    return _joined(q, b, *_attend(q[b], k, v, seen[:, None, None, :]), s)


def _plain_pages(s):
    case, pool, lens, p = s["case"], s["pool"], s["lens"].long(), s["case"]["page"]
    heads, d = case["kv_heads"], case["d"]
    q = s["q"].float().view(len(lens), heads, -1, d)
    per = BLOCK // p
    counts = s["counts"].long()
    host = np.minimum(-(-s["host_lens"] // p), case["budget"])
    b, first = _blocks(counts[:, 0], host, per)
    at = first[:, None] + torch.arange(per, device=q.device)  # [n][per], places in the lists
    there = at[:, :, None] < counts[b][:, None, :]  # [n][per][Hkv]
    j = s["lists"][b[:, None], :, at.clamp_max(case["budget"] - 1)].long()
    j = torch.where(there, j, 0)
    ids = s["table"][b[:, None, None], j].long()
    token = j[..., None] * p + torch.arange(p, device=q.device)
    seen = (there[..., None] & (token < lens[b][:, None, None, None])).transpose(1, 2).reshape(len(b), heads, 1, per * p)
    head = torch.arange(heads, device=q.device)
    k = _widened(pool["k"], pool["k_scales"], (ids, head), case, True).transpose(1, 2).reshape(len(b), heads, per * p, d)
    v = _widened(pool["v"], pool["v_scales"], (ids, head), case, False).transpose(1, 2).reshape(len(b), heads, per * p, d)
    return _joined(q, b, *_attend(q[b], k, v, seen), s)


def _token_places(s, total):
    """Of every token of a write: its sequence, its number in the write, its page and its slot."""
    counts, p = s["counts"].long(), s["case"]["page"]
    b = torch.repeat_interleave(torch.arange(len(counts), device=counts.device), counts, output_size=total)
    i = torch.arange(total, device=counts.device) - (torch.cumsum(counts, 0) - counts)[b]
    t = (s["lens"].long() - counts)[b] + i
    return b, i, s["table"][b, t // p].long(), t % p


def _plain_store(s):
    """Whole pages: widened to codes and scales, the tokens put into them, and laid out again."""
    case, pool, p, d, heads = s["case"], s["pool"], s["case"]["page"], s["case"]["d"], s["case"]["kv_heads"]
    total = int(s["host_counts"].sum())
    b, i, ids, slot = _token_places(s, total)
    n = pool["k"].shape[0]
    power, codes = _key_bytes(s["k_new"][b, i].float().view(total, heads, d // 32, 32))
    k = pool["k"][..., :p * d // 2].view(n, heads, d // 32, p, 16)
    k[ids, :, :, slot] = _pairs(codes)
    pool["k"][..., p * d // 2:].view(n, heads, d // 32, p // 16, 4, 4)[ids, :, :, slot // 16, slot % 4, slot % 16 // 4] = power.to(torch.uint8)
    scale, codes = _value_bytes(s["v_new"][b, i].float().view(total, heads, d // 64, 64))
    packed = pool["v"][..., :p * d // 2].view(n, heads, d, p // 2)
    wide = torch.stack([packed & 15, packed >> 4], dim=-1).view(n, heads, d, p)
    wide[ids, :, :, slot] = codes.view(total, heads, d)
    pool["v"][..., :p * d // 2] = _pairs(wide).view(n, heads, -1)
    pool["v"][..., p * d // 2:].view(torch.bfloat16).view(n, heads, d // 64, p)[ids, :, :, slot] = scale
    # and back
    k = _halves(k[ids, :, :, slot])
    power = pool["k"][..., p * d // 2:].view(n, heads, d // 32, p // 16, 4, 4)[ids, :, :, slot // 16, slot % 4, slot % 16 // 4]
    s["k_out"][b, i] = (k * (power.int() << 23).view(torch.float32)[..., None]).view(total, heads, d).to(torch.bfloat16)
    packed = pool["v"][..., :p * d // 2].view(n, heads, d, p // 2)[ids, :, :, slot // 2]
    v = _halves(packed[..., None])[torch.arange(total, device=ids.device), :, :, slot % 2].view(total, heads, d // 64, 64)
    scale = pool["v"][..., p * d // 2:].view(torch.bfloat16).view(n, heads, d // 64, p)[ids, :, :, slot]
    s["v_out"][b, i] = (v * scale.float()[..., None]).view(total, heads, d).to(torch.bfloat16)
    return {"k": s["k_out"], "v": s["v_out"]}


def _put_bounds(bounds, ids, high, low, case):
    """Bounds of the pages ids from their largest and smallest values [n][Hkv][d], 32 bits: the quotients by a scale, in
    32 bits, rounded away from each other."""
    heads, d = case["kv_heads"], case["d"]
    scale = (torch.maximum(high.abs(), low.abs()).amax(dim=2).double() / 127.0).float().clamp_min(TINY)
    of = scale.double()[..., None]
    edge = torch.stack([(high.double() / of).float().ceil(), (low.double() / of).float().floor()], dim=2)
    bounds[ids, :heads * 2 * d] = edge.clamp(-127, 127).to(torch.int8).view(torch.uint8).view(len(ids), -1)
    bounds[ids, heads * 2 * d:heads * (2 * d + 4)] = scale.contiguous().view(torch.uint8)


def _plain_bounds(s):
    case, p = s["case"], s["case"]["page"]
    counts, lens = s["counts"].long(), s["lens"].long()
    host_first = s["host_base"] // p
    touched = np.where(s["host_counts"] > 0, -(-(s["host_base"] + s["host_counts"]) // p) - host_first, 0)
    total = int(touched.sum())
    first = (lens - counts) // p
    n = torch.where(counts > 0, -(-lens // p) - first, 0)
    b = torch.repeat_interleave(torch.arange(len(counts), device=lens.device), n, output_size=total)
    j = first[b] + torch.arange(total, device=lens.device) - (torch.cumsum(n, 0) - n)[b]
    ids = s["table"][b, j].long()
    k = _widened(s["pool"]["k"], s["pool"]["k_scales"], ids, case, True)
    k = torch.where(torch.isnan(k), 0.0, k.clamp(-BF16_MAX, BF16_MAX))
    seen = (torch.arange(p, device=lens.device) < (lens[b] - j * p)[:, None])[:, None, :, None]
    high, low = torch.where(seen, k, -math.inf).amax(dim=2), torch.where(seen, k, math.inf).amin(dim=2)
    _put_bounds(s["bounds"], ids, high, low, case)
    return _bounds_of(s["bounds"], case)


def _plain_select(s):
    case, lens, p = s["case"], s["lens"].long(), s["case"]["page"]
    heads, d, budget = case["kv_heads"], case["d"], case["budget"]
    b, width = s["table"].shape
    n = -(-lens // p)
    q = s["q"].float().view(b, heads, -1, d)
    step = (q.abs().amax(dim=3).double() / 127.0).float().clamp_min(TINY)
    q = (q.double() / step.double()[..., None]).float().round()  # whole numbers; ties to even
    q = torch.cat([q.clamp_min(0.0), q.clamp_max(0.0)], dim=3)
    held = _bounds_of(s["bounds"], case)
    edge = held["edge"][s["table"].long()].view(b, width, heads, 2 * d).permute(0, 2, 3, 1).float().contiguous()
    # products of whole numbers, below 2^24 in any order
    score = (torch.matmul(q, edge) * step[..., None]).amax(dim=2) * held["scale"][s["table"].long()].transpose(1, 2) + 0.0
    at = torch.arange(width, device=lens.device)
    live = (at < n[:, None])[:, None, :].expand(b, heads, width)
    s["scores"].copy_(torch.where(live, score, s["scores"]))
    kept = (at < case["sinks"]) | (at >= (n - case["recent"])[:, None])  # [B][width]
    rank = torch.where(kept[:, None, :], math.inf, score)
    rank = torch.where(live, rank, -math.inf)
    # those that are kept come first, those that are not there last, equal ones by their number
    group = torch.where(live, torch.where(kept[:, None, :], 0, 1), 2)
    order = torch.sort(rank, dim=2, descending=True, stable=True).indices
    order = order.gather(2, torch.sort(group.gather(2, order), dim=2, stable=True).indices)
    order = torch.nn.functional.pad(order[:, :, :budget], (0, max(0, budget - width)), value=width)
    count = n.clamp_max(budget)
    chosen = torch.where(torch.arange(budget, device=lens.device) < count[:, None, None], order, 1 << 30).sort(dim=2).values
    s["lists"].copy_(torch.where(chosen < (1 << 30), chosen, s["lists"].long()))
    s["counts"].copy_(count[:, None].expand(b, heads))
    return {"lists": s["lists"], "counts": s["counts"], "scores": s["scores"]}


# ---------------------------------------------------------------------------
# what a pass cannot do without, and what it gives in 64 bits
# ---------------------------------------------------------------------------

def work(case):
    row = case["kv_heads"] * case["d"]  # values of one token's K (or V)
    held = {"bf16": 2.0, "fp8": 1.0, "fp4": 17 / 32}.get(case.get("dtype"))  # bytes of one
    scales = 8 if case.get("dtype") == "fp8" else 0  # of a page
    record = case["kv_heads"] * (2 * case["d"] + 4)
    if case["kind"] in ("store4", "bounds"):
        counts = _counts(case)
        base = _rng(case).integers(0, 64 * case["page"], case["seqs"])
        first = base // case["page"] * case["page"]
        pages = int(np.where(counts > 0, -(-(base + counts - first) // case["page"]), 0).sum())
        if case["kind"] == "store4":  # each token read, stored, read again and given out
            return {"bytes": int(counts.sum()) * 2 * row * (2 + 2 * held + 2) + 4 * pages + 8 * case["seqs"], "flops": 0}
        tokens = int(np.where(counts > 0, base + counts - first, 0).sum())
        return {"bytes": tokens * row * held + pages * (record + 4 + scales // 2) + 8 * case["seqs"], "flops": 0}
    lens = _lengths(case)
    n = -(-lens // case["page"])
    rows = 2 * case["seqs"] * case["q_heads"] * case["d"] * 2 + 4 * case["seqs"]
    if case["kind"] == "select":  # bounds and table entries read, scores and lists written
        count = int(np.minimum(n, case["budget"]).sum())
        pages = int(n.sum())
        size = pages * (record + 4 + 4 * case["kv_heads"]) + 4 * case["kv_heads"] * (count + case["seqs"])
        return {"bytes": size + rows // 2, "flops": 4 * pages * case["q_heads"] * case["d"]}
    if case["kind"] == "decode4":
        tokens, pages, entries = int(lens.sum()), int(n.sum()), 0
    else:  # the tokens of each list (the last page, which may be partly filled, is in it), its entries
        pages = int(np.minimum(n, case["budget"]).sum())
        tokens = int(np.where(lens > 0, lens - (n - np.minimum(n, case["budget"])) * case["page"], 0).sum())
        entries = 4 * case["kv_heads"] * (pages + case["seqs"])
    return {"bytes": tokens * 2 * row * held + pages * (scales + 4) + entries + rows, "flops": 4 * tokens * case["q_heads"] * case["d"]}


def exact(case, seed):
    s = prepare(case, seed)
    return {"decode4": _exact_attention, "pages": _exact_attention, "store4": _exact_store, "bounds": _exact_bounds, "select": _exact_select}[case["kind"]](s)


def _value_of(code):
    """What an E2M1 code stands for, from its sign, exponent and mantissa."""
    code = code.long()
    e, m = (code >> 1) & 3, (code & 1).double()
    x = torch.where(e > 0, (1 + m / 2) * torch.pow(torch.tensor(2.0, dtype=torch.float64, device=code.device), (e - 1).double()), m / 2)
    return torch.where(code >= 8, -x, x)


def _tokens64(s, ids, slot, head, key):
    """K or V of tokens by page and slot, of one KV head: [t][d], 64 bits."""
    case, p, d = s["case"], s["case"]["page"], s["case"]["d"]
    pages = s["pool"]["k" if key else "v"]
    if case["dtype"] != "fp4":
        x = pages[ids, head, :, slot] if key else pages[ids, head][torch.arange(len(ids), device=ids.device), :, slot]
        if case["dtype"] == "fp8":
            scale = s["pool"]["k_scales" if key else "v_scales"][ids].double()
            return x.view(torch.float8_e4m3fn).float().double().reshape(len(ids), d) * scale[:, None]
        return x.double().reshape(len(ids), d)
    tile, dim = pages[ids, head], torch.arange(d, device=ids.device)
    t = torch.arange(len(ids), device=ids.device)[:, None]
    if key:
        at = (dim // 32 * p + slot[:, None]) * 32 + dim % 32
        scale = tile[t, p * d // 2 + dim // 32 * p + (slot // 16 * 16 + slot % 4 * 4 + slot % 16 // 4)[:, None]].double() - 127
        scale = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=ids.device), scale)
    else:
        at = dim * p + slot[:, None]
        where = p * d // 2 + 2 * (dim // 64 * p + slot[:, None])
        bits = tile[t, where].int() | (tile[t, where + 1].int() << 8)
        scale = (bits << 16).view(torch.float32).double()
    return _value_of((tile[t, at // 2] >> (4 * (at % 2)).to(torch.uint8)) & 15) * scale


def _exact_attention(s):
    """Sequence by sequence and head by head, in 64 bits: the tokens by their numbers, each read from its page and slot."""
    case, p = s["case"], s["case"]["page"]
    heads, d = case["kv_heads"], case["d"]
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    q = s["q"].double().view(len(s["host_lens"]), heads, -1, d)
    lists = s["lists"].cpu().numpy() if case["kind"] == "pages" else None
    counts = s["counts"].cpu().numpy() if case["kind"] == "pages" else None
    for b, length in enumerate(s["host_lens"].tolist()):
        t = torch.arange(length, device="cuda")
        for h in range(heads):
            if lists is not None:
                t = (torch.from_numpy(lists[b, h, :counts[b, h]].astype(np.int64)).cuda()[:, None] * p + torch.arange(p, device="cuda")).flatten()
                t = t[t < length]
            if not len(t):
                continue
            ids, slot = s["table"][b, t // p].long(), t % p
            x = torch.matmul(q[b, h], _tokens64(s, ids, slot, h, True).T.contiguous()) * d ** -0.5
            g = q.shape[2]
            out[b, h * g:(h + 1) * g] = torch.matmul(torch.softmax(x, dim=1), _tokens64(s, ids, slot, h, False))
    return out


def _nearest(y):
    """y, 64 bits, at the nearest E2M1 value; a tie goes to the one with an even code."""
    grid = torch.tensor(E2M1, dtype=torch.float64, device=y.device)
    far = (y.abs()[..., None] - grid).abs()
    best = far.amin(dim=-1, keepdim=True)
    near = far == best
    even = near & (torch.arange(8, device=y.device) % 2 == 0)
    pick = torch.where(even.any(dim=-1, keepdim=True), even, near)
    return torch.copysign(grid[pick.to(torch.uint8).argmax(dim=-1)], y)


def _exact_store(s):
    """Each new token at the nearest values that its blocks' scales give.  (A scale is a rounded number that is held: a
    key's power of two is exact, a value's is the bf16 number next to a sixth of its largest.)"""
    case, d = s["case"], s["case"]["d"]
    out = {}
    for name, width in (("k", 32), ("v", 64)):
        x = s[name + "_new"].double()
        y = x.view(x.shape[:3] + (d // width, width))
        top = y.abs().amax(dim=-1, keepdim=True)
        if name == "k":
            mantissa, e = torch.frexp(top)  # top = mantissa 2^e, a half <= mantissa < 1
            e = torch.where(mantissa >= 0.875, e + 1, e) - 3
            scale = torch.pow(torch.tensor(2.0, dtype=torch.float64, device=x.device), e.clamp(-126, 125).double())
            scale = torch.where(top > 0, scale, TINY)
        else:
            scale = (top / 6).to(torch.float32).to(torch.bfloat16).double().clamp_min(TINY)
        near = (_nearest(y / scale) * scale).view(x.shape)
        live = torch.arange(case["tokens"], device=x.device)[None, :] < s["counts"][:, None]
        out[name] = torch.where(live[:, :, None, None], near, 0.0)
    return out


def _exact_bounds(s):
    """The scales of the bounds, page by page; the bounds themselves are whole numbers."""
    case, p = s["case"], s["case"]["page"]
    heads = case["kv_heads"]
    scale = torch.zeros((s["bounds"].shape[0], heads), dtype=torch.float64, device="cuda")
    if int((-(-s["host_counts"] // p)).sum()) > 20000:
        return None
    b = np.repeat(np.arange(len(s["host_counts"])), s["host_counts"])
    # every token of every page that holds a new one
    b, t = [], []
    for i, (start, n) in enumerate(zip(s["host_base"].tolist(), s["host_counts"].tolist())):
        if n:
            t.append(np.arange(start // p * p, start + n))
            b.append(np.full(len(t[-1]), i))
    if not b:
        return {"edge": None, "scale": scale}
    b, t = _dev(np.concatenate(b), np.int64), _dev(np.concatenate(t), np.int64)
    ids, slot = s["table"][b, t // p].long(), t % p
    for h in range(heads):
        top = torch.zeros(len(ids), dtype=torch.float64, device="cuda")
        step = 1 << 18
        for i in range(0, len(ids), step):
            top[i:i + step] = _tokens64(s, ids[i:i + step], slot[i:i + step], h, True).abs().amax(dim=1)
        scale[:, h] = scale[:, h].index_reduce(0, ids, top / 127, "amax")
    return {"edge": None, "scale": scale}


def _exact_select(s):
    """The scores in 64 bits, from the numbers that the queries and the bounds are held in."""
    case, p = s["case"], s["case"]["page"]
    heads, d = case["kv_heads"], case["d"]
    held = _bounds_of(s["bounds"], case)
    score = torch.zeros(s["scores"].shape, dtype=torch.float64, device="cuda")
    q = s["q"].double().view(len(s["host_lens"]), heads, -1, d)
    step = (q.abs().amax(dim=3, keepdim=True) / 127).float().clamp_min(TINY).double()
    q = torch.round((q / step).float().double())
    for b, length in enumerate(s["host_lens"].tolist()):
        n = -(-length // p)
        ids = s["table"][b, :n].long()
        edge = held["edge"][ids].double().view(n, heads, 2, d)
        for h in range(heads):
            high, low = q[b, h, :, None, :] * edge[:, h, 0], q[b, h, :, None, :] * edge[:, h, 1]
            x = torch.maximum(high, low).sum(dim=2) * step[b, h]  # [G][n]
            score[b, h, :n] = x.amax(dim=0) * held["scale"][ids, h].double()
    return {"lists": None, "counts": None, "scores": score}
