"""Cases and plain forms of what a decoding step does with long paged caches besides reading all of them once per sequence:
the attention of a batch whose sequences share a long prefix, and the attention over the pages that a cheap score selects (the
bounds of every page's keys, the score of a query against them, the selection, the attention over what was selected).

`run` computes an operator in elementary torch operations, or, where `own` is true, through the calls that a user makes of
`paper_2512_21571_b200.binding`.  `exact` is the same operator from its definition in 64 bits, sequence by sequence.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1}
ROOM = 1 << 29   # cache values of one kind (keys or values) that a call may hold
GATHERED = 1 << 30   # values of one kind that the plain form of an attention may lay out at a time


# ---- cases -----------------------------------------------------------------------------------------------------------

def _prefix(name, groups, members, heads, group, head_dim, page, shared, tail, kv, dtype, ragged):
    return {"name": name, "op": "prefix", "groups": groups, "members": members, "heads": heads, "group": group, "head_dim": head_dim,
            "page": page, "shared": shared, "tail": tail, "kv": kv, "dtype": dtype, "ragged": ragged}


def _pages(name, op, seqs, heads, group, head_dim, page, length, take, kv, dtype, ragged):
    """take: new tokens of each sequence ("bounds"), pages a KV head ("select", "selected"); "score" has no use for it."""
    return {"name": name, "op": op, "seqs": seqs, "heads": heads, "group": group, "head_dim": head_dim, "page": page,
            "length": length, "take": take, "kv": kv, "dtype": dtype, "ragged": ragged}


def listed():
    return [
        # a few answers being sampled from one short prompt
        _prefix("prefix few", 1, 3, 2, 4, 128, 16, 496, 40, "bf16", "bf16", True),
        # a serving batch of the 8B shape behind one system prompt, each sequence some hundred tokens into its own turn
        _prefix("prefix batch", 1, 64, 8, 4, 128, 64, 8192, 700, "bf16", "bf16", True),
        # many questions about one long document, small heads with many queries a key head
        _prefix("prefix document fp16", 1, 48, 2, 12, 64, 128, 65536, 300, "fp16", "fp16", False),
        # several prompts with answers of their own, on a quantised cache
        _prefix("prefix groups e4m3", 5, 12, 8, 4, 128, 32, 6000, 900, "e4m3", "bf16", True),
        # a decoding step's new rows: the bounds of the page that each of 48 sequences writes to
        _pages("bounds one token each", "bounds", 48, 8, 4, 128, 64, 9000, 1, "bf16", "bf16", True),
        # prompts that have just been written
        _pages("bounds prompts", "bounds", 4, 8, 4, 128, 64, 16384, 16384, "bf16", "bf16", False),
        # one long document: every page's score for the 8B shape's query heads
        _pages("score one", "score", 1, 8, 4, 128, 32, 131071, 0, "bf16", "fp32", False),
        # a batch of long sequences, small pages
        _pages("score batch", "score", 32, 8, 4, 128, 16, 32768, 0, "bf16", "bf16", True),
        # the selection that goes with one document
        _pages("select one", "select", 1, 8, 4, 128, 32, 131071, 128, "bf16", "bf16", False),
        # and with a batch
        _pages("select batch", "select", 32, 8, 4, 128, 16, 32768, 256, "bf16", "bf16", True),
        # a batch of long sequences that each attend to 64 pages a KV head
        _pages("selected batch", "selected", 32, 8, 4, 128, 64, 16000, 64, "bf16", "bf16", False),
        # quantised cache, small pages, results in 32 bits
        _pages("selected e4m3", "selected", 20, 4, 8, 64, 16, 30011, 200, "e4m3", "fp32", True),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["prefix", "prefix", "prefix", "bounds", "score", "select", "selected", "selected"])
    head_dim, heads, page = rng.choice([64, 128]), rng.choice([1, 2, 4, 8]), rng.choice([16, 32, 64, 128, 256])
    kv = rng.choice(["bf16", "fp16", "e4m3"])
    group = rng.randint(1, 16)
    if op == "prefix":
        dtype = "bf16" if kv == "bf16" else "fp16" if kv == "fp16" else rng.choice(["bf16", "fp16"])
        groups = rng.choice([1, 1, 1, _spread(rng, 2, 8)])
        members = _spread(rng, 1, 96 // groups)
        most = GATHERED // (groups * members * heads * head_dim)
        shared = max(page, min(_spread(rng, page, 65536), most * 7 // 8 // page * page))
        tail = max(1, min(_spread(rng, 1, 4000), most - shared))
        c = _prefix("", groups, members, heads, group, head_dim, page, shared, tail, kv, dtype, rng.random() < 0.6)
    else:
        dtype = rng.choice(["fp32", "bf16" if kv == "e4m3" else kv])
        seqs = _spread(rng, 1, 64)
        most = min(ROOM // (seqs * heads * head_dim), 131072)
        length = max(1, min(_spread(rng, 16, 131072), most))
        if op == "select":   # there is something to leave out
            length = max(length, 9 * page)
        columns = -(-length // page)
        if op == "bounds":
            take = rng.choice([1, _spread(rng, 1, length)])
        else:
            take = max(4, min(_spread(rng, 4, 512), GATHERED // (seqs * heads * head_dim * page), max(4, columns // 2)))
        c = _pages("", op, seqs, heads, group, head_dim, page, length, take, kv, dtype, rng.random() < 0.6)
    del c["name"]
    return c


def _lengths(case):
    """(lengths, first sequence of each group and the end, shared positions of each group); sequences of one group follow one
    another.  Cases without groups have a group of no shared positions for each sequence."""
    if case["op"] != "prefix":
        n, longest = case["seqs"], case["length"]
        r = random.Random(1000003 * n + longest)
        got = [r.randint(1, longest) for _ in range(n)] if case["ragged"] else [longest] * n
        got[r.randrange(n)] = longest
        return got, list(range(n + 1)), [0] * n
    r = random.Random(1000003 * case["members"] + case["shared"] + case["tail"])
    page = case["page"]
    lens, starts, shared = [], [0], []
    for g in range(case["groups"]):
        members = r.randint(max(1, case["members"] // 4), case["members"]) if case["ragged"] and g else case["members"]
        most = case["shared"] // page
        shared.append(page * (r.randint(max(1, most // 3), most) if case["ragged"] and g else most))
        lens += [shared[-1] + (r.randint(1, case["tail"]) if case["ragged"] else case["tail"]) for _ in range(members)]
        starts.append(len(lens))
    return lens, starts, shared


def _columns(case):
    return -(-max(_lengths(case)[0]) // case["page"]) + 1


def work(case):
    lens, starts, shared = _lengths(case)
    d, heads, page, n = case["head_dim"], case["heads"], case["page"], len(lens)
    values = d * SIZE[case["kv"]]
    row = 2 * heads * (values + (1 if case["kv"] == "e4m3" else 0))      # a cached position: key and value rows
    q = n * heads * case["group"]
    bound = 2 * 2 * heads * d                                            # a page's two bounds, 16 bits
    if case["op"] == "prefix":
        rows = sum(shared) + sum(x - shared[g] for g in range(len(shared)) for x in lens[starts[g]:starts[g + 1]])
        return {"bytes": rows * row + 2 * q * d * SIZE[case["dtype"]] + 4 * q + 4 * n + 4 * -(-rows // page),
                "flops": 4 * sum(lens) * heads * case["group"] * d}
    pages = [-(-x // page) for x in lens]
    if case["op"] == "bounds":
        touched = [p - max(0, x - case["take"]) // page for x, p in zip(lens, pages)]
        rows = sum(x - max(0, x - case["take"]) // page * page for x in lens)
        return {"bytes": rows * row // 2 + sum(touched) * bound + 8 * n + 4 * sum(touched), "flops": 2 * rows * heads * d}
    if case["op"] == "score":
        return {"bytes": sum(pages) * (bound + 4) + 4 * heads * _columns(case) * n + q * d * SIZE[case["dtype"]] + 4 * n,
                "flops": 4 * sum(pages) * heads * case["group"] * d}
    if case["op"] == "select":
        return {"bytes": 4 * heads * (sum(pages) + n * (case["take"] + 1)) + 4 * n, "flops": heads * sum(pages)}
    rows = sum(min(x, case["take"] * page) for x in lens)                # (a last page that is not full: counted as full)
    return {"bytes": rows * row + 2 * q * d * SIZE[case["dtype"]] + 4 * q + 4 * n + 4 * heads * n * (case["take"] + 1),
            "flops": 4 * rows * heads * case["group"] * d}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _normal(shape, g, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if dtype is torch.float32 else torch.bfloat16).to(dtype)


def _power(e):
    """2^e for whole e within +-126, from its bits: a power function may be off in the last place."""
    return (e.int() + 127 << 23).view(torch.float32)


def _to_codes(x):
    """E4M3 codes and biased exponents of x's rows: the smallest 2^e with max|x| <= 448 * 2^e, 0 for a row of zeros."""
    x = x.float()
    f, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(f > 0, (e - 9 + (f > 0.875).int()).clamp(-60, 60), 0)
    return (x * _power(-e)).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _fill(pool, scale, g):
    """Rows of normal values about a mean of each column's own, as key rows have; codes with scales of slowly varying size."""
    total, heads, page, d = pool.shape
    mean = torch.randn((heads, 1, d), generator=g, device="cuda")
    step = max(1, (1 << 26) // (heads * page * d))
    for lo in range(0, total, step):
        n = min(step, total - lo)
        x = _normal((n, heads, page, d), g, torch.bfloat16).add_(mean)
        if scale is None:
            pool[lo:lo + n] = x
        else:
            codes, e = _to_codes(x * torch.rand((n, heads, page, 1), generator=g, device="cuda"))
            pool[lo:lo + n].view(torch.uint8).copy_(codes.view(torch.uint8))
            scale[lo:lo + n] = e[..., 0]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    op, d, heads, page, kv = (case[x] for x in ("op", "head_dim", "heads", "page", "kv"))
    lens, starts, shared = _lengths(case)
    s = {"case": case, "max_len": max(lens), "lens": torch.tensor(lens, dtype=torch.int32, device="cuda")}
    if op == "select":   # scores as sums of many products have them
        s["scores"] = 40 + 12 * torch.randn((len(lens), heads, _columns(case)), generator=g, device="cuda")
        return s
    # pages were handed out in no order; a group's sequences have its shared pages in common; entries past a sequence's last
    # page hold -1
    r = random.Random(seed)
    own_pages = [-(-x // page) - shared[i] // page for i in range(len(shared)) for x in lens[starts[i]:starts[i + 1]]]
    total = sum(own_pages) + sum(x // page for x in shared) + 3
    order = torch.tensor(r.sample(range(total), total), dtype=torch.int32)
    table = torch.full((len(lens), _columns(case)), -1, dtype=torch.int32)
    at = 0
    for i, positions in enumerate(shared):
        common = order[at:at + positions // page]
        at += len(common)
        for b in range(starts[i], starts[i + 1]):
            table[b, :len(common)] = common
            table[b, len(common):len(common) + own_pages[b]] = order[at:at + own_pages[b]]
            at += own_pages[b]
    s["table"] = table.cuda()
    shape = (total, heads, page, d)
    store = torch.float8_e4m3fn if kv == "e4m3" else TYPES[kv]
    s["k"], s["v"] = (torch.empty(shape, dtype=store, device="cuda") for _ in range(2))
    s["k_scale"], s["v_scale"] = (torch.empty(shape[:3], dtype=torch.uint8, device="cuda") if kv == "e4m3" else None for _ in range(2))
    if op != "score":
        _fill(s["k"], s["k_scale"], g)
        _fill(s["v"], s["v_scale"], g)
    if op in ("bounds", "score"):   # [pages][KV heads][lowest, highest][head_dim]
        middle = _normal((total, heads, 1, d), g, torch.float32)
        reach = 2 * torch.rand((total, heads, 2, d), generator=g, device="cuda") * torch.tensor([[-1.0], [1.0]], device="cuda")
        s["bounds"] = (middle + reach).to(torch.float16 if kv == "fp16" else torch.bfloat16)
    if op == "bounds":
        s["first"] = torch.tensor([max(0, x - case["take"]) for x in lens], dtype=torch.int32, device="cuda")
        return s
    s["q"] = _normal((len(lens), heads * case["group"], d), g, TYPES[case["dtype"]])
    if op == "prefix":
        s["starts"], s["shared"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (starts, shared))
    if op == "selected":   # a selection as scores make it: the first and the last page, and others without an order in their scores
        n = -(-s["lens"].long() // page)[:, None, None]
        order = torch.rand((len(lens), heads, _columns(case)), generator=g, device="cuda")
        column = torch.arange(_columns(case), device="cuda")
        order = torch.where(column >= n, -1.0, torch.where((column == 0) | (column == n - 1), 2.0, order))
        take = min(case["take"], _columns(case))
        pages = order.topk(take, -1).indices
        pages = torch.where(pages < n, pages, 1 << 30).sort(-1).values
        s["pages"] = torch.full((len(lens), heads, case["take"]), -1, dtype=torch.int32, device="cuda")
        s["pages"][..., :take] = torch.where(pages < n, pages, -1)
        s["counts"] = n.clamp(max=take).expand(-1, heads, 1)[..., 0].int().contiguous()
    return s


# ---- the operators ---------------------------------------------------------------------------------------------------

def _kept(s, name, make):
    """What a user's program makes once and keeps: the handle of the cache, a scratch buffer."""
    if name not in s:
        s[name] = make()
    return s[name]


def _values(rows, scale):
    """Rows taken from a pool, as 32-bit values."""
    if scale is None:
        return rows.float()
    return rows.view(torch.float8_e4m3fn).float() * _power(scale.int()[..., None] - 127)


def _pool(x):
    return x.view(torch.uint8) if x.dtype is torch.float8_e4m3fn else x


def _take(s, which, *at):
    scale = s[which + "_scale"]
    return _values(_pool(s[which])[at], None if scale is None else scale[at])


def _softmax(s, k, v, live):
    """k, v [sequences][KV heads][positions][head_dim]; live [sequences][KV heads or 1][positions]."""
    c = s["case"]
    q = s["q"].float().unflatten(1, (c["heads"], c["group"]))
    score = (q @ k.transpose(-1, -2) * c["head_dim"] ** -0.5).masked_fill(~live[:, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top.clamp(min=-3e38))
    total = p.sum(-1, keepdim=True)
    out = p @ v.masked_fill(~live[..., None], 0.0) / total.clamp(min=1e-38)
    lse = (top + torch.log(total))[..., 0]
    return {"out": out.flatten(1, 2).to(s["q"].dtype), "lse": lse.flatten(1, 2)}


def _prefix_plain(s):
    table = s["table"].long().clamp(min=0)
    k, v = (_take(s, x, table).transpose(1, 2).flatten(2, 3) for x in "kv")
    live = torch.arange(k.shape[2], device="cuda") < s["lens"][:, None]
    return _softmax(s, k, v, live[:, None])


def _selected_plain(s):
    page = s["case"]["page"]
    listed_ = torch.arange(s["pages"].shape[2], device="cuda") < s["counts"][..., None]
    pages = s["pages"].long().clamp(min=0)
    seq = torch.arange(pages.shape[0], device="cuda")[:, None, None]
    head = torch.arange(pages.shape[1], device="cuda")[:, None]
    at = s["table"][seq, pages].long().clamp(min=0)
    pos = pages[..., None] * page + torch.arange(page, device="cuda")
    live = (listed_[..., None] & (pos < s["lens"][:, None, None, None])).flatten(2)
    k, v = (_take(s, x, at, head).flatten(2, 3) for x in "kv")
    return _softmax(s, k, v, live)


def _bounds_plain(s):
    page, lens, first = s["case"]["page"], s["lens"].long()[:, None], s["first"].long()[:, None]
    column = torch.arange(s["table"].shape[1], device="cuda")
    seq, column = torch.nonzero((column >= first // page) & (column * page < lens), as_tuple=True)
    at = s["table"][seq, column].long()
    k = _take(s, "k", at)
    live = ((column[:, None] * page + torch.arange(page, device="cuda")) < lens[seq])[:, None, :, None]
    s["bounds"][at, :, 0] = k.masked_fill(~live, math.inf).amin(2).to(s["bounds"].dtype)
    s["bounds"][at, :, 1] = k.masked_fill(~live, -math.inf).amax(2).to(s["bounds"].dtype)
    return s["bounds"]


def _score_plain(s):
    c = s["case"]
    q = s["q"].float().unflatten(1, (c["heads"], c["group"]))                       # [sequences][KV heads][group][d]
    bounds = s["bounds"].float()[s["table"].long().clamp(min=0)].transpose(1, 2)    # [sequences][KV heads][columns][2][d]
    # q * lowest where q < 0, q * highest elsewhere: the most that a key between the two can give
    score = q.clamp(max=0) @ bounds[..., 0, :].transpose(-1, -2) + q.clamp(min=0) @ bounds[..., 1, :].transpose(-1, -2)
    there = torch.arange(s["table"].shape[1], device="cuda") * c["page"] < s["lens"][:, None]
    return score.amax(2).masked_fill(~there[:, None], -math.inf)


def _select_plain(s):
    c, scores = s["case"], s["scores"]
    n = -(-s["lens"].long() // c["page"])[:, None, None]
    column = torch.arange(scores.shape[2], device="cuda")
    rank = torch.where((column == 0) | (column == n - 1), math.inf, scores).masked_fill(column >= n, -math.inf)
    # the stable descending order puts the lowest index first among equal scores
    take = min(c["take"], scores.shape[2])
    pages = rank.sort(dim=-1, descending=True, stable=True).indices[..., :take]
    counts = n.clamp(max=take).expand(-1, scores.shape[1], 1)
    kept = torch.where(torch.arange(take, device="cuda") < counts, pages, 1 << 30).sort(-1).values
    out = torch.full((*scores.shape[:2], c["take"]), -1, dtype=torch.int32, device="cuda")
    out[..., :take] = torch.where(kept < 1 << 30, kept, -1)
    return {"pages": out, "counts": counts[..., 0].int()}


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2512_21571_b200 import binding
        if c["op"] == "select":
            pages, counts = binding.op_select_pages(s["scores"], s["lens"], c["page"], c["take"])
            return {"pages": pages, "counts": counts}
        cache = _kept(s, "cache", lambda: binding.PagedKV(s["k"], s["v"], s["table"], s["k_scale"], s["v_scale"]))
        if c["op"] == "bounds":
            return binding.op_page_bounds(cache, s["bounds"], s["lens"], s["first"])
        if c["op"] == "score":
            return binding.op_score_pages(s["q"], cache, s["bounds"], s["lens"])
        if c["op"] == "selected":
            scratch = _kept(s, "scratch", binding.attn_paged_scratch)
            out, lse = binding.op_attn_selected_paged(s["q"], cache, s["lens"], s["pages"], s["counts"], scratch=scratch, want_lse=True)
        else:
            scratch = _kept(s, "scratch", lambda: binding.attn_prefix_scratch(*s["q"].shape))
            out, lse = binding.op_attn_prefix_paged(s["q"], cache, s["lens"], s["starts"], s["shared"], scratch=scratch, want_lse=True)
        return {"out": out, "lse": lse}
    return {"prefix": _prefix_plain, "bounds": _bounds_plain, "score": _score_plain, "select": _select_plain, "selected": _selected_plain}[c["op"]](s)


# ---- the operators from their definitions, in 64 bits -------------------------------------------------------------------

def _e4m3_table():
    """The 256 values of E4M3: sign, four exponent bits of bias 7, three mantissa bits; 0x7f and 0xff are NaN."""
    got = []
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        x = math.nan if code & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        got.append(-x if code >> 7 else x)
    return torch.tensor(got, dtype=torch.float64, device="cuda")


def _exact_pages(s, which, pages, head=slice(None)):
    """Rows of the pages, in 64 bits."""
    pages = pages.long()
    if s[which + "_scale"] is None:
        return s[which][pages, head].double()
    unit = (s[which + "_scale"][pages, head].long() + 1023 - 127 << 52).view(torch.float64)   # 2^(byte - 127), exactly
    return _e4m3_table()[s[which].view(torch.uint8)[pages, head].long()] * unit[..., None]


def _exact_head(q, k, v):
    """One KV head: q [group][d], k, v [positions][d]; output rows and log-sum-exps."""
    score = q @ k.T / math.sqrt(q.shape[1])
    return torch.softmax(score, -1) @ v, torch.logsumexp(score, -1)


def exact(case, seed):
    s = prepare(case, seed)
    op, page, heads, group = case["op"], case["page"], case["heads"], case["group"]
    if op == "select":
        return None
    lens = _lengths(case)[0]
    if op == "bounds":
        got = s["bounds"].double()
        for b, n in enumerate(lens):
            for column in range(max(0, n - case["take"]) // page, -(-n // page)):
                at = s["table"][b, column]
                rows = _exact_pages(s, "k", at)[:, :min(page, n - column * page)]
                got[at.long(), :, 0], got[at.long(), :, 1] = rows.amin(1), rows.amax(1)
        return got
    if op == "score":
        got = torch.full((len(lens), heads, s["table"].shape[1]), -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            columns = -(-n // page)
            q = s["q"][b].double().reshape(heads, group, 1, -1)
            for lo in range(0, columns, 1024):
                bounds = s["bounds"][s["table"][b, lo:min(lo + 1024, columns)].long()].double().transpose(0, 1)[:, None]
                got[b, :, lo:min(lo + 1024, columns)] = torch.maximum(q * bounds[..., 0, :], q * bounds[..., 1, :]).sum(-1).amax(1)
        return got
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, n in enumerate(lens):
        for h in range(heads):
            at = slice(h * group, (h + 1) * group)
            columns = torch.arange(-(-n // page), device="cuda") if op == "prefix" else s["pages"][b, h, :int(s["counts"][b, h])].long()
            live = (columns[:, None] * page + torch.arange(page, device="cuda") < n).flatten()
            k, v = (_exact_pages(s, x, s["table"][b, columns], h).flatten(0, 1)[live] for x in "kv")
            out[b, at], lse[b, at] = _exact_head(s["q"][b, at].double(), k, v)
    return {"out": out, "lse": lse}
