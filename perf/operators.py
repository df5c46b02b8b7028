"""Cases and plain forms of the paged key-value cache's operators: rotary positions, writing and reading the cache
(16-bit rows, or E4M3 codes with a power-of-two scale per row), and the attention of one new token over it.

`run` computes an operator in elementary torch operations, or, where `own` is true, through the calls that a user makes of
`paper_2512_21571_b200.binding`.  `exact` is the same operator from its definition in 64 bits, sequence by sequence.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SCRATCH_BYTES = 16 << 20   # NNC_ATTN_PAGED_SCRATCH_BYTES
ROOM = 32 * 8192 * 8 * 128   # cache values of one kind (keys or values) that a call may hold: 32 sequences of 8192, 8 heads of 128


# ---- cases -----------------------------------------------------------------------------------------------------------

def _rope(name, tokens, heads, head_dim, rotary_dim, interleaved, inverse, dtype, scaling, far):
    return {"name": name, "op": "rope", "tokens": tokens, "heads": heads, "head_dim": head_dim, "rotary_dim": rotary_dim,
            "interleaved": interleaved, "inverse": inverse, "dtype": dtype, "scaling": scaling, "far": far}


def _store(name, op, seqs, heads, head_dim, page, length, new, kv, dtype, ragged):
    return {"name": name, "op": op, "seqs": seqs, "heads": heads, "head_dim": head_dim, "page": page, "length": length,
            "new": new, "kv": kv, "dtype": dtype, "ragged": ragged}


def _attn(name, seqs, heads, group, head_dim, page, length, kv, dtype, window, ragged):
    return {"name": name, "op": "attn", "seqs": seqs, "heads": heads, "group": group, "head_dim": head_dim, "page": page,
            "length": length, "kv": kv, "dtype": dtype, "window": window, "ragged": ragged}


def listed():
    return [
        # one new token of the 8B shape: its 32 query and 8 key heads turned together
        _rope("rope one token", 1, 40, 128, 128, False, False, "bf16", "none", 4096),
        # a prompt of 4 sequences of 2048 of the same shape
        _rope("rope prompt", 8192, 40, 128, 128, False, False, "bf16", "none", 2048),
        # the gradient of the rotation: neighbouring pairs, half of an odd-sized head, stretched for a long context
        _rope("rope gradient far", 4099, 24, 96, 48, True, True, "fp32", "ramp", 1 << 20),
        # a batch of 32 sequences that each append one token
        _store("write one token each", "write", 32, 8, 128, 64, 500, 1, "bf16", "bf16", True),
        # a prompt chunk quantised into the cache and taken back for the chunk's own attention
        _store("write and read chunk", "turn", 4, 8, 128, 64, 4000, 2048, "e4m3", "bf16", False),
        # a cached prefix that several prompts share, read back in ragged lengths
        _store("read prefixes", "read", 7, 8, 128, 32, 8191, 8191, "e4m3", "bf16", True),
        # the shortest useful call: one sequence, a few tokens in
        _attn("attend short", 1, 8, 2, 128, 16, 19, "bf16", "bf16", 0, False),
        # single-sequence decoding of the 8B shape at 4096 positions
        _attn("attend one sequence", 1, 8, 4, 128, 64, 4097, "bf16", "bf16", 0, False),
        # batched decoding of the 8B shape
        _attn("attend batch", 32, 8, 4, 128, 64, 8192, "bf16", "bf16", 0, False),
        # ragged serving batch on a quantised cache
        _attn("attend ragged e4m3", 61, 8, 4, 128, 64, 9000, "e4m3", "bf16", 0, True),
        # small heads, many queries a key head, sliding window
        _attn("attend window fp16", 48, 2, 12, 64, 128, 20000, "fp16", "fp16", 4096, True),
        # one long document on a quantised cache, queries and results in 32 bits
        _attn("attend long e4m3", 1, 4, 8, 128, 256, 131071, "e4m3", "fp32", 0, False),
    ]


def _spread(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    op = rng.choice(["rope", "write", "turn", "read", "attn", "attn", "attn"])
    if op == "rope":
        head_dim = rng.choice([64, 80, 96, 128, 192, 256])
        tokens = _spread(rng, 1, 16384)
        heads = max(1, min(_spread(rng, 1, 64), 8192 * 40 * 128 // (tokens * head_dim)))
        c = _rope("", tokens, heads, head_dim, head_dim // rng.choice([1, 1, 2, 4]) // 2 * 2, rng.random() < 0.5, rng.random() < 0.4,
                  rng.choice(["bf16", "fp16", "fp32"]), rng.choice(["none", "linear", "ramp"]), _spread(rng, 16, 1 << 22))
    elif op == "attn":
        head_dim, heads, seqs = rng.choice([64, 128]), rng.choice([1, 2, 4, 8]), _spread(rng, 1, 96)
        length = max(1, min(_spread(rng, 1, 131072), ROOM // (seqs * heads * head_dim)))
        kv = rng.choice(["bf16", "fp16", "e4m3"])
        c = _attn("", seqs, heads, rng.randint(1, 16), head_dim, rng.choice([16, 32, 64, 128, 256]), length, kv,
                  rng.choice([kv if kv != "e4m3" else "bf16", "fp16" if kv == "e4m3" else kv, "fp32"]),
                  rng.choice([0, 0, _spread(rng, 1, 8192)]), rng.random() < 0.6)
    else:
        head_dim, heads, seqs = rng.choice([64, 128]), rng.choice([1, 2, 4, 8]), _spread(rng, 1, 48)
        length = max(1, min(_spread(rng, 1, 16384), ROOM // 16 // (seqs * heads * head_dim)))
        kv = {"write": rng.choice(["bf16", "fp16"]), "turn": "e4m3", "read": rng.choice(["bf16", "fp16", "e4m3"])}[op]
        c = _store("", op, seqs, heads, head_dim, rng.choice([16, 32, 64, 128, 256]), length,
                   length if op == "read" else _spread(rng, 1, length), kv, rng.choice(["bf16", "fp16", "fp32"]), rng.random() < 0.5)
    del c["name"]
    return c


def _lengths(case):
    """Cached positions of each sequence after the call; a ragged batch holds an empty sequence when it has ten or more."""
    n, longest = case["seqs"], case["length"]
    if not case["ragged"]:
        return [longest] * n
    r = random.Random(1000003 * n + longest)
    got = [r.randint(1, longest) for _ in range(n)]
    got[r.randrange(n)] = longest
    if n >= 10:
        at = r.randrange(n)
        got[at] = 0 if got[at] != longest else longest
    return got


def _tokens(case):
    """(sequence, position) of each token that a call on the cache's rows names: the last `new` of every sequence."""
    seq, pos = [], []
    for b, n in enumerate(_lengths(case)):
        first = max(0, n - case["new"])
        seq += [b] * (n - first)
        pos += range(first, n)
    return seq, pos


def _attended(case):
    return sum(min(n, case["window"]) if case["window"] else n for n in _lengths(case))


def work(case):
    size = {"bf16": 2, "fp16": 2, "fp32": 4, "e4m3": 1}
    d = case["head_dim"]
    if case["op"] == "rope":
        n = case["tokens"] * case["heads"] * d
        return {"bytes": 2 * n * size[case["dtype"]] + 4 * case["tokens"] + 4 * case["rotary_dim"],
                "flops": 3 * case["tokens"] * case["heads"] * case["rotary_dim"]}
    row = 2 * case["heads"] * (d * size[case["kv"]] + (1 if case["kv"] == "e4m3" else 0))   # a cached position: key and value rows
    if case["op"] == "attn":
        n, q = _attended(case), case["seqs"] * case["heads"] * case["group"]
        return {"bytes": n * row + 2 * q * d * size[case["dtype"]] + 4 * q + 4 * case["seqs"] + 4 * sum(-(-x // case["page"]) for x in _lengths(case)),
                "flops": 4 * n * case["heads"] * case["group"] * d}
    n = len(_tokens(case)[0])
    outside = 2 * case["heads"] * d * size[case["dtype"]]
    return {"bytes": n * (8 + (2 if case["op"] == "turn" else 1) * (row + outside)), "flops": 2 * n * case["heads"] * d}


# ---- inputs ----------------------------------------------------------------------------------------------------------

def _normal(shape, g, dtype):
    return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32 if dtype is torch.float32 else torch.bfloat16).to(dtype)


def _frequencies(case):
    """Angle per position of each pair, 64 bits: theta 1e6; stretched by 8 from an original context of 4096 positions, all pairs
    alike, or only those that turn seldom."""
    half = case["rotary_dim"] // 2
    f = 1e6 ** (-torch.arange(half, dtype=torch.float64) / half)
    if case["scaling"] == "linear":
        f = f / 8
    elif case["scaling"] == "ramp":
        keep = ((4096 * f / (2 * math.pi) - 1) / 31).clamp(0, 1)
        f = f * (keep + (1 - keep) / 8)
    return f


def _power(e):
    """2^e for whole e within +-126, from its bits: a power function may be off in the last place, which moves ties."""
    return (e.int() + 127 << 23).view(torch.float32)


def _to_codes(x):
    """E4M3 codes and biased exponents of x's rows: the smallest 2^e with max|x| <= 448 * 2^e, e within +-60, 0 for a row of zeros."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    f, e = torch.frexp(top)
    e = torch.where(top > 0, (e - 9 + (f > 0.875).int()).clamp(-60, 60), 0)
    return (x * _power(-e)).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    d, dtype = case["head_dim"], TYPES[case["dtype"]]
    s = {"case": case}
    if case["op"] == "rope":
        s["x"] = _normal((case["tokens"], case["heads"], d), g, dtype)
        s["pos"] = torch.randint(0, case["far"], (case["tokens"],), generator=g, device="cuda", dtype=torch.int32)
        s["freq"] = _frequencies(case).cuda()
        s["amplitude"] = 0.1 * math.log(8) + 1 if case["scaling"] == "ramp" else 1.0
        return s
    lens, page, heads = _lengths(case), case["page"], case["heads"]
    used = [-(-n // page) for n in lens]
    total = sum(used) + 3                                   # a pool with a few pages free
    # pages were handed out in no order; a table's entries past a sequence's last page hold -1
    table = torch.full((len(lens), max(used) + 1), -1, dtype=torch.int32)
    r = random.Random(seed)
    order = r.sample(range(total), total)
    at = 0
    for b, n in enumerate(used):
        table[b, :n] = torch.tensor(order[at:at + n], dtype=torch.int32)
        at += n
    s["table"] = table.cuda()
    s["max_len"] = max(lens)
    kv = case["kv"]
    shape = (total, heads, page, d)
    s["k_scale"] = s["v_scale"] = None
    if kv == "e4m3":
        # pools of codes, as rows of normal values of slowly varying size leave them
        s["k"], s["v"] = (torch.empty(shape, dtype=torch.float8_e4m3fn, device="cuda") for _ in range(2))
        s["k_scale"], s["v_scale"] = (torch.empty(shape[:3], dtype=torch.uint8, device="cuda") for _ in range(2))
        for pool, scale in ((s["k"], s["k_scale"]), (s["v"], s["v_scale"])):
            step = max(1, (1 << 26) // (heads * page * d))
            for lo in range(0, total, step):
                x = _normal((min(step, total - lo), heads, page, d), g, torch.bfloat16)
                codes, e = _to_codes(x * torch.rand((x.shape[0], heads, page, 1), generator=g, device="cuda"))
                pool[lo:lo + step].view(torch.uint8).copy_(codes.view(torch.uint8))
                scale[lo:lo + step] = e[..., 0]
    else:
        s["k"], s["v"] = _normal(shape, g, TYPES[kv]), _normal(shape, g, TYPES[kv])
    if case["op"] == "attn":
        s["q"] = _normal((case["seqs"], heads * case["group"], d), g, dtype)
        s["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        s["scratch"] = torch.zeros(SCRATCH_BYTES, dtype=torch.uint8, device="cuda")
        return s
    seq, pos = _tokens(case)
    s["seq"], s["pos"] = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in (seq, pos))
    if case["op"] != "read":
        s["k_new"], s["v_new"] = (_normal((len(seq), heads, d), g, dtype) for _ in range(2))
    return s


# ---- the operators ---------------------------------------------------------------------------------------------------

def _cache(s):
    """The framework's handle of this state's cache, which a user's program makes once, when it lays the cache out."""
    if "handle" not in s:
        from paper_2512_21571_b200 import binding
        s["handle"] = binding.PagedKV(s["k"], s["v"], s["table"], s["k_scale"], s["v_scale"])
    return s["handle"]


def _rope_plain(s):
    c, x = s["case"], s["x"].float()
    angle = s["pos"].double()[:, None] * s["freq"]
    cos, sin = (s["amplitude"] * f(angle).float()[:, None] for f in (torch.cos, torch.sin))
    if c["inverse"]:
        sin = -sin
    rot = c["rotary_dim"]
    if c["interleaved"]:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., rot:]], -1).to(s["x"].dtype)


def _rows(s):
    """Pool indices (page, slot) of the call's tokens."""
    page = s["case"]["page"]
    pos = s["pos"].long()
    return s["table"][s["seq"].long(), pos // page].long(), pos % page


def _write_plain(s):
    at, slot = _rows(s)
    for_k, for_v = s["k_new"].float(), s["v_new"].float()
    if s["case"]["kv"] == "e4m3":
        (k, ke), (v, ve) = _to_codes(for_k), _to_codes(for_v)
        s["k"].view(torch.uint8)[at, :, slot] = k.view(torch.uint8)
        s["v"].view(torch.uint8)[at, :, slot] = v.view(torch.uint8)
        s["k_scale"][at, :, slot] = ke[..., 0]
        s["v_scale"][at, :, slot] = ve[..., 0]
    else:
        s["k"][at, :, slot] = for_k.to(s["k"].dtype)
        s["v"][at, :, slot] = for_v.to(s["v"].dtype)


def _values(rows, scale):
    """Rows taken from a pool, as 32-bit values."""
    if scale is None:
        return rows.float()
    return rows.view(torch.float8_e4m3fn).float() * _power(scale.int()[..., None] - 127)


def _pool(x):
    return x.view(torch.uint8) if x.dtype is torch.float8_e4m3fn else x


def _read_plain(s):
    at, slot = _rows(s)
    scale = lambda x: None if x is None else x[at, :, slot]
    dtype = TYPES[s["case"]["dtype"]]
    return {"k": _values(_pool(s["k"])[at, :, slot], scale(s["k_scale"])).to(dtype),
            "v": _values(_pool(s["v"])[at, :, slot], scale(s["v_scale"])).to(dtype)}


def _attn_plain(s):
    c, page = s["case"], s["case"]["page"]
    columns = -(-s["max_len"] // page)
    table = s["table"][:, :columns].long().clamp(min=0)
    laid = lambda x: x.transpose(1, 2).flatten(2, 3)         # [seqs][heads][positions][head_dim]
    k = laid(_values(_pool(s["k"])[table], None if s["k_scale"] is None else s["k_scale"][table]))
    v = laid(_values(_pool(s["v"])[table], None if s["v_scale"] is None else s["v_scale"][table]))
    q = s["q"].float().unflatten(1, (c["heads"], c["group"]))
    pos = torch.arange(columns * page, device="cuda")
    n = s["lens"].long()[:, None]
    live = pos < n
    if c["window"]:
        live &= pos >= n - c["window"]
    score = (q @ k.transpose(-1, -2) * c["head_dim"] ** -0.5).masked_fill(~live[:, None, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - top.clamp(min=-3e38))
    total = p.sum(-1, keepdim=True)
    out = p @ v.masked_fill(~live[:, None, :, None], 0.0) / total.clamp(min=1e-38)
    lse = (top + torch.log(total))[..., 0]
    return {"out": out.flatten(1, 2).to(s["q"].dtype), "lse": lse.flatten(1, 2)}


def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2512_21571_b200 import binding
        if c["op"] == "rope":
            return binding.op_rope(s["x"], s["pos"], s["freq"], interleaved=c["interleaved"], amplitude=s["amplitude"], inverse=c["inverse"])
        cache = _cache(s)
        if c["op"] == "attn":
            out, lse = binding.op_attn_decode_paged(s["q"], cache, s["lens"], window=c["window"], scratch=s["scratch"], want_lse=True)
            return {"out": out, "lse": lse}
        if c["op"] != "read":
            binding.op_kv_write_paged(cache, s["k_new"], s["v_new"], s["pos"], s["seq"])
        if c["op"] == "write":
            return {"k": s["k"], "v": s["v"]}
        k, v = binding.op_kv_read_paged(cache, s["pos"], s["seq"], dtype=TYPES[c["dtype"]])
        return {"k": k, "v": v}
    if c["op"] == "rope":
        return _rope_plain(s)
    if c["op"] == "attn":
        return _attn_plain(s)
    if c["op"] != "read":
        _write_plain(s)
    if c["op"] == "write":
        return {"k": s["k"], "v": s["v"]}
    return _read_plain(s)


# ---- the operators from their definitions, in 64 bits -------------------------------------------------------------------

def _power64(e):
    """2^e for whole e, exactly."""
    return (e.long() + 1023 << 52).view(torch.float64)


def _e4m3_table():
    """The 256 values of E4M3: sign, four exponent bits of bias 7, three mantissa bits; 0x7f and 0xff are NaN."""
    got = []
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        x = math.nan if code & 127 == 127 else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        got.append(-x if code >> 7 else x)
    return torch.tensor(got, dtype=torch.float64, device="cuda")


def _exact_row(s, which, b, first, end):
    """Cached positions [first, end) of sequence b: [heads][positions][head_dim] in 64 bits."""
    page, pool, scale = s["case"]["page"], s[which], s[which + "_scale"]
    pages = s["table"][b, first // page:-(-end // page)].long()
    x = pool.view(torch.uint8)[pages] if scale is not None else pool[pages]
    if scale is not None:
        x = _e4m3_table()[x.long()] * _power64(scale[pages].long()[..., None] - 127)
    x = x.double().permute(1, 0, 2, 3).reshape(pool.shape[1], -1, pool.shape[3])
    skip = first // page * page
    return x[:, first - skip:end - skip]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        rot = case["rotary_dim"]
        x = s["x"].double()
        turn = torch.polar(torch.full((), s["amplitude"], dtype=torch.float64, device="cuda"),
                           (-1 if case["inverse"] else 1) * s["pos"].double()[:, None, None] * s["freq"])
        pair = (x[..., :rot].unflatten(-1, (rot // 2, 2)) if case["interleaved"] else x[..., :rot].unflatten(-1, (2, rot // 2)).transpose(-1, -2))
        z = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
        x[..., :rot] = (z if case["interleaved"] else z.transpose(-1, -2)).flatten(-2)
        return x
    if case["op"] == "attn":
        lens = _lengths(case)
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            first = max(0, n - case["window"]) if case["window"] else 0
            if n == first:
                continue
            k, v = _exact_row(s, "k", b, first, n), _exact_row(s, "v", b, first, n)
            q = s["q"][b].double().reshape(case["heads"], case["group"], -1)
            score = torch.einsum("hgd,hnd->hgn", q, k) / math.sqrt(case["head_dim"])
            out[b] = torch.einsum("hgn,hnd->hgd", torch.softmax(score, -1), v).reshape(out[b].shape)
            lse[b] = torch.logsumexp(score, -1).reshape(-1)
        return {"out": out, "lse": lse}
    if case["op"] == "write":
        k, v = s["k"].double(), s["v"].double()
        at, slot = _rows(s)
        k[at, :, slot], v[at, :, slot] = s["k_new"].double(), s["v_new"].double()
        return {"k": k, "v": v}
    if case["op"] == "turn":
        return {"k": _exact_turn(s["k_new"]), "v": _exact_turn(s["v_new"])}
    seq, pos = _tokens(case)
    runs = [(b, n) for b, n in enumerate(_lengths(case)) if n]
    take = lambda which: torch.cat([_exact_row(s, which, b, max(0, n - case["new"]), n).transpose(0, 1) for b, n in runs])
    return {"k": take("k"), "v": take("v")}


def _exact_turn(x):
    """What a row becomes through the cache: the nearest E4M3 multiple of its scale, ties to the even code."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(top, -60)
    for step in range(-60, 60):
        e = torch.where(top > 448 * 2.0 ** step, step + 1.0, e)      # the smallest e whose largest code reaches the row
    e = torch.where(top > 0, e, 0.0)
    y = x / _power64(e)
    unit = _power64(torch.frexp(y.abs().clamp(min=2.0 ** -6))[1] - 4)
    return torch.round(y / unit) * unit * _power64(e)
