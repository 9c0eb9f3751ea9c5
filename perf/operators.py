"""Performance cases of the 8-bit paged cache and what goes round it: rotary positions, storing rows, attention over
the cache, and the management of its pages.

A case is a dict of plain values; `listed()` holds the fixed ones, `draw(rng)` makes one more of the same ranges,
`prepare` builds what a program has in hand before the call, `run` makes one pass, `work` says what a pass cannot do
without, `exact` is the same pass in 64 bits.

Kinds of cases (`op`):
  rotary     q, k and v of a pass out of the projection's output: rotation of q and k, all three to the operand type
  attention  rows of a pass against the cached tokens of their sequences and against one another (tree or causal)
  store      rows of K and V go into the pages of all layers; the rows of the touched pages are read back
  fork       answers of one prompt: sequences share its pages, take room for new tokens, are dropped again
  turnover   a sequence leaves, the pool is compacted, a new sequence is admitted

With `own` false a pass is elementary torch operations in 32 bits on the same tensors, rounded once at the end.

The cache's tensors: codes uint8 [layer][kv head][page][K|V][16 * D], scales float32 [layer][kv head][page][K|V],
page_table int32 [sequence][page], refs int32 [page] (sequences that hold the page), lens int32 [sequence]. A K block is
[token / 8][dim / 16][token % 8][dim % 16], a V block [dim][place of the token] with PLACE below; a value is code * scale, codes being
int8 or e4m3 bytes.
"""
import math
import random

import torch

own = False                                     # false: plain forms; true: the framework's kernels

DEVICE = "cuda:0"
PAGE = 16
PLACE = [4 * ((t % 8) // 2) + 2 * (t // 8) + t % 2 for t in range(PAGE)]
QMAX = {"int8": 127.0, "e4m3": 448.0}
FLUSH = 2.0 ** -100                             # a page whose largest magnitude is below this is stored as zeros, scale 0
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}

# head shapes of the repository's configurations: (query heads, kv heads, head dim)
WIDE = dict(heads=32, kv=32, hd=128)
GROUPED = dict(heads=32, kv=8, hd=128)
MEDIUM = dict(heads=16, kv=4, hd=64)


def _attention(name, shape, batch, lo, hi, rows, mask="tree", fmt="int8", dtype="bf16"):
    c = dict(op="attention", **shape, batch=batch, lo=lo, hi=hi, rows=rows, mask=mask, fmt=fmt, dtype=dtype)
    return dict(name=name, **c) if name else c


def listed():
    return [
        # projections' output of one 64-node tree: launch and latency
        dict(name="rotary_tree64", op="rotary", **WIDE, rows=64, rot=128, layout="half", scaling="none", source="fp32", dtype="bf16", span=8192),
        # a long prompt, grouped heads, table stretched for long contexts
        dict(name="rotary_prompt_4096", op="rotary", **GROUPED, rows=4096, rot=128, layout="half", scaling="yarn", source="bf16", dtype="bf16", span=32768),
        # the next token of one short sequence: latency
        _attention("attention_token_short", MEDIUM, 1, 300, 300, 1, mask="causal"),
        # next tokens of sixteen ragged sequences served together, grouped heads
        _attention("attention_tokens_batch16", GROUPED, 16, 128, 8192, 1, mask="causal"),
        # a 64-node tree far into a long context, 7B heads: what the verification of the long configuration reads
        _attention("attention_tree64_8192", WIDE, 1, 8192, 8192, 64),
        # three sequences of odd lengths with 23-node trees, heads of 64, e4m3 codes
        _attention("attention_tree23_batch3", MEDIUM, 3, 37, 2411, 23, fmt="e4m3"),
        # second half of a 4096-token prompt: 2048 rows, causal, 2048 tokens cached
        _attention("attention_prompt_2048", WIDE, 1, 2048, 2048, 2048, mask="causal"),
        # accepted paths of sixteen sequences into the cache of all 32 layers
        dict(name="store_accepted_batch16", op="store", **WIDE, layers=32, batch=16, lo=128, hi=2048, rows=64, count_lo=1, count_hi=5, fmt="int8", dtype="bf16"),
        # a prompt's rows into an empty cache, eight layers
        dict(name="store_prompt_2048", op="store", **WIDE, layers=8, batch=1, lo=0, hi=0, rows=2048, count_lo=2048, count_hi=2048, fmt="e4m3", dtype="bf16"),
        # twenty answers to one prompt: shared pages, copies of the last one, and all dropped again
        dict(name="fork_20_answers", op="fork", **WIDE, layers=32, batch=20, lo=2041, hi=2041, count=5),
        # two answers to a short prompt, grouped heads: latency
        dict(name="fork_2_answers", op="fork", **MEDIUM, layers=6, batch=2, lo=411, hi=411, count=5),
        # continuous serving: one of eight sequences leaves, the pool is compacted, another is admitted
        dict(name="turnover_batch8", op="turnover", **GROUPED, layers=16, batch=8, lo=512, hi=2048),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng: random.Random):
    op = rng.choices(["attention", "rotary", "store", "fork", "turnover"], [6, 2, 2, 1, 1])[0]
    shape = rng.choice([WIDE, GROUPED, MEDIUM, dict(heads=12, kv=4, hd=128), dict(heads=8, kv=1, hd=64)])
    fmt, dtype = rng.choice(["int8", "int8", "e4m3"]), rng.choice(["bf16", "bf16", "fp16"])
    if op == "rotary":
        rot = rng.choice([shape["hd"], shape["hd"], shape["hd"] // 2, shape["hd"] // 4])
        return dict(op=op, **shape, rows=_log(rng, 1, 4096), rot=rot, layout=rng.choice(["half", "interleaved"]),
                    scaling=rng.choice(["none", "linear", "ntk", "yarn"]), source=rng.choice(["fp32", "bf16"]), dtype=dtype, span=_log(rng, 4096, 65536))
    if op == "store":
        if rng.random() < 0.6:
            return dict(op=op, **shape, layers=rng.randint(1, 32), batch=_log(rng, 1, 16), lo=0, hi=_log(rng, 16, 2048), rows=rng.randint(5, 64),
                        count_lo=1, count_hi=5, fmt=fmt, dtype=dtype)
        rows = _log(rng, 16, 2048)
        return dict(op=op, **shape, layers=rng.randint(1, 8), batch=1, lo=0, hi=_log(rng, 1, 500), rows=rows, count_lo=rows, count_hi=rows, fmt=fmt, dtype=dtype)
    if op == "fork":
        n = _log(rng, 16, 4000)
        return dict(op=op, **shape, layers=rng.randint(1, 32), batch=_log(rng, 1, 32), lo=n, hi=n, count=rng.randint(1, 40))
    if op == "turnover":
        hi = _log(rng, 64, 2048)
        return dict(op=op, **shape, layers=rng.randint(1, 16), batch=rng.randint(2, 12), lo=max(16, hi // 8), hi=hi)
    kind = rng.choice(["token", "tree", "tree", "prompt"])
    if kind == "prompt":
        return _attention("", shape, 1, 0, _log(rng, 16, 2048), _log(rng, 65, 2048), mask="causal", fmt=fmt, dtype=dtype)
    batch = rng.choice([1, 1, rng.randint(2, 4), rng.randint(2, 16)])
    hi = _log(rng, 16, 16384 if batch == 1 else 4096)
    return _attention("", shape, batch, hi if batch == 1 else max(1, hi // 8), hi, 1 if kind == "token" else rng.choice([16, 32, 64, 128, rng.randint(2, 128)]),
                      mask="causal" if kind == "token" else "tree", fmt=fmt, dtype=dtype)


# ---------------------------------------------------------------- inputs
def _lens(case):
    """Cached tokens of each sequence: spread over [lo, hi], in no order."""
    B, lo, hi = case["batch"], case["lo"], case["hi"]
    return [hi - (hi - lo) * ((b * 5) % B) // max(B - 1, 1) for b in range(B)]


def _counts(case):
    lo, hi = case["count_lo"], case["count_hi"]
    return [lo + (b * 3 + 1) % (hi - lo + 1) for b in range(case["batch"])]


def _pages(tokens):
    return -(-tokens // PAGE)


def _scale_of(amax, fmt):
    return torch.where(amax < FLUSH, torch.zeros_like(amax), amax / QMAX[fmt])


def _fill(g, case, layers, n_pages, fmt):
    """Codes and scales of a pool: rows as a cache holds them (channels of unequal size, pages of unequal size), quantised page by page."""
    kv, D = case["kv"], case["hd"]
    channel = torch.exp(0.5 * torch.randn((kv, 2, D), generator=g, device=DEVICE))
    codes = torch.empty((layers, kv, n_pages, 2, PAGE * D), dtype=torch.uint8, device=DEVICE)
    scales = torch.empty((layers, kv, n_pages, 2), device=DEVICE)
    for l in range(layers):
        x = torch.randn((kv, n_pages, 2, PAGE, D), generator=g, device=DEVICE)
        x *= channel[:, None, :, None, :] * torch.exp(0.2 * torch.randn((kv, n_pages, 2, 1, 1), generator=g, device=DEVICE))
        s = _scale_of(x.abs().amax(dim=(-1, -2)), fmt)
        x /= s[..., None, None]
        codes[l] = _pack(x, fmt)
        scales[l] = s
    return codes, scales


def _pack(x, fmt):
    """[..., K|V, 16, D] values in units of the scale -> bytes in the order of the pool."""
    lead, D = x.shape[:-3], x.shape[-1]
    k = x[..., 0, :, :].reshape(*lead, 2, 8, D // 16, 16).transpose(-2, -3).reshape(*lead, PAGE * D)
    order = torch.tensor([PLACE.index(p) for p in range(PAGE)], device=x.device)
    v = x[..., 1, :, :].index_select(-2, order).transpose(-1, -2).reshape(*lead, PAGE * D)
    y = torch.stack([k, v], dim=-2)
    if fmt == "int8":
        return y.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _unpack(codes, fmt):
    """Inverse of _pack: bytes [..., K|V, 16 * D] -> float32 [..., K|V, 16, D] in units of the scale."""
    lead, D = codes.shape[:-2], codes.shape[-1] // PAGE
    y = (codes.view(torch.int8) if fmt == "int8" else codes.view(torch.float8_e4m3fn)).float()
    k = y[..., 0, :].reshape(*lead, 2, D // 16, 8, 16).transpose(-2, -3).reshape(*lead, PAGE, D)
    v = y[..., 1, :].reshape(*lead, D, PAGE).index_select(-1, torch.tensor(PLACE, device=y.device)).transpose(-1, -2)
    return torch.stack([k, v], dim=-3)


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device=DEVICE)


def _state_of_cache(s, case, g, layers, lens, room, fmt, spare=0):
    """A pool in which every sequence holds pages for `room` tokens, scattered over the pool as after some time of use."""
    need = [_pages(r) for r in room]
    n_pages = sum(need) + spare
    order = torch.randperm(n_pages, generator=g, device=DEVICE).to(torch.int32)
    width = max(need + [1])
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device=DEVICE)
    refs = torch.zeros(n_pages, dtype=torch.int32, device=DEVICE)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    refs[order[:at].long()] = 1
    codes, scales = _fill(g, case, layers, n_pages, fmt)
    s.update(codes=codes, scales=scales, page_table=table, refs=refs, lens=_int(lens), fmt=fmt)


def _tree(nodes, rng):
    """Ancestor sets of a random candidate tree, as bit words: node i sees itself and the nodes on its path to the root."""
    sees, out = [], []
    for i in range(nodes):
        up = sees[rng.randrange(max(0, i - 12), i)] if i else 0
        sees.append(up | (1 << i))
    words = -(-nodes // 32)
    for m in sees:
        out.append([(m >> (32 * w)) & 0xFFFFFFFF for w in range(words)])
    return [[v - (1 << 32) if v >= 1 << 31 else v for v in row] for row in out]


def _inv_freq(case, dtype):
    """Angular step of each pair, with the scaling for long contexts."""
    rot, base, factor, original = case["rot"], 1e6, 4.0, 8192
    if case["scaling"] == "ntk":
        base = base * factor ** (rot / (rot - 2))
    f = base ** (-torch.arange(0, rot, 2, dtype=dtype, device=DEVICE) / rot)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "yarn":
        turn = lambda beta: rot * math.log(original / (beta * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        low, high = max(math.floor(turn(32.0)), 0), min(math.ceil(turn(1.0)), rot - 1)
        ramp = ((torch.arange(rot // 2, dtype=dtype, device=DEVICE) - low) / max(high - low, 1e-3)).clamp(0, 1)
        f = f * (1 - ramp) + f / factor * ramp
    return f, (0.1 * math.log(factor) + 1.0 if case["scaling"] == "yarn" else 1.0)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    rng = random.Random(seed)
    op, s = case["op"], {"case": dict(case), "scale": 1.0 / math.sqrt(case["hd"])}
    kv, D, H = case["kv"], case["hd"], case["heads"]
    dt = TYPES.get(case.get("dtype", "bf16"))
    if op == "rotary":
        R = case["rows"]
        s["qkv"] = torch.randn((R, (H + 2 * kv) * D), generator=g, device=DEVICE).to(TYPES[case["source"]])
        start = rng.randrange(case["span"] - R + 1) if case["span"] > R else 0
        # positions of a tree repeat: depths 0, 1, 1, 2, ... after the sequence's length; a prompt's run on
        offs = [i if R > 128 else int(math.log2(i + 1)) for i in range(R)]
        s["positions"] = _int([min(start + o, case["span"] - 1) for o in offs])
        f, gain = _inv_freq(case, torch.float64)
        a = torch.arange(case["span"], dtype=torch.float64, device=DEVICE)[:, None] * f
        s["table"] = (torch.stack([a.cos(), a.sin()], dim=-1) * gain).float().contiguous()
        return s
    lens, B = _lens(case), case["batch"]
    if op == "attention":
        _state_of_cache(s, case, g, 1, lens, lens, case["fmt"], spare=3)
        R = case["rows"]
        # queries as peaked as a trained model's: scores spread over several units
        s["q"] = (2.0 * torch.randn((B * R, H, D), generator=g, device=DEVICE)).to(dt)
        s["k"] = torch.randn((B * R, kv, D), generator=g, device=DEVICE).to(dt)
        s["v"] = torch.randn((B * R, kv, D), generator=g, device=DEVICE).to(dt)
        s["mask"] = _int([w for _ in range(B) for w in _tree(R, rng)]) if case["mask"] == "tree" else None
    elif op == "store":
        counts, C = _counts(case), case["count_hi"]
        _state_of_cache(s, case, g, case["layers"], [n + c for n, c in zip(lens, counts)], [n + c for n, c in zip(lens, counts)], case["fmt"], spare=3)
        R = case["rows"]
        s["k"] = (1.5 * torch.randn((case["layers"], B * R, kv, D), generator=g, device=DEVICE)).to(dt)
        s["v"] = (1.5 * torch.randn((case["layers"], B * R, kv, D), generator=g, device=DEVICE)).to(dt)
        s["counts"] = _int(counts)
        s["path"] = _int([sorted(rng.sample(range(R), C)) for _ in range(B)])
        s["start"] = _int([n // PAGE * PAGE for n in lens])
        s["window"] = max(_pages(n + c) - n // PAGE for n, c in zip(lens, counts)) * PAGE
    elif op == "fork":
        n, C = case["lo"], case["count"]
        _state_of_cache(s, case, g, case["layers"], [n], [n], "int8", spare=B * (_pages(n + C) - n // PAGE) + 5)
        width = _pages(n + C)
        table = torch.full((B + 1, width), -1, dtype=torch.int32, device=DEVICE)
        table[0, :_pages(n)] = s["page_table"][0]
        s.update(page_table=table, lens=_int([n] + [0] * B), src=_int([0] * B), dst=_int(list(range(1, B + 1))), counts=_int([C] * B))
    elif op == "turnover":
        _state_of_cache(s, case, g, case["layers"], lens, lens, "int8", spare=max(_pages(n) for n in lens))
        s.update(turn=0, slots=[_int([b]) for b in range(B)], new=[_int([n]) for n in lens])
    if own and op != "rotary":
        from paper_2503_14153_b200 import SpecCache
        s["cache"] = SpecCache.from_tensors(s["codes"], s["scales"], s["page_table"], s["refs"], s["lens"], fmt=s["fmt"])
    return s


# ---------------------------------------------------------------- one pass
def run(s):
    case = s["case"]
    if not own:
        return {"rotary": _plain_rotary, "attention": _plain_attention, "store": _plain_store, "fork": _plain_fork, "turnover": _plain_turnover}[case["op"]](s, case)
    if case["op"] == "rotary":
        from paper_2503_14153_b200 import spec_rotary
        R, H, kv, D = case["rows"], case["heads"], case["kv"], case["hd"]
        q, k, v = s["qkv"].view(R, H + 2 * kv, D).split((H, kv, kv), dim=1)
        return spec_rotary(q, k, v, s["positions"], s["table"], interleaved=case["layout"] == "interleaved", dtype=TYPES[case["dtype"]])
    cache = s["cache"]
    if case["op"] == "attention":
        return cache.attention(0, s["q"], s["k"], s["v"], batch=case["batch"], mask=s["mask"], scale=s["scale"], lse=True)
    if case["op"] == "store":
        cache.store(s["k"], s["v"], s["counts"], path=s["path"])
        k, v = cache.read(s["start"], s["window"], batch=case["batch"], dtype=TYPES[case["dtype"]])
        return k, v, cache.scales
    if case["op"] == "fork":
        cache.fork(s["src"], s["dst"])
        granted = cache.reserve(s["counts"], seqs=s["dst"])
        taken, refs, lens = cache.page_table.clone(), cache.refs.clone(), cache.lens.clone()
        cache.truncate(seqs=s["dst"])
        return granted, taken, refs, lens, cache.page_table, cache.refs, cache.lens, cache.codes
    t = s["turn"] % case["batch"]
    s["turn"] += 1
    cache.truncate(seqs=s["slots"][t])
    used = cache.compact()
    granted = cache.reserve(s["new"][t], seqs=s["slots"][t])
    return used, granted, cache.page_table, cache.refs, cache.lens, cache.codes


def _plain_rotary(s, case):
    R, H, kv, D, rot = case["rows"], case["heads"], case["kv"], case["hd"], case["rot"]
    x = s["qkv"].view(R, H + 2 * kv, D).float()
    cs = s["table"][s["positions"].long()][:, None]
    c, n = cs[..., 0], cs[..., 1]
    qk = x[:, :H + kv]
    if case["layout"] == "half":
        a, b = qk[..., :rot // 2], qk[..., rot // 2:rot]
        y = torch.cat([a * c - b * n, b * c + a * n, qk[..., rot:]], dim=-1)
    else:
        a, b = qk[..., 0:rot:2], qk[..., 1:rot:2]
        y = torch.cat([torch.stack([a * c - b * n, b * c + a * n], dim=-1).flatten(-2), qk[..., rot:]], dim=-1)
    dt = TYPES[case["dtype"]]
    return y[:, :H].to(dt), y[:, H:].to(dt), x[:, H + kv:].to(dt)


def _cached_rows(s, case, N):
    """Cached K and V of all sequences, [2][batch, kv head, N, D] float32 (N rounded up to pages; rows past a sequence's end are whatever is there)."""
    B, kv, D, P = case["batch"], case["kv"], case["hd"], _pages(N)
    pages = s["page_table"][:, :P].clamp(min=0).long()
    x = _unpack(s["codes"][0][:, pages], s["fmt"]) * s["scales"][0][:, pages][..., None, None]       # [kv, B, P, 2, 16, D]
    return x.permute(3, 1, 0, 2, 4, 5).reshape(2, B, kv, P * PAGE, D)


def _plain_attention(s, case):
    B, R, H, kv, D = case["batch"], case["rows"], case["heads"], case["kv"], case["hd"]
    G, N = H // kv, max(_lens(case))
    new = lambda x: x.float().view(B, R, kv, D).transpose(1, 2)  # noqa: E731
    K, V = _cached_rows(s, case, N)
    NP = K.shape[2]
    K, V = torch.cat([K, new(s["k"])], dim=2), torch.cat([V, new(s["v"])], dim=2)
    q = s["q"].float().view(B, R, kv, G, D).permute(0, 2, 1, 3, 4).reshape(B, kv, R * G, D)
    z = torch.matmul(q, K.transpose(-1, -2)) * s["scale"]
    at = torch.arange(R, device=DEVICE)
    if s["mask"] is None:
        sees = (at[None, :] <= at[:, None]).expand(B, R, R)
    else:
        sees = ((s["mask"].view(B, R, -1)[:, :, at // 32] >> (at % 32)) & 1).bool()
    old = (torch.arange(NP, device=DEVICE) < s["lens"][:, None])[:, None, :].expand(B, R, NP)
    keep = torch.cat([old, sees], dim=2)[:, None, :, None].expand(B, kv, R, G, NP + R).reshape(B, kv, R * G, NP + R)
    z = torch.where(keep, z, torch.full_like(z, -math.inf))
    top = z.amax(dim=-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(z - top)
    total = p.sum(dim=-1, keepdim=True)
    o = torch.matmul(p, V) / torch.where(total > 0, total, torch.ones_like(total))
    rows = lambda x: x.view(B, kv, R, G, -1).permute(0, 2, 1, 3, 4).reshape(B * R, H, -1)  # noqa: E731
    return rows(o).to(s["q"].dtype), rows(top + torch.log(total)).squeeze(-1)


def _plain_store(s, case):
    B, R, kv, D, L = case["batch"], case["rows"], case["kv"], case["hd"], case["layers"]
    W, fmt = s["window"], s["fmt"]
    PT = W // PAGE
    page = s["start"].long()[:, None] // PAGE + torch.arange(PT, device=DEVICE)                # [B, PT]
    ids = torch.where(page < s["page_table"].shape[1], s["page_table"].gather(1, page.clamp(max=s["page_table"].shape[1] - 1)), -1).long()
    first = (s["lens"] - s["counts"]).long()
    pos = (page[..., None] * PAGE + torch.arange(PAGE, device=DEVICE)).view(B, W)
    fresh = (pos >= first[:, None]) & (pos < s["lens"][:, None])
    held = pos < first[:, None]
    row = s["path"].long().gather(1, (pos - first[:, None]).clamp(0, s["path"].shape[1] - 1)) + torch.arange(B, device=DEVICE)[:, None] * R
    x = torch.stack([s["k"], s["v"]], dim=1)[:, :, row].float()                                # [L, 2, B, W, kv, D]
    x = torch.where(fresh[:, :, None, None], x, torch.zeros_like(x)).view(L, 2, B, PT, PAGE, kv, D).permute(0, 5, 2, 3, 1, 4, 6)
    got = ids.clamp(min=0)
    was = s["scales"][:, :, got] * held.view(B, PT, PAGE)[..., :1]                             # [L, kv, B, PT, 2]
    now = torch.maximum(was, _scale_of(x.abs().amax(dim=(-1, -2)), fmt))
    div = torch.where(now > 0, now, torch.ones_like(now))[..., None, None]
    old = _unpack(s["codes"][:, :, got], fmt) * (was[..., None, None] / div)
    code = _pack(torch.where(held.view(B, PT, 1, PAGE, 1), old, x / div), fmt)
    touched = fresh.view(B, PT, PAGE).any(dim=-1)
    s["codes"][:, :, ids[touched]] = code[:, :, touched]
    s["scales"][:, :, ids[touched]] = now[:, :, touched]
    y = _unpack(s["codes"][:, :, got], fmt) * s["scales"][:, :, got][..., None, None]           # [L, kv, B, PT, 2, 16, D]
    y = y.permute(4, 0, 2, 3, 5, 1, 6).reshape(2, L, B, W, kv, D)
    y = torch.where((pos < s["lens"][:, None])[:, :, None, None], y, torch.zeros_like(y)).to(TYPES[case["dtype"]])
    return y[0], y[1], s["scales"]


def _free_pages(s, count):
    """The `count` lowest free pages."""
    return torch.sort((s["refs"] > 0).int(), stable=True)[1][:count]


def _plain_fork(s, case):
    B, n, C = case["batch"], case["lo"], case["count"]
    table, refs, lens = s["page_table"], s["refs"], s["lens"]
    held, need = _pages(n), _pages(n + C)
    dst, src = s["dst"].long(), s["src"].long()
    table[dst, :held] = table[src, :held]
    refs.index_add_(0, table[dst, :held].reshape(-1).long(), torch.ones(B * held, dtype=torch.int32, device=DEVICE))
    lens[dst] = lens[src]
    first = n // PAGE if n % PAGE else held                     # a partial last page is shared: every answer gets its own
    if need > first:
        take = _free_pages(s, B * (need - first)).view(B, need - first)
        if held > first:
            old = table[dst, first].long()
            s["codes"][:, :, take[:, 0]] = s["codes"][:, :, old]
            s["scales"][:, :, take[:, 0]] = s["scales"][:, :, old]
            refs.index_add_(0, old, torch.full((B,), -1, dtype=torch.int32, device=DEVICE))
        table[dst, first:need] = take.to(torch.int32)
        refs[take.reshape(-1)] = 1
    lens[dst] += s["counts"]
    granted = s["counts"].clone()
    taken, counted, long = table.clone(), refs.clone(), lens.clone()
    refs.index_add_(0, table[dst, :need].reshape(-1).long(), torch.full((B * need,), -1, dtype=torch.int32, device=DEVICE))
    table[dst] = -1
    lens[dst] = 0
    return granted, taken, counted, long, table, refs, lens, s["codes"]


def _plain_turnover(s, case):
    t = s["turn"] % case["batch"]
    s["turn"] += 1
    table, refs, lens, n = s["page_table"], s["refs"], s["lens"], _lens(case)[t]
    P = _pages(n)
    refs[table[t, :P].long()] -= 1
    table[t] = -1
    lens[t] = 0
    held = refs > 0
    used = held.sum()
    at = torch.arange(refs.numel(), device=DEVICE)
    src, dst = (held & (at >= used)).nonzero().view(-1), (~held & (at < used)).nonzero().view(-1)
    s["codes"][:, :, dst] = s["codes"][:, :, src]
    s["scales"][:, :, dst] = s["scales"][:, :, src]
    to = at.clone()
    to[src] = dst
    table.copy_(torch.where(table >= 0, to[table.clamp(min=0).long()].to(torch.int32), table))
    refs[dst], refs[src] = refs[src], 0
    take = _free_pages(s, P)
    table[t, :P] = take.to(torch.int32)
    refs[take] = 1
    lens[t] = n
    return used.to(torch.int32).view(1), s["new"][t].clone(), table, refs, lens, s["codes"]


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    kv, D, H = case["kv"], case["hd"], case["heads"]
    size = lambda t: {"fp32": 4}.get(t, 2)  # noqa: E731
    block = PAGE * D + 4                                        # codes and scale of a page, one head, K or V
    if case["op"] == "rotary":
        n = case["rows"] * (H + 2 * kv) * D
        return {"bytes": n * (size(case["source"]) + size(case["dtype"])) + case["rows"] * (4 * case["rot"] + 4), "flops": 3 * case["rows"] * (H + kv) * case["rot"]}
    lens = _lens(case)
    if case["op"] == "attention":
        R, B = case["rows"], case["batch"]
        own_keys = R * (R + 1) // 2 if case["mask"] == "causal" else R * min(R, 6)
        cached = sum(n * D + 4 * _pages(n) for n in lens) * 2 * kv
        return {"bytes": cached + B * R * (4 * H + 4 * kv) * D + 4 * B * R * H, "flops": 4 * H * D * (R * sum(lens) + B * own_keys)}
    L = case["layers"]
    if case["op"] == "store":
        rows = pages = window = 0
        for n, c in zip(lens, _counts(case)):
            rows += c
            pages += _pages(n + c) - n // PAGE
            window += n + c - n // PAGE * PAGE
        partial = sum(1 for n in lens if n % PAGE)
        out = max(_pages(n + c) - n // PAGE for n, c in zip(lens, _counts(case))) * PAGE * case["batch"]
        return {"bytes": L * kv * 2 * (rows * D * 2 + (partial + pages) * block + out * D * 2), "flops": 4 * L * kv * 2 * window * D}
    if case["op"] == "fork":
        B, n = case["batch"], case["lo"]
        copies = B if n % PAGE else 0
        return {"bytes": L * kv * 2 * 2 * block * copies + 8 * B * _pages(n + case["count"]) * 2, "flops": 0}
    # the pages of one sequence of middling length are what others move into
    return {"bytes": L * kv * 2 * 2 * block * _pages(sum(lens) // len(lens)) + 4 * sum(_pages(n) for n in lens), "flops": 0}


# ---------------------------------------------------------------- the definition in 64 bits
def _values64(block, scale, fmt, D):
    """A page's 16 rows of K (or V, by `kind`) in 64 bits, read byte by byte from the definition of the layout."""
    tok, dim = torch.meshgrid(torch.arange(PAGE, device=DEVICE), torch.arange(D, device=DEVICE), indexing="ij")
    at_k = (tok // 8) * 8 * D + (dim // 16) * 128 + (tok % 8) * 16 + dim % 16
    at_v = dim * PAGE + torch.tensor(PLACE, device=DEVICE)[tok]
    b = block.long()
    if fmt == "int8":
        val = ((b + 128) % 256 - 128).double()
    else:
        sign, e, m = 1.0 - 2.0 * (b // 128), (b // 8) % 16, (b % 8).double()
        val = sign * torch.where(e > 0, (1 + m / 8) * torch.exp2((e - 7).double()), m / 8 * 2.0 ** -6)
    val = val * scale.double()[..., None]
    return val[..., 0, :][..., at_k], val[..., 1, :][..., at_v]


def exact(case, seed):
    op, D, kv, H = case["op"], case["hd"], case["kv"], case["heads"]
    if op in ("fork", "turnover"):
        return None                                             # whole numbers and copies
    s = prepare(case, seed)
    if op == "rotary":
        R, rot = case["rows"], case["rot"]
        x = s["qkv"].double().view(R, H + 2 * kv, D)
        f, gain = _inv_freq(case, torch.float64)
        turn = torch.polar(torch.full((R, rot // 2), gain, dtype=torch.float64, device=DEVICE), s["positions"].double()[:, None] * f)[:, None]
        y = x.clone()
        lo, hi = (slice(0, rot // 2), slice(rot // 2, rot)) if case["layout"] == "half" else (slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(x[:, :H + kv, lo], x[:, :H + kv, hi]) * turn
        y[:, :H + kv, lo], y[:, :H + kv, hi] = z.real, z.imag
        return y[:, :H], y[:, H:H + kv], y[:, H + kv:]
    if op == "attention":
        R, G, o, lse = case["rows"], H // kv, [], []
        for b, n in enumerate(_lens(case)):
            pages = s["page_table"][b, :_pages(n)].long()
            k, v = _values64(s["codes"][0][:, pages], s["scales"][0][:, pages], s["fmt"], D)
            for h in range(H):
                mine = slice(b * R, (b + 1) * R)
                K = torch.cat([k[h // G].reshape(-1, D)[:n], s["k"][mine, h // G].double()])
                V = torch.cat([v[h // G].reshape(-1, D)[:n], s["v"][mine, h // G].double()])
                z = s["q"][mine, h].double() @ K.T * s["scale"]
                if s["mask"] is None:
                    z[:, n:] += torch.full((R, R), -math.inf, dtype=torch.float64, device=DEVICE).triu(1)
                else:
                    bits = s["mask"][mine].long()
                    for j in range(R):
                        z[(bits[:, j // 32] >> (j % 32)) & 1 == 0, n + j] = -math.inf
                lse.append(torch.logsumexp(z, dim=1))
                o.append(torch.softmax(z, dim=1) @ V)
        shape = lambda xs: torch.stack(xs).view(case["batch"], H, R, -1).transpose(1, 2).reshape(case["batch"] * R, H, -1)  # noqa: E731
        return shape(o), shape(lse).squeeze(-1)
    R, L, Q, W = case["rows"], case["layers"], QMAX[case["fmt"]], s["window"]
    out = torch.zeros((2, L, case["batch"], W, kv, D), dtype=torch.float64, device=DEVICE)
    scales = s["scales"].double()
    for b, (n, c) in enumerate(zip(_lens(case), _counts(case))):
        rows = s["path"][b, :c].long() + b * R
        x = torch.stack([s["k"][:, rows], s["v"][:, rows]]).double()
        for p in range(n // PAGE, _pages(n + c)):
            lo, hi = max(p * PAGE, n), min((p + 1) * PAGE, n + c)
            page = int(s["page_table"][b, p])
            new = x[:, :, lo - n:hi - n]                        # [2, L, rows, kv, D]
            old = torch.zeros((2, L, lo - p * PAGE, kv, D), dtype=torch.float64, device=DEVICE)
            step = new.abs().amax(dim=(2, 4)) / Q               # [2, L, kv]
            if lo > p * PAGE:
                pair = _values64(s["codes"][:, :, page], s["scales"][:, :, page], case["fmt"], D)
                old = torch.stack(pair)[:, :, :, :lo - p * PAGE].transpose(2, 3)
                step = torch.maximum(step, s["scales"][:, :, page].double().permute(2, 0, 1))
            y = torch.cat([old, new], dim=2) / step[:, :, None, :, None]
            y = y.round() if case["fmt"] == "int8" else y.float().to(torch.float8_e4m3fn).double()
            at = p * PAGE - n // PAGE * PAGE
            out[:, :, b, at:at + hi - p * PAGE] = y * step[:, :, None, :, None]
            scales[:, :, page] = step.permute(1, 2, 0)
    return out[0], out[1], scales
