"""Operators of decoding with trees of drafts and drawn tokens, as measurable cases.

A case is a dict of plain values.  `kind` says which operator a pass runs:

  attend    attention of the rows of a drafted tree (or chain, or of one token) over a cache
  sample    a token per row of logits: temperature, top-k, top-p, min-p, from given random numbers
  fork      sequences of a cache that go on as copies of others, in place
  compact   the rows of an accepted path moved right behind the cached ones, in place

`run` is the operator in plain torch operations while `own` is false, and the library's entry point while it is true."""
import math
import random

import torch

own = False

BF16, F16, F32 = "bf16", "f16", "f32"
DTYPES = {BF16: torch.bfloat16, F16: torch.float16, F32: torch.float32}
V32K = 32768


def _attend(name, B, T, H, Hkv, dh, n, cap, dtype=BF16, layout="heads", tree=True, ragged=False):
    return dict(name=name, kind="attend", B=B, T=T, H=H, Hkv=Hkv, dh=dh, n_lo=n[0], n_hi=n[1], cap=cap, dtype=dtype, layout=layout,
                tree=tree, ragged=ragged)


def _sample(name, rows, vocab, dtype, temperature, top_k, top_p, min_p):
    return dict(name=name, kind="sample", rows=rows, vocab=vocab, dtype=dtype, t_lo=temperature[0], t_hi=temperature[1], top_k=top_k,
                top_p=top_p, min_p=min_p)


def _cache(name, kind, layers, B, heads, dh, n, cap, layout="heads", **more):
    return dict(dict(name=name, kind=kind, layers=layers, B=B, heads=heads, dh=dh, n_lo=n[0], n_hi=n[1], cap=cap, layout=layout), **more)


def listed():
    return [
        # one user, one token, the big verifier's heads and arena: latency is all there is
        _attend("attend one token, 16 heads of 64", 1, 1, 16, 16, 64, (224, 224), 288, tree=False),
        # a batch with a tree of 25 drafts each at the big verifier's sizes (k = 25 is the paper's best block), ragged
        _attend("attend 32 trees of 26, 16 heads of 64", 32, 26, 16, 16, 64, (0, 245), 288, ragged=True),
        # one user far into a long text, plain decoding, grouped heads: one sequence has to fill the GPU
        _attend("attend one token, 65536 cached, 32 / 8 heads of 128", 1, 1, 32, 8, 128, (65536, 65536), 65600, layout="rows", tree=False),
        # a service with long ragged contexts and the largest trees, few key heads: most operations a byte
        _attend("attend 16 trees of 61, long ragged, 32 / 4 heads of 128", 16, 61, 32, 4, 128, (1000, 16000), 16064, dtype=F16, ragged=True),
        # the token one user waits for
        _sample("sample one row", 1, V32K, F32, (0.8, 0.8), 50, 0.95, 0.0),
        # a batch of mixed requests on half-precision logits, an odd vocabulary
        _sample("sample 128 rows, mixed, 32003", 128, 32003, BF16, (0.0, 1.5), -1, -1.0, -1.0),
        # every row of a full verification batch (128 sequences x 11 rows), nucleus sampling on the fp32 logits of the pass
        _sample("sample 1408 rows, top-p", 1408, V32K, F32, (0.7, 1.0), 0, 0.9, 0.0),
        # a large vocabulary, temperature and min-p alone
        _sample("sample 96 rows, 131072, min-p", 96, 131072, F16, (1.0, 1.3), 0, 1.0, 0.05),
        # four outputs for each of eight sources, right behind the prefix, the base verifier's arenas
        _cache("fork 32, 6 layers, 8 heads of 64", "fork", 6, 32, 8, 64, (10, 120), 160, samples=4),
        # four long prompts, four outputs each
        _cache("fork 16, 4096 rows, 8 heads of 128", "fork", 8, 16, 8, 128, (2000, 4096), 4096, layout="rows", samples=4),
        # the accepted path of one tree, the base verifier: latency
        _cache("compact 1, 6 layers, 8 heads of 64", "compact", 6, 1, 8, 64, (57, 57), 160, T=26, path=6),
        # the same for a full batch of the big verifier
        _cache("compact 128, 6 layers, 16 heads of 64", "compact", 6, 128, 16, 64, (48, 64), 160, T=32, path=7),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(lo * (hi / lo) ** rng.random()))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "sample", "sample", "fork", "compact"])
    if kind == "attend":
        G = rng.choice([1, 1, 2, 3, 4, 8])
        Hkv = rng.choice([1, 2, 4, 8, 12, 16])
        dh = rng.choice([64, 128])
        T = rng.choice([1, 1, rng.randrange(2, 12), rng.randrange(12, 33), rng.randrange(33, 65)])
        n_hi = _log_int(rng, 1, 65536)
        rows = 16 * 16000 * 4 * 128 // (Hkv * dh)                      # key rows of a batch that cost no more than the largest listed
        flop_rows = int(16 * 16000 * 61 * 32 * 128 / (T * G * Hkv * dh))
        B = max(1, min(_log_int(rng, 1, 128), min(rows, flop_rows) // (n_hi + 64)))
        while n_hi + 64 > min(rows, flop_rows):
            n_hi //= 2
        cap = n_hi + T + rng.choice([0, 1, 7, 64])
        return _attend(None, B, T, G * Hkv, Hkv, dh, (rng.choice([n_hi, n_hi // 2, 0]), n_hi), cap, dtype=rng.choice([BF16, F16]),
                       layout=rng.choice(["heads", "rows"]), tree=rng.random() < 0.7, ragged=rng.random() < 0.5) | {"seed": rng.randrange(1 << 30)}
    if kind == "sample":
        vocab = _log_int(rng, 1000, 160000)
        rows = max(1, min(_log_int(rng, 1, 1408), 1408 * V32K // vocab))
        t = rng.choice([(0.0, 1.5), (0.6, 1.0), (1.0, 1.0)])
        return _sample(None, rows, vocab, rng.choice([F32, BF16, F16]), t, rng.choice([0, 1, 40, -1, vocab // 2]),
                       rng.choice([1.0, 0.5, 0.9, 0.999, -1.0]), rng.choice([0.0, 0.02, 0.1, -1.0])) | {"seed": rng.randrange(1 << 30)}
    layers, heads, dh = rng.choice([1, 2, 6, 12]), rng.choice([2, 8, 16]), rng.choice([64, 128])
    n_hi = _log_int(rng, 4, 4096)
    most = 16 * 8 * 4096 * 8 * 128 // (layers * heads * dh)            # rows of all sequences
    if kind == "fork":
        samples = rng.choice([2, 3, 4, 8])
        most = most * 2 // 3
        while n_hi * samples > most:
            n_hi //= 2
        B = samples * max(1, min(_log_int(rng, 1, 128), most // n_hi) // samples)
        cap = n_hi + rng.choice([0, 5, 31])
        return _cache(None, kind, layers, B, heads, dh, (n_hi // rng.choice([1, 2, 8]), n_hi), cap, layout=rng.choice(["heads", "rows"]),
                      samples=samples) | {"seed": rng.randrange(1 << 30)}
    T = rng.randrange(2, 65)
    while n_hi + T > most and n_hi > 1:
        n_hi //= 2
    B = max(1, min(_log_int(rng, 1, 128), most // (n_hi + T)))
    return _cache(None, kind, layers, B, heads, dh, (n_hi // 2, n_hi), n_hi + T, layout=rng.choice(["heads", "rows"]), T=T,
                  path=rng.randrange(1, min(T, 12) + 1)) | {"seed": rng.randrange(1 << 30)}


# ---------------------------------------------------------------------------------------------------------------- inputs
def _lengths(rng, lo, hi, B):
    out = [rng.randint(lo, hi) for _ in range(B)]
    out[rng.randrange(B)] = hi
    return out


def _randn(gen, shape, dtype):
    """Normal values; the largest tensors are drawn in pieces, so that no fp32 copy of all of it is made."""
    out = torch.empty(shape, dtype=dtype, device="cuda")
    flat = out.view(-1)
    for i in range(0, flat.numel(), 1 << 27):
        piece = flat[i:i + (1 << 27)]
        piece.copy_(torch.randn(piece.numel(), generator=gen, device="cuda"))
    return out


def _i32(a):
    return torch.tensor(a, dtype=torch.int32, device="cuda")


def _arena(gen, case, dtype, lead):
    """Keys or values [lead.., B, heads, cap, dh]: rows of a head together, or rows of all heads."""
    heads = case.get("Hkv", case.get("heads"))
    if case["layout"] == "heads":
        return _randn(gen, (*lead, case["B"], heads, case["cap"], case["dh"]), dtype)
    return _randn(gen, (*lead, case["B"], case["cap"], heads, case["dh"]), dtype).transpose(-2, -3)


def _tree_masks(rng, T):
    """Row i sees itself and its ancestors: bit s of mask i.  Rows are numbered level by level, as drafters fill them."""
    masks, level, first = [1], 0, 0
    while len(masks) < T:
        level, first, last = level + 1, len(masks), first
        width = min(T - first, rng.choice([1, 2, 4, 6]))
        for _ in range(width):
            masks.append(masks[rng.randrange(last, first)] | 1 << len(masks))
    return [m - (1 << 64) if m >> 63 else m for m in masks]


def _path(rng, T, most):
    """Rows of an accepted path: the first drafts of a chain, then a branch stored beyond the path's length (a second move of the
    same path leaves every row where it is, so passes repeat)."""
    n = rng.randint(1, most)
    along = rng.randint(1, n)
    rest = sorted(rng.sample(range(n, T), min(n - along, T - n)))
    return list(range(along)) + rest


def prepare(case, seed):
    """What a decoding program holds when it makes the call: queries, caches and their lengths, logits, masks, outputs."""
    seed = seed * 7919 + case.get("seed", 0)
    rng, kind = random.Random(seed), case["kind"]
    gen = torch.Generator(device="cuda").manual_seed(seed)
    st = dict(case=case, kind=kind)
    if kind == "attend":
        B, T, H, dh, dtype = case["B"], case["T"], case["H"], case["dh"], DTYPES[case["dtype"]]
        st["q"] = _randn(gen, (B, T, H, dh), dtype)
        st["k"], st["v"] = _arena(gen, case, dtype, ()), _arena(gen, case, dtype, ())
        st["n"] = _i32(_lengths(rng, case["n_lo"], case["n_hi"], B))
        st["rows"] = _i32(_lengths(rng, 1, T, B)) if case["ragged"] else None
        st["visible"] = torch.tensor([_tree_masks(rng, T) for _ in range(B)], dtype=torch.int64, device="cuda") if case["tree"] else None
        st["scale"] = 1.0 / math.sqrt(dh)
        st["out"] = torch.zeros((B, T, H, dh), dtype=dtype, device="cuda")
    elif kind == "sample":
        rows, vocab = case["rows"], case["vocab"]
        # a language model's row: most tokens far below a few likely ones; two special tokens never come
        x = 2.0 * torch.randn((rows, vocab), generator=gen, device="cuda")
        x += 0.25 * torch.randn((rows, vocab), generator=gen, device="cuda").clamp_(min=0).pow_(3)
        x[:, [1, vocab - 1]] = -math.inf
        st["logits"] = x.to(DTYPES[case["dtype"]])

        def column(value, mixed, dtype):   # a negative setting: every request has its own
            row = [rng.choice(mixed) if value < 0 else value for _ in range(rows)]
            return torch.tensor(row, dtype=dtype, device="cuda")
        t = [0.0 if case["t_lo"] == 0.0 and rng.random() < 0.2 else rng.uniform(max(case["t_lo"], 0.2), case["t_hi"]) for _ in range(rows)]
        st["temperature"] = torch.tensor(t, dtype=torch.float32, device="cuda")
        st["top_k"] = column(case["top_k"], [0, 1, 5, 50, 1000], torch.int32)
        st["top_p"] = column(case["top_p"], [1.0, 0.5, 0.9, 0.95], torch.float32)
        st["min_p"] = column(case["min_p"], [0.0, 0.05, 0.2], torch.float32)
        st["u"] = torch.rand(rows, generator=gen, device="cuda")
        st["token"] = torch.zeros(rows, dtype=torch.int32, device="cuda")
        st["logprob"] = torch.zeros(rows, dtype=torch.float32, device="cuda")
    else:
        B = case["B"]
        st["k"], st["v"] = (_arena(gen, case, torch.bfloat16, (case["layers"],)) for _ in range(2))
        n = _lengths(rng, case["n_lo"], case["n_hi"], B)
        if kind == "fork":
            groups = [list(range(i, min(i + case["samples"], B))) for i in range(0, B, case["samples"])]
            src = [b for g in groups for b in [rng.choice(g)] * len(g)]
            st["src"], st["n"] = _i32(src), _i32(n)
        else:
            T = case["T"]
            paths = [_path(rng, T, case["path"]) for _ in range(B)]
            st["first"] = _i32([min(j, case["cap"] - T) for j in n])
            st["count"] = _i32([len(p) for p in paths])
            st["path"] = _i32([p + [0] * (case["path"] - len(p)) for p in paths])
    if own:
        from paper_2203_16487_amd import binding as sd
        st["sd"], st["ctx"] = sd, sd.specdec_create(1, 1, 1, 1)
        if kind == "attend":
            st["desc"] = sd.tree_attn_desc(st["q"], st["k"], st["v"], st["out"], st["scale"])
            st["ws"] = torch.empty(sd.specdec_tree_attention_bytes(st["ctx"], st["desc"]), dtype=torch.uint8, device="cuda")
        elif kind != "sample":
            st["desc"] = sd.cache_desc(st["k"], st["v"])
    return st


# ---------------------------------------------------------------------------------------------------------------- one pass
def run(st):
    kind = st["kind"]
    if not own:
        return _PLAIN[kind](st)
    sd, ctx = st["sd"], st["ctx"]
    if kind == "attend":
        sd.specdec_tree_attention(ctx, st["desc"], st["q"], st["k"], st["v"], st["n"], st["visible"], st["rows"], st["out"], st["ws"])
        return st["out"]
    if kind == "sample":
        sd.specdec_sample(ctx, st["logits"], st["temperature"], st["top_k"], st["top_p"], st["min_p"], st["u"], st["token"], st["logprob"])
        return {"token": st["token"], "logprob": st["logprob"]}
    if kind == "fork":
        sd.specdec_fork_cache(ctx, st["desc"], st["k"], st["v"], st["src"], st["n"])
    else:
        sd.specdec_compact_cache(ctx, st["desc"], st["k"], st["v"], st["first"], st["path"], st["count"])
    return [st["k"], st["v"]]


def _plain_attend(st):
    q, k, v, n = st["q"], st["k"], st["v"], st["n"].long()
    B, T, H, dh = q.shape
    Hkv, cap = k.shape[1], k.shape[2]
    rows = st["rows"].long() if st["rows"] is not None else torch.full_like(n, T)
    place = torch.arange(cap, device="cuda")[None] - n[:, None]                                     # of a key among the tree's rows
    if st["visible"] is None:
        row = (place[:, None] <= torch.arange(T, device="cuda")[None, :, None])
    else:
        row = (st["visible"][:, :, None] >> place.clamp(0, 63)[:, None]) & 1 == 1
    seen = (place < 0)[:, None] | (row & ((place >= 0) & (place < rows[:, None]))[:, None])          # [B, T, cap]
    qf = (q.float() * st["scale"]).view(B, T, Hkv, H // Hkv, dh).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, dh)
    s = torch.matmul(qf, k.float().transpose(-1, -2).contiguous()).view(B, Hkv, H // Hkv, T, cap)
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(top == -math.inf, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(B, Hkv, -1, cap), v.float().contiguous()).view(B, Hkv, H // Hkv, T, dh)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).permute(0, 3, 1, 2, 4).reshape(B, T, H, dh)
    there = torch.arange(T, device="cuda")[None] < rows[:, None]
    st["out"].copy_(torch.where(there[:, :, None, None], o.to(q.dtype), st["out"]))
    return st["out"]


def _plain_sample(st):
    x = st["logits"].double()
    x = torch.where(torch.isnan(x), torch.full_like(x, -math.inf), x)
    t, p, least = (st[name].double()[:, None] for name in ("temperature", "top_p", "min_p"))
    k = st["top_k"].long()[:, None]
    k = torch.where(k > 0, k, torch.full_like(k, x.shape[1]))
    top = x.amax(-1, keepdim=True)
    d = torch.where(x == top, torch.zeros_like(x), (x - top) / torch.where(t > 0, t, torch.ones_like(t)))
    w = torch.exp(d)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    ws = torch.gather(w, 1, order)
    at = torch.arange(x.shape[1], device="cuda")[None]
    ws = torch.where(at < k, ws, torch.zeros_like(ws))
    before = torch.cumsum(ws, -1) - ws
    keep = (at < k) & ((p >= 1) | (before < p * ws.sum(-1, keepdim=True))) & (ws >= least) | (at == 0)
    kept = torch.zeros_like(keep).scatter_(1, order, keep)
    total = torch.cumsum(torch.where(kept, w, torch.zeros_like(w)), -1)
    Z = total[:, -1:]
    drawn = (total <= st["u"].double()[:, None] * Z).sum(-1, keepdim=True)
    best = torch.where(x == top, at, torch.full_like(at, x.shape[1])).amin(-1, keepdim=True)
    greedy = ~(t > 0)
    token = torch.where(greedy, best, drawn)
    logprob = torch.where(greedy, torch.zeros_like(t), torch.gather(d, 1, token) - torch.log(Z))
    st["token"].copy_(token[:, 0])
    st["logprob"].copy_(logprob[:, 0])
    return {"token": st["token"], "logprob": st["logprob"]}


def _plain_fork(st):
    src, n = st["src"].long(), st["n"].long()
    for cache in (st["k"], st["v"]):
        copied = torch.arange(cache.shape[3], device="cuda")[None] < n[src][:, None]
        cache.copy_(torch.where(copied[None, :, None, :, None], cache[:, src], cache))
    return [st["k"], st["v"]]


def _plain_compact(st):
    first, path, count = st["first"].long(), st["path"].long(), st["count"].long()
    i = torch.arange(path.shape[1], device="cuda")[None]
    live = i < count[:, None]
    dst = first[:, None] + torch.where(live, i, torch.zeros_like(i))
    src = first[:, None] + torch.where(live, path, path[:, :1])     # (rows beyond the count: the first one onto its own place)
    b = torch.arange(first.shape[0], device="cuda")[:, None]
    for cache in (st["k"], st["v"]):
        cache[:, b, :, dst] = cache[:, b, :, src]
    return [st["k"], st["v"]]


_PLAIN = {"attend": _plain_attend, "sample": _plain_sample, "fork": _plain_fork, "compact": _plain_compact}


# ---------------------------------------------------------------------------------------------------------------- in 64 bits
def exact(case, seed):
    """The definitions, sequence after sequence and row after row in 64 bits."""
    st = prepare(case, seed)
    if case["kind"] == "attend":
        out = st["out"].double()
        B, T, H, dh = out.shape
        G, n = H // case["Hkv"], st["n"].tolist()
        rows = st["rows"].tolist() if case["ragged"] else [T] * B
        masks = st["visible"].tolist() if case["tree"] else [[(1 << (i + 1)) - 1 for i in range(T)]] * B
        for b in range(B):
            tree = torch.tensor([[bool(masks[b][i] >> s & 1) for s in range(rows[b])] for i in range(rows[b])], device="cuda")
            hidden = torch.cat([torch.zeros((rows[b], n[b]), dtype=torch.bool, device="cuda"), ~tree], 1).repeat_interleave(G, 0)
            for h in range(case["Hkv"]):
                K, V = (st[name][b, h, :n[b] + rows[b]].double() for name in "kv")
                Q = st["q"][b, :rows[b], h * G:(h + 1) * G].reshape(-1, dh).double()
                P = torch.softmax((Q @ K.T.contiguous() * st["scale"]).masked_fill_(hidden, -math.inf), -1)
                out[b, :rows[b], h * G:(h + 1) * G] = (P @ V).view(rows[b], G, dh)
        return out
    if case["kind"] == "sample":
        tokens, logprobs = [], []
        cols = {name: st[name].tolist() for name in ("temperature", "top_k", "top_p", "min_p", "u")}
        for r in range(case["rows"]):
            x = st["logits"][r].double()
            best = int(torch.nonzero(x == x.max())[0])
            if not cols["temperature"][r] > 0:
                tokens.append(best)
                logprobs.append(0.0)
                continue
            z = (x - x[best]) / cols["temperature"][r]
            ranked = torch.argsort(x, descending=True, stable=True)
            if cols["top_k"][r] > 0:
                ranked = ranked[:cols["top_k"][r]]
            mass = torch.exp(z[ranked])
            keep = mass >= cols["min_p"][r]
            if cols["top_p"][r] < 1:
                reached = torch.cumsum(mass, 0)
                keep[1:] &= reached[:-1] < cols["top_p"][r] * reached[-1]
            keep[0] = True
            index = torch.sort(ranked[keep]).values
            steps = torch.cumsum(torch.exp(z[index]), 0)
            token = index[torch.searchsorted(steps, cols["u"][r] * steps[-1], right=True).clamp(max=len(index) - 1)]
            tokens.append(int(token))
            logprobs.append(float(z[token] - torch.log(steps[-1])))
        return {"token": torch.tensor(tokens, dtype=torch.int32, device="cuda"), "logprob": torch.tensor(logprobs, dtype=torch.float64, device="cuda")}
    caches = []
    for old in (st["k"], st["v"]):
        new = old.clone()
        for b in range(case["B"]):
            if case["kind"] == "fork":
                a = int(st["src"][b])
                new[:, b, :, :int(st["n"][a])] = old[:, a, :, :int(st["n"][a])]
            else:
                for i in range(int(st["count"][b])):
                    new[:, b, :, int(st["first"][b]) + i] = old[:, b, :, int(st["first"][b]) + int(st["path"][b, i])]
        caches.append(new)
    return caches


def work(case):
    """Each input once, each output once: of caches only what is cached."""
    n = (case.get("n_lo", 0) + case.get("n_hi", 0)) / 2
    if case["kind"] == "attend":
        B, T, H, Hkv, dh = (case[name] for name in ("B", "T", "H", "Hkv", "dh"))
        rows = (1 + T) / 2 if case["ragged"] else T
        seen = n + (rows + 1) / 2
        return {"bytes": 2.0 * B * (2 * (n + rows) * Hkv * dh + 2 * rows * H * dh) + (8.0 * B * T if case["tree"] else 0.0),
                "flops": 4.0 * B * rows * H * dh * seen}
    if case["kind"] == "sample":
        values = case["rows"] * case["vocab"]
        return {"bytes": float(values * (4 if case["dtype"] == F32 else 2) + 28 * case["rows"]), "flops": 2.0 * values}
    row = 2 * 2 * case["layers"] * case["heads"] * case["dh"]            # bytes of one position, keys and values
    if case["kind"] == "fork":
        groups = -(-case["B"] // case["samples"])
        return {"bytes": float(row * n * (groups + case["B"] - groups)), "flops": 0.0}   # (one read a group, one write a copy)
    return {"bytes": 2.0 * row * case["B"] * (case["path"] - 1) / 4, "flops": 0.0}       # (mean number of rows that move)
