"""Operators around drafted tokens on a key/value cache, as cases to be timed and checked.

Four operators that a program with speculative decoding runs in turn, all on the cache layout of the decode block
([batch, kv head, row, head dimension]), held as fp16, or as int8 or e4m3 with one fp32 scale per cached row of a head:

  append   the fused projection of the new tokens (a prompt, a tree of drafted tokens, one token): queries and keys are rotated for
           their positions, queries written out, keys and values written to the cache in its format
  attend   attention of every drafted token over the cached rows and its own ancestors in the tree, optionally with scores
           capped by a tanh, a bias that falls with the distance, and a sliding window
  keep     after verification: the cache rows of the accepted tokens moved to where the sequence goes on
  read     cached rows back as fp16

Head counts and head dimensions are those of cf_inputs.py's shapes, batches up to its 16, cached lengths up to its 32768; drawn
cases take any other of the same ranges.  `own` chooses between plain torch operations and the library.
"""
import ctypes
import math
import random

import torch

own = False
DEV = "cuda"
FORMATS = {"f16": 0, "e4m3": 1, "int8": 2}
LARGEST = {"e4m3": 448.0, "int8": 127.0}       # the largest value a code stands for, before the row's scale


# ---- the cases -------------------------------------------------------------------------------------------------

def _case(name, op, fmt, heads, batch, kv, tokens, **more):
    n_q, n_kv, d, base = heads
    return {"name": name, "op": op, "format": fmt, "n_q": n_q, "n_kv": n_kv, "head_dim": d, "rope_base": base, "batch": batch,
            "kv": kv, "tokens": tokens, "ragged": False, "tree": True, "cap": 0.0, "window": 0, "bias": False, **more}


H7B, H8B, H70B = (32, 32, 128, 10000.0), (32, 8, 128, 500000.0), (64, 8, 128, 10000.0)
HODD = (14, 7, 64, 10000.0)


def listed():
    return [
        # one user, one new token on a 7B model: launch latency is nearly all there is
        _case("append int8 7b b1 t1", "append", "int8", H7B, 1, 4096, 1, tree=False),
        # two prompts of different lengths, padded to one, written into an empty 8-bit cache
        _case("append int8 8b prompts 8192", "append", "int8", H8B, 2, 0, 8192, tree=False, ragged=True),
        # a single drafted token over a short cache, head dimension 64: the smallest attention
        _case("attend f16 odd b1 t1 kv256", "attend", "f16", HODD, 1, 256, 1),
        # a tree of 64 drafts of one user over a chat
        _case("attend e4m3 7b b1 t64 kv4096", "attend", "e4m3", H7B, 1, 4096, 64),
        # four users with trees and lengths of their own, on the decode block's fp16 caches
        _case("attend f16 8b b4 t16 kv8192", "attend", "f16", H8B, 4, 8192, 16, ragged=True),
        # a capped, windowed and biased model of odd sizes that drafts chains of seven
        _case("attend f16 odd b3 t7 window", "attend", "f16", HODD, 3, 5000, 7, tree=False, cap=30.0, window=1024, bias=True),
        # one token, long context, the largest model's heads: all of it is reading the 8-bit cache
        _case("attend e4m3 70b b1 t1 kv32768", "attend", "e4m3", H70B, 1, 32768, 1),
        # a full batch with trees of 64: the products are what takes the time
        _case("attend int8 8b b16 t64 kv8192", "attend", "int8", H8B, 16, 8192, 64),
        # the accepted path of a small tree, one user
        _case("keep f16 7b b1 t16", "keep", "f16", H7B, 1, 4096, 16),
        # the accepted paths of a full batch, trees of 64
        _case("keep int8 8b b16 t64", "keep", "int8", H8B, 16, 4096, 64, ragged=True),
        # a piece of an odd 8-bit cache handed to code that takes fp16
        _case("read int8 odd b3 777", "read", "int8", HODD, 3, 777, 1),
        # all of a full batch's 8-bit cache
        _case("read e4m3 8b b16 4096", "read", "e4m3", H8B, 16, 4096, 1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_BYTES, MOST_FLOPS = 400e6, 137.9e9      # of a drawn pass: the largest listed ones have these
MOST_HELD = 400e6      # values that a drawn case's keys may have in its cache


def draw(rng):
    while True:
        op = rng.choice(["append", "attend", "attend", "attend", "keep", "read"])
        n_kv = rng.choice([rng.randint(1, 32), 8, 32])
        heads = (n_kv * rng.choice([1, 2, 4, 8]), n_kv, rng.choice([64, 128, 128]), rng.choice([10000.0, 500000.0]))
        if heads[0] > 128:
            continue
        case = _case("", op, rng.choice(["f16", "e4m3", "int8"]), heads, _log(rng, 1, 16), _log(rng, 1, 32768), 1,
                     ragged=rng.random() < 0.5, tree=rng.random() < 0.7)
        if op == "append":
            case["tokens"] = _log(rng, 1, 8192)
            case["tree"] = case["tree"] and case["tokens"] <= 64
        elif op == "attend":
            case["tokens"] = rng.choice([1, _log(rng, 1, 64), _log(rng, 2, 128)])
            if rng.random() < 0.3:
                case.update(cap=rng.choice([0.0, 20.0, 50.0]), window=rng.choice([0, _log(rng, 16, 4096)]), bias=rng.random() < 0.5)
        elif op == "keep":
            case["tokens"] = _log(rng, 12, 64)
        elif op == "read" and case["format"] == "f16":
            continue
        del case["name"]
        if case["batch"] * n_kv * (case["kv"] + case["tokens"]) * heads[2] > MOST_HELD:
            continue
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return case


# ---- inputs ----------------------------------------------------------------------------------------------------

class State:
    pass


def _lengths(case):
    """Cached tokens of every batch row: one length, or spread between half of it and all of it."""
    B, L = case["batch"], case["kv"]
    return [L - (b * L) // (2 * B) for b in range(B)] if case["ragged"] else [L] * B


def _counts(case):
    """New tokens of every batch row: all, or padded rows with down to half of them."""
    B, T = case["batch"], case["tokens"]
    return [T - (b * T) // (2 * B) for b in range(B)] if case["ragged"] else [T] * B


def _kept(case):
    """Accepted tokens of every batch row."""
    return [max(1, min(n // 3, 1 + (5 + 3 * b) % 7 if case["ragged"] else 5)) for b, n in enumerate(_counts(case))]


def _encode(x, fmt):
    """fp16 rows as codes and scales: scale = largest magnitude / largest code, code = x / scale rounded to nearest, ties to even.
    A row of zeros has scale 0, a row with an infinity or a NaN has scale NaN and codes 0."""
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    usable = (top > 0) & (top < math.inf)
    y = torch.where(usable, x * LARGEST[fmt] / top, torch.zeros_like(x))     # (products exact; a quotient is on a border only where the exact one is)
    codes = torch.round(y).to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)
    scale = torch.where(top < math.inf, top / LARGEST[fmt], torch.full_like(top, math.nan))
    return codes, scale.squeeze(-1)


def _stored(x, fmt):
    return (x, None) if fmt == "f16" else _encode(x, fmt)


def prepare(case, seed):
    st, g, rng = State(), torch.Generator(device=DEV).manual_seed(seed), random.Random(seed)

    def drafted(tokens):
        """Depths and ancestor masks (64 tokens a word, a token counts as its own ancestor) of a drafted tree: every token continues one
        of the tokens before it, most often a late one."""
        words = (tokens + 63) // 64
        depth, masks = [0] * tokens, [1] + [0] * (tokens - 1)
        for t in range(1, tokens):
            parent = max(rng.randrange(t), rng.randrange(t)) if t > 3 else 0
            depth[t], masks[t] = depth[parent] + 1, masks[parent] | 1 << t
        signed = [[(m >> 64 * w) & (1 << 64) - 1 for w in range(words)] for m in masks]
        return depth, [[x - (1 << 64) if x >> 63 else x for x in row] for row in signed]

    B, T, nq, nkv, d, L = (case[k] for k in ("batch", "tokens", "n_q", "n_kv", "head_dim", "kv"))
    st.case, st.call = case, None
    st.max_seq = L + T + 9
    st.row_len = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)
    st.row_tokens = torch.tensor(_counts(case), dtype=torch.int32, device=DEV)
    st.depth = st.tree = None
    st.per_row = case["ragged"]
    if case["tree"] and case["op"] in ("append", "attend"):
        trees = [drafted(T) for _ in range(B if st.per_row else 1)]
        st.depth = torch.tensor([t[0] for t in trees], dtype=torch.int32, device=DEV)
        st.tree = torch.tensor([t[1] for t in trees], dtype=torch.int64, device=DEV)

    def rows(n):        # cached rows: normal values, rows of different size
        x = torch.randn((B, nkv, n, d), generator=g, device=DEV) * torch.exp(0.3 * torch.randn((B, nkv, n, 1), generator=g, device=DEV))
        return x.half()
    held = L + T if case["op"] in ("attend", "keep") else L
    st.cache = {}
    for name in ("k", "v"):
        x, scale = _stored(rows(held), case["format"])
        kept = torch.zeros((B, nkv, st.max_seq, d), dtype=x.dtype, device=DEV)
        kept.view(torch.uint8 if x.dtype != torch.float16 else x.dtype)[:, :, :held] = x.view(torch.uint8 if x.dtype != torch.float16 else x.dtype)
        st.cache[name] = kept
        if scale is not None:
            st.cache[name + "_scale"] = torch.zeros((B, nkv, st.max_seq), device=DEV)
            st.cache[name + "_scale"][:, :, :held] = scale
    st.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / nq) for h in range(nq)], device=DEV) if case["bias"] else None
    if case["op"] == "append":
        st.qkv = torch.randn((B, T, (nq + 2 * nkv) * d), generator=g, device=DEV).half()
        st.q = torch.zeros((B, T, nq, d), dtype=torch.float16, device=DEV)
    elif case["op"] == "attend":
        st.q = torch.randn((B, T, nq, d), generator=g, device=DEV).half()
        st.out = torch.zeros((B, T, nq, d), dtype=torch.float16, device=DEV)
    elif case["op"] == "keep":
        picks = []      # the root, and tokens behind the places that are written: a second pass moves the same rows
        for n, a in zip(_counts(case), _kept(case)):
            picks.append([0] + sorted(rng.sample(range(a, n), a - 1)) + [0] * (T - a))
        st.kept = torch.tensor(picks, dtype=torch.int32, device=DEV)
        st.n_kept = torch.tensor(_kept(case), dtype=torch.int32, device=DEV)
        st.new_len = torch.zeros(B, dtype=torch.int32, device=DEV)
    else:
        st.first, st.rows = L // 7, L - L // 7
        st.k_out, st.v_out = (torch.zeros((B, nkv, st.rows, d), dtype=torch.float16, device=DEV) for _ in range(2))
    return st


# ---- the plain forms -------------------------------------------------------------------------------------------

def _half(x):
    """fp64 to fp16, rounded once: by way of fp32 the value is first moved off an even fp32 neighbour that it does not equal."""
    f = x.float()
    rest = x - f.double()
    bits = f.view(torch.int32)
    move = (rest != 0) & (f != 0) & (bits % 2 == 0) & torch.isfinite(f)
    return torch.where(move, bits + torch.where((rest > 0) == (f > 0), 1, -1).int(), bits).view(torch.float32).half()


def _positions(st):
    T = st.case["tokens"]
    depth = st.depth if st.depth is not None else torch.arange(T, dtype=torch.int32, device=DEV)[None]
    return st.row_len[:, None] + depth                                   # [B, T]


def _turned(x, positions, base):
    """Pairs (i, i + d/2) of the heads of x [B, T, heads, d] turned by position * base^(-2i/d), rounded to fp16."""
    d = x.shape[-1]
    theta = torch.tensor([math.pow(base, -2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device=DEV)
    angle = positions.double()[..., None, None] * theta
    c, s = torch.cos(angle), torch.sin(angle)
    lo, hi = x[..., :d // 2].double(), x[..., d // 2:].double()
    return _half(torch.cat([lo * c - hi * s, hi * c + lo * s], -1))


def _bytes_of(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x


def _write(st, name, new, valid, at):
    """Rows `new` [B, T, heads, d] written to rows at[b, t] of every head's slice of the cache, where valid[b, t]."""
    codes, scale = _stored(new, st.case["format"])
    b = torch.arange(new.shape[0], device=DEV)[:, None].expand_as(at)[valid]
    _bytes_of(st.cache[name])[b, :, at[valid]] = _bytes_of(codes)[valid]
    if scale is not None:
        st.cache[name + "_scale"][b, :, at[valid]] = scale[valid]


def _plain_append(st):
    case = st.case
    nq, nkv, d = case["n_q"], case["n_kv"], case["head_dim"]
    q, k, v = st.qkv.unflatten(-1, (nq + 2 * nkv, d)).split([nq, nkv, nkv], 2)
    positions = _positions(st)
    t = torch.arange(case["tokens"], device=DEV)
    valid = t[None] < st.row_tokens[:, None]
    at = st.row_len[:, None].long() + t[None]
    q = torch.where(valid[..., None, None], _turned(q, positions, case["rope_base"]), torch.zeros_like(q))
    _write(st, "k", _turned(k, positions, case["rope_base"]), valid, at)
    _write(st, "v", v, valid, at)
    return {"q": q, **st.cache}


def _values(st, name, n):
    x = st.cache[name][:, :, :n].float()
    scale = st.cache.get(name + "_scale")
    return x if scale is None else x * scale[:, :, :n, None]


def _seen(st, n):
    """[B, T, n]: which cache rows a drafted token attends to, and its distance from them."""
    case = st.case
    T, L = case["tokens"], st.row_len[:, None, None].long()
    t = torch.arange(T, device=DEV)
    row = torch.arange(n, device=DEV)[None, None]
    place = row - L                                                       # of a drafted token in the tree
    inside = (place >= 0) & (place < T)
    place = place.clamp(0, T - 1)
    if st.tree is not None:
        words = st.tree.expand(case["batch"], -1, -1)
        word = torch.gather(words, 2, (place // 64).expand(-1, T, -1))
        mine = (word >> (place % 64)) & 1 != 0
    else:
        mine = place <= t[None, :, None]
    at = _positions(st).long()
    key_at = torch.where(inside, torch.gather(at.expand(case["batch"], -1), 1, place[:, 0])[:, None], row)
    distance = at.expand(case["batch"], -1)[..., None] - key_at
    seen = (row < L) | (inside & (place < st.row_tokens[:, None, None]) & mine)
    if case["window"]:
        seen = seen & (distance < case["window"])
    return seen, distance


def _plain_attend(st):
    case = st.case
    B, T, nq, nkv, d = (case[k] for k in ("batch", "tokens", "n_q", "n_kv", "head_dim"))
    n = case["kv"] + T
    k, v = _values(st, "k", n), _values(st, "v", n)
    q = st.q.float().reshape(B, T, nkv, nq // nkv, d).permute(0, 2, 3, 1, 4).reshape(B, nkv, -1, d)
    s = (q @ k.transpose(2, 3).contiguous() / math.sqrt(d)).reshape(B, nq, T, n)
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    seen, distance = _seen(st, n)
    if st.slopes is not None:
        s = s - st.slopes[:, None, None] * distance[:, None].float()
    s = s.masked_fill(~seen[:, None], -math.inf)
    p = torch.exp(s - s.amax(-1, keepdim=True).clamp(min=-1e30))
    p = p / p.sum(-1, keepdim=True).clamp(min=1e-30)
    out = (p.reshape(B, nkv, -1, n) @ v).reshape(B, nq, T, d).transpose(1, 2)
    valid = torch.arange(T, device=DEV)[None] < st.row_tokens[:, None]
    return {"out": torch.where(valid[..., None, None], out, torch.zeros_like(out)).half()}


def _plain_keep(st):
    t = torch.arange(st.case["tokens"], device=DEV)
    valid = t[None] < st.n_kept[:, None]
    b = torch.arange(st.case["batch"], device=DEV)[:, None].expand_as(valid)[valid]
    start = st.row_len[:, None].long()
    source, target = (start + st.kept)[valid], (start + t[None])[valid]

    def moved(x):
        x = _bytes_of(x) if x.dim() == 4 else x
        x[b, :, target] = x[b, :, source]
        return 0
    [moved(x) for x in st.cache.values()]
    return {"new_len": st.row_len + st.n_kept, **st.cache}


def _plain_read(st):
    end = st.first + st.rows
    return {"k": _values(st, "k", end)[:, :, st.first:].half(), "v": _values(st, "v", end)[:, :, st.first:].half()}


# ---- the library's calls ---------------------------------------------------------------------------------------

_handles = {}       # a program keeps one for a model


def _library_call(st):
    """What a program sets up once for its buffers, and the call that it then makes for every step."""
    import paper_2508_18850_amd as lib
    case = st.case
    B, T = case["batch"], case["tokens"]
    cfg = (case["n_q"], case["n_kv"], case["head_dim"], 16, st.max_seq, FORMATS[case["format"]], case["rope_base"])
    address = lambda x: x.data_ptr() if x is not None else 0  # noqa: E731
    cache = lib.cache_pointers(*(address(st.cache.get(k)) for k in ("k", "v", "k_scale", "v_scale")))
    draft = lib.draft(T, case["kv"], row_len=address(st.row_len), row_tokens=address(st.row_tokens) if case["ragged"] else 0,
                      depth=address(st.depth), tree=address(st.tree), per_row=st.per_row)
    if case["op"] == "attend":
        key = cfg + (T, case["cap"], case["window"])
        if key not in _handles:
            _handles[key] = lib.TreeAttention(*cfg, T, score_cap=case["cap"], window=case["window"])
        handle, q, slopes, out = _handles[key], address(st.q), address(st.slopes), address(st.out)
        st.outputs = {"out": st.out}
        return lambda stream: handle.attend(B, q, cache, draft, slopes, out, stream)
    kv = lib.KvCache(*cfg)
    if case["op"] == "append":
        qkv, q = address(st.qkv), address(st.q)
        st.outputs = {"q": st.q, **st.cache}
        return lambda stream: kv.append(B, qkv, cache, draft, q, stream)
    if case["op"] == "keep":
        kept, n_kept, new_len = address(st.kept), address(st.n_kept), address(st.new_len)
        st.outputs = {"new_len": st.new_len, **st.cache}
        return lambda stream: kv.keep(B, cache, draft, kept, n_kept, new_len, stream)
    first, rows, k_out, v_out = st.first, st.rows, address(st.k_out), address(st.v_out)
    st.outputs = {"k": st.k_out, "v": st.v_out}
    return lambda stream: kv.read(B, cache, first, rows, k_out, v_out, stream)


def run(state):
    if own:
        if state.call is None:
            state.call = _library_call(state)
        state.call(torch.cuda.current_stream().cuda_stream)
        return state.outputs
    return {"append": _plain_append, "attend": _plain_attend, "keep": _plain_keep, "read": _plain_read}[state.case["op"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(case):
    T, nq, nkv, d = (case[k] for k in ("tokens", "n_q", "n_kv", "head_dim"))
    lengths, counts = _lengths(case), _counts(case)
    row = 2 * nkv * (2 * d if case["format"] == "f16" else d + 4)          # a cached token, key and value, with its scales
    if case["op"] == "append":
        n = sum(counts)
        return {"bytes": n * (2 * d * (2 * nq + 2 * nkv) + row), "flops": n * 3 * d * (nq + nkv)}
    if case["op"] == "read":
        n = case["batch"] * (case["kv"] - case["kv"] // 7)
        return {"bytes": n * (row + 4 * nkv * d), "flops": 0 if case["format"] == "f16" else 2 * n * nkv * d}
    if case["op"] == "keep":
        return {"bytes": sum(2 * (a - 1) * row for a in _kept(case)) + 12 * case["batch"], "flops": 0}
    reach = case["window"] or case["kv"] + T
    keys = sum(min(n, reach) + c for n, c in zip(lengths, counts))
    pairs = sum(c * (min(n, reach) + c / 2) for n, c in zip(lengths, counts))
    return {"bytes": keys * row + sum(counts) * nq * 4 * d, "flops": int(pairs * nq * 4 * d)}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)
    B, T, nq, nkv, d = (case[k] for k in ("batch", "tokens", "n_q", "n_kv", "head_dim"))
    lengths, counts = _lengths(case), _counts(case)

    def values(name):
        x = st.cache[name].to(torch.float32).double()
        return x if name + "_scale" not in st.cache else x * st.cache[name + "_scale"].double()[..., None]

    def depths(b):
        return st.depth[b if st.per_row else 0].tolist() if st.depth is not None else list(range(T))

    def seen(b):        # which of the drafted tokens each of them sees
        if st.tree is None:
            return [[u <= t for u in range(counts[b])] for t in range(counts[b])]
        masks = [sum((w & (1 << 64) - 1) << 64 * i for i, w in enumerate(row)) for row in st.tree[b if st.per_row else 0].tolist()]
        return [[masks[t] >> u & 1 != 0 for u in range(counts[b])] for t in range(counts[b])]

    def attend():       # head by head: scores, and a softmax over what each token sees
        out = torch.zeros((B, T, nq, d), dtype=torch.float64, device=DEV)
        keys, vals = values("k"), values("v")
        for b, (L, c) in enumerate(zip(lengths, counts)):
            at = torch.tensor(list(range(L)) + [L + x for x in depths(b)[:c]], dtype=torch.float64)
            distance = at[L:, None] - at[None]
            see = torch.cat([torch.ones((c, L), dtype=torch.bool), torch.tensor(seen(b))], 1)
            if case["window"]:
                see &= distance < case["window"]
            see, distance = see.to(DEV), distance.to(DEV)
            for h in range(nq):
                s = st.q[b, :c, h].double() @ keys[b, h * nkv // nq, :L + c].T.contiguous() * d ** -0.5
                if case["cap"]:
                    s = torch.tanh(s / case["cap"]) * case["cap"]
                if case["bias"]:
                    s = s - distance * st.slopes[h].double()
                w = torch.where(see, torch.exp(s - torch.where(see, s, -1e300).amax(1, keepdim=True)), 0.0)
                total = w.sum(1, keepdim=True)
                out[b, :c, h] = torch.where(total > 0, w @ vals[b, h * nkv // nq, :L + c] / total.clamp(min=1e-300), 0.0)
        return {"out": out}

    def nearest(x, digits, smallest):       # ties to even, steps not below `smallest`
        step = torch.ldexp(torch.ones_like(x), torch.frexp(x)[1] - digits).clamp(min=smallest)
        return torch.round(x / step) * step

    def code(rows):
        top, most = rows.abs().amax(-1, keepdim=True), LARGEST[case["format"]]
        y = torch.where(top > 0, rows * most / top.clamp(min=1e-300), 0.0)
        return torch.round(y).to(torch.int8) if case["format"] == "int8" else nearest(y, 4, 2.0 ** -9), (top / most).squeeze(-1)

    def append():       # pairs of dimensions as complex numbers
        result = {"q": torch.zeros((B, T, nq, d), dtype=torch.float64, device=DEV)}
        result.update({k: x.clone() if x.dtype == torch.int8 else x.float().double() for k, x in st.cache.items()})
        turns = torch.tensor([math.pow(case["rope_base"], -2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device=DEV)
        for b, (L, c) in enumerate(zip(lengths, counts)):
            heads = st.qkv[b, :c].double().reshape(c, nq + 2 * nkv, d)
            at = torch.tensor([L + x for x in depths(b)[:c]], dtype=torch.float64, device=DEV)
            z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), at[:, None] * turns)[:, None]
            turned = torch.complex(heads[:, :nq + nkv, :d // 2].contiguous(), heads[:, :nq + nkv, d // 2:].contiguous()) * z
            turned = torch.cat([turned.real, turned.imag], -1)
            result["q"][b, :c] = turned[:, :nq]
            for name, rows in (("k", turned[:, nq:]), ("v", heads[:, nq + nkv:])):
                rows = rows.transpose(0, 1)
                if case["format"] == "f16":
                    result[name][b, :, L:L + c] = rows
                else:       # what an fp16 cache would hold, as codes
                    result[name][b, :, L:L + c], result[name + "_scale"][b, :, L:L + c] = code(nearest(rows, 11, 2.0 ** -24))
        return result

    def keep():
        result = {k: x.clone() if x.dtype == torch.int8 else x.float().double() for k, x in st.cache.items()}
        for b, (L, a) in enumerate(zip(lengths, _kept(case))):
            source = [L + i for i in st.kept[b, :a].tolist()]
            for x in result.values():
                x[b, :, L:L + a] = x[b, :, source].clone()
        return {"new_len": None, **result}

    def read():
        return {k: values(k)[:, :, st.first:st.first + st.rows] for k in ("k", "v")}
    return {"append": append, "attend": attend, "keep": keep, "read": read}[case["op"]]()
