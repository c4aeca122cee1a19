"""Operators of a quantised step with drafted tokens, as cases to be timed and checked.

A program that verifies drafts, or fills a cache from prompts, runs these in turn around its own choice of tokens:

  quantize  rows of fp16 (hidden states, attention results, once the weights) as int8 codes with one scale a row
  product   the integer product of such rows with weights quantised by output channel, scaled and rounded to fp16
  append    queries and keys of the fused projection normalised head by head and rotated, queries written out, keys and values
            written to the cache in its format; a cache that holds codes is read back as fp16 for what attends over the prompt itself
  attend    attention of every drafted token over a cache held in 4 bits and its own ancestors in the tree

The 4-bit format: e2m1 codes (0 .5 1 1.5 2 3 4 6 and a sign), one power of two for every 32 adjacent values of a row.  Head counts, model and
feed-forward widths are those of cf_inputs.py's shapes, batches up to its 16, cached lengths up to its 32768; drawn cases take any
other of the same ranges.  `own` chooses between plain torch operations and the library.
"""
import ctypes
import math
import random

import torch

own = False
DEV = "cuda"
FORMATS = {"f16": 0, "e4m3": 1, "int8": 2, "mxfp4": 4}
LARGEST = {"e4m3": 448.0, "int8": 127.0}       # the largest value a code stands for, before the row's scale
EPS = 1e-6


# ---- the cases -------------------------------------------------------------------------------------------------

def _rows(name, rows, n):
    return {"name": name, "op": "quantize", "rows": rows, "n": n}


def _product(name, rows, n, out):
    return {"name": name, "op": "product", "rows": rows, "n": n, "out": out}


def _tokens(name, op, fmt, heads, batch, kv, tokens, **more):
    n_q, n_kv, d, base = heads
    return {"name": name, "op": op, "format": fmt, "n_q": n_q, "n_kv": n_kv, "head_dim": d, "rope_base": base, "batch": batch,
            "kv": kv, "tokens": tokens, "ragged": False, "tree": True, "cap": 0.0, "window": 0, "bias": False, **more}


H7B, H8B, H70B = (32, 32, 128, 10000.0), (32, 8, 128, 500000.0), (64, 8, 128, 10000.0)
HODD = (14, 7, 64, 10000.0)


def listed():
    return [
        # the hidden state of one user's one token on a 7B model: launch latency
        _rows("quantize 7b b1 t1", 1, 4096),
        # the hidden states of prompts on a 70B model
        _rows("quantize 70b prompts 8192", 8192, 8192),
        # three tokens through the projection of the odd model: the smallest product
        _product("product odd t3", 3, 896, 1792),
        # one token through the fused projection of a 7B model: all of it is reading the weights
        _product("product 7b qkv t1", 1, 4096, 12288),
        # four users with trees of 16 drafts through the fused projection of an 8B model
        _product("product 8b qkv t64", 64, 4096, 6144),
        # prompts through the fused projection of a 70B model: the matrix units' rate
        _product("product 70b qkv prompts 8192", 8192, 8192, 10240),
        # one new token on a 7B model's fp16 cache
        _tokens("append f16 7b b1 t1", "append", "f16", H7B, 1, 4096, 1, tree=False),
        # two prompts of different lengths, padded to one, into an empty 4-bit cache, and back for the prompt's own attention
        _tokens("append mxfp4 8b prompts 4096", "append", "mxfp4", H8B, 2, 0, 4096, tree=False, ragged=True),
        # a single drafted token over a short cache, head dimension 64: the smallest attention
        _tokens("attend mxfp4 odd b1 t1 kv256", "attend", "mxfp4", HODD, 1, 256, 1),
        # four users with trees and lengths of their own
        _tokens("attend mxfp4 8b b4 t16 kv8192", "attend", "mxfp4", H8B, 4, 8192, 16, ragged=True),
        # one token, long context, the largest model's heads: all of it is reading the cache
        _tokens("attend mxfp4 70b b1 t1 kv32768", "attend", "mxfp4", H70B, 1, 32768, 1),
        # a full batch with trees of 64: the products are what takes the time
        _tokens("attend mxfp4 8b b16 t64 kv8192", "attend", "mxfp4", H8B, 16, 8192, 64),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MOST_BYTES, MOST_FLOPS = 400e6, {"product": 1.38e12, "attend": 137.9e9}      # of a drawn pass: the largest listed ones have these
MOST_HELD = 400e6      # values that a drawn case's keys may have in its cache


def draw(rng):
    while True:
        op = rng.choice(["quantize", "product", "product", "append", "attend", "attend"])
        width = 16 * _log(rng, 4, 1792)
        if op == "quantize":
            case = _rows("", _log(rng, 1, 16384), width)
        elif op == "product":
            case = _product("", rng.choice([_log(rng, 1, 64), _log(rng, 1, 8192)]), width, 8 * _log(rng, 8, 3584))
        else:
            n_kv = rng.choice([rng.randint(1, 32), 8, 32])
            heads = (n_kv * rng.choice([1, 2, 4, 8]), n_kv, rng.choice([64, 128, 128]), rng.choice([10000.0, 500000.0]))
            if heads[0] > 128:
                continue
            case = _tokens("", op, "mxfp4", heads, _log(rng, 1, 16), _log(rng, 1, 32768), 1, ragged=rng.random() < 0.5,
                           tree=rng.random() < 0.7)
            if op == "append":
                case["format"] = rng.choice(["f16", "e4m3", "int8", "mxfp4"])
                case["tokens"] = _log(rng, 1, 4096)
                case["tree"] = case["tree"] and case["tokens"] <= 64
            else:
                case["tokens"] = rng.choice([1, _log(rng, 1, 64), _log(rng, 2, 128)])
                if rng.random() < 0.3:
                    case.update(cap=rng.choice([0.0, 20.0, 50.0]), window=rng.choice([0, _log(rng, 16, 4096)]), bias=rng.random() < 0.5)
            if case["batch"] * n_kv * (case["kv"] + case["tokens"]) * heads[2] > MOST_HELD:
                continue
        del case["name"]
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS.get(op, math.inf):
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


def _first(case):
    """First row that an append reads back: everything from the shortest row's new tokens on."""
    return min(_lengths(case))


def _encode(x, fmt):
    """fp16 rows as codes and scales.  8 bits: scale = largest magnitude / largest code, code = x / scale rounded to nearest, ties to even; a
    row of zeros has scale 0, a row with an infinity or a NaN has scale NaN and codes 0.  4 bits: see _encode4."""
    if fmt == "mxfp4":
        return _encode4(x)
    x = x.float()
    top = x.abs().amax(-1, keepdim=True)
    usable = (top > 0) & (top < math.inf)
    y = torch.where(usable, x * LARGEST[fmt] / top, torch.zeros_like(x))     # (products exact; a quotient is on a border only where the exact one is)
    codes = torch.round(y).to(torch.int8) if fmt == "int8" else y.to(torch.float8_e4m3fn)
    scale = torch.where(top < math.inf, top / LARGEST[fmt], torch.full_like(top, math.nan))
    return codes, scale.squeeze(-1)


def _encode4(x):
    """Every 32 adjacent values: 2^e, the smallest power of two with (largest magnitude) <= 6 * 2^e that lies in 2^-23 .. 2^13, held as
    e + 127 (255 where one of the values is no finite number); codes nearest to x / 2^e, ties to the even one, two to a byte, the
    first in the low half."""
    x = x.float().unflatten(-1, (-1, 32))
    top = x.abs().amax(-1, keepdim=True)
    part, power = torch.frexp(top)
    power = torch.where(top > 0, power - torch.where(part <= 0.75, 3, 2), -23).clamp(-23, 13)
    fine = top < math.inf
    y = torch.where(fine, torch.ldexp(x, -power), torch.zeros_like(x))
    a = y.abs()
    code = (a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    code = (code + 8 * torch.signbit(y)).flatten(-2).unflatten(-1, (-1, 2))
    scale = torch.where(fine, power + 127, torch.full_like(power, 255))
    return (code[..., 0] | code[..., 1] << 4).to(torch.uint8), scale.squeeze(-1).to(torch.uint8)


def _stored(x, fmt):
    return (x, None) if fmt == "f16" else _encode(x, fmt)


def prepare(case, seed):
    st, g, rng = State(), torch.Generator(device=DEV).manual_seed(seed), random.Random(seed)
    st.case, st.call = case, None

    def normal(*shape):
        return torch.randn(shape, generator=g, device=DEV)
    if case["op"] in ("quantize", "product"):       # rows of different size, and in each a few dimensions that are larger than the rest
        M, K = case["rows"], case["n"]
        x = normal(M, K)
        x *= torch.exp(0.5 * normal(M, 1))
        x *= 1 + 7 * (torch.rand((1, K), generator=g, device=DEV) < 0.004)
        st.x = x.half()
        if case["op"] == "quantize":
            st.codes, st.scale = torch.zeros((M, K), dtype=torch.int8, device=DEV), torch.zeros(M, device=DEV)
        else:
            st.x, st.x_scale = _encode(st.x, "int8")
            st.w, st.w_scale = _encode((0.02 * normal(case["out"], K)).half(), "int8")
            st.out = torch.zeros((M, case["out"]), dtype=torch.float16, device=DEV)
        return st

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
    st.max_seq = L + T + 9
    st.row_len = torch.tensor(_lengths(case), dtype=torch.int32, device=DEV)
    st.row_tokens = torch.tensor(_counts(case), dtype=torch.int32, device=DEV)
    st.depth = st.tree = None
    st.per_row = case["ragged"]
    if case["tree"]:
        trees = [drafted(T) for _ in range(B if st.per_row else 1)]
        st.depth = torch.tensor([t[0] for t in trees], dtype=torch.int32, device=DEV)
        st.tree = torch.tensor([t[1] for t in trees], dtype=torch.int64, device=DEV)

    held = L + T if case["op"] == "attend" else L
    st.cache = {}
    for name in ("k", "v"):
        x, scale = _stored((normal(B, nkv, held, d) * torch.exp(0.3 * normal(B, nkv, held, 1))).half(), case["format"])
        kept = torch.zeros((B, nkv, st.max_seq, x.shape[-1]), dtype=x.dtype, device=DEV)
        _bytes_of(kept)[:, :, :held] = _bytes_of(x)
        st.cache[name] = kept
        if scale is not None:
            st.cache[name + "_scale"] = torch.zeros((B, nkv, st.max_seq) + scale.shape[3:], dtype=scale.dtype, device=DEV)
            st.cache[name + "_scale"][:, :, :held] = scale
    st.slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / nq) for h in range(nq)], device=DEV) if case["bias"] else None
    if case["op"] == "append":
        st.qkv = (normal(B, T, (nq + 2 * nkv) * d) * torch.exp(0.5 * normal(B, T, 1))).half()
        st.q_weight, st.k_weight = ((1 + 0.2 * normal(d)).half() for _ in range(2))
        st.q = torch.zeros((B, T, nq, d), dtype=torch.float16, device=DEV)
        if case["format"] != "f16":
            st.first = _first(case)
            st.rows = L + T - st.first
            st.k_out, st.v_out = (torch.zeros((B, nkv, st.rows, d), dtype=torch.float16, device=DEV) for _ in range(2))
    else:
        st.q = normal(B, T, nq, d).half()
        st.out = torch.zeros((B, T, nq, d), dtype=torch.float16, device=DEV)
    return st


# ---- the plain forms -------------------------------------------------------------------------------------------

def _half(x):
    """fp64 to fp16, rounded once: by way of fp32 the value is first moved off an even fp32 neighbour that it does not equal."""
    f = x.float()
    rest = x - f.double()
    bits = f.view(torch.int32)
    move = (rest != 0) & (f != 0) & (bits % 2 == 0) & torch.isfinite(f)
    return torch.where(move, bits + torch.where((rest > 0) == (f > 0), 1, -1).int(), bits).view(torch.float32).half()


def _plain_quantize(st):
    codes, scale = _encode(st.x, "int8")
    return {"codes": codes, "scale": scale}


def _plain_product(st):
    out = st.x.float() @ st.w.float().T
    return {"out": (out * st.x_scale[:, None] * st.w_scale).half()}


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
    lo, hi = x[..., :d // 2], x[..., d // 2:]
    return _half(torch.cat([lo * c - hi * s, hi * c + lo * s], -1))


def _normed(x, weight):
    x = x.double()
    return x / torch.sqrt((x * x).mean(-1, keepdim=True) + EPS) * weight.double()


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
    q = torch.where(valid[..., None, None], _turned(_normed(q, st.q_weight), positions, case["rope_base"]), torch.zeros_like(q))
    _write(st, "k", _turned(_normed(k, st.k_weight), positions, case["rope_base"]), valid, at)
    _write(st, "v", v, valid, at)
    if case["format"] == "f16":
        return {"q": q, **st.cache}
    end = st.first + st.rows
    return {"q": q, "k_back": _values(st, "k", st.first, end).half(), "v_back": _values(st, "v", st.first, end).half()}


def _values(st, name, first, end):
    x, scale = st.cache[name][:, :, first:end], st.cache.get(name + "_scale")
    if st.case["format"] == "mxfp4":
        level = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=DEV)
        level = torch.cat([level, -level])
        x = torch.stack([level[(x & 15).long()], level[(x >> 4).long()]], -1).flatten(-2)
        power = scale[:, :, first:end].int()
        unit = torch.where(power < 255, torch.ldexp(torch.ones((), device=DEV), power - 127), torch.full((), math.nan, device=DEV))
        return (x.unflatten(-1, (-1, 32)) * unit[..., None]).flatten(-2)
    return x.float() if scale is None else x.float() * scale[:, :, first:end, None]


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
    k, v = _values(st, "k", 0, n), _values(st, "v", 0, n)
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


# ---- the library's calls ---------------------------------------------------------------------------------------

_handles = {}       # a program keeps one for a model


def _kept(key, make):
    if key not in _handles:
        _handles[key] = make()
    return _handles[key]


def _library_call(st):
    """What a program sets up once for its buffers, and the call that it then makes for every step."""
    import paper_2508_18850_amd as lib
    case = st.case
    address = lambda x: x.data_ptr() if x is not None else 0  # noqa: E731
    if case["op"] == "quantize":
        M, K, x, codes, scale = case["rows"], case["n"], address(st.x), address(st.codes), address(st.scale)
        st.outputs = {"codes": st.codes, "scale": st.scale}
        return lambda stream: lib.quantize_rows(M, K, x, codes, scale, stream)
    if case["op"] == "product":
        M, sizes = case["rows"], (case["n"], case["out"], case["rows"])
        handle = _kept(sizes, lambda: lib.Int8Linear(*sizes))
        x, x_scale, w, w_scale, out = (address(t) for t in (st.x, st.x_scale, st.w, st.w_scale, st.out))
        st.outputs = {"out": st.out}
        return lambda stream: handle.forward(M, x, x_scale, w, w_scale, out, stream)
    B, T = case["batch"], case["tokens"]
    cfg = (case["n_q"], case["n_kv"], case["head_dim"], 16, st.max_seq, FORMATS[case["format"]], case["rope_base"])
    cache = lib.cache_pointers(*(address(st.cache.get(k)) for k in ("k", "v", "k_scale", "v_scale")))
    draft = lib.draft(T, case["kv"], row_len=address(st.row_len), row_tokens=address(st.row_tokens) if case["ragged"] else 0,
                      depth=address(st.depth), tree=address(st.tree), per_row=st.per_row)
    if case["op"] == "attend":
        key = cfg + (T, case["cap"], case["window"])
        handle = _kept(key, lambda: lib.TreeAttention(*cfg, T, score_cap=case["cap"], window=case["window"]))
        q, slopes, out = address(st.q), address(st.slopes), address(st.out)
        st.outputs = {"out": st.out}
        return lambda stream: handle.attend(B, q, cache, draft, slopes, out, stream)
    kv = lib.KvCache(*cfg)
    qkv, q, q_weight, k_weight = (address(t) for t in (st.qkv, st.q, st.q_weight, st.k_weight))
    if case["format"] == "f16":
        st.outputs = {"q": st.q, **st.cache}
        return lambda stream: kv.append_normed(B, qkv, q_weight, k_weight, EPS, cache, draft, q, stream)
    first, rows, k_out, v_out = st.first, st.rows, address(st.k_out), address(st.v_out)
    st.outputs = {"q": st.q, "k_back": st.k_out, "v_back": st.v_out}

    def append_and_read(stream):
        kv.append_normed(B, qkv, q_weight, k_weight, EPS, cache, draft, q, stream)
        kv.read(B, cache, first, rows, k_out, v_out, stream)
    return append_and_read


def run(state):
    if own:
        if state.call is None:
            state.call = _library_call(state)
        state.call(torch.cuda.current_stream().cuda_stream)
        return state.outputs
    return {"quantize": _plain_quantize, "product": _plain_product, "append": _plain_append, "attend": _plain_attend}[state.case["op"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(case):
    if case["op"] == "quantize":
        M, K = case["rows"], case["n"]
        return {"bytes": 3 * M * K + 4 * M, "flops": 2 * M * K}
    if case["op"] == "product":
        M, K, N = case["rows"], case["n"], case["out"]
        return {"bytes": M * K + N * K + 4 * (M + N) + 2 * M * N, "flops": 2 * M * K * N}
    T, nq, nkv, d = (case[k] for k in ("tokens", "n_q", "n_kv", "head_dim"))
    lengths, counts = _lengths(case), _counts(case)
    row = 2 * nkv * {"f16": 2 * d, "mxfp4": d // 2 + d // 32}.get(case["format"], d + 4)     # a cached token, key and value, with its scales
    if case["op"] == "append":
        n = sum(counts)
        back = 0 if case["format"] == "f16" else case["batch"] * (case["kv"] + T - _first(case)) * 4 * nkv * d
        return {"bytes": n * (2 * d * (2 * nq + 2 * nkv) + row) + back, "flops": n * 7 * d * (nq + nkv)}
    reach = case["window"] or case["kv"] + T
    keys = sum(min(n, reach) + c for n, c in zip(lengths, counts))
    pairs = sum(c * (min(n, reach) + c / 2) for n, c in zip(lengths, counts))
    return {"bytes": keys * row + sum(counts) * nq * 4 * d, "flops": int(pairs * nq * 4 * d)}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    st = prepare(case, seed)

    def power(e):       # 2^e for whole numbers in e, put together from its bits
        return ((e.long() + 1023) << 52).view(torch.float64)

    def exponent(x):       # of x >= 2^-1022: 2^e <= x < 2^(e + 1)
        return (x.clamp(min=2.0 ** -1022).view(torch.int64) >> 52) - 1023

    def nearest(x, digits, smallest):       # ties to even, steps not below 2^smallest
        step = power((exponent(x.abs()) + 1 - digits).clamp(min=smallest))
        return torch.round(x / step) * step

    def whole_codes(x):
        x = x.double()
        top = x.abs().amax(-1, keepdim=True)
        return torch.round(torch.where(top > 0, x * 127 / top.clamp(min=1e-300), 0.0)).to(torch.int8), (top / 127).squeeze(-1)

    if case["op"] == "quantize":
        codes, scale = whole_codes(st.x)
        return {"codes": codes, "scale": scale}
    if case["op"] == "product":
        x, w = st.x.double() * st.x_scale.double()[:, None], st.w.double() * st.w_scale.double()[:, None]
        return {"out": x @ w.T.contiguous()}

    B, T, nq, nkv, d = (case[k] for k in ("batch", "tokens", "n_q", "n_kv", "head_dim"))
    lengths, counts = _lengths(case), _counts(case)

    def values(name):
        x, scale = st.cache[name], st.cache.get(name + "_scale")
        if case["format"] != "mxfp4":
            x = x.to(torch.float32).double()
            return x if scale is None else x * scale.double()[..., None]
        result = torch.zeros(x.shape[:-1] + (d,), dtype=torch.float64, device=DEV)
        for half in (0, 1):
            code = x >> 4 * half & 15
            low, steps = (code & 7).double(), code & 7
            size = torch.where(steps < 4, low / 2, torch.where(steps < 6, low - 2, 2 * low - 8))
            result[..., half::2] = torch.where(code > 7, -size, size)
        return result * power(scale.int() - 127).repeat_interleave(32, -1)

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

    def held(rows):        # fp16 rows as the cache gives them back
        if case["format"] == "mxfp4":
            x = rows.unflatten(-1, (-1, 32))
            top = x.abs().amax(-1, keepdim=True)
            e = exponent(top / 6)
            e = torch.where(6 * power(e) < top, e + 1, e).clamp(-23, 13)
            step = power(torch.maximum(exponent(x.abs()), e) - 1)        # two levels to a power of two, and as far apart below the first
            return (torch.round(x / step) * step).clamp(-6 * power(e), 6 * power(e)).flatten(-2)
        top, most = rows.abs().amax(-1, keepdim=True), LARGEST[case["format"]]
        y = torch.where(top > 0, rows * most / top.clamp(min=1e-300), 0.0)
        return (torch.round(y) if case["format"] == "int8" else nearest(y, 4, -9)) * (top / most)

    def append():       # pairs of dimensions as complex numbers
        q = torch.zeros((B, T, nq, d), dtype=torch.float64, device=DEV)
        cache = {n: values(n) for n in ("k", "v")}
        turns = torch.tensor([math.pow(case["rope_base"], -2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device=DEV)
        for b, (L, c) in enumerate(zip(lengths, counts)):
            heads = st.qkv[b, :c].double().reshape(c, nq + 2 * nkv, d)
            norm = heads[:, :nq + nkv] * (heads[:, :nq + nkv].square().sum(-1, keepdim=True) / d + EPS).rsqrt()
            norm[:, :nq] *= st.q_weight.double()
            norm[:, nq:] *= st.k_weight.double()
            at = torch.tensor([L + x for x in depths(b)[:c]], dtype=torch.float64, device=DEV)
            z = torch.polar(torch.ones((), dtype=torch.float64, device=DEV), at[:, None] * turns)[:, None]
            turned = torch.complex(norm[..., :d // 2].contiguous(), norm[..., d // 2:].contiguous()) * z
            turned = torch.cat([turned.real, turned.imag], -1)
            q[b, :c] = turned[:, :nq]
            for name, rows in (("k", turned[:, nq:]), ("v", heads[:, nq + nkv:])):
                rows = rows.transpose(0, 1)
                cache[name][b, :, L:L + c] = rows if case["format"] == "f16" else held(nearest(rows, 11, -24))
        if case["format"] == "f16":
            return {"q": q, **cache}
        return {"q": q, **{n + "_back": x[:, :, st.first:st.first + st.rows] for n, x in cache.items()}}
    return {"append": append, "attend": attend}[case["op"]]()
