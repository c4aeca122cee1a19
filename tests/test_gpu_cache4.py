"""The cache calls in 4 bits, and the append with norms in every format, through the C ABI against oracle/quantized_step.py.

In 4 bits nothing has a tolerance but what depends on the norm: rotated values are the fp64 ones rounded once to fp16, codes the nearest ones,
read values exact.  With norms kernel and oracle take the same steps in fp64 in another order, so that a value which lies within some 2^-45
of a border between two fp16 numbers may go either way: one in 10^9, none among the inputs below (they are as drawn)."""
import numpy as np
import pytest

from draft_cases import FORMATS as OTHERS
from oracle import draft_block as base
from oracle import quantized_step as orc
from quant_cases import FILL, FORMATS, MXFP4, Buffers

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _append(fmt, nq, nkv, d, B, T, lens, counts=None, depth=None, per_row=False, rope=10000.0, seed=0, special=None, eps=None, run=None):
    """eps: with norms."""
    import paper_2508_18850_amd as lib
    print("append: %s %d/%d x %d batch %d tokens %d lens %s eps %s" % (fmt, nq, nkv, d, B, T, lens, eps), flush=True)
    rng = np.random.default_rng(seed)
    bound, rows = max(lens), max(lens) + T + 3
    qkv = (rng.standard_normal((B, T, nq + 2 * nkv, d)) * np.exp(rng.standard_normal((B, T, nq + 2 * nkv, 1)))).astype(np.float16)
    weight = (1 + 0.3 * rng.standard_normal((2, d))).astype(np.float16)
    if special:
        special(qkv)
    buf = Buffers(B, nkv, rows, d, fmt)
    n_new = [T] * B if counts is None else counts
    q_want = np.full((B, T, nq, d), 7.0, np.float16)
    for b in range(B):
        for t in range(n_new[b]):
            at = lens[b] + (t if depth is None else int(depth[b, t] if per_row else depth[t]))
            x = qkv[b, t, :nq + nkv].astype(np.float64)
            if eps is not None:
                x = np.concatenate([orc.head_norm(x[:nq], weight[0], eps), orc.head_norm(x[nq:], weight[1], eps)])
            with np.errstate(over="ignore", invalid="ignore"):
                turned = base.rotate(x, at, rope).astype(np.float16)
            q_want[b, t] = turned[:nq]
            buf.put("k", b, lens[b] + t, turned[nq:, None])
            buf.put("v", b, lens[b] + t, qkv[b, t, nq + nkv:, None])
    q, x, w = _dev(np.full((B, T, nq, d), 7.0, np.float16)), _dev(qkv), _dev(weight)
    dl, dc = _dev(np.array(lens, np.int32)), _dev(np.array(n_new, np.int32))
    dd = None if depth is None else _dev(np.asarray(depth, np.int32))
    draft = lib.draft(T, bound, row_len=dl.data_ptr(), row_tokens=dc.data_ptr() if counts is not None else 0,
                      depth=dd.data_ptr() if dd is not None else 0, per_row=per_row)
    kv = lib.KvCache(nq, nkv, d, B, rows, FORMATS[fmt], rope)

    def call(stream):
        if eps is None:
            kv.append(B, x.data_ptr(), buf.pointers(), draft, q.data_ptr(), stream)
        else:
            kv.append_normed(B, x.data_ptr(), w[0].data_ptr(), w[1].data_ptr(), eps, buf.pointers(), draft, q.data_ptr(), stream)
    if run:
        run(call, buf, q)
    else:
        call(_stream())
    torch.cuda.synchronize()
    assert np.array_equal(q.cpu().numpy(), q_want, equal_nan=True)
    buf.same()


SHAPES = [(1, 1, 64), (14, 7, 64), (3, 3, 128), (32, 8, 128), (33, 11, 64)]


@pytest.mark.parametrize("nq,nkv,d", SHAPES, ids=str)
@pytest.mark.parametrize("B,T", [(1, 1), (3, 5)], ids=str)
def test_append_4_bits(nq, nkv, d, B, T):
    _append("mxfp4", nq, nkv, d, B, T, [11 * b + 2 for b in range(B)], seed=nq + T)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("nq,nkv,d", SHAPES, ids=str)
@pytest.mark.parametrize("eps", [1e-6, 0.0, 0.5])
def test_append_with_norms(fmt, nq, nkv, d, eps):
    _append(fmt, nq, nkv, d, 1, 1, [9], seed=nq, eps=eps)
    _append(fmt, nq, nkv, d, 3, 4, [0, 7, 31], counts=[4, 0, 3], seed=nq + 1, eps=eps)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("eps", [None, 1e-5])
def test_append_a_prompt(fmt, eps):
    """Enough tokens for four of them to a workgroup; prompts of different lengths, one empty, into an empty cache."""
    if eps is None and fmt in OTHERS:
        pytest.skip("test_gpu_cache.py has it")
    _append(fmt, 4, 2, 64, 4, 701, [0, 0, 0, 0], counts=[701, 1, 0, 698], seed=5, eps=eps)
    _append(fmt, 2, 1, 128, 1, 2050, [3], seed=6, eps=eps)


@pytest.mark.parametrize("eps", [None, 1e-6])
def test_append_a_tree_far_out(eps):
    depth = np.array([0, 1, 1, 2, 5, 2, 3], np.int32)
    _append("mxfp4", 4, 2, 128, 2, 7, [32000, 31], depth=depth, rope=500000.0, seed=7, eps=eps)
    _append("mxfp4", 4, 2, 64, 2, 7, [32000, 0], counts=[7, 4], depth=np.stack([depth, depth[::-1]]), per_row=True, seed=8, eps=eps)


def test_every_fp16_number_as_a_value():
    """All 63488 finite ones as values of V heads, and every block with a top of its own: codes, signs of zeros and scales to the bit."""
    x = np.arange(65536, dtype=np.uint16).view(np.float16)
    x = np.random.default_rng(1).permutation(x[np.isfinite(x)])
    for d in (64, 128):
        for shrink in (0, 1):                                       # blocks whose tops are small as well
            rows = x.reshape(-1, d)
            if shrink:
                rows = (rows.astype(np.float64) * 2.0 ** -np.random.default_rng(2).integers(0, 32, (rows.shape[0], 1))).astype(np.float16)

            def fill(qkv):                                          # the value head of a token each
                qkv[0, :, 2] = rows
            _append("mxfp4", 1, 1, d, 1, rows.shape[0], [0], seed=3, special=fill)


@pytest.mark.parametrize("eps", [None, 1e-6, 0.0])
@pytest.mark.parametrize("fmt", ["f16", "mxfp4"])
def test_append_special_rows(fmt, eps):
    """Zeros, the smallest and the largest values, infinities and NaN in one block of a value head, in a query and in a key."""
    def special(x):                                             # heads: 2 queries, 2 keys, 2 values
        x[0, 0, 4] = 0
        x[0, 1, 4] = np.float16(2.0 ** -24)
        x[0, 1, 5] = np.float16(-65504)
        x[0, 2, 4] = np.arange(64) - 31
        x[0, 2, 5] = np.arange(64) / 8 - 0.5
        x[0, 3, 4, 7] = np.inf
        x[0, 3, 5, 40] = 1.0 if fmt == "f16" else np.nan        # (fp16 keeps the bits of a NaN, which numpy's arrays compare as equal in values only)
        x[0, 4, 4] = -0.0
        x[0, 5, 4] = np.float16(2.0 ** -24) * np.arange(64)
        x[0, 5, :4] = np.float16(2.0 ** -24) * (1 + np.arange(64))
        x[0, 6, :4] = 0
        x[0, 7, 0:4] = 65504
    if eps != 0.0:
        _append(fmt, 2, 2, 64, 1, 8, [3], seed=9, special=special, eps=eps)
    else:
        with np.errstate(invalid="ignore"):
            _append("mxfp4", 2, 2, 64, 1, 8, [3], seed=9, special=special, eps=eps)


def test_norm_of_infinite_and_nan_heads():
    """By the formula: all of a head with a NaN is NaN; of a head with an infinity that dimension and its partner of the rotation, zeros elsewhere."""
    import paper_2508_18850_amd as lib
    x = torch.ones((1, 2, 3, 64), dtype=torch.float16, device="cuda")
    x[0, 0, 0, 5], x[0, 1, 0, 7] = float("nan"), float("-inf")
    w, q = torch.ones(64, dtype=torch.float16, device="cuda"), torch.zeros((1, 2, 1, 64), dtype=torch.float16, device="cuda")
    buf = Buffers(1, 1, 5, 64, "f16")
    lib.KvCache(1, 1, 64, 1, 5, 0, 10000.0).append_normed(1, x.data_ptr(), w.data_ptr(), w.data_ptr(), 1e-6, buf.pointers(), lib.draft(2, 3), q.data_ptr(), _stream())
    torch.cuda.synchronize()
    assert q[0, 0, 0].isnan().all()
    assert q[0, 1, 0].isnan().nonzero().flatten().tolist() == [7, 39] and (q[0, 1, 0].nan_to_num() == 0).all()


@pytest.mark.parametrize("eps", [None, 1e-6])
def test_append_on_a_stream_and_captured(eps):
    """On a stream of its own, then three replays of a captured call into cleared buffers."""
    def run(call, buf, q):
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        call(s.cuda_stream)
        s.synchronize()
        first = {n: x.clone() for n, x in buf.dev.items()}
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            call(torch.cuda.current_stream().cuda_stream)
        for _ in range(3):
            for x in buf.dev.values():
                x.fill_(FILL)
            q.fill_(7.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for n, x in buf.dev.items():
                assert torch.equal(x, first[n])
    _append("mxfp4", 6, 3, 64, 2, 9, [5, 2], counts=[9, 3], run=run, eps=eps)


@pytest.mark.parametrize("nkv,d,B,first,rows", [(1, 64, 1, 0, 1), (3, 64, 2, 5, 77), (2, 128, 3, 1, 300), (1, 128, 1, 9, 1031), (2, 64, 1, 3, 0)], ids=str)
def test_read(nkv, d, B, first, rows):
    """Every code under every scale that the format has."""
    import paper_2508_18850_amd as lib
    print("read: %d heads x %d batch %d rows %d from %d" % (nkv, d, B, rows, first), flush=True)
    rng = np.random.default_rng(rows)
    buf = Buffers(B, nkv, first + rows + 2, d, "mxfp4")
    for n in ("k", "v"):
        buf.host[n] = rng.integers(0, 256, buf.host[n].shape).astype(np.uint8)
        scale = rng.integers(104, 142, buf.host[n + "_scale"].shape)
        buf.host[n + "_scale"] = np.where(scale == 141, 255, scale).astype(np.uint8)
    buf.upload()
    outs = {n: torch.full((B, nkv, rows + 1, d), 7.0, dtype=torch.float16, device="cuda") for n in ("k", "v")}
    lib.KvCache(nkv, nkv, d, B, first + rows + 2, MXFP4, 10000.0).read(B, buf.pointers(), first, rows, outs["k"].data_ptr(), outs["v"].data_ptr(), _stream())
    torch.cuda.synchronize()
    for n, out in outs.items():
        flat = out.cpu().numpy().reshape(-1)
        got, rest = flat[:B * nkv * rows * d].reshape(B, nkv, rows, d), flat[B * nkv * rows * d:]
        want = orc.decode4(orc.unpack4(buf.host[n][:, :, first:first + rows]), buf.host[n + "_scale"][:, :, first:first + rows])
        assert np.array_equal(got.astype(np.float64), want, equal_nan=True) and (rest == 7.0).all()
    buf.same()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,counts,kept", [
    ([4], [6], [[0, 2, 5]]), ([0], [1], [[0]]), ([7], [5], [[]]), ([3, 9, 0], [8, 8, 8], [[7, 6, 5, 4, 3, 2, 1, 0], [0, 0, 3, 3], [1]]),
    ([2, 5], [64, 11], [list(range(1, 64, 2)), [10, 0, 10]]), ([1], [256], [list(range(255, -1, -1))])], ids=["path", "one", "none", "ragged", "two", "reversed"])
def test_keep(d, lens, counts, kept):
    import paper_2508_18850_amd as lib
    B, T, nkv = len(lens), max(counts), 3
    print("keep: d %d lens %s of %s" % (d, lens, counts), flush=True)
    rng = np.random.default_rng(T)
    buf = Buffers(B, nkv, max(lens) + T + 2, d, "mxfp4")
    for n in buf.host:
        buf.host[n] = rng.integers(0, 256, buf.host[n].shape).astype(np.uint8)
    buf.upload()
    pad = np.full((B, T), 10 ** 6, np.int32)                        # not looked at
    for b, rows in enumerate(kept):
        pad[b, :len(rows)] = rows
        for x in buf.host.values():
            x[b, :, lens[b]:lens[b] + len(rows)] = x[b][:, [lens[b] + r for r in rows]]
    dl, dc, dk = _dev(np.array(lens, np.int32)), _dev(np.array(counts, np.int32)), _dev(pad)
    dn, new = _dev(np.array([len(r) for r in kept], np.int32)), torch.full((B + 1,), -1, dtype=torch.int32, device="cuda")
    kv = lib.KvCache(6, nkv, d, B, max(lens) + T + 2, MXFP4, 10000.0)
    kv.keep(B, buf.pointers(), lib.draft(T, max(lens), row_len=dl.data_ptr(), row_tokens=dc.data_ptr()), dk.data_ptr(), dn.data_ptr(), new.data_ptr(), _stream())
    torch.cuda.synchronize()
    buf.same()
    assert new.tolist() == [L + len(r) for L, r in zip(lens, kept)] + [-1]


def test_slices_beyond_32_bits():
    """The last head's slice starts beyond 4 GiB: 67 heads of 2^20 rows of 64 bytes."""
    import paper_2508_18850_amd as lib
    nkv, rows, d = 67, 1 << 20, 128
    k, v = (torch.zeros((nkv, rows, d // 2), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((nkv, rows, d // 32), dtype=torch.uint8, device="cuda") for _ in range(2))
    cache = lib.cache_pointers(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr())
    kv = lib.KvCache(nkv, nkv, d, 1, rows, MXFP4, 10000.0)
    tree = lib.TreeAttention(nkv, nkv, d, 1, rows, MXFP4, 10000.0, 2, window=1)
    qkv = torch.randn((1, 2, 3 * nkv, d), device="cuda").half()
    q, a = (torch.empty((1, 2, nkv, d), dtype=torch.float16, device="cuda") for _ in range(2))
    draft = lib.draft(2, rows - 2)
    kv.append(1, qkv.data_ptr(), cache, draft, q.data_ptr(), _stream())
    out = torch.empty((2, nkv, 2, d), dtype=torch.float16, device="cuda")
    kv.read(1, cache, rows - 2, 2, out[0].data_ptr(), out[1].data_ptr(), _stream())
    tree.attend(1, q.data_ptr(), cache, draft, 0, a.data_ptr(), _stream())        # a window of one: each token's result is its own value
    torch.cuda.synchronize()
    code, scale = orc.encode4(qkv[0, :, 2 * nkv:].transpose(0, 1).cpu().numpy())
    want = orc.decode4(code, scale)
    assert np.array_equal(out[1].cpu().numpy().astype(np.float64), want)
    assert np.abs(a[0].transpose(0, 1).cpu().numpy() - want).max() <= 2.0 ** -10 * np.abs(want).max()
    before = k[-1, -1].clone(), v[-1, -1].clone(), vs[-1, -1].clone()
    kept, n_kept = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda")
    kv.keep(1, cache, draft, kept.data_ptr(), n_kept.data_ptr(), 0, _stream())
    torch.cuda.synchronize()
    assert torch.equal(k[-1, -2], before[0]) and torch.equal(v[-1, -2], before[1]) and torch.equal(vs[-1, -2], before[2])
    assert not v[0, :rows - 2].any() and not v[-1, :rows - 2].any()
    tree.close()
