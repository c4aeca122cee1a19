"""cf_cache_append, cf_cache_read and cf_cache_keep against oracle/draft_block.py, through the C ABI.

Nothing here has a tolerance: rotated values are the fp64 ones rounded once to fp16, codes the nearest ones, scales one fp32 division,
read values one fp32 product and one rounding, and what a call does not own keeps its bytes."""
import numpy as np
import pytest

from draft_cases import FORMATS, code_bytes
from oracle import draft_block as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu
FILL = 0x5a


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


class Buffers:
    """A cache on the GPU, filled with a pattern, and its copy on the host."""

    def __init__(self, B, nkv, rows, d, fmt):
        import paper_2508_18850_amd as lib
        size = 2 if fmt == "f16" else 1
        self.fmt, self.shape = fmt, (B, nkv, rows, d)
        self.host = {n: np.full((B, nkv, rows, d * size), FILL, np.uint8) for n in ("k", "v")}
        self.host.update({n: np.full((B, nkv, rows), 1234.5, np.float32) for n in ("k_scale", "v_scale")})
        self.upload()
        self.lib = lib

    def upload(self):
        self.dev = {n: _dev(x) for n, x in self.host.items()}

    def pointers(self):
        return self.lib.cache_pointers(*(self.dev[n].data_ptr() for n in ("k", "v", "k_scale", "v_scale")))

    def put(self, name, b, first, rows):
        """fp16 rows [heads, n, d] into the host copy, in the cache's format."""
        n = rows.shape[1]
        if self.fmt == "f16":
            self.host[name][b, :, first:first + n] = np.ascontiguousarray(rows).view(np.uint8)
        else:
            code, scale = orc.encode(rows, self.fmt)
            self.host[name][b, :, first:first + n] = code_bytes(code, self.fmt)
            self.host[name + "_scale"][b, :, first:first + n] = scale

    def same(self):
        for n, x in self.host.items():
            got = self.dev[n].cpu().numpy()
            if x.dtype == np.float32:
                assert np.array_equal(got, x, equal_nan=True), n
            else:
                assert np.array_equal(got, x), (n, np.argwhere(got != x)[:4])


def _append(fmt, nq, nkv, d, B, T, lens, counts=None, depth=None, per_row=False, base=10000.0, seed=0, special=None, max_len=None,
            run=None):
    import paper_2508_18850_amd as lib
    print("append: %s %d/%d x %d batch %d tokens %d lens %s" % (fmt, nq, nkv, d, B, T, lens), flush=True)
    rng = np.random.default_rng(seed)
    bound = max(lens) if max_len is None else max_len
    rows = bound + T + 3
    qkv = rng.standard_normal((B, T, nq + 2 * nkv, d)).astype(np.float16)
    if special:
        special(qkv)
    buf = Buffers(B, nkv, rows, d, fmt)
    n_new = [T] * B if counts is None else counts
    q_want = np.full((B, T, nq, d), 7.0, np.float16)
    for b in range(B):
        for t in range(n_new[b]):
            at = lens[b] + (t if depth is None else int(depth[b, t] if per_row else depth[t]))
            with np.errstate(over="ignore", invalid="ignore"):
                turned = orc.rotate(qkv[b, t, :nq + nkv], at, base).astype(np.float16)
            q_want[b, t] = turned[:nq]
            buf.put("k", b, lens[b] + t, turned[nq:, None])
            buf.put("v", b, lens[b] + t, qkv[b, t, nq + nkv:, None])
    q = _dev(np.full((B, T, nq, d), 7.0, np.float16))
    x = _dev(qkv)
    dl, dc = _dev(np.array(lens, np.int32)), _dev(np.array(n_new, np.int32))
    dd = None if depth is None else _dev(np.asarray(depth, np.int32))
    draft = lib.draft(T, bound, row_len=dl.data_ptr(), row_tokens=dc.data_ptr() if counts is not None else 0,
                      depth=dd.data_ptr() if dd is not None else 0, per_row=per_row)
    kv = lib.KvCache(nq, nkv, d, B, rows, FORMATS[fmt], base)
    call = lambda stream: kv.append(B, x.data_ptr(), buf.pointers(), draft, q.data_ptr(), stream)  # noqa: E731
    if run:
        run(call, buf, q)
    else:
        call(torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert np.array_equal(q.cpu().numpy(), q_want, equal_nan=True)
    buf.same()


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("nq,nkv,d", [(1, 1, 64), (14, 7, 64), (3, 3, 128), (32, 8, 128), (33, 11, 64)], ids=str)
@pytest.mark.parametrize("B,T", [(1, 1), (3, 5)], ids=str)
def test_append(fmt, nq, nkv, d, B, T):
    _append(fmt, nq, nkv, d, B, T, [11 * b + 2 for b in range(B)], seed=nq + T)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_a_prompt(fmt):
    """Enough tokens for four of them to a workgroup; prompts of different lengths, one empty, into an empty cache."""
    _append(fmt, 4, 2, 64, 4, 701, [0, 0, 0, 0], counts=[701, 1, 0, 698], seed=5)
    _append(fmt, 2, 1, 128, 1, 2050, [3], seed=6)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_a_tree_far_out(fmt):
    """Positions where fp32 angles would be off; depths that are not the token's number, of all rows or of each."""
    depth = np.array([0, 1, 1, 2, 5, 2, 3], np.int32)
    _append(fmt, 4, 2, 128, 2, 7, [32000, 31], depth=depth, base=500000.0, seed=7)
    _append(fmt, 4, 2, 64, 2, 7, [32000, 0], counts=[7, 4], depth=np.stack([depth, depth[::-1]]), per_row=True, seed=8)


@pytest.mark.parametrize("fmt", FORMATS)
def test_append_special_rows(fmt):
    """Zeros, the smallest and the largest values, ties of the rounding, infinities and NaN (of a V head: a K head turns them)."""
    def special(x):                                             # heads: 2 queries, 2 keys, 2 values
        x[0, 0, 4] = 0
        x[0, 1, 4] = np.float16(2.0 ** -24)
        x[0, 1, 5] = np.float16(-65504)
        x[0, 2, 4] = np.arange(64) - 31                         # top 32
        x[0, 2, 5] = np.arange(64) / 8 - 0.5
        x[0, 3, 4, 7] = np.inf
        x[0, 3, 5, 9] = np.nan
        x[0, 4, 4] = -0.0
        x[0, 5, 4] = np.float16(2.0 ** -24) * np.arange(64)
        x[0, 5, 2:4] = np.float16(2.0 ** -24) * np.arange(64)   # keys turned within the subnormal numbers
        x[0, 6, 2:4] = 0
        x[0, 7, 0:4] = 65504                                    # turned beyond the largest fp16: infinite
    if fmt == "f16":
        def special_f16(x):
            special(x)
            x[0, 3, 5, 9] = 1
        _append(fmt, 2, 2, 64, 1, 8, [3], seed=9, special=special_f16)
    else:
        _append(fmt, 2, 2, 64, 1, 8, [3], seed=9, special=special)


def test_append_on_a_stream_and_captured():
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
            for n, x in buf.dev.items():
                x.copy_(_dev(np.full_like(buf.host[n], FILL if x.dtype == torch.uint8 else 1234.5)))
            q.fill_(7.0)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            for n, x in buf.dev.items():
                assert torch.equal(x, first[n])
    _append("int8", 6, 3, 64, 2, 9, [5, 2], counts=[9, 3], run=run)


def test_row_lengths_are_clamped():
    """Entries outside their range count as the nearest one inside."""
    import paper_2508_18850_amd as lib
    kv = lib.KvCache(2, 1, 64, 2, 20, 0, 10000.0)
    x = torch.randn(2, 4, 4 * 64, device="cuda").half()
    got = []
    for lens, counts in (((-5, 900), (77, -1)), ((0, 10), (4, 0))):
        buf = Buffers(2, 1, 20, 64, "f16")
        q = torch.zeros(2, 4, 2, 64, dtype=torch.float16, device="cuda")
        dl, dc = (_dev(np.array(v, np.int32)) for v in (lens, counts))
        kv.append(2, x.data_ptr(), buf.pointers(), lib.draft(4, 10, row_len=dl.data_ptr(), row_tokens=dc.data_ptr()), q.data_ptr(),
                  torch.cuda.current_stream().cuda_stream)
        torch.cuda.synchronize()
        got.append([q] + list(buf.dev.values()))
    assert all(torch.equal(a, b) for a, b in zip(*got))


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("nkv,d,B,first,rows", [(1, 64, 1, 0, 1), (3, 64, 2, 5, 77), (2, 128, 3, 1, 300), (1, 128, 1, 9, 1031), (2, 64, 1, 3, 0)], ids=str)
def test_read(fmt, nkv, d, B, first, rows):
    import paper_2508_18850_amd as lib
    print("read: %s %d heads x %d batch %d rows %d from %d" % (fmt, nkv, d, B, rows, first), flush=True)
    rng = np.random.default_rng(rows)
    buf = Buffers(B, nkv, first + rows + 2, d, fmt)
    for name in ("k", "v"):
        if fmt == "f16":
            buf.host[name] = rng.integers(0, 256, buf.host[name].shape).astype(np.uint8)
        else:                                                       # every code that the library writes, scales of all sizes
            raw = rng.integers(0, 256, buf.host[name].shape).astype(np.uint8)
            raw[(raw & 0x7f) == 0x7f] = 0x80 if fmt == "int8" else 0
            if fmt == "int8":
                raw[raw == 0x80] = 0
            buf.host[name] = raw
            buf.host[name + "_scale"] = np.exp(6 * rng.standard_normal(buf.host[name + "_scale"].shape)).astype(np.float32)
            buf.host[name + "_scale"][:, :, first::5] = 0
            buf.host[name + "_scale"][:, :, first + 1::7] = np.nan
    buf.upload()
    outs = {n: torch.full((B, nkv, rows + 1, d), 7.0, dtype=torch.float16, device="cuda") for n in ("k", "v")}
    lib.KvCache(nkv, nkv, d, B, first + rows + 2, FORMATS[fmt], 10000.0).read(
        B, buf.pointers(), first, rows, outs["k"].data_ptr(), outs["v"].data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    for n, out in outs.items():
        flat = out.cpu().numpy().reshape(-1)
        got, rest = flat[:B * nkv * rows * d].reshape(B, nkv, rows, d), flat[B * nkv * rows * d:]
        raw = buf.host[n][:, :, first:first + rows]
        if fmt == "f16":
            assert np.array_equal(got.view(np.uint8).reshape(raw.shape), raw)
        else:
            value = raw.view(np.int8).astype(np.float32) if fmt == "int8" else orc.E4M3.astype(np.float32)[raw]
            with np.errstate(over="ignore"):
                want = (value * buf.host[n + "_scale"][:, :, first:first + rows, None]).astype(np.float16)
            assert np.array_equal(got, want, equal_nan=True)
        assert (rest == 7.0).all()
    buf.same()


KEEP = [  # lens, new tokens, kept rows
    ([4], [6], [[0, 2, 5]]),
    ([0], [1], [[0]]),
    ([7], [5], [[]]),
    ([3, 9, 0], [8, 8, 8], [[7, 6, 5, 4, 3, 2, 1, 0], [0, 0, 3, 3], [1]]),          # backwards; twice the same; one
    ([2, 5], [64, 11], [list(range(1, 64, 2)), [10, 0, 10]]),
    ([1], [256], [list(range(255, -1, -1))]),
]


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("lens,counts,kept", KEEP, ids=["path", "one", "none", "ragged", "two", "reversed"])
def test_keep(fmt, d, lens, counts, kept):
    import paper_2508_18850_amd as lib
    B, T, nkv = len(lens), max(counts), 2
    print("keep: %s d %d lens %s of %s" % (fmt, d, lens, counts), flush=True)
    rng = np.random.default_rng(T)
    buf = Buffers(B, nkv, max(lens) + T + 2, d, fmt)
    for n in buf.host:
        buf.host[n] = rng.integers(0, 200, buf.host[n].shape).astype(buf.host[n].dtype)
    buf.upload()
    pad = np.full((B, T), 10 ** 6, np.int32)                        # not looked at
    for b, rows in enumerate(kept):
        pad[b, :len(rows)] = rows
        for n, x in buf.host.items():
            if fmt != "f16" or x.dtype == np.uint8:
                x[b, :, lens[b]:lens[b] + len(rows)] = x[b][:, [lens[b] + r for r in rows]]
    dl, dc, dk = _dev(np.array(lens, np.int32)), _dev(np.array(counts, np.int32)), _dev(pad)
    dn, new = _dev(np.array([len(r) for r in kept], np.int32)), torch.full((B + 1,), -1, dtype=torch.int32, device="cuda")
    kv = lib.KvCache(4, nkv, d, B, max(lens) + T + 2, FORMATS[fmt], 10000.0)
    kv.keep(B, buf.pointers(), lib.draft(T, max(lens), row_len=dl.data_ptr(), row_tokens=dc.data_ptr()), dk.data_ptr(), dn.data_ptr(),
            new.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    buf.same()
    assert new.tolist() == [L + len(r) for L, r in zip(lens, kept)] + [-1]


def test_keep_clamps_and_needs_no_new_len():
    import paper_2508_18850_amd as lib
    buf = Buffers(1, 1, 12, 64, "int8")
    buf.host["k"][:] = np.arange(12, dtype=np.uint8)[:, None]
    buf.upload()
    buf.host["k"][0, 0, 4:8] = np.array([7, 4, 7, 5], np.uint8)[:, None]     # rows 4 + (9 -> 3), 4 + (-1 -> 0), 4 + 3, 4 + 1; n_kept 50 -> 4
    kept, n_kept = _dev(np.array([[9, -1, 3, 1]], np.int32)), _dev(np.array([50], np.int32))
    lib.KvCache(1, 1, 64, 1, 12, 2, 10000.0).keep(1, buf.pointers(), lib.draft(4, 4), kept.data_ptr(), n_kept.data_ptr(), 0,
                                                   torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    buf.same()


def test_slices_beyond_32_bits():
    """The last head's slice starts beyond 4 GiB: 33 heads of 2^20 rows of 128 codes."""
    import paper_2508_18850_amd as lib
    nkv, rows, d = 33, 1 << 20, 128
    k, v = (torch.zeros((nkv, rows, d), dtype=torch.uint8, device="cuda") for _ in range(2))
    ks, vs = (torch.zeros((nkv, rows), device="cuda") for _ in range(2))
    cache = lib.cache_pointers(k.data_ptr(), v.data_ptr(), ks.data_ptr(), vs.data_ptr())
    kv = lib.KvCache(nkv, nkv, d, 1, rows, 2, 10000.0)
    qkv = torch.randn((1, 2, 3 * nkv, d), device="cuda").half()
    q = torch.empty((1, 2, nkv, d), dtype=torch.float16, device="cuda")
    s = torch.cuda.current_stream().cuda_stream
    draft = lib.draft(2, rows - 2)
    kv.append(1, qkv.data_ptr(), cache, draft, q.data_ptr(), s)
    out = torch.empty((2, nkv, 2, d), dtype=torch.float16, device="cuda")
    kv.read(1, cache, rows - 2, 2, out[0].data_ptr(), out[1].data_ptr(), s)
    torch.cuda.synchronize()
    want = qkv[0, :, 2 * nkv:].transpose(0, 1).float()
    assert ((out[1].float() - want).abs().amax(-1) <= want.abs().amax(-1) * (0.5 / 127 + 2.0 ** -11)).all()
    before = k[-1, -1].clone(), v[-1, -1].clone()
    kept, n_kept = torch.tensor([[1, 0]], dtype=torch.int32, device="cuda"), torch.tensor([1], dtype=torch.int32, device="cuda")
    kv.keep(1, cache, draft, kept.data_ptr(), n_kept.data_ptr(), 0, s)
    torch.cuda.synchronize()
    assert torch.equal(k[-1, -2], before[0]) and torch.equal(v[-1, -2], before[1]) and vs[-1, -2] == vs[-1, -1]
    assert not v[0, :rows - 2].any() and not v[-1, :rows - 2].any()
