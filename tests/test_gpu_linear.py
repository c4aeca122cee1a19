"""cf_linear_quantize and cf_linear_forward against oracle/quantized_step.py, through the C ABI.

Nothing has a tolerance: codes are the correctly rounded ones, scales one fp32 division, sums whole numbers, and the result three fp32
roundings and one to fp16 in a fixed order."""
import numpy as np
import pytest

from oracle import draft_block as base
from oracle import quantized_step as orc

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _stream():
    return torch.cuda.current_stream().cuda_stream


# ---- rows to codes ------------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("rows", [1, 3, 130])
@pytest.mark.parametrize("n", [16, 64, 496, 512, 1376, 4096, 4112, 11008, 16384, 16400, 28672, 40000])
def test_rows_to_codes(rows, n):
    import paper_2508_18850_amd as lib
    print("quantize: %d x %d" % (rows, n), flush=True)
    rng = np.random.default_rng(n + rows)
    x = (rng.standard_normal((rows, n)) * np.exp(2 * rng.standard_normal((rows, 1)))).astype(np.float16)
    x[0, n - 1] = -60000                                            # the largest at the end
    if rows > 2:
        x[1], x[2, 5] = 0, np.float16(2.0 ** -24)
    if rows > 100:
        x[50, 3], x[60, n - 2], x[70] = np.nan, -np.inf, (np.arange(n) % 255 - 127).astype(np.float16)
        x[80] = ((np.arange(n) % 510 - 254.0) / 2).astype(np.float16)       # every border between two codes
        x[80, 0] = 127
        x[90] = np.float16(2.0 ** -24) * (np.arange(n) % 300)
    code, scale = base.encode(x, "int8")
    xd, codes, scales = _dev(x), torch.full((rows + 1, n), 77, dtype=torch.int8, device="cuda"), torch.full((rows + 1,), 5.0, device="cuda")
    lib.quantize_rows(rows, n, xd.data_ptr(), codes.data_ptr(), scales.data_ptr(), _stream())
    torch.cuda.synchronize()
    assert np.array_equal(codes[:rows].cpu().numpy(), code.astype(np.int8)) and np.array_equal(scales[:rows].cpu().numpy(), scale, equal_nan=True)
    assert (codes[rows:] == 77).all() and scales[rows] == 5.0


def test_every_fp16_number_under_some_tops():
    import paper_2508_18850_amd as lib
    x = np.arange(32768, dtype=np.uint16).view(np.float16)
    x = x[np.isfinite(x)]
    tops = np.array([65504, 1, 0.1, 127, 254, 2.0 ** -14, 3.0 ** -9], np.float16)
    rows = np.stack([np.where(x <= t, x, -t) for t in tops])
    code, scale = base.encode(rows, "int8")
    xd, codes, scales = _dev(rows), torch.zeros(rows.shape, dtype=torch.int8, device="cuda"), torch.zeros(len(tops), device="cuda")
    lib.quantize_rows(len(tops), rows.shape[1], xd.data_ptr(), codes.data_ptr(), scales.data_ptr(), _stream())
    torch.cuda.synchronize()
    assert np.array_equal(codes.cpu().numpy(), code.astype(np.int8)) and np.array_equal(scales.cpu().numpy(), scale)


# ---- products -----------------------------------------------------------------------------------------------------------------

class Product:
    def __init__(self, M, K, N, seed=0, max_rows=None, full=False):
        import paper_2508_18850_amd as lib
        print("product: %d x %d x %d" % (M, K, N), flush=True)
        g = torch.Generator(device="cuda").manual_seed(seed + M + K + N)
        codes = lambda *shape: torch.randint(-128 if full else -127, 128, shape, generator=g, device="cuda", dtype=torch.int32).to(torch.int8)  # noqa: E731
        self.x, self.w = codes(M, K), codes(N, K)
        self.xs = torch.rand(M, generator=g, device="cuda") * 0.01 + 1e-4
        self.ws = torch.rand(N, generator=g, device="cuda") * 0.001 + 1e-6
        self.out = torch.full((M + 1, N), 7.0, dtype=torch.float16, device="cuda")
        self.M, self.linear = M, lib.Int8Linear(K, N, max_rows or M)

    def call(self, stream=None):
        self.linear.forward(self.M, self.x.data_ptr(), self.xs.data_ptr(), self.w.data_ptr(), self.ws.data_ptr(), self.out.data_ptr(),
                            _stream() if stream is None else stream)

    def want(self):
        # whole numbers below 2^53: exact in fp64 in any order
        total = self.x.double() @ self.w.double().T.contiguous()
        return (total.float() * self.xs[:, None] * self.ws).half()

    def check(self):
        self.out.fill_(7.0)
        self.call()
        torch.cuda.synchronize()
        assert torch.equal(self.out[:self.M], self.want()), (self.out[:self.M] != self.want()).nonzero()[:4]
        assert (self.out[self.M:] == 7.0).all(), "rows behind the last were written"
        return self.out[:self.M].clone()


ROWS = [1, 2, 3, 8, 15, 16, 17, 31, 32, 33, 48, 63, 64, 65, 100, 127, 128, 129, 200, 255, 256, 257, 300]


@pytest.mark.parametrize("M", ROWS)
def test_rows(M):
    Product(M, 512, 256).check()
    Product(M, 80, 72).check()


@pytest.mark.parametrize("K", [16, 32, 48, 64, 112, 128, 144, 240, 256, 272, 496, 512, 896, 1008, 1376, 2048, 2064, 11008])
def test_lengths_of_the_sum(K):
    for M in (1, 20, 70, 300):
        Product(M, K, 136).check()


@pytest.mark.parametrize("N", [8, 16, 24, 56, 64, 72, 120, 128, 136, 248, 256, 264, 520, 1000, 4104])
def test_outputs(N):
    for M in (1, 20, 70, 300):
        Product(M, 208, N).check()


@pytest.mark.parametrize("M,K,N", [(1, 4096, 12288), (4, 8192, 10240), (16, 11008, 4096), (64, 4096, 6144), (77, 28672, 8192), (128, 14336, 4096),
                                   (500, 4096, 6144), (1024, 1376, 512), (2048, 4096, 4096), (3000, 896, 1792)], ids=str)
def test_shapes_of_models(M, K, N):
    Product(M, K, N).check()


def test_against_the_oracle():
    """The same in numpy's integers, and codes of -128."""
    for M, K, N in ((5, 96, 40), (130, 272, 200)):
        c = Product(M, K, N, full=True)
        total, out = orc.int8_product(*(t.cpu().numpy() for t in (c.x, c.xs, c.w, c.ws)))
        assert np.array_equal(c.check().cpu().numpy(), out)


@pytest.mark.parametrize("M", [1, 40, 300])
def test_largest_sums(M):
    """-128 times -128 as often as there may be inputs: 131056 of them are 2^31 - 2^18, the most that 32 bits hold."""
    c = Product(M, 131056, 16)
    c.x.fill_(-128)
    c.w.fill_(-128)
    c.w[3] = 127
    c.xs.fill_(2.0 ** -9)
    c.ws.fill_(2.0 ** -9)
    c.check()


@pytest.mark.parametrize("M", [2, 70, 300])
def test_special_scales(M):
    """NaN rows stay apart, zeros and results beyond fp16."""
    c = Product(M, 256, 128)
    c.xs[0], c.xs[1] = float("nan"), 0.0
    c.ws[5], c.ws[6] = float("inf"), 1e30
    c.call()
    torch.cuda.synchronize()
    want = c.want()
    assert torch.equal(torch.nan_to_num(c.out[:M], 3.0, 4.0, 5.0), torch.nan_to_num(want, 3.0, 4.0, 5.0))
    assert want[0].isnan().all() and c.out[0].isnan().all()


def test_one_handle_for_calls_of_different_sizes():
    """And the same bits again, whatever ran before on the handle."""
    big = Product(300, 1024, 256, max_rows=300)
    first = {}
    for M in (300, 1, 64, 17, 300, 1, 64, 17, 128):
        big.M = M
        got = big.x[:M], big.check_rows(M)
        assert M not in first or torch.equal(first[M], got[1])
        first[M] = got[1]


def _check_rows(self, M):
    self.out.fill_(7.0)
    self.call()
    torch.cuda.synchronize()
    want = ((self.x[:M].double() @ self.w.double().T.contiguous()).float() * self.xs[:M, None] * self.ws).half()
    assert torch.equal(self.out[:M], want) and (self.out[M:] == 7.0).all()
    return want


Product.check_rows = _check_rows


@pytest.mark.parametrize("M", [1, 33, 200])
def test_captured_and_replayed(M):
    """Three replays with eager calls and changed inputs between them."""
    c = Product(M, 4096, 512)
    want = c.check()
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.call(torch.cuda.current_stream().cuda_stream)
    for replay in range(3):
        c.out.fill_(7.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(c.out[:M], want), replay
        c.x.neg_()
        want = -want
        c.check()


def test_two_handles_on_two_streams():
    cases = [Product(64, 8192, 512, seed=i) for i in range(2)]
    want = [c.check() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    for c in cases:
        c.out.fill_(7.0)
    torch.cuda.synchronize()
    for _ in range(20):
        for c, s in zip(cases, streams):
            c.call(s.cuda_stream)
    torch.cuda.synchronize()
    for c, w in zip(cases, want):
        assert torch.equal(c.out[:64], w)


def test_one_handle_on_two_streams():
    """It has no workspace: two streams, and two graphs with calls on it, at the same time."""
    cases = [Product(16, 4096, 512, seed=i) for i in range(2)]
    want = [c.check() for c in cases]
    cases[1].linear = cases[0].linear
    streams = [torch.cuda.Stream() for _ in cases]
    graphs = [torch.cuda.CUDAGraph() for _ in cases]
    for c, g in zip(cases, graphs):
        with torch.cuda.graph(g):
            for _ in range(4):
                c.call(torch.cuda.current_stream().cuda_stream)
    for replayed in (False, True):
        for c in cases:
            c.out.fill_(7.0)
        torch.cuda.synchronize()
        for _ in range(10):
            for c, s, g in zip(cases, streams, graphs):
                if replayed:
                    with torch.cuda.stream(s):
                        g.replay()
                else:
                    c.call(s.cuda_stream)
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert torch.equal(c.out[:len(w)], w), replayed


def test_offsets_beyond_32_bits():
    """Codes and results of more than 4 GiB; the last rows against a product of their own."""
    M, K, N = 300000, 16384, 8192
    import paper_2508_18850_amd as lib
    x = torch.zeros((M, K), dtype=torch.int8, device="cuda")
    x[-300:].copy_(torch.randint(-127, 128, (300, K), device="cuda", dtype=torch.int32))
    w = torch.randint(-127, 128, (N, K), device="cuda", dtype=torch.int32).to(torch.int8)
    xs, ws = torch.full((M,), 0.01, device="cuda"), torch.full((N,), 0.001, device="cuda")
    out = torch.full((M, N), 7.0, dtype=torch.float16, device="cuda")
    linear = lib.Int8Linear(K, N, M)
    linear.forward(M, x.data_ptr(), xs.data_ptr(), w.data_ptr(), ws.data_ptr(), out.data_ptr(), _stream())
    torch.cuda.synchronize()
    want = ((x[-300:].double() @ w.double().T.contiguous()).float() * xs[-300:, None] * ws).half()
    assert torch.equal(out[-300:], want) and not out[:1000].any() and not out[150000:151000].any()


def test_refusals():
    """Each differs from a call that runs in what is refused."""
    import paper_2508_18850_amd as lib
    linear = lib.Int8Linear(64, 32, 8)
    buf = torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = (buf.data_ptr() + 255) // 256 * 256
    X, XS, W, WS, OUT = (p + 8192 * i for i in range(5))
    call = lambda rows=8, x=X, xs=XS, w=W, ws=WS, out=OUT: linear.forward_rc(rows, x, xs, w, ws, out, _stream())  # noqa: E731
    assert call() == 0 and call(rows=1) == 0 and call(xs=XS + 4) == 0 and call(x=W) == 0      # (inputs may share memory)
    for over in (dict(rows=0), dict(rows=-1), dict(rows=9), dict(x=0), dict(xs=0), dict(w=0), dict(ws=0), dict(out=0), dict(x=X + 8), dict(w=W + 4), dict(out=OUT + 2),
                 dict(xs=XS + 2), dict(ws=WS + 1), dict(out=X), dict(out=X + 496), dict(out=X - 496), dict(out=W), dict(out=W + 2032), dict(out=XS), dict(out=XS + 16),
                 dict(out=WS), dict(out=WS + 112)):
        assert call(**over) == -1, over
    assert call(out=X + 512) == 0 and call(out=W + 2048) == 0 and call(out=WS + 128) == 0
    torch.cuda.synchronize()
    linear.close()
