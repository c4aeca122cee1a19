"""cf_tree_attend over a cache in 4 bits, against oracle/draft_block.py on the values that the cache stands for.  Those are fp16 numbers, which enter
the products as such, so that the bound is the one of an fp16 cache (draft_cases.bound)."""
import numpy as np
import pytest

from draft_cases import random_tree
from oracle import draft_block as base
from oracle import quantized_step as orc
from quant_cases import MXFP4, store
import test_gpu_tree

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


class Case(test_gpu_tree.Case):
    """The same inputs, held in 4 bits."""

    def __init__(self, nq, nkv, d, lens, T, max_tokens=None, **more):
        print("attend: %d/%d x %d lens %s T %d %s" % (nq, nkv, d, lens, T, {k: v for k, v in more.items() if np.ndim(v) == 0}), flush=True)
        super().__init__("f16", nq, nkv, d, lens, T, max_tokens=max_tokens, **more)
        self.tree.close()
        self.fmt = "mxfp4"
        self.tree = self.lib.TreeAttention(nq, nkv, d, self.B, self.rows, MXFP4, 10000.0, max_tokens or T, self.cap, self.window)
        self.hold(self.k, self.v)

    def hold(self, k, v):
        """fp16 rows as the cache's codes, scales and values."""
        self.k, self.ks, self.kv = store(k, "mxfp4")
        self.v, self.vs, self.vv = store(v, "mxfp4")

    def poison_rest(self):
        for b in range(self.B):
            end = self.lens[b] + self.counts[b]
            self.ks[b, :, end:], self.vs[b, :, end:] = 255, 255

    def want(self):
        return base.attend(self.q, self.kv, self.vv, self.lens, self.counts, self.depth, self.mask, self.slopes, self.cap, self.window)


@pytest.mark.parametrize("L", [0, 1, 15, 31, 32, 33, 63, 64, 127, 250, 511])
def test_lengths(L):
    Case(4, 2, 64, [L], 3, seed=1).check()
    Case(4, 1, 128, [L], 5, seed=2).check()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [1, 2, 7, 16, 17, 31, 33, 63, 64, 65, 100, 128, 129, 256])
def test_drafts(d, T):
    c = Case(2, 1, d, [75], T, seed=3)
    c.poison_rest()
    c.check()


@pytest.mark.parametrize("nq,nkv", [(1, 1), (3, 1), (5, 5), (8, 1), (16, 1), (12, 4), (64, 8), (24, 1)], ids=str)
def test_heads(nq, nkv):
    for T in (1, 6):
        Case(nq, nkv, 64 if nq % 2 else 128, [90], T, seed=4).check()


@pytest.mark.parametrize("per_row", [True, False])
def test_ragged_batches(per_row):
    """Lengths and counts of their own, a row without cached tokens, one without new ones, a bound above all lengths; what lies
    behind is NaN."""
    for d, T in ((128, 9), (64, 90)):
        c = Case(8, 2, d, [300, 0, 77, 140], T, counts=[T, 4, 0, 1], per_row=per_row, seed=5, max_len=333)
        c.poison_rest()
        c.check()


@pytest.mark.parametrize("cap,window,slopes", [(5.0, 0, False), (0.0, 40, False), (0.0, 0, True), (20.0, 100, True), (0.0, 1, False),
                                               (0.0, 10000, True)], ids=str)
def test_forms_of_the_score(cap, window, slopes):
    Case(6, 2, 64, [190, 23], 12, cap=cap, window=window, slopes=slopes, seed=6, q_size=3.0).check()
    Case(4, 2, 128, [333], 70, chain=True, cap=cap, window=window, slopes=slopes, seed=7).check()
    Case(8, 1, 128, [0, 65], 4, counts=[4, 2], cap=cap, window=window, slopes=slopes, seed=8).check()
    Case(4, 4, 64, [500], 40, cap=cap, window=window, slopes=slopes, seed=9).check()


@pytest.mark.parametrize("T", [3, 80])
def test_rows_that_see_nothing(T):
    """An empty cache and empty masks; a window that reaches no key."""
    mask = np.zeros((2, T, T), bool)
    mask[:, 2, 1] = mask[:, 1, 0] = True
    depth = np.tile(np.arange(T, dtype=np.int32) % 5 * 3, (2, 1))
    got = Case(2, 1, 64, [0, 3], T, mask=mask, depth=depth, seed=10).check()
    assert not got[0, 0].any() and got[0, 2].any(-1).all() and got[1].any(-1).all()
    got = Case(2, 1, 128, [6, 40], T, mask=mask, depth=depth, window=2, seed=11).check()
    assert not got[0, 1].any() and not got[1, 1].any() and got[0, 0].any()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T", [6, 20, 40, 140])
def test_masked_rows_may_be_nan(d, T):
    """A drafted token's key and value are NaN, whole or one block: whoever does not see it gets the result without it, to the bit.  And a
    cached row outside the window of some tokens."""
    depth, mask = random_tree(np.random.default_rng(3), T)
    mask[:, 3] = False
    mask[3, 3] = mask[5, 3] = True
    c = Case(4, 2, d, [70], T, mask=mask[None], depth=depth[None], seed=12)
    clean = c.run()
    blind = [t for t in range(T) if not mask[t, 3]]
    c.vs[0, :, 73, 1] = 255                                         # one block of the value: its dimensions alone
    got = c.run()
    assert np.array_equal(got[:, blind], clean[:, blind])
    assert np.isnan(got[0, [3, 5], :, 32:64]).all()
    keep = [i for i in range(d) if not 32 <= i < 64]
    assert np.array_equal(got[..., keep], clean[..., keep])
    c.ks[0, :, 73], c.vs[0, :, 73] = 255, 255
    got = c.run()
    assert np.array_equal(got[:, blind], clean[:, blind]) and np.isnan(got[0, [3, 5]]).all()
    chain = Case(2, 1, d, [50], T, chain=True, window=10, seed=13)
    clean = chain.run()
    chain.ks[0, :, 42], chain.vs[0, :, 42] = 255, 255               # distance of token t: 8 + t
    got = chain.run()
    assert np.array_equal(got[0, 2:], clean[0, 2:]) and np.isnan(got[0, :2]).all()


@pytest.mark.parametrize("T", [2, 30, 140])
@pytest.mark.parametrize("splits", [0, 1, 4])
def test_visible_nan_at_any_weight(T, splits):
    """A cached value block that is NaN shows in its dimensions for everybody, also where the key's weight is nothing."""
    c = Case(2, 1, 128, [600], T, seed=15)
    k, v = (orc.decode4(orc.unpack4(x), s).astype(np.float16) for x, s in ((c.k, c.ks), (c.v, c.vs)))
    c.q[..., 0] = 100
    k[0, 0, 11], k[0, 0, 11, 0] = 0, -6000                           # a score of -53000
    c.hold(k, v)
    c.tree.set_splits(splits)
    clean = c.run()
    c.vs[0, 0, 11, 2] = 255
    got = c.run()
    assert np.isnan(got[..., 64:96]).all()
    keep = [i for i in range(128) if not 64 <= i < 96]
    assert np.array_equal(got[..., keep], clean[..., keep])


@pytest.mark.parametrize("power", [-23, -12, 0, 9, 13])
def test_blocks_of_any_size(power):
    """Scales over all of the format: keys of one size and values of another, blocks of all sizes in a row."""
    rng = np.random.default_rng(1)
    for T in (3, 70):
        c = Case(4, 1, 128, [200], T, seed=16, q_size=1e-3 if power > 5 else 1.0)
        c.vs = np.clip(127 + power + rng.integers(-6, 7, c.vs.shape), 104, 140).astype(np.uint8)
        c.ks = np.clip(127 + min(power, 4) + rng.integers(-6, 7, c.ks.shape), 104, 140).astype(np.uint8)
        c.kv, c.vv = orc.decode4(orc.unpack4(c.k), c.ks), orc.decode4(orc.unpack4(c.v), c.vs)
        c.check()


@pytest.mark.parametrize("q_size", [30.0, 1000.0])
def test_peaked_and_growing_scores(q_size):
    c = Case(4, 1, 64, [257], 3, seed=17, q_size=q_size)
    c.check()
    c.q[:] = np.abs(c.q)
    k = np.abs(c.kv) * np.linspace(0, 1, c.rows)[:, None]
    c.hold(k.astype(np.float16), c.vv.astype(np.float16))
    c.check()


@pytest.mark.parametrize("T", [1, 5, 40, 130])
def test_splits_do_not_matter(T):
    """Any limit on the parts: within the bound, and the same bits again."""
    c = Case(8, 2, 128, [1000, 333], T, seed=18)
    for splits in (1, 2, 3, 7, 64, 0):
        c.tree.set_splits(splits)
        first = c.run()
        c.check(first)
        c.out.fill_(7.0)
        c.call()
        torch.cuda.synchronize()
        assert np.array_equal(first, c.out.cpu().numpy())


@pytest.mark.parametrize("T", [1, 9, 20])
def test_rows_of_very_different_lengths(T):
    lens = [3000, 1, 0, 40, 900, 33, 0, 64, 2000, 31]
    counts = [T, T, T, 0, T, max(T - 2, 0), 1, T, T, T]
    for window in (0, 300):
        c = Case(2, 1, 64, lens, T, counts=counts, window=window, seed=26)
        c.poison_rest()
        first = c.check()
        assert np.array_equal(first, c.run())
        c.tree.set_splits(3)
        c.check()


@pytest.mark.parametrize("nq,nkv,d,L,T,window", [(4, 2, 128, 380, 4, 0), (4, 2, 128, 381, 4, 0), (8, 2, 128, 900, 1, 0), (32, 32, 128, 1100, 16, 0),
                                                 (16, 2, 128, 600, 16, 0), (8, 1, 64, 2500, 9, 0), (1, 1, 64, 70000, 1, 0), (8, 1, 64, 66000, 4, 0),
                                                 (8, 2, 64, 3000, 2, 2900), (8, 2, 64, 3000, 20, 1300), (8, 1, 128, 20000, 33, 0)], ids=str)
def test_every_way_to_divide(nq, nkv, d, L, T, window):
    c = Case(nq, nkv, d, [L], T, window=window, seed=41)
    c.poison_rest()
    first = c.check()
    c.call()                                                        # (the counters of the row blocks are as they were)
    torch.cuda.synchronize()
    assert np.array_equal(first, c.out.cpu().numpy())


@pytest.mark.parametrize("nq,nkv,B,rows,T", [(1, 1, 1, 200, 1), (8, 1, 1, 1000, 40), (4, 2, 3, 400, 17), (64, 8, 1, 5000, 4), (2, 1, 1, 3000, 130)], ids=str)
def test_workspaces_hold_every_division(nq, nkv, B, rows, T):
    """Handles as small as their largest call, at every limit on the parts, with and without forms of the score."""
    for window in (0, rows):
        c = Case(nq, nkv, 64, [rows - T] * B, T, window=window, seed=60, extra=0)
        for splits in (0, 64, 2):
            c.tree.set_splits(splits)
            c.check()


@pytest.mark.parametrize("T", [1, 40])
def test_captured_and_replayed(T):
    """Three replays with eager calls and changed lengths between them: the lengths are read on the device."""
    c = Case(8, 2, 128, [900, 500], T, seed=22, max_len=901)
    eager = c.run()
    s = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        c.call(torch.cuda.current_stream().cuda_stream)
    for replay in range(3):
        c.out.fill_(7.0)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert np.array_equal(c.out.cpu().numpy(), eager), replay
        c.call()
    c.t["lens"].copy_(torch.tensor([321, 0], dtype=torch.int32))
    g.replay()
    torch.cuda.synchronize()
    c.lens = [321, 0]
    c.check(c.out.cpu().numpy())


def test_a_stream_of_its_own():
    c = Case(8, 2, 64, [300], 4, seed=23)
    want = c.run()
    s = torch.cuda.Stream()
    c.out.fill_(7.0)
    s.wait_stream(torch.cuda.current_stream())
    c.call(s.cuda_stream)
    s.synchronize()
    assert np.array_equal(want, c.out.cpu().numpy())


def test_refusals():
    """Each differs from a call that runs in what is refused."""
    import paper_2508_18850_amd as lib
    tree = lib.TreeAttention(4, 2, 64, 2, 100, MXFP4, 10000.0, 8)
    buf = torch.zeros(1 << 17, dtype=torch.uint8, device="cuda")
    p = (buf.data_ptr() + 255) // 256 * 256
    K, V, KS, VS, Q, OUT = (p + 16384 * i for i in range(6))          # rows of 2 x 2 heads x 100 x 64 values: 12800 bytes, scales 800
    call = lambda batch=2, q=Q, out=OUT, k=K, v=V, ks=KS, vs=VS, tokens=8, length=50: tree.attend_rc(  # noqa: E731
        batch, q, lib.cache_pointers(k, v, ks, vs), lib.draft(tokens, length), 0, out, _stream())
    assert call() == 0 and call(batch=1) == 0 and call(length=92) == 0 and call(ks=KS + 4) == 0
    for over in (dict(batch=0), dict(batch=3), dict(q=0), dict(out=0), dict(k=0), dict(v=0), dict(ks=0), dict(vs=0), dict(k=K + 8), dict(ks=KS + 2), dict(vs=VS + 1),
                 dict(tokens=9), dict(tokens=0), dict(length=93), dict(length=-1), dict(out=Q), dict(out=K), dict(out=V + 12800 - 16), dict(out=KS + 784), dict(out=VS)):
        assert call(**over) == -1, over
    assert call(out=KS + 800) == 0
    torch.cuda.synchronize()
    tree.close()


def _stream():
    return torch.cuda.current_stream().cuda_stream
