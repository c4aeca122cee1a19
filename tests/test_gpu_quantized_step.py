"""The operators of a quantised step together, as a program runs them: hidden states to codes, projection, norms and rotation into a 4-bit cache,
attention of a drafted tree, the result to codes, output projection, accepted rows kept, and the next tree."""
import numpy as np
import pytest

from draft_cases import bound, mask_words, random_tree
from oracle import draft_block as base
from oracle import quantized_step as orc
from quant_cases import MXFP4, store

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _dev(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _half(shape):
    return torch.zeros(shape, dtype=torch.float16, device="cuda")


class Quantized:
    """Rows on the GPU and, by the oracle, on the host."""

    def __init__(self, x):
        import paper_2508_18850_amd as lib
        rows, n = x.shape
        self.codes, self.scale = torch.zeros((rows, n), dtype=torch.int8, device="cuda"), torch.zeros(rows, device="cuda")
        lib.quantize_rows(rows, n, x.data_ptr(), self.codes.data_ptr(), self.scale.data_ptr(), torch.cuda.current_stream().cuda_stream)
        code, scale = base.encode(x.cpu().numpy(), "int8")
        assert np.array_equal(self.codes.cpu().numpy(), code.astype(np.int8)) and np.array_equal(self.scale.cpu().numpy(), scale)


def _product(linear, x, w, out):
    """Checked to the bit: the inputs are the GPU's own."""
    linear.forward(out.shape[0], x.codes.data_ptr(), x.scale.data_ptr(), w.codes.data_ptr(), w.scale.data_ptr(), out.data_ptr(),
                   torch.cuda.current_stream().cuda_stream)
    want = orc.int8_product(*(t.cpu().numpy() for t in (x.codes, x.scale, w.codes, w.scale)))[1]
    assert np.array_equal(out.cpu().numpy(), want)


@pytest.mark.parametrize("d,T,window", [(64, 11, 0), (128, 20, 0), (64, 9, 40)], ids=str)
def test_prompt_drafts_and_kept_rows(d, T, window):
    import paper_2508_18850_amd as lib
    B, nq, nkv, prompt, steps, D = 2, 4, 2, 37, 3, 512
    rng = np.random.default_rng(d + T)
    rows, width = prompt + 64, (nq + 2 * nkv) * d
    s = torch.cuda.current_stream().cuda_stream
    w_qkv, w_o = (Quantized(_dev((rng.standard_normal(shape) / np.sqrt(shape[1])).astype(np.float16))) for shape in ((width, D), (D, nq * d)))
    project, out_project = lib.Int8Linear(D, width, B * prompt), lib.Int8Linear(nq * d, D, B * T)
    weight = (1 + 0.2 * rng.standard_normal((2, d))).astype(np.float16)
    wd, eps = _dev(weight), 1e-6
    t = {n: torch.zeros((B, nkv, rows, d // 2), dtype=torch.uint8, device="cuda") for n in ("k", "v")}
    sc = {n: torch.zeros((B, nkv, rows, d // 32), dtype=torch.uint8, device="cuda") for n in ("k", "v")}
    cache = lib.cache_pointers(t["k"].data_ptr(), t["v"].data_ptr(), sc["k"].data_ptr(), sc["v"].data_ptr())
    kv = lib.KvCache(nq, nkv, d, B, rows, MXFP4, 10000.0)
    tree = lib.TreeAttention(nq, nkv, d, B, rows, MXFP4, 10000.0, T, window=window)
    host = {n: np.zeros((B, nkv, rows, d)) for n in ("k", "v")}
    lens = torch.zeros(B, dtype=torch.int32, device="cuda")

    def append(n, counts, depth, now):
        x = Quantized(_dev(rng.standard_normal((B * n, D)).astype(np.float16)))
        qkv, q = _half((B * n, width)), _half((B, n, nq, d))
        _product(project, x, w_qkv, qkv)
        cd, dd = _dev(np.array(counts, np.int32)), _dev(depth.astype(np.int32))
        dr = lib.draft(n, rows - n, row_len=lens.data_ptr(), row_tokens=cd.data_ptr(), depth=dd.data_ptr(), per_row=True)
        kv.append_normed(B, qkv.data_ptr(), wd[0].data_ptr(), wd[1].data_ptr(), eps, cache, dr, q.data_ptr(), s)
        heads = qkv.cpu().numpy().reshape(B, n, nq + 2 * nkv, d)
        for b in range(B):
            for i in range(counts[b]):
                normed = np.concatenate([orc.head_norm(heads[b, i, :nq], weight[0], eps), orc.head_norm(heads[b, i, nq:nq + nkv], weight[1], eps)])
                turned = base.rotate(normed, now[b] + depth[b, i], 10000.0).astype(np.float16)
                assert np.array_equal(q[b, i].cpu().numpy(), turned[:nq])
                host["k"][b, :, now[b] + i], host["v"][b, :, now[b] + i] = store(turned[nq:], "mxfp4")[2], store(heads[b, i, nq + nkv:], "mxfp4")[2]
        return q

    now = [prompt, prompt - 9]
    append(prompt, now, np.tile(np.arange(prompt), (B, 1)), [0, 0])
    lens.copy_(_dev(np.array(now, np.int32)))
    for step in range(steps):
        trees = [random_tree(rng, T) for _ in range(B)]
        depth, mask, counts = np.stack([x[0] for x in trees]), np.stack([x[1] for x in trees]), [T, T - 3]
        q = append(T, counts, depth, now)
        md, dd, cd = _dev(mask_words(mask).view(np.int64)), _dev(depth), _dev(np.array(counts, np.int32))
        out = _half((B, T, nq, d))
        dr = lib.draft(T, rows - T, row_len=lens.data_ptr(), row_tokens=cd.data_ptr(), depth=dd.data_ptr(), tree=md.data_ptr(), per_row=True)
        tree.attend(B, q.data_ptr(), cache, dr, 0, out.data_ptr(), s)
        want, size, reach, flat = base.attend(q.cpu().numpy(), host["k"], host["v"], now, counts, depth, mask, window=window)
        tol = bound(want, size, reach, flat, d, rows)
        got = out.cpu().numpy().astype(np.float64)
        for b in range(B):
            assert (np.abs(got[b, :counts[b]] - want[b, :counts[b]]) <= tol[b, :counts[b]]).all(), (step, b)
            assert not got[b, counts[b]:].any()
        _product(out_project, Quantized(out.reshape(B * T, nq * d)), w_o, _half((B * T, D)))
        kept, n_kept = np.zeros((B, T), np.int32), []
        for b in range(B):                                      # a deepest path
            leaf = int(np.argmax(depth[b, :counts[b]]))
            path = np.nonzero(mask[b, leaf, :leaf + 1])[0]
            kept[b, :len(path)] = path
            n_kept.append(len(path))
            for n in ("k", "v"):
                host[n][b, :, now[b]:now[b] + len(path)] = host[n][b][:, now[b] + path]
        kd, nd, new = _dev(kept), _dev(np.array(n_kept, np.int32)), torch.zeros(B, dtype=torch.int32, device="cuda")
        kv.keep(B, cache, dr, kd.data_ptr(), nd.data_ptr(), new.data_ptr(), s)
        lens.copy_(new)
        now = [a + b for a, b in zip(now, n_kept)]
        torch.cuda.synchronize()
        assert lens.tolist() == now
    n = min(now)
    back = {k: _half((B, nkv, n, d)) for k in ("k", "v")}
    kv.read(B, cache, 0, n, back["k"].data_ptr(), back["v"].data_ptr(), s)
    torch.cuda.synchronize()
    for k in ("k", "v"):
        assert np.array_equal(back[k].cpu().numpy().astype(np.float64), host[k][:, :, :n])
