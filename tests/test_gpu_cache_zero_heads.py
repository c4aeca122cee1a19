"""cf_cache_append_normed with heads of zeros, infinities and NaN and eps 0, into caches of every format, against oracle/quantized_step.py.

A head of zeros has no norm then and becomes NaN; so does all of its row in a cache that holds codes.  Heads beside it keep their values.  Nothing
has a tolerance (what a value within some 2^-45 of a border does, test_gpu_cache4.py says); an fp16 cache is compared by values, since the bits of a NaN
are not given.  So are 4 bits of a key with an infinity: its finite values become zeros, and the formula does not give their signs.  (x / sqrt(inf) is a zero of
x's sign, and the rotation then a difference of two zeros, +0 unless the first is -0 and the second +0; taken the other way round, x c - y s times
1 / sqrt(inf), it is a zero with the sign of the difference.  Both are 0.)"""
import numpy as np
import pytest

from oracle import draft_block as base
from oracle import quantized_step as orc
from quant_cases import FORMATS, Buffers

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [6, 2050], ids=["a token to a workgroup", "four tokens to a workgroup"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("fmt", FORMATS)
def test_heads_of_zeros_without_eps(fmt, d, tokens):
    import paper_2508_18850_amd as lib
    print("append: %s x %d tokens %d" % (fmt, d, tokens), flush=True)
    nq, nkv, at = 4, 2, 5
    rng = np.random.default_rng(d + tokens)
    qkv = rng.standard_normal((tokens, nq + 2 * nkv, d)).astype(np.float16)
    weight = (1 + 0.3 * rng.standard_normal((2, d))).astype(np.float16)
    qkv[1, 0], qkv[2, nq], qkv[3, nq + 1], qkv[tokens - 1, nq + 1] = 0, 0, -0.0, 0      # a query, keys
    qkv[4, nq, 9], qkv[4, nq + 1, 1], qkv[4, 2, 7] = np.inf, np.nan, -np.inf
    with np.errstate(invalid="ignore"):
        x = np.concatenate([orc.head_norm(qkv[:, :nq], weight[0], 0.0), orc.head_norm(qkv[:, nq:nq + nkv], weight[1], 0.0)], 1)
        turned = np.stack([base.rotate(x[t], at + t, 10000.0) for t in range(tokens)]).astype(np.float16)
    assert np.isnan(turned[1, 0]).all() and np.isnan(turned[2, nq]).all() and np.isnan(turned[tokens - 1, nq + 1]).all() and not np.isnan(turned[2, nq + 1]).any()
    buf = Buffers(1, nkv, at + tokens + 2, d, fmt)
    with np.errstate(invalid="ignore"):
        buf.put("k", 0, at, turned[:, nq:].transpose(1, 0, 2))
    buf.put("v", 0, at, qkv[:, nq + nkv:].transpose(1, 0, 2))
    q = torch.full((tokens, nq, d), 7.0, dtype=torch.float16, device="cuda")
    dev = [torch.from_numpy(np.ascontiguousarray(a)).cuda() for a in (qkv, weight[0], weight[1])]
    lib.KvCache(nq, nkv, d, 1, at + tokens + 2, FORMATS[fmt], 10000.0).append_normed(
        1, dev[0].data_ptr(), dev[1].data_ptr(), dev[2].data_ptr(), 0.0, buf.pointers(), lib.draft(tokens, at), q.data_ptr(), torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert np.array_equal(q.cpu().numpy(), turned[:, :nq], equal_nan=True)
    if fmt == "f16":
        for n in ("k", "v"):
            got, want = (np.ascontiguousarray(a).view(np.float16) for a in (buf.dev[n].cpu().numpy(), buf.host[n]))
            assert np.array_equal(got, want, equal_nan=True), n
        return
    if fmt == "mxfp4":
        row = (0, slice(None), at + 4)
        codes, scales = (buf.dev[n].cpu().numpy()[row] for n in ("k", "k_scale"))
        assert np.array_equal(orc.decode4(orc.unpack4(codes), scales), orc.decode4(orc.unpack4(buf.host["k"][row]), buf.host["k_scale"][row]), equal_nan=True)
        buf.host["k"][row] = codes
    buf.same()
