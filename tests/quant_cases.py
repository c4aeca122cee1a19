"""What the tests of the 4-bit cache, of the append with norms and of the integer products share."""
import numpy as np

from oracle import draft_block as base
from oracle import quantized_step as orc
from draft_cases import code_bytes

MXFP4 = 4
FORMATS = {"f16": 0, "e4m3": 1, "int8": 2, "mxfp4": MXFP4}
FILL = 0x5a


def row_bytes(fmt, d):
    return {"f16": 2 * d, "mxfp4": d // 2}.get(fmt, d)


def store(rows, fmt):
    """fp16 rows [..., d] -> (bytes [..., row bytes], scales or None, the fp64 values that they stand for)."""
    if fmt == "f16":
        return np.ascontiguousarray(rows).view(np.uint8), None, rows.astype(np.float64)
    if fmt == "mxfp4":
        code, scale = orc.encode4(rows)
        return orc.pack4(code), scale, orc.decode4(code, scale)
    code, scale = base.encode(rows, fmt)
    return code_bytes(code, fmt), scale, code * scale.astype(np.float64)[..., None]


class Buffers:
    """A cache on the GPU, filled with a pattern, and its copy on the host."""

    def __init__(self, B, nkv, rows, d, fmt):
        self.fmt = fmt
        self.host = {n: np.full((B, nkv, rows, row_bytes(fmt, d)), FILL, np.uint8) for n in ("k", "v")}
        scale = np.full((B, nkv, rows, d // 32), FILL, np.uint8) if fmt == "mxfp4" else np.full((B, nkv, rows), 1234.5, np.float32)
        self.host.update({n: scale.copy() for n in ("k_scale", "v_scale")})
        self.upload()

    def upload(self):
        import torch
        self.dev = {n: torch.from_numpy(x).cuda() for n, x in self.host.items()}

    def pointers(self):
        import paper_2508_18850_amd as lib
        return lib.cache_pointers(*(self.dev[n].data_ptr() for n in ("k", "v", "k_scale", "v_scale")))

    def put(self, name, b, first, rows):
        """fp16 rows [heads, n, d] into the host copy, in the cache's format."""
        raw, scale, _ = store(rows, self.fmt)
        self.host[name][b, :, first:first + rows.shape[1]] = raw
        if scale is not None:
            self.host[name + "_scale"][b, :, first:first + rows.shape[1]] = scale

    def same(self):
        for n, x in self.host.items():
            got = self.dev[n].cpu().numpy()
            assert np.array_equal(got, x, equal_nan=x.dtype == np.float32), (n, np.argwhere(got != x)[:4])
