"""A 4-bit cache on the device with its token-major copy on the host, for the GPU tests."""
import numpy as np
import torch

from oracle import fp4

from gpu_common import kv

T = {"f32": torch.float32, "bf16": torch.bfloat16}


class Cache:
    """Pages of `lengths` tokens with room for `rows` more each, scattered over a pool. Slots that no token fills and
    pages of nobody hold NaN (scale byte 255). sizes: the factors that tokens' values are drawn from."""

    def __init__(self, nq, nkv, d, lengths, rows=None, layers=2, seed=0, spare=3, sizes=(1.0,)):
        rng = np.random.default_rng(seed)
        self.m, self.shape, self.layers, self.lengths = kv(), (nq, nkv, d), layers, list(lengths)
        want = [-(-(n + r) // 16) for n, r in zip(lengths, rows or [0] * len(lengths))]
        self.pages, self.width = sum(want) + spare, max(want + [1]) + 1
        ids = rng.permutation(self.pages)
        self.table = np.full((len(lengths), self.width), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(want):
            self.table[b, :n] = ids[at:at + n]
            at += n
        filled = np.zeros((self.pages, 16), dtype=bool)
        for b, n in enumerate(lengths):
            for p in range(-(-n // 16)):
                filled[self.table[b, p], :min(16, n - 16 * p)] = True
        self.code, self.scale = [], []
        for _ in (0, 1):
            x = rng.normal(size=(layers, self.pages, nkv, 16, d))
            x *= rng.choice(sizes, size=(layers, self.pages, nkv, 16, 1))
            code, scale = fp4.encode(x)
            scale[np.broadcast_to(~filled[None, :, None, :, None], scale.shape)] = 255
            self.code.append(code)
            self.scale.append(scale)
        self.upload()
        self.h = self.m.kvprm_create(self.m.make_desc(layers, 64 * nq, nq, nkv, d, 64, kv_dtype="fp4"))

    def upload(self):
        self.pool = [torch.from_numpy(np.stack([fp4.store(c[l], s[l], part) for l in range(self.layers)])).cuda()
                     for part, (c, s) in enumerate(zip(self.code, self.scale))]
        self.dtab = torch.from_numpy(self.table).cuda()
        self.dlen = torch.tensor(self.lengths, dtype=torch.int32).cuda()
        self.cache = self.m.make_cache(self.pool[0].data_ptr(), self.pool[1].data_ptr(), self.pages)
        self.batch = self.m.make_batch(len(self.lengths), self.dtab.data_ptr(), self.width, self.dlen.data_ptr(),
                                       self.lengths)

    def cached(self, part, layer, b):
        return fp4.cached(self.code[part][layer], self.scale[part][layer], self.table[b], self.lengths[b])

    def check(self):
        """The device's pools are the host's, byte for byte."""
        for part in (0, 1):
            got = self.pool[part].cpu().numpy()
            for l in range(self.layers):
                want = fp4.store(self.code[part][l], self.scale[part][l], part)
                assert np.array_equal(got[l], want), (part, l, np.argwhere(got[l] != want)[:4])

    def __del__(self):
        self.m.kvprm_destroy(self.h)
