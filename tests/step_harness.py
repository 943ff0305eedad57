"""What the tests of the calls around attention share: a pool whose pages are read and written as logical images."""
import numpy as np
import torch

from oracle import paged_attention as orc
from paper_2607_23815_b200 import kvattn

NAN_BITS = 0x7FC1


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def bits(x):
    """float64/float32 values as bf16 bit patterns, rounded to nearest even by torch."""
    return torch.tensor(np.asarray(x, np.float64)).to(torch.float32).to(torch.bfloat16).view(torch.int16).numpy().view(np.uint16)


def to_gpu(b):
    return torch.from_numpy(np.ascontiguousarray(b).view(np.int16)).cuda().view(torch.bfloat16)


def from_gpu(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


def randn_bits(rng, *shape):
    return bits(rng.standard_normal(shape))


def _places(d):
    slot, x = np.arange(16)[:, None], np.arange(d)[None, :]
    return ((slot // 8) * (8 * d * 2) + (x // 64) * 1024 + (slot % 8) * 128 + ((((x % 64) // 8) ^ (slot % 8)) * 16) + (x % 8) * 2) // 2


class Pages:
    """A pool of `n` pages over buffers of its own, with an oracle image of the same bits (not numbers, to begin with)."""

    def __init__(self, n, heads, d, fill=NAN_BITS):
        self.n, self.heads, self.d = n, heads, d
        self.host = orc.PagePool(n, 16, heads, d, fill=fill)
        self.k, self.v = (torch.full((n, heads, 16 * d), fill, dtype=torch.int16, device="cuda") for _ in range(2))
        self.pool = kvattn.kv_pool_create_ex(n, 16, heads, d, self.k, self.v)

    def upload(self):
        place = _places(self.d).reshape(-1)
        for buf, image in ((self.k, self.host.k), (self.v, self.host.v)):
            raw = np.empty((self.n, self.heads, 16 * self.d), np.uint16)
            raw[:, :, place] = image.reshape(self.n, self.heads, -1)
            buf.copy_(torch.from_numpy(raw.view(np.int16)))

    def image(self):
        place = _places(self.d).reshape(-1)
        return [b.cpu().numpy().view(np.uint16)[:, :, place].reshape(self.n, self.heads, 16, self.d) for b in (self.k, self.v)]

    def status(self):
        return kvattn.kv_last_async_status(self.pool)


def guarded(shape, dtype, fill):
    """A tensor with a band of `fill` on both sides; check() says whether the bands are as they were."""
    n = int(np.prod(shape))
    whole = torch.full((n + 128,), fill, dtype=dtype, device="cuda")
    t = whole[64:64 + n].view(shape)
    ref = whole.clone()

    def check():
        same = lambda a, b: torch.equal(a.view(torch.uint8), b.view(torch.uint8))
        return same(whole[:64], ref[:64]) and same(whole[64 + n:], ref[64 + n:])
    return t, check
