"""A refused rotary append reports nothing on the device, and neither does one row with strides that only a next row would need."""
import ctypes as C

import pytest
import torch

from paper_2607_23815_b200 import kvattn
from step_harness import Pages, i32

pytestmark = pytest.mark.gpu


def test_the_status_stays_clear():
    pages, lib = Pages(3, 2, 64), kvattn.lib()
    t, zeros = torch.zeros(4096, dtype=torch.bfloat16, device="cuda"), i32([0] * 64)
    p, z = (lambda off=0: C.c_void_p(t.data_ptr() + off)), C.c_void_p(zeros.data_ptr())
    good = dict(pool=pages.pool.handle, q=p(), qs=256, k=p(), ks=128, v=p(), vs=128, hq=4, slots=z, pos=z, axes=1, inv=z, axis=None, rot=64, nb=0, total=2,
                out=p(4096), os=256)
    call = lambda **kw: lib.kv_append_rotary(*{**good, **kw}.values(), None)
    for kw in (dict(out=None), dict(qs=255), dict(ks=120), dict(q=p(2)), dict(rot=24), dict(axes=2), dict(slots=None)):
        assert call(**kw) in (kvattn.KV_ERR_INVALID, kvattn.KV_ERR_UNSUPPORTED)
    assert call(total=1, qs=3, ks=0, vs=1, os=5) == 0                           # (one row has no next one)
    torch.cuda.synchronize()
    assert pages.status() == 0
