"""Whole numbers beyond an int are an error of the binding and not cut to their lower 32 bits (no GPU needed)."""
import pytest
import torch

from paper_2607_23815_b200 import kvattn


class _NoPool:
    ptr = None


def _mixed(n):
    kvattn.attn_mixed(_NoPool, n, 1.0, None, None, None, 0)


def _host(n):
    t, i = torch.zeros(2, 4, 64, dtype=torch.bfloat16), torch.zeros(2, 8, dtype=torch.int32)
    kvattn.attn_extend_host(_NoPool, t, t, t, i[0], i, i[0], i[0], 1, n, 1.0, torch.zeros_like(t), torch.zeros(2, 4), None, 0)


@pytest.mark.parametrize("call", [_mixed, _host])
def test_integers_that_no_int_holds(call):
    for n in (2 ** 31, 2 ** 32 + 64, -2 ** 31 - 1, 2 ** 63 - 1, -2 ** 63, 2 ** 64 + 8, 2 ** 100):
        with pytest.raises(OverflowError):
            call(n)
    for n in (8, 2 ** 31 - 1, -2 ** 31):
        with pytest.raises(kvattn.KvError):                                    # no pool: refused by the library itself
            call(n)
    with pytest.raises(TypeError):
        call("8")
