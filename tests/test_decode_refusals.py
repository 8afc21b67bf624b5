"""What the decode entry points refuse on the host, before anything touches CUDA: called through the C ABI with addresses that nothing
may follow.  Only where there is no device: a call that is not refused then ends with STR_ERR_CUDA."""
import ctypes

import pytest
import torch

from paper_2603_00198_b200 import binding

pytestmark = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real")
INVALID, NO_DEVICE = -1, -4


class Call:
    """One call's arguments; every buffer its own stretch of addresses, far from the others."""

    def __init__(self):
        self.ctx = ctypes.create_string_buffer(4096)
        self.shape = binding.Kv4Shape(2, 64, 3, 128, 32)
        self.next = 1 << 20
        self.cache, self.out = self.caches(), self.caches()

    def buffer(self):
        self.next += 1 << 28
        return self.next

    def caches(self):
        return binding.Kv4CachePtrs(*(self.buffer() for _ in range(6)))

    def attn(self, scale=0.1, n_q=1):
        return binding.lib().str_kv4_attn(ctypes.addressof(self.ctx), ctypes.addressof(self.shape), 1, 12, n_q, self.buffer(), ctypes.addressof(self.cache),
                                          self.buffer(), scale, self.buffer(), self.buffer(), self.buffer(), 1 << 27, None)


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf"), 3.0e38, -3.0e38])
@pytest.mark.parametrize("n_q", [0, 1])
def test_attention_refuses_a_scale_that_is_not_finite(scale, n_q):
    assert Call().attn(scale, n_q) == INVALID


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45, -1.0, 2.0e38])
def test_attention_takes_every_finite_scale(scale):
    assert Call().attn(scale) == NO_DEVICE
