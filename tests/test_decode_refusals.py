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

    def evict(self, keep=16, cap_out=32, **at):
        """`at` puts an argument at an address; the caches' parts are named k_codes, out_k_codes and so on."""
        for prefix, c in (("out_", self.out), ("", self.cache)):
            for name, _ in c._fields_:
                if prefix + name in at:
                    setattr(c, name, at.pop(prefix + name))
        a = dict(lens=self.buffer(), n_evictable=None, lens_out=self.buffer(), kept=self.buffer())
        a.update(at)
        return binding.lib().str_kv4_evict(ctypes.addressof(self.ctx), ctypes.addressof(self.shape), ctypes.addressof(self.cache), a["lens"], keep, min(4, keep),
                                           a["n_evictable"], cap_out, ctypes.addressof(self.out), a["lens_out"], a["kept"], None, 0, None)


@pytest.mark.parametrize("scale", [float("nan"), float("inf"), float("-inf"), 3.0e38, -3.0e38])
@pytest.mark.parametrize("n_q", [0, 1])
def test_attention_refuses_a_scale_that_is_not_finite(scale, n_q):
    assert Call().attn(scale, n_q) == INVALID


@pytest.mark.parametrize("scale", [0.0, -0.0, 1e-45, -1.0, 2.0e38])
def test_attention_takes_every_finite_scale(scale):
    assert Call().attn(scale) == NO_DEVICE


def test_eviction_refuses_outputs_that_share_memory():
    """Each pair of a buffer that is written and another, overlapping by a little or the same; touching is allowed."""
    c = Call()
    rows, rows_out, words = 2 * 3 * 64, 2 * 3 * 32, 16
    size = dict(k_codes=rows * 64, v_codes=rows * 64, k_scales=rows * words, v_scales=rows * words, weight=rows * 4, pos=2 * 64 * 4, lens=8, n_evictable=8)
    size_out = dict(out_k_codes=rows_out * 64, out_v_codes=rows_out * 64, out_k_scales=rows_out * words, out_v_scales=rows_out * words,
                    out_weight=rows_out * 4, out_pos=2 * 32 * 4, lens_out=8, kept=2 * 16 * 4)
    assert c.evict(n_evictable=c.buffer()) == NO_DEVICE
    for written, n in size_out.items():
        for other, m in list(size.items()) + [kv for kv in size_out.items() if kv[0] != written]:
            step = 4 if min(n, m) < 16 or {written, other} & {"lens", "n_evictable", "lens_out", "kept"} else 16      # caches are 16-byte aligned
            at = c.buffer()
            for gap, want in ((0, INVALID), (m - step, INVALID), (m, NO_DEVICE), (step - n, INVALID), (-n, NO_DEVICE)):
                if (at + gap) % 16 and written.startswith("out_"):
                    continue
                assert Call().evict(**{other: at, written: at + gap}) == want, (written, other, gap)


def test_eviction_of_no_rows_or_without_optional_parts():
    assert Call().evict(keep=0, kept=None) == NO_DEVICE
    assert Call().evict(out_pos=None, out_weight=None) == NO_DEVICE
    assert Call().evict(pos=None, out_pos=None) == NO_DEVICE
    assert Call().evict(pos=None) == INVALID
    assert Call().evict(weight=None) == INVALID
