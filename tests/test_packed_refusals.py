"""What the entry points on packed sequences refuse on the host, before anything touches CUDA: through the C ABI with addresses that nothing may
follow, and through the module that marshals them with host tensors."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2603_00198_b200 import binding

INVALID, UNSUPPORTED, NO_DEVICE = -1, -2, -4
no_device = pytest.mark.skipif(torch.cuda.is_available(), reason="the addresses are not real")


class Call:
    def __init__(self):
        self.ctx = ctypes.create_string_buffer(4096)
        self.next = 1 << 20

    def buffer(self):
        self.next += 1 << 34
        return self.next

    def _args(self, names, given):
        a = {n: self.buffer() for n in names}
        a.update({n: given.pop(n) for n in list(given) if n in a})
        assert not given, given
        return a

    def conv(self, step=False, dtype=1, n_seq=3, rows=50, H=4, p=16, n=8, G=2, W=4, ctx=True, **at):
        a = self._args(("zx", "w", "b", "bias", "start", "window", "x", "B", "C", "dt", "wout"), at)
        f = binding.lib().str_mamba_conv_step if step else binding.lib().str_mamba_conv_packed
        ptrs = [a[k] for k in ("zx", "w", "b", "bias")] + ([] if step else [a["start"]]) + [a[k] for k in ("window", "x", "B", "C", "dt", "wout")]
        return f(ctypes.addressof(self.ctx) if ctx else None, dtype, n_seq, rows, H, p, n, G, W, *ptrs, None)

    def scan(self, n_seq=3, rows=50, H=4, p=16, n=8, G=2, dtype=1, **at):
        a = self._args(("x", "dt", "A", "B", "C", "D", "start", "init", "y", "final"), at)
        s = binding.SsdPackedShape(n_seq, rows, H, p, n, G, dtype)
        return binding.lib().str_mamba2_prefill_packed(ctypes.addressof(self.ctx), ctypes.addressof(s), *(a[k] for k in ("x", "dt", "A", "B", "C", "D", "start", "init", "y", "final")),
                                                       None, 0, None)

    def attn(self, n_seq=3, rows_q=50, rows_k=50, Hq=4, Hkv=2, d=64, dtype=1, scale=0.1, **at):
        a = self._args(("q", "k", "v", "qs", "ks", "o"), at)
        s = binding.AttnPackedShape(n_seq, rows_q, rows_k, Hq, Hkv, d, dtype)
        need = binding.lib().str_attn_prefill_packed_workspace_size(ctypes.addressof(s))
        return binding.lib().str_attn_prefill_packed(ctypes.addressof(self.ctx), ctypes.addressof(s), *(a[k] for k in ("q", "k", "v", "qs", "ks")), scale, a["o"],
                                                     self.buffer() if need else None, need, None)

    def rope(self, rows=9, Hq=4, Hkv=2, d=64, dtype=1, at=None, **desc):
        a = self._args(("pos", "qkv", "q", "k", "v"), dict(at or {}))
        r = dict(rot_dim=32, layout=0, scaling=0, trained_len=100, theta=1e4, factor=2.0, turns_low=1.0, turns_high=32.0, amplitude=1.0)
        r.update(desc)
        s = binding.RopeDesc(**r)
        return binding.lib().str_rope_split_ex(ctypes.addressof(self.ctx), ctypes.addressof(s), dtype, rows, Hq, Hkv, d, *(a[k] for k in ("pos", "qkv", "q", "k", "v")), None)


@no_device
@pytest.mark.parametrize("step", [False, True])
def test_convolution(step):
    assert Call().conv(step) == NO_DEVICE
    for bad in (dict(n_seq=0), dict(rows=-1), dict(H=0), dict(p=0), dict(n=0), dict(G=0), dict(G=3), dict(W=0), dict(dtype=2), dict(ctx=False), dict(w=None), dict(b=None),
                dict(bias=None), dict(zx=None), dict(x=None), dict(B=None), dict(C=None), dict(dt=None)):
        assert Call().conv(step, **bad) == INVALID, bad
    for bad in (dict(W=1), dict(W=5)):
        assert Call().conv(step, **bad) == UNSUPPORTED, bad
    size = 3 * 3 * 96 * 2                                   # bytes of the windows
    assert Call().conv(step, window=1 << 40, wout=(1 << 40) + size - 2) == INVALID
    assert Call().conv(step, window=1 << 40, wout=(1 << 40) + size) == NO_DEVICE
    assert Call().conv(step, window=1 << 40, wout=1 << 40) == (NO_DEVICE if step else INVALID)
    if step:
        assert Call().conv(step, window=None) == INVALID and Call().conv(step, wout=None) == INVALID and Call().conv(step, rows=0) == INVALID
        assert Call().conv(step, n_seq=1, rows=1 << 28, H=8) == UNSUPPORTED and Call().conv(step, n_seq=1, rows=1 << 28) == NO_DEVICE
    else:
        assert Call().conv(window=None) == NO_DEVICE and Call().conv(wout=None) == NO_DEVICE and Call().conv(start=None) == INVALID
        assert Call().conv(rows=0, zx=None, x=None, B=None, C=None, dt=None) == NO_DEVICE
        assert Call().conv(n_seq=65536) == UNSUPPORTED and Call().conv(rows=(1 << 30) + 1) == UNSUPPORTED


@no_device
def test_scan():
    assert Call().scan() == NO_DEVICE
    for bad in (dict(n_seq=0), dict(rows=-1), dict(H=0), dict(p=0), dict(n=0), dict(G=0), dict(G=3), dict(dtype=3), dict(x=None), dict(dt=None), dict(A=None), dict(B=None),
                dict(C=None), dict(start=None), dict(y=None)):
        assert Call().scan(**bad) == INVALID, bad
    for bad in (dict(n=257), dict(n_seq=65536), dict(rows=(1 << 30) + 1)):
        assert Call().scan(**bad) == UNSUPPORTED, bad
    for free in (dict(D=None), dict(init=None), dict(final=None), dict(rows=0, x=None, dt=None, B=None, C=None, y=None)):
        assert Call().scan(**free) == NO_DEVICE, free
    at, size = 1 << 40, 3 * 4 * 16 * 8 * 4
    assert Call().scan(init=at, final=at) == NO_DEVICE and Call().scan(init=at, final=at + 4) == INVALID and Call().scan(init=at, final=at + size) == NO_DEVICE
    for name in ("x", "B", "C"):
        assert Call().scan(**{name: at, "y": at}) == INVALID, name


@no_device
def test_scan_workspace():
    """Long sequences of few heads ask for one; too small, missing, misaligned or shared with another tensor it is refused."""
    names = ("x", "dt", "A", "B", "C", "D", "start", "init", "y", "final")

    def call(ws, given, **at):
        c = Call()
        s = binding.SsdPackedShape(1, 2000, 4, 64, 128, 2, 1)
        need = binding.lib().str_mamba2_prefill_packed_workspace_size(ctypes.addressof(s))
        assert need > 0
        return binding.lib().str_mamba2_prefill_packed(ctypes.addressof(c.ctx), ctypes.addressof(s), *(at.get(n) or c.buffer() for n in names), ws, need + given, None)

    at = 1 << 44
    assert call(at, 0) == NO_DEVICE and call(at, -1) == -3 and call(None, 0) == INVALID and call(at + 128, 0) == INVALID
    for name in ("x", "dt", "B", "C", "init", "y", "final"):
        assert call(at, 0, **{name: at + 256}) == INVALID, name
    for shape in ((1, 1000, 4, 64, 128, 2, 1), (1, 24576, 128, 64, 128, 8, 1), (1, 100, 4, 64, 128, 2, 0), (200, 20000, 4, 64, 128, 2, 1), (1, 0, 4, 64, 128, 2, 1), (0, 2000, 4, 64, 128, 2, 1),
                  (1, 2000, 4, 64, 257, 2, 1)):
        s = binding.SsdPackedShape(*shape)
        assert binding.lib().str_mamba2_prefill_packed_workspace_size(ctypes.addressof(s)) == 0, shape
    assert binding.lib().str_mamba2_prefill_packed_workspace_size(None) == 0


@no_device
def test_attention():
    assert Call().attn() == NO_DEVICE
    for bad in (dict(n_seq=0), dict(rows_q=-1), dict(rows_k=-1), dict(Hq=0), dict(Hkv=0), dict(Hq=3), dict(d=0), dict(dtype=2), dict(q=None), dict(k=None), dict(v=None),
                dict(o=None), dict(qs=None), dict(ks=None, rows_k=49)):
        assert Call().attn(**bad) == INVALID, bad
    for scale in (0.0, -1.0, float("nan"), float("inf"), 3.0e38):
        assert Call().attn(scale=scale) == INVALID, scale
    for bad in (dict(d=129), dict(Hq=129, Hkv=1), dict(n_seq=32769), dict(rows_q=(1 << 30) + 1), dict(rows_k=(1 << 30) + 1)):
        assert Call().attn(**bad) == UNSUPPORTED, bad
    assert Call().attn(ks=None) == NO_DEVICE and Call().attn(rows_k=0, k=None, v=None) == NO_DEVICE
    assert Call().attn(rows_q=0) == 0
    at = 1 << 40
    for name in ("q", "k", "v"):
        assert Call().attn(**{name: at, "o": at}) == INVALID, name


@no_device
def test_attention_workspace():
    """Few queries over many keys ask for one; too small, missing, misaligned or shared with the output or an input it is refused."""
    def call(ws, given, o=1 << 45, **at):
        c = Call()
        s = binding.AttnPackedShape(1, 10, 5000, 4, 2, 64, 1)
        need = binding.lib().str_attn_prefill_packed_workspace_size(ctypes.addressof(s))
        assert need > 0
        return binding.lib().str_attn_prefill_packed(ctypes.addressof(c.ctx), ctypes.addressof(s), *(at.get(n) or c.buffer() for n in ("q", "k", "v", "qs", "ks")), 0.1, o, ws, need + given, None)

    at = 1 << 44
    assert call(at, 0) == NO_DEVICE and call(at, -1) == -3 and call(None, 0) == INVALID and call(at + 128, 0) == INVALID and call(1 << 45, 0) == INVALID
    for name in ("q", "k", "v"):
        assert call(at, 0, **{name: at + 256}) == INVALID, name
    for shape in ((1, 10, 5000, 4, 2, 64, 0), (1, 5000, 5000, 4, 2, 64, 1), (1, 10, 900, 4, 2, 64, 1), (1, 10, 5000, 4, 2, 63, 1), (0, 10, 5000, 4, 2, 64, 1), (1, 0, 0, 4, 2, 64, 1)):
        s = binding.AttnPackedShape(*shape)
        assert binding.lib().str_attn_prefill_packed_workspace_size(ctypes.addressof(s)) == 0, shape
    assert binding.lib().str_attn_prefill_packed_workspace_size(None) == 0


@no_device
def test_rotary():
    assert Call().rope() == NO_DEVICE
    for bad in (dict(rot_dim=0), dict(rot_dim=33), dict(rot_dim=66), dict(layout=2), dict(scaling=3), dict(theta=0.0), dict(theta=float("nan")), dict(amplitude=float("inf")),
                dict(scaling=1, factor=0.0), dict(scaling=2, factor=-1.0), dict(scaling=2, trained_len=0), dict(scaling=2, turns_low=32.0), dict(scaling=2, turns_high=float("nan")),
                dict(rows=-1), dict(Hq=0), dict(Hkv=0), dict(d=0), dict(dtype=2), dict(at=dict(pos=None)), dict(at=dict(qkv=None)), dict(at=dict(v=None)),
                dict(at=dict(qkv=1 << 40, q=1 << 40)), dict(at=dict(qkv=1 << 40, v=(1 << 40) + 64))):
        assert Call().rope(**bad) == INVALID, bad
    assert Call().rope(d=300, rot_dim=258) == UNSUPPORTED and Call().rope(d=65, layout=1) == UNSUPPORTED and Call().rope(d=65) == NO_DEVICE
    assert Call().rope(rows=0, at=dict(pos=None, qkv=None, q=None, k=None, v=None)) == 0


def test_the_description_of_a_rotary_embedding_is_checked():
    with pytest.raises(ValueError, match="layout"):
        binding.Rope(1e4, 64, "quarters")
    with pytest.raises(ValueError, match="scaling"):
        binding.Rope(1e4, 64, scaling="square")


def test_tensors_are_checked():
    m, i32 = binding._marshal(), lambda *s: torch.zeros(s, dtype=torch.int32)
    for f, n in ((m.rope, 8), (m.conv_packed, 17), (m.conv_step, 14), (m.scan_packed, 12), (m.attn_packed, 9)):
        with pytest.raises(TypeError, match="arguments"):
            f(1, 2)
    q, w = torch.zeros(5, 2, 64), torch.zeros(2 * 16 + 2 * 8, 4)
    r = binding.Rope(1e4, 64)
    with pytest.raises(ValueError, match="expected a tensor on cuda:0, got cpu"):
        m.attn_packed(0, 0, q, q, q, i32(2), None, 0.1, None)
    with pytest.raises(ValueError, match="q_start: expected n_seq"):
        m.attn_packed(0, 0, q, q, q, i32(1), None, 0.1, None)
    with pytest.raises(ValueError, match="q: expected 3 dimensions"):
        m.attn_packed(0, 0, q[0], q, q, i32(2), None, 0.1, None)
    with pytest.raises(TypeError, match="unsupported dtype"):
        m.attn_packed(0, 0, q.half(), q, q, i32(2), None, 0.1, None)
    with pytest.raises(ValueError, match="expected a tensor on cuda:0, got cpu"):
        m.rope(0, 0, r.desc_ref, torch.zeros(3, 4 * 64), i32(3), 2, 1, 64)
    with pytest.raises(ValueError, match="Hq: 0 is out of range"):
        m.rope(0, 0, r.desc_ref, torch.zeros(3, 4 * 64), i32(3), 0, 1, 64)
    zx = torch.zeros(6, 2 * 32 + 2 * 8 + 2)
    with pytest.raises(ValueError, match="expected a tensor on cuda:0, got cpu"):
        m.conv_packed(0, 0, zx, w, w[:, 0], w[:2, 0], 2, 16, 8, 1, i32(2), None, None, None, None, None, None)
    with pytest.raises(ValueError, match="expected a tensor on cuda:0, got cpu"):
        m.conv_step(0, 0, zx, w, w[:, 0], w[:2, 0], 2, 16, 8, 1, zx, 2, 3, zx)
    with pytest.raises(ValueError, match="expected a tensor on cuda:0, got cpu"):
        m.scan_packed(0, 0, q, q, q, q, q, i32(2), None, None, None, None)


def test_a_call_before_setup_is_refused():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = ("import torch\nfrom paper_2603_00198_b200 import _marshal as m\n"
            "for f in (lambda: m.rope(*[0] * 8), lambda: m.setup_packed(*[0] * 7)):\n"
            "    try:\n        f()\n    except RuntimeError as e:\n        assert 'setup' in str(e)\n        print('refused')\n"
            "m.setup(print, 0, *[1] * 7)\n"
            "try:\n    m.setup_packed(*[0] * 7)\nexcept ValueError:\n    print('refused')\n")
    res = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.split() == ["refused"] * 3, res.stderr[-3000:]


@no_device
@pytest.mark.parametrize("step", [False, True])
def test_convolution_whose_outputs_share_memory_with_its_inputs(step):
    """Rows that one block writes are another's history: every input against every output, whole and by the last element."""
    at, rows = 1 << 40, 150 if step else 50
    ch, cols = 4 * 16 + 2 * 2 * 8, 2 * 4 * 16 + 2 * 2 * 8 + 4
    inputs = dict(zx=rows * cols * 2, window=3 * 3 * ch * 2, w=ch * 4 * 4, b=ch * 4, bias=4 * 4)
    if not step:
        inputs["start"] = 4 * 4
    for i, size in inputs.items():
        for o in ("x", "B", "C", "dt", "wout"):
            in_place = step and (i, o) == ("window", "wout")
            assert Call().conv(step, **{i: at, o: at}) == (NO_DEVICE if in_place else INVALID), (i, o)
            assert Call().conv(step, **{i: at, o: at + size - 2}) == INVALID, (i, o)
            assert Call().conv(step, **{i: at, o: at + size}) == NO_DEVICE, (i, o)


@no_device
def test_scan_whose_outputs_share_memory():
    """y and the final state against every input and against each other, whole and by the last element."""
    at = 1 << 40
    x, B, state, head = 50 * 4 * 16 * 2, 50 * 2 * 8 * 2, 3 * 4 * 16 * 8 * 4, 4 * 4
    inputs = dict(x=x, dt=50 * 4 * 4, A=head, B=B, C=B, D=head, start=4 * 4, init=state)
    for o in ("y", "final"):
        for i, size in (*inputs.items(), *((("y", x),) if o == "final" else ())):
            same = (i, o) == ("init", "final")
            assert Call().scan(**{i: at, o: at}) == (NO_DEVICE if same else INVALID), (i, o)
            assert Call().scan(**{i: at, o: at + size - 2}) == INVALID and Call().scan(**{i: at, o: at + size}) == NO_DEVICE, (i, o)


@no_device
def test_rotary_descriptions_beyond_what_an_angle_or_an_output_holds():
    """An amplitude that fp32 has not, and frequencies whose quarter turns a 64-bit number does not count any more."""
    for bad in (dict(amplitude=1e39), dict(amplitude=-1e300), dict(theta=1e-300), dict(scaling=1, factor=1e-200), dict(scaling=1, factor=1e-8), dict(scaling=2, factor=5e-324)):
        assert Call().rope(**bad) == INVALID, bad
    for good in (dict(amplitude=-3e38), dict(theta=1e300), dict(theta=1e-6), dict(scaling=1, factor=1e-6), dict(scaling=2, factor=1e300)):
        assert Call().rope(**good) == NO_DEVICE, good


@no_device
def test_rotary_outputs_share_no_memory():
    at, q, k = 1 << 40, 9 * 4 * 64 * 2, 9 * 2 * 64 * 2
    for i, size in (("qkv", 9 * 8 * 64 * 2), ("pos", 9 * 4), ("q", q), ("k", k), ("v", k)):
        for o in ("q", "k", "v"):
            if i != o:
                assert Call().rope(at={i: at, o: at}) == INVALID and Call().rope(at={i: at, o: at + size - 2}) == INVALID, (i, o)
                assert Call().rope(at={i: at, o: at + size}) == NO_DEVICE, (i, o)


@no_device
def test_attention_starts_that_share_memory_with_what_is_written():
    at = 1 << 40
    for name in ("qs", "ks"):
        assert Call().attn(**{name: at, "o": at}) == INVALID and Call().attn(**{name: at, "o": at + 12}) == INVALID and Call().attn(**{name: at, "o": at + 16}) == NO_DEVICE, name
    c, s = Call(), binding.AttnPackedShape(1, 10, 5000, 4, 2, 64, 1)
    need = binding.lib().str_attn_prefill_packed_workspace_size(ctypes.addressof(s))
    for n in (3, 4):                                       # the starts' places among the arguments, in the workspace's last 256 bytes and behind it
        for shift, want in ((-256, INVALID), (0, NO_DEVICE)):
            p = [c.buffer() for _ in range(5)]
            p[n] = at + need + shift
            assert binding.lib().str_attn_prefill_packed(ctypes.addressof(c.ctx), ctypes.addressof(s), *p, 0.1, c.buffer(), at, need, None) == want, (n, shift)
