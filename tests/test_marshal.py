"""The extension module that marshals the decode calls: what it refuses, and how, without a GPU.  (The calls themselves, their
outputs and the refusals of tensors on a device are tested with the operators.)"""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

from paper_2603_00198_b200 import binding


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


class _Shape:
    def __init__(self):
        self.s = binding.Kv4Shape(2, 32, 2, 64, 32)
        self.c = binding.Kv4CachePtrs()
        self.args = (0, 0, ctypes.addressof(self.s), ctypes.addressof(self.c))


def test_wrong_argument_counts_and_types_are_refused():
    m, sh = binding._marshal(), _Shape()
    for f in (m.append, m.read, m.attn, m.evict, m.step):
        with pytest.raises(TypeError, match="arguments"):
            f(1, 2)
    with pytest.raises(TypeError, match="k: expected a tensor, got list"):
        m.append(*sh.args, [1.0], None, None, None, None)
    with pytest.raises(TypeError, match="q: expected a tensor, got NoneType"):
        m.attn(*sh.args, None, _i32(2), 0.1, None)
    with pytest.raises(TypeError):
        m.read("handle", *sh.args[1:], _i32(2), 1, torch.float32, None)
    with pytest.raises(TypeError, match="dtype"):
        m.read(*sh.args, _i32(2), 1, "float32", None)
    with pytest.raises(TypeError, match="unsupported dtype"):
        m.read(*sh.args, _i32(2), 1, torch.float16, None)
    with pytest.raises(TypeError, match="unsupported dtype"):
        m.attn(*sh.args, torch.zeros(2, 1, 2, 64, dtype=torch.float64), _i32(2), 0.1, None)


def test_sizes_out_of_range_are_refused():
    m, sh = binding._marshal(), _Shape()
    for T in (-1, 1 << 31, 1 << 70):
        with pytest.raises((ValueError, OverflowError)):
            m.read(*sh.args, _i32(2), T, torch.float32, None)
    for keep, recent in ((1 << 31, 0), (0, 1 << 31), (0, -(1 << 40))):
        with pytest.raises(ValueError, match="out of range"):
            m.evict(*sh.args, _i32(2), keep, recent, None, 32, sh.args[3])
    for bad in (torch.zeros(2, 1, 64), torch.zeros(64)):
        with pytest.raises(ValueError, match="dimensions"):
            m.attn(*sh.args, bad, _i32(2), 0.1, None)
        with pytest.raises(ValueError, match="dimensions"):
            m.append(*sh.args, bad, bad, _i32(2), None, None)
        with pytest.raises(ValueError, match="dimensions"):
            m.step(0, 0, bad, bad, bad, bad, bad, bad, None, bad)


def test_host_tensors_are_refused():
    m, sh = binding._marshal(), _Shape()
    q, lens = torch.zeros(2, 1, 2, 64), _i32(2)
    x, B, st = torch.zeros(2, 1, 4, 16), torch.zeros(2, 1, 1, 16), torch.zeros(2, 4, 16, 16)
    for call in (lambda: m.append(*sh.args, q, q, lens, None, None), lambda: m.attn(*sh.args, q, lens, 0.1, None),
                 lambda: m.read(*sh.args, lens, 1, torch.float32, None), lambda: m.evict(*sh.args, lens, 8, 0, None, 32, sh.args[3]),
                 lambda: m.step(0, 0, x, torch.zeros(2, 1, 4), torch.zeros(4), B, B, st, None, st)):
        with pytest.raises(ValueError, match="expected a tensor on cuda:0, got cpu"):
            call()


def test_refused_calls_hold_no_references():
    m, sh = binding._marshal(), _Shape()
    q, lens = torch.zeros(2, 1, 2, 64), _i32(2)
    before = sys.getrefcount(q), sys.getrefcount(lens), sys.getrefcount(binding._check)
    for _ in range(50):
        with pytest.raises(ValueError):
            m.attn(*sh.args, q, lens, 0.1, None)
    assert (sys.getrefcount(q), sys.getrefcount(lens), sys.getrefcount(binding._check)) == before


def test_a_call_before_setup_is_refused():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    code = ("import torch\nfrom paper_2603_00198_b200 import _marshal as m\n"
            "try:\n    m.step(*[0] * 10)\nexcept RuntimeError as e:\n    assert 'setup' in str(e)\n    print('refused')\n"
            "try:\n    m.setup(print, 0, *[0] * 7)\nexcept ValueError:\n    print('refused')\n")
    res = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and res.stdout.split() == ["refused", "refused"], res.stderr[-3000:]


class _Fake:
    """What Kv4Cache looks at in a tensor on a device."""

    def __init__(self, shape, dtype, at):
        self.shape, self.dtype, self.device, self.at = shape, dtype, torch.device("cuda", 0), at

    def dim(self):
        return len(self.shape)

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return self.at


def test_a_cache_asks_for_the_addresses_of_its_tensors_anew(monkeypatch):
    """An attribute that names another tensor than before: the next call gets that one's address."""

    class Module:
        @staticmethod
        def cache(ptrs, shape, device, *tensors):
            assert device == 0
            p = ctypes.cast(ptrs, ctypes.POINTER(binding.Kv4CachePtrs)).contents
            for (name, _), t in zip(binding.Kv4CachePtrs._fields_, tensors):
                setattr(p, name, t.data_ptr() if t is not None else None)

    monkeypatch.setattr(binding, "_MARSHAL", Module)
    codes, words = ((2, 2, 32, 32), torch.uint8), ((2, 2, 32, 2), torch.int32)
    cache = binding.Kv4Cache(_Fake(*codes, 0x100), _Fake(*codes, 0x200), _Fake(*words, 0x300), _Fake(*words, 0x400),
                             _Fake((2, 32), torch.int32, 0x500), _Fake((2, 2, 32), torch.float32, 0x600))

    def names():
        p = ctypes.cast(cache.ptrs_ref, ctypes.POINTER(binding.Kv4CachePtrs)).contents
        return [getattr(p, n) for n, _ in binding.Kv4CachePtrs._fields_]

    assert names() == [0x100, 0x200, 0x300, 0x400, 0x500, 0x600]
    cache.weight, cache.pos = _Fake((2, 2, 32), torch.float32, 0x700), None
    assert names() == [0x100, 0x200, 0x300, 0x400, None, 0x700]
    cache.k_codes.at = 0x800                                 # the tensor itself was given other memory
    assert names() == [0x800, 0x200, 0x300, 0x400, None, 0x700]


def test_the_tensors_of_a_cache_are_checked_at_every_call():
    m, sh = binding._marshal(), _Shape()
    codes, words = torch.zeros(2, 2, 32, 32, dtype=torch.uint8), torch.zeros(2, 2, 32, 2, dtype=torch.int32)
    with pytest.raises(TypeError, match="Kv4Cache.k_codes: expected a tensor, got NoneType"):
        m.cache(sh.args[3], sh.args[2], 0, None, codes, words, words, None, None)
    with pytest.raises(TypeError, match="Kv4Cache.k_codes: expected Byte"):
        m.cache(sh.args[3], sh.args[2], 0, words, codes, words, words, None, None)
    with pytest.raises(ValueError, match="Kv4Cache.k_codes: expected a tensor on cuda:0, got cpu"):
        m.cache(sh.args[3], sh.args[2], 0, codes, codes, words, words, None, None)
    assert sh.c.k_codes is None                              # nothing is stored before all have been checked


def test_a_module_built_for_another_torch_is_refused(monkeypatch):
    m = binding._marshal()
    assert m.built_for == torch.__version__
    monkeypatch.setattr(binding, "_MARSHAL", None)
    monkeypatch.setattr(torch, "__version__", "0.0.0")
    with pytest.raises(ImportError, match="built for torch"):
        binding._marshal()


def test_the_module_is_built_anew_for_another_torch(monkeypatch, tmp_path):
    from paper_2603_00198_b200 import build
    build.build()
    commands = []

    def run(cmd, **kw):
        commands.append(cmd)
        return subprocess.CompletedProcess(cmd, 0, "", "")

    monkeypatch.setattr(build.subprocess, "run", run)
    build._build_marshal(False)
    assert not commands                                      # up to date
    stamp = tmp_path / "marshal.torch"
    stamp.write_text("0.0.0")
    monkeypatch.setattr(build, "BUILT_FOR", str(stamp))
    build._build_marshal(False)
    assert len(commands) == 1 and stamp.read_text() == torch.__version__
    build._build_marshal(False)
    assert len(commands) == 1
    stamp.unlink()
    build._build_marshal(False)
    assert len(commands) == 2


@pytest.mark.gpu
def test_outputs_are_new_tensors_and_threads_may_call_at_once():
    """Four threads, each on its own stream, step their own states: the lock is free during a call, and no two share a buffer."""
    import threading
    ctx = binding.Context(0)
    Bz, H, p, n = 2, 4, 16, 32
    g = torch.Generator().manual_seed(3)
    x, dt, A = torch.randn(Bz, 1, H, p, generator=g).cuda(), torch.rand(Bz, 1, H, generator=g).cuda(), -torch.rand(H, generator=g).cuda()
    B, C = torch.randn(Bz, 1, 1, n, generator=g).cuda(), torch.randn(Bz, 1, 1, n, generator=g).cuda()
    torch.cuda.synchronize()
    res, errors = [None] * 4, []

    def work(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()):
                st = torch.zeros(Bz, H, p, n, device="cuda")
                ys = [binding.str_mamba2_step(ctx, x, dt, A, B, C, st)[0] for _ in range(200)]
                torch.cuda.current_stream().synchronize()
                assert len({y.data_ptr() for y in ys}) == 200
                res[i] = (torch.stack(ys).cpu(), st.cpu())
        except Exception as e:                               # reported by the test's own thread
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join(120)
    assert not errors, errors
    for ys, st in res[1:]:
        assert torch.equal(ys, res[0][0]) and torch.equal(st, res[0][1])
    ctx.check_status()


@pytest.mark.gpu
def test_a_refused_eviction_allocates_nothing_for_its_rows():
    ctx = binding.Context(0)
    cache, out = binding.Kv4Cache.empty(ctx, 2, 32, 2, 64), binding.Kv4Cache.empty(ctx, 2, 16, 2, 64)
    lens = torch.full((2,), 20, dtype=torch.int32, device="cuda")
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    for keep in (-1, 17, 33, (1 << 31) - 1):                 # more than the target, the source, any memory holds
        with pytest.raises(binding.StrError):
            binding.str_kv4_evict(ctx, cache, lens, keep, 0, out)
    assert torch.cuda.max_memory_allocated() - before < 4096


@pytest.mark.gpu
def test_calls_use_the_tensors_that_a_cache_names_now():
    """Attributes given other tensors, and a tensor given other memory, between two calls: nothing goes to where they were."""
    ctx = binding.Context(0)
    g = torch.Generator(device="cuda").manual_seed(4)
    rows = lambda: torch.randn(2, 20, 2, 64, device="cuda", generator=g)  # noqa: E731
    k, v, q = rows(), rows(), torch.randn(2, 1, 4, 64, device="cuda", generator=g)
    start, lens = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.full((2,), 20, dtype=torch.int32, device="cuda")
    cache, same = (binding.Kv4Cache.empty(ctx, 2, 32, 2, 64) for _ in range(2))
    for c in (cache, same):
        binding.str_kv4_append(ctx, c, k, v, start)
        binding.str_kv4_attn(ctx, c, q, lens, 0.125, weight_out=c.weight)
    first = cache.weight
    kept = first.clone()
    cache.weight = cache.weight * 0.5                        # a decay written as one would
    same.weight.mul_(0.5)
    for c in (cache, same):
        binding.str_kv4_attn(ctx, c, q, lens, 0.125, weight_out=c.weight)
    assert torch.equal(cache.weight, same.weight) and torch.equal(first, kept)
    old, at = cache.v_codes, cache.v_codes.data_ptr()
    before = old.clone()
    cache.v_codes = torch.zeros_like(old)
    binding.str_kv4_append(ctx, cache, k, v, start)
    binding.str_kv4_append(ctx, same, k, v, start)
    assert torch.equal(cache.v_codes, same.v_codes) and torch.equal(old, before)
    moved = torch.zeros_like(cache.k_codes)
    cache.k_codes.set_(moved)                                # the same tensor object, other memory
    assert cache.k_codes.data_ptr() == moved.data_ptr() != at
    binding.str_kv4_append(ctx, cache, k, v, start)
    assert torch.equal(moved, same.k_codes)
    out, out_same = (binding.Kv4Cache.empty(ctx, 2, 16, 2, 64) for _ in range(2))
    out.pos, held = None, out.pos
    held.fill_(-3)
    cache.weight, same.weight = (torch.rand(2, 2, 32, device="cuda", generator=g),) * 2
    assert torch.equal(binding.str_kv4_evict(ctx, cache, lens, 9, 2, out)[1], binding.str_kv4_evict(ctx, same, lens, 9, 2, out_same)[1])
    assert (held == -3).all() and torch.equal(out.k_codes, out_same.k_codes)
    for name, bad in (("weight", torch.zeros(2, 2, 16, device="cuda")), ("weight", torch.zeros(2, 2, 32)), ("pos", torch.zeros(2, 32, device="cuda")),
                      ("k_scales", None), ("v_codes", torch.zeros(2, 2, 64, 32, dtype=torch.uint8, device="cuda")[:, :, ::2])):
        good = getattr(cache, name)
        setattr(cache, name, bad)
        with pytest.raises((TypeError, ValueError), match="Kv4Cache." + name):
            binding.str_kv4_append(ctx, cache, k, v, start)
        setattr(cache, name, good)
    cache.weight.resize_(2, 2, 16)
    with pytest.raises(ValueError, match="Kv4Cache.weight"):
        binding.str_kv4_attn(ctx, cache, q, lens, 0.125)
    cache.weight = None
    with pytest.raises(binding.StrError):
        binding.str_kv4_attn(ctx, cache, q, lens, 0.125, weight_out=kept)
    ctx.check_status()
