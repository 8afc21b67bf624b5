"""Pins of the decode-side oracle, and the host-side refusals of the decode entry points (no GPU needed)."""
import ctypes

import numpy as np
import pytest

import oracle
from oracle import decode
from paper_2603_00198_b200 import binding, build

pytestmark = pytest.mark.filterwarnings("ignore::RuntimeWarning")


def test_bf16_rounding_helpers():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal(4000) * 10.0 ** rng.integers(-20, 20, 4000)).astype(np.float32)
    f, r = decode.bf16_floor(x), decode.bf16_round(x)
    assert np.all(f <= x) and np.all((x - f) <= 2.0 ** -7 * np.abs(x))            # at most one step below
    assert np.all(np.abs(r - x) <= 2.0 ** -8 * np.abs(x) * 1.0000001)              # at most half a step away
    assert np.array_equal(decode.bf16_floor(f), f) and np.array_equal(decode.bf16_round(f), f)
    assert np.array_equal(r, oracle.round_to_bf16(x).astype(np.float32))


@pytest.mark.parametrize("d,group", [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)])
def test_quantisation_is_within_half_a_step_and_packing_inverts(d, group):
    rng = np.random.default_rng(d + group)
    x = (rng.standard_normal((50, d)) * 3 + 7 * rng.standard_normal((50, 1))).astype(np.float32)
    code, zero, scale = decode.kv4_quantise(x, group)
    err = np.abs(decode.kv4_values(code, zero, scale, group) - x).reshape(50, -1, group)
    # half a step, plus what the rounded scale takes from the top code: 15 steps x 2^-9, plus fp32's own
    assert np.all(err <= scale[..., None] * (0.5 + 15 * 2.0 ** -9 + 1e-5))
    assert code.min() == 0 and code.max() == 15
    for keys in (True, False):
        assert np.array_equal(decode.kv4_unpack(decode.kv4_pack(code, keys), keys), code)
        assert sorted(decode.kv4_element_nibble(d, keys)) == list(range(d))


def test_quantisation_of_constant_and_unusable_groups():
    x = np.full((4, 64), 1.7, dtype=np.float32)
    x[1, 3], x[2, 40], x[3, :2] = np.nan, np.inf, (3e38, -3e38)
    code, zero, scale = decode.kv4_quantise(x, 32)
    v = decode.kv4_values(code, zero, scale, 32)
    assert np.all(code[0] <= 15) and np.all(np.abs(v[0] - 1.7) <= 1.7 * 2.0 ** -7)
    assert np.isnan(v[1, :32]).all() and not np.isnan(v[1, 32:]).any()
    assert np.isnan(v[2, 32:]).all() and not np.isnan(v[2, :32]).any()
    assert np.isnan(scale[3, 0]) or np.isfinite(v[3, :32]).all()
    ones = np.full((1, 32), np.float32(1.5))                                      # on the bf16 grid: exact, scale 0
    code, zero, scale = decode.kv4_quantise(ones, 32)
    assert scale[0, 0] == 0 and zero[0, 0] == 1.5 and not code.any()


def test_attention_closed_forms():
    rng = np.random.default_rng(3)
    k, v = rng.standard_normal((2, 9, 64)), rng.standard_normal((2, 9, 64))
    o, drawn = decode.kv4_attention(np.zeros((1, 4, 64)), k, v, 0.1)               # zero query: the mean of the values
    assert np.allclose(o[0, 0], v[0].mean(0)) and np.allclose(o[0, 3], v[1].mean(0)) and np.allclose(drawn, 2 / 9)
    q = rng.standard_normal((3, 4, 64))
    o, drawn = decode.kv4_attention(q, k, v, 0.125)
    assert np.allclose(drawn.sum(1), 6)                                            # 3 tokens x 2 heads per key head
    ref = oracle.attention_forward(np.concatenate([np.zeros((6, 4, 64)), q]), np.swapaxes(k, 0, 1), np.swapaxes(v, 0, 1), 0.125)
    assert np.allclose(o, ref[-3:])                                                # the last rows of causal attention
    o, drawn = decode.kv4_attention(rng.standard_normal((5, 2, 64)), k[:, :2], v[:, :2], 1.0)
    assert not o[:3].any() and o[3:].any(-1).all() and np.allclose(drawn.sum(), 2 * 2)


def test_evict_closed_forms():
    w = np.array([[1, 5, 0, 5, 2, 9, 0, 0]], dtype=np.float32)
    assert decode.kv4_evict(w, 6, 3, 0).tolist() == [1, 3, 5]
    assert decode.kv4_evict(w, 6, 2, 1).tolist() == [1, 5]                         # ties: the lower row
    assert decode.kv4_evict(w, 6, 3, 3).tolist() == [3, 4, 5]
    assert decode.kv4_evict(w, 6, 9, 2).tolist() == [0, 1, 2, 3, 4, 5]
    assert decode.kv4_evict(w, 0, 4, 2).tolist() == []
    assert decode.kv4_evict(w, 6, 3, 0, n_evictable=4).tolist() == [1, 4, 5]
    assert decode.kv4_evict(w, 6, 3, 0, n_evictable=1).tolist() == [3, 4, 5]       # more protected than fit: the newest
    w2 = np.array([[1, np.nan, 3], [1, 1, np.inf]], dtype=np.float32)
    assert decode.kv4_evict(w2, 3, 2, 0).tolist() == [0, 2]


def test_step_is_the_recurrence():
    rng = np.random.default_rng(5)
    T, H, p, n, G = 7, 4, 3, 5, 2
    x, B, C = rng.standard_normal((T, H, p)), rng.standard_normal((T, G, n)), rng.standard_normal((T, G, n))
    dt, A, D = rng.uniform(0.001, 0.1, (T, H)), -rng.uniform(1, 16, H), rng.standard_normal(H)
    S0 = rng.standard_normal((H, p, n))
    y, S = decode.mamba2_step(x, dt, A, B, C, S0, D)
    yr, Sr = oracle.mamba2_recurrence(x, dt, A, B, C, D=D, init_state=S0)
    assert np.allclose(y, yr, rtol=1e-10) and np.allclose(S, Sr, rtol=1e-10)


# ---------------------------------------------------------------- refusals on the host
@pytest.fixture(scope="module")
def libstr():
    build.build()
    return binding.lib()


def _cache_ptrs(**kw):
    base = dict(k_codes=4096, v_codes=8192, k_scales=16384, v_scales=32768, pos=65536, weight=131072)
    base.update(kw)
    return binding.Kv4CachePtrs(*(base[k] for k, _ in binding.Kv4CachePtrs._fields_))


class _FakeCtx(ctypes.Structure):
    """Enough zeroed memory to stand for a context in calls that must be refused before they touch it."""
    _fields_ = [("bytes", ctypes.c_char * 4096)]


OK = dict(Bz=1, cap=64, Hkv=2, d=128, group=32)
BAD_SHAPES = [(dict(Bz=0), -1), (dict(cap=0), -1), (dict(Hkv=-1), -1), (dict(d=0), -1), (dict(group=0), -1), (dict(d=96), -2), (dict(d=256), -2),
              (dict(group=16), -2), (dict(d=64, group=128), -2), (dict(cap=60), -2), (dict(Bz=70000), -2)]


def _addr(s):
    return ctypes.addressof(s)


@pytest.mark.parametrize("change,code", BAD_SHAPES)
def test_cache_shapes_are_refused(libstr, change, code):
    ctx, s, c, c2 = _FakeCtx(), binding.Kv4Shape(**{**OK, **change}), _cache_ptrs(), _cache_ptrs(k_codes=1 << 20, v_codes=1 << 21, k_scales=1 << 22,
                                                                                            v_scales=1 << 23, pos=1 << 24, weight=1 << 25)
    a, p = _addr, 1 << 26
    assert libstr.str_kv4_append(a(ctx), a(s), 1, 1, p, p, None, p, None, a(c), None) == code
    assert libstr.str_kv4_read(a(ctx), a(s), 1, 1, p, None, a(c), p, p, None) == code
    assert libstr.str_kv4_attn(a(ctx), a(s), 1, 4, 1, p, a(c), p, 0.1, p, None, p, 1 << 40, None) == code
    assert libstr.str_kv4_evict(a(ctx), a(s), a(c), p, 16, 0, None, 16, a(c2), p + 64, p, p, 1 << 40, None) == code
    assert libstr.str_kv4_attn_workspace_size(a(s), 4, 1, 1) == 0 and libstr.str_kv4_evict_workspace_size(a(s), 16) == 0


def test_cache_arguments_are_refused(libstr):
    ctx, s, c, a, p = _FakeCtx(), binding.Kv4Shape(**OK), _cache_ptrs(), _addr, 1 << 26
    c2 = _cache_ptrs(k_codes=1 << 20, v_codes=1 << 21, k_scales=1 << 22, v_scales=1 << 23, pos=1 << 24, weight=1 << 25)
    assert libstr.str_kv4_append(None, a(s), 1, 1, p, p, None, p, None, a(c), None) == -1
    assert libstr.str_kv4_append(a(ctx), None, 1, 1, p, p, None, p, None, a(c), None) == -1
    assert libstr.str_kv4_append(a(ctx), a(s), 7, 1, p, p, None, p, None, a(c), None) == -1                 # dtype
    assert libstr.str_kv4_append(a(ctx), a(s), 1, -1, p, p, None, p, None, a(c), None) == -1
    assert libstr.str_kv4_append(a(ctx), a(s), 1, 1, None, p, None, p, None, a(c), None) == -1
    assert libstr.str_kv4_append(a(ctx), a(s), 1, 1, p + 8, p, None, p, None, a(c), None) == -1             # alignment
    assert libstr.str_kv4_append(a(ctx), a(s), 1, 1, p, p, None, None, None, a(c), None) == -1
    assert libstr.str_kv4_append(a(ctx), a(s), 1, 1, p, p, None, p, None, ctypes.byref(_cache_ptrs(v_scales=None)), None) == -1
    assert libstr.str_kv4_append(a(ctx), a(s), 1, 1, p, p, None, p, None, ctypes.byref(_cache_ptrs(k_codes=4100)), None) == -1
    assert libstr.str_kv4_append(a(ctx), a(s), 1, 0, None, None, None, None, None, a(c), None) == 0          # no tokens: nothing to do
    assert libstr.str_kv4_read(a(ctx), a(s), 1, 0, None, None, a(c), None, None, None) == 0
    assert libstr.str_kv4_read(a(ctx), a(s), 1, 4, p, None, a(c), None, p, None) == -1
    big = 1 << 40
    assert libstr.str_kv4_attn(a(ctx), a(s), 1, 3, 1, p, a(c), p, 0.1, p, None, p, big, None) == -1          # 3 heads over 2
    assert libstr.str_kv4_attn(a(ctx), a(s), 1, 0, 1, p, a(c), p, 0.1, p, None, p, big, None) == -1
    assert libstr.str_kv4_attn(a(ctx), a(s), 1, 4, -1, p, a(c), p, 0.1, p, None, p, big, None) == -1
    assert libstr.str_kv4_attn(a(ctx), a(s), 1, 4, 1, p, a(c), None, 0.1, p, None, p, big, None) == -1
    assert libstr.str_kv4_attn(a(ctx), a(s), 1, 4, 1, p, ctypes.byref(_cache_ptrs(weight=None)), p, 0.1, p, p, p, big, None) == -1
    assert libstr.str_kv4_attn(a(ctx), a(s), 1, 4, 0, None, a(c), p, 0.1, None, None, None, 0, None) == 0
    need = libstr.str_kv4_attn_workspace_size(a(s), 4, 1, 1)
    assert need > 0
    assert libstr.str_kv4_attn(a(ctx), a(s), 1, 4, 1, p, a(c), p, 0.1, p, p, p, need - 1, None) == -3
    assert libstr.str_kv4_attn(a(ctx), a(s), 1, 4, 1, p, a(c), p, 0.1, p, p, None, need, None) == -1
    ev = lambda cache=c, out=c2, keep=16, recent=0, cap_out=16, lens=p, lens_out=p + 64, kept=p, ws=p, nb=big: libstr.str_kv4_evict(  # noqa: E731
        a(ctx), a(s), a(cache), lens, keep, recent, None, cap_out, a(out), lens_out, kept, ws, nb, None)
    assert ev(keep=65, cap_out=80) == -1 and ev(keep=17) == -1 and ev(recent=17) == -1 and ev(keep=-1) == -1 and ev(recent=-1) == -1
    assert ev(cap_out=20) == -2 and ev(kept=None) == -1 and ev(lens_out=p) == -1
    assert ev(cache=_cache_ptrs(weight=131076)) == -1                                                       # alignment
    assert libstr.str_kv4_evict_workspace_size(a(s), 16) == 0
    s.cap = 200000                                                                                          # a row over many CTAs: needs a workspace
    far = _cache_ptrs(**{k: 1 << (36 + i) for i, (k, _) in enumerate(binding.Kv4CachePtrs._fields_)})
    ev2 = lambda ws=p, nb=big, cache=c: ev(cache=cache, out=far, ws=ws, nb=nb)  # noqa: E731
    need = libstr.str_kv4_evict_workspace_size(a(s), 16)
    assert need >= 200000 * 4 and ev2(nb=need - 1) == -3 and ev2(ws=None) == -1 and ev2(ws=p + 128) == -1
    assert ev2(cache=_cache_ptrs(v_codes=far.v_codes + 1024), nb=need - 1) == -1                             # buffers that overlap in part
    s.cap = 64
    assert ev(cache=_cache_ptrs(weight=None)) == -1 and ev(cache=_cache_ptrs(pos=None)) == -1
    for shared in ("k_codes", "v_codes", "k_scales", "v_scales", "pos", "weight"):
        assert ev(cache=_cache_ptrs(**{shared: getattr(c2, shared)})) == -1


def test_step_arguments_are_refused(libstr):
    ctx, a, p = _FakeCtx(), _addr, 1 << 26
    ok = dict(Bz=1, T=1, H=4, p=8, n=16, G=2, Q=0, dtype=1)
    call = lambda args=(p,) * 5, D=None, state=p, y=p, out=p, **kw: libstr.str_mamba2_step(  # noqa: E731
        a(ctx), ctypes.byref(binding.SsdShape(**{**ok, **kw})), *args, D, state, y, out, None)
    assert libstr.str_mamba2_step(None, ctypes.byref(binding.SsdShape(**ok)), p, p, p, p, p, None, p, p, p, None) == -1
    for kw in (dict(Bz=0), dict(T=0), dict(T=-2), dict(H=3), dict(p=0), dict(n=0), dict(G=0), dict(dtype=5)):
        assert call(**kw) == -1, kw
    assert call(state=None) == -1 and call(y=None) == -1 and call(out=None) == -1
    for i in range(5):
        assert call(args=tuple(None if j == i else p for j in range(5))) == -1
    assert call(n=513) == -2 and call(H=65536, G=1) == -2
