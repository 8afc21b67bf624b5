"""GPU parity of the decode-side operators (4-bit cache: append, read, attention, eviction; Mamba-2 step) against the plain
fp64 oracle, at the sizes, masks and values where they can go wrong.

Tolerances are bounds worked out from the data of each case.  Attention: with e = 2^-24 (half a step of fp32), a score
s = scale * sum_j q_j k_j formed in fp32 is off by at most ds = (d + 64) e * scale * sum_j |q_j| |k_j| (d sequential
additions, and the roundings of the factors, of the group terms and of the exponent's scaling); a softmax weight
p = exp(s - m) / sum is then off by at most 2 ds + 32 e + n e relative (numerator and denominator, the exponential's
2^-22, and the sum of n terms), and o = sum p v by that times max |v|, plus the rounding of the factor p * scale of the
matrix product: 2^-11 of 15 scale for bf16 storage (one fp16 factor, half a step), 2^-22 of it for fp32 storage (two),
plus the storage type's own half step (bf16 2^-8, fp32 2^-24) of |o|.
"""
import numpy as np
import pytest
import torch

import oracle
from oracle import decode
from paper_2603_00198_b200 import binding, inputs
from util_gpu import dev

pytestmark = [pytest.mark.gpu, pytest.mark.filterwarnings("ignore::RuntimeWarning")]
E = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": E}
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
SHAPES = [(64, 32), (64, 64), (128, 32), (128, 64), (128, 128)]


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.check_status()
    c.close()


def _i32(a):
    return dev(np.asarray(a, dtype=np.int32))


def _rows(g, shape, dtype, keys):
    x = g.standard_normal(shape)
    if keys:
        x = x + np.where(g.random(shape[-1]) < 0.1, 6.0, 0.0) * g.standard_normal(shape[-1])
    return inputs.to_grid(x, dtype)


class Filled:
    """A cache filled from host data, with the logical content kept on the host.  Rows of a sequence from lens[b] on hold
    rubbish: codes of all ones, NaN scales and zeros, weights of 1e30."""

    def __init__(self, g, lens, cap, Hkv, d, group, k=None, v=None):
        Bz = len(lens)
        self.lens, self.cap, self.Hkv, self.d, self.group = lens, cap, Hkv, d, group
        k = _rows(g, (Bz, Hkv, cap, d), "f32", True) if k is None else k
        v = _rows(g, (Bz, Hkv, cap, d), "f32", False) if v is None else v
        parts = []
        self.k = self.v = None
        for x, keys in ((k, True), (v, False)):
            code, zero, scale = decode.kv4_quantise(x, group)
            vals = decode.kv4_values(code, zero, scale, group)
            packed, words = decode.kv4_pack(code, keys), decode.kv4_words(zero, scale)
            for b, n in enumerate(lens):
                packed[b, :, n:], words[b, :, n:] = 0xFF, 0xFFFFFFFF
            parts.append((packed, words.view(np.int32)))
            if keys:
                self.k, self.k_scale = vals, scale
            else:
                self.v, self.v_scale = vals, scale
        self.weight = np.abs(g.standard_normal((Bz, Hkv, cap))).astype(np.float32)
        self.pos = np.cumsum(g.integers(1, 4, (Bz, cap)), axis=1).astype(np.int32)
        for b, n in enumerate(lens):
            self.weight[b, :, n:] = 1e30
        self.cache = binding.Kv4Cache(dev(parts[0][0]), dev(parts[1][0]), dev(parts[0][1]), dev(parts[1][1]), dev(self.pos), dev(self.weight))


# ---------------------------------------------------------------- rows in and out
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("Bz,T,Hkv,cap", [(1, 1, 1, 16), (3, 7, 5, 48), (2, 33, 8, 64), (1, 257, 2, 272)])
def test_append_stores_the_definition_and_read_returns_it(ctx, dtype, d, group, Bz, T, Hkv, cap):
    g = np.random.default_rng([d, group, Bz, T])
    k, v = _rows(g, (Bz, T, Hkv, d), dtype, True), _rows(g, (Bz, T, Hkv, d), dtype, False)
    k[0, 0, 0, :group] = 1.5                                        # a constant group: scale 0
    start = g.integers(0, cap - T + 1, Bz)
    n_new = g.integers(0, T + 1, Bz)
    n_new[0] = T
    pos = g.integers(0, 1 << 30, (Bz, T)).astype(np.int32)
    cache = binding.Kv4Cache.empty(ctx, Bz, cap, Hkv, d, group)
    for t in (cache.k_codes, cache.v_codes):
        t.fill_(0xA5)
    for t in (cache.k_scales, cache.v_scales, cache.pos):
        t.fill_(-7)
    cache.weight.fill_(3.0)
    want = {n: getattr(cache, n).cpu().numpy().copy() for n in ("k_codes", "v_codes", "k_scales", "v_scales", "pos", "weight")}
    binding.str_kv4_append(ctx, cache, dev(k, dtype), dev(v, dtype), _i32(start), positions=dev(pos), n_new=_i32(n_new))
    vals = {}
    for name, x, keys in (("k", k, True), ("v", v, False)):
        code, zero, scale = decode.kv4_quantise(np.swapaxes(x, 1, 2), group)           # [Bz, Hkv, T, d]
        vals[name] = np.swapaxes(decode.kv4_values(code, zero, scale, group), 1, 2)
        for b in range(Bz):
            at = slice(start[b], start[b] + n_new[b])
            want[name + "_codes"][b, :, at] = decode.kv4_pack(code, keys)[b, :, :n_new[b]]
            want[name + "_scales"][b, :, at] = decode.kv4_words(zero, scale).view(np.int32)[b, :, :n_new[b]]
    for b in range(Bz):
        want["pos"][b, start[b]:start[b] + n_new[b]] = pos[b, :n_new[b]]
        want["weight"][b, :, start[b]:start[b] + n_new[b]] = 0.0
    for n, w in want.items():                                       # bit for bit, and nothing beside the new rows
        assert np.array_equal(getattr(cache, n).cpu().numpy(), w), n
    kr, vr = binding.str_kv4_read(ctx, cache, _i32(start), T, TORCH[dtype], n_rows=_i32(n_new))
    for name, r in (("k", kr), ("v", vr)):
        r = r.float().cpu().numpy()
        for b in range(Bz):
            ref = vals[name][b, :n_new[b]]
            assert np.all(np.abs(r[b, :n_new[b]] - ref) <= (HALF[dtype] + 2 * E) * np.abs(ref))
            assert not r[b, n_new[b]:].any()
    ctx.check_status()


def test_append_values_that_are_not_finite_poison_their_group_only(ctx):
    x = np.ones((1, 3, 1, 64), dtype=np.float32) * np.linspace(-1, 1, 64, dtype=np.float32)
    x[0, 0, 0, 5], x[0, 1, 0, 40], x[0, 2, 0, 1] = np.nan, np.inf, -np.inf
    cache = binding.Kv4Cache.empty(ctx, 1, 16, 1, 64, 32)
    binding.str_kv4_append(ctx, cache, dev(x), dev(x[:, ::-1].copy()), _i32([0]))
    k, v = (t.cpu().numpy()[0, :, 0] for t in binding.str_kv4_read(ctx, cache, _i32([0]), 3, torch.float32))
    for r, order in ((k, (0, 1, 2)), (v, (2, 1, 0))):
        bad = np.isnan(r[list(order)]).reshape(3, 2, 32)
        assert bad.all(-1).tolist() == [[True, False], [False, True], [True, False]] and bad.sum() == 96
    big = np.full((1, 1, 1, 64), 3e38, dtype=np.float32)            # finite, but its range is not
    big[..., ::2] *= -1
    binding.str_kv4_append(ctx, cache, dev(big), dev(big), _i32([4]))
    want = decode.kv4_words(*decode.kv4_quantise(big[:, 0], 32)[1:]).view(np.int32)
    assert np.array_equal(cache.k_scales[0, :, 4].cpu().numpy(), want[0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,group", SHAPES)
def test_append_a_non_finite_element_anywhere_poisons_its_group_only(ctx, dtype, d, group):
    """Row t has one NaN, inf or -inf at element t (values: at element d - 1 - t): every lane and piece in turn."""
    g = np.random.default_rng([7, d, group])
    k, v = _rows(g, (1, d, 2, d), dtype, True), _rows(g, (1, d, 2, d), dtype, False)
    words = []
    for x, at in ((k, np.arange(d)), (v, np.arange(d)[::-1])):
        x[0, np.arange(d), 1, at] = np.where(np.arange(d) % 3 == 0, np.nan, np.where(np.arange(d) % 3 == 1, np.inf, -np.inf))
        clean = np.where(np.isfinite(x), x, 0.0)
        code, zero, scale = decode.kv4_quantise(np.swapaxes(clean, 1, 2), group)
        w = decode.kv4_words(zero, scale).view(np.int32)[0]                           # [Hkv, d, d / group]
        w[1, np.arange(d), at // group] = 0x7FFF0000
        words.append(w)
    cache = binding.Kv4Cache.empty(ctx, 1, d, 2, d, group)
    binding.str_kv4_append(ctx, cache, dev(k, dtype), dev(v, dtype), _i32([0]))
    assert np.array_equal(cache.k_scales[0].cpu().numpy(), words[0])
    assert np.array_equal(cache.v_scales[0].cpu().numpy(), words[1])
    ctx.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_at_sixteen_byte_addresses(ctx, dtype):
    """The alignment that the interface asks for and no more: inputs and outputs 16 bytes behind a 256-byte boundary."""
    g = np.random.default_rng(11)
    T, Hkv, d = 19, 3, 64
    off = 16 // (2 if dtype == "bf16" else 4)
    k, v = (dev(_rows(g, (1, T, Hkv, d), dtype, keys), dtype) for keys in (True, False))
    shift = lambda t: torch.cat([torch.zeros(off, dtype=t.dtype, device="cuda"), t.flatten()])[off:].view(t.shape)
    ks, vs = shift(k), shift(v)
    assert ks.data_ptr() % 32 == 16 and vs.data_ptr() % 32 == 16
    caches = [binding.Kv4Cache.empty(ctx, 1, 32, Hkv, d) for _ in range(2)]
    start = _i32([5])
    binding.str_kv4_append(ctx, caches[0], k, v, start)
    binding.str_kv4_append(ctx, caches[1], ks, vs, start)
    for n in ("k_codes", "v_codes", "k_scales", "v_scales"):
        assert torch.equal(getattr(caches[0], n), getattr(caches[1], n)), n
    want = binding.str_kv4_read(ctx, caches[0], start, T, TORCH[dtype])
    buf = [torch.full((k.numel() + 2 * off,), 7.0, dtype=TORCH[dtype], device="cuda") for _ in range(2)]
    rc = binding.lib().str_kv4_read(ctx.handle, caches[0].shape_ref, binding._dt(k), T, start.data_ptr(), None, caches[0].ptrs_ref,
                                    buf[0][off:].data_ptr(), buf[1][off:].data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    for b, w in zip(buf, want):
        assert torch.equal(b[off:off + k.numel()].view(k.shape), w) and (b[:off] == 7.0).all() and (b[off + k.numel():] == 7.0).all()
    ctx.check_status()


def test_append_and_read_outside_the_capacity_are_skipped_and_reported(ctx):
    cache = binding.Kv4Cache.empty(ctx, 2, 16, 1, 64, 32)
    x = dev(np.ones((2, 4, 1, 64), dtype=np.float32))
    binding.str_kv4_append(ctx, cache, x, x, _i32([14, -2]))
    with pytest.raises(binding.StrError) as e:
        ctx.check_status()
    assert e.value.code == -1
    ctx.check_status()                                              # reported once
    used = (cache.k_scales[:, 0, :, 0] != 0).cpu().numpy()
    assert np.flatnonzero(used[0]).tolist() == [14, 15] and np.flatnonzero(used[1]).tolist() == [0, 1]
    k, _ = binding.str_kv4_read(ctx, cache, _i32([14, -2]), 4, torch.float32)
    with pytest.raises(binding.StrError):
        ctx.check_status()
    assert np.array_equal(k[:, :, 0, 0].cpu().numpy(), [[1, 1, 0, 0], [0, 0, 1, 1]])


@pytest.mark.parametrize("counts", [[5, 2], [2, -1], [-(1 << 31), (1 << 31) - 1]])
def test_counts_of_append_and_read_outside_their_range_are_held_to_it_and_reported(ctx, counts):
    cache = binding.Kv4Cache.empty(ctx, 2, 32, 3, 64, 32)
    x = dev(np.ones((2, 4, 3, 64), dtype=np.float32))
    held = [min(max(n, 0), 4) for n in counts]
    binding.str_kv4_append(ctx, cache, x, x, _i32([3, 8]), n_new=_i32(counts))
    with pytest.raises(binding.StrError) as e:
        ctx.check_status()
    assert e.value.code == -1
    used = (cache.k_scales[:, :, :, 0] != 0).cpu().numpy()
    for b, start in enumerate((3, 8)):
        assert all(np.flatnonzero(used[b, h]).tolist() == list(range(start, start + held[b])) for h in range(3))
    binding.str_kv4_append(ctx, cache, x, x, _i32([3, 8]), n_new=_i32([4, 0]))
    binding.str_kv4_append(ctx, cache, x, x, _i32([3, 8]))
    ctx.check_status()                                              # 0 and T_new are inside
    k, _ = binding.str_kv4_read(ctx, cache, _i32([3, 8]), 4, torch.float32, n_rows=_i32(counts))
    with pytest.raises(binding.StrError):
        ctx.check_status()
    assert np.array_equal((k[:, :, 1, 0] == 1).sum(1).cpu().numpy(), held) and np.array_equal((k != 0).sum((1, 2, 3)).cpu().numpy(), [64 * 3 * n for n in held])
    binding.str_kv4_read(ctx, cache, _i32([3, 8]), 4, torch.float32, n_rows=_i32([4, 0]))
    ctx.check_status()


# ---------------------------------------------------------------- attention
def _attention_reference(f, q, scale):
    """(o, drawn, bound of o without the output rounding, bound of drawn) per sequence."""
    out = []
    n_q, Hq, d = q.shape[1:]
    R = Hq // f.Hkv
    for b, n in enumerate(f.lens):
        k, v = f.k[b, :, :n], f.v[b, :, :n]
        o, drawn = decode.kv4_attention(q[b], k, v, scale)
        ds = np.zeros(f.Hkv)
        for h in range(f.Hkv):
            if n:
                ds[h] = (d + 64) * E * abs(scale) * (np.abs(k[h]) @ np.abs(q[b].reshape(n_q, f.Hkv, R, d)[:, h].reshape(-1, d).T.astype(np.float64))).max()
        rel = 2 * ds + (32 + n) * E                                 # of every softmax weight
        vmax = np.abs(v).max((1, 2)) if n else np.zeros(f.Hkv)
        smax = f.v_scale[b, :, :n].max((1, 2)) if n else np.zeros(f.Hkv)
        out.append((o, drawn, np.repeat(rel * vmax, R), np.repeat(15.0 * smax, R), rel[:, None] * drawn))
    return out


def check_attention(ctx, f, q, dtype, scale, weights, got=None, got_w=None):
    if got is None:
        w_out = torch.full(f.weight.shape, -5.0, device="cuda") if weights else None
        got = binding.str_kv4_attn(ctx, f.cache, dev(q, dtype), _i32(f.lens), scale, weight_out=w_out)
        ctx.check_status()
        got_w = w_out.cpu().numpy() if weights else None
    got = got.float().cpu().numpy()
    factor = 2.0 ** -11 if dtype == "bf16" else 2.0 ** -22
    for b, (o, drawn, tol, vscale, wtol) in enumerate(_attention_reference(f, q, scale)):
        n = f.lens[b]
        bound = (tol + factor * vscale)[None, :, None] + HALF[dtype] * np.abs(o)
        assert np.all(np.abs(got[b] - o) <= bound), (b, n, float((np.abs(got[b] - o) / np.maximum(bound, 1e-300)).max()))
        if weights:
            ref = f.weight[b, :, :n] + drawn
            assert np.all(np.abs(got_w[b, :, :n] - ref) <= wtol + 2 * E * ref), (b, n)
            assert np.all(got_w[b, :, n:] == -5.0)                  # rows behind the sequence are left as they were


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("Hq,Hkv,n_q", [(1, 1, 1), (8, 2, 1), (6, 2, 5), (21, 7, 2), (16, 1, 3)])
def test_attention_over_ragged_lengths(ctx, dtype, d, group, Hq, Hkv, n_q):
    g = np.random.default_rng([d, group, Hq, n_q])
    lens = [0, 1, 2, 15, 16, 17, 31, 33, 64, 127, 129, 255, 300, 304]
    f = Filled(g, lens, 304, Hkv, d, group)
    q = inputs.to_grid(g.standard_normal((len(lens), n_q, Hq, d)), dtype)
    check_attention(ctx, f, q, dtype, d ** -0.5, True)
    check_attention(ctx, f, q, dtype, d ** -0.5, False)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Bz,n,Hq,Hkv,d,group,n_q", [(1, 4999, 32, 8, 128, 32, 1), (2, 3001, 8, 2, 64, 64, 8), (1, 9000, 4, 1, 128, 64, 16),
                                                     (5, 1500, 12, 3, 128, 128, 1), (1, 2100, 40, 1, 128, 32, 1)])
def test_attention_over_long_rows(ctx, dtype, Bz, n, Hq, Hkv, d, group, n_q):
    g = np.random.default_rng([n, Hq, d])
    lens = [max(0, n - 700 * b - b) for b in range(Bz)]
    f = Filled(g, lens, (n + 15) // 16 * 16 + 32, Hkv, d, group)
    q = inputs.to_grid(g.standard_normal((Bz, n_q, Hq, d)), dtype)
    check_attention(ctx, f, q, dtype, d ** -0.5, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kq,vq", [(1.0, 1.0), (40.0, 1.0), (1e-12, 1e-20), (1e12, 1e-12), (1e-15, 1e18), (3e4, 3e30)])
def test_attention_of_large_and_small_values(ctx, dtype, kq, vq):
    """Queries of size kq against keys of size 1 / kq (or, at 40, scores of hundreds: one row takes all), values of size vq."""
    g = np.random.default_rng(int(abs(np.log2(kq * vq)) * 10) + 1)
    d, lens, Hkv, Hq = 128, [700, 33], 2, 8
    size = 1.0 if kq == 40.0 else 1.0 / kq
    k = _rows(g, (2, Hkv, 704, d), "f32", True) * np.float32(size)
    v = (_rows(g, (2, Hkv, 704, d), "f32", False) * np.exp2(g.integers(-6, 7, (2, Hkv, 704, 1)))).astype(np.float32) * np.float32(vq)
    f = Filled(g, lens, 704, Hkv, d, 32, k=k, v=v)
    q = inputs.to_grid(g.standard_normal((2, 1, Hq, d)) * np.float32(kq), dtype)
    check_attention(ctx, f, q, dtype, d ** -0.5, True)


def test_attention_scale_may_be_negative_or_zero(ctx):
    g = np.random.default_rng(9)
    f = Filled(g, [100, 7], 112, 2, 64, 32)
    q = inputs.to_grid(g.standard_normal((2, 2, 4, 64)), "bf16")
    check_attention(ctx, f, q, "bf16", -0.3, True)
    check_attention(ctx, f, q, "bf16", 0.0, True)
    check_attention(ctx, f, np.zeros_like(q), "bf16", 1.0, True)
    check_attention(ctx, f, np.zeros_like(q), "bf16", 0.0, True)
    check_attention(ctx, f, q, "f32", 1e-30, False)
    check_attention(ctx, f, (q * np.float32(1e-25)), "f32", 1e-20, True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scale", [0.41, 0.47, 0.53, -0.93])
@pytest.mark.parametrize("top", [1e6, 1.8e7, 2.6e7, 4.5e7, 1e8])
def test_attention_of_scores_whose_neighbours_lie_far_apart(ctx, dtype, scale, top):
    """Rows 0-15 of a sequence share a score of about `top` (log2 units), rows 16-31 one that is a few units higher.

    A raw score S = 32 (z0 + z1) is formed exactly (groups of equal elements, scale 0; q all ones), its product with the scale is
    rounded once: off by at most half a step, 2^-24 of it, and the scale's own product with log2(e) moves a difference D by 2^-23 D.
    The weight of the second rows, 1 / (1 + 2^-D), then lies between those of D -+ both scores' half steps, and the output between
    the two means of the values."""
    d, cap, Bz = 64, 32, 96
    g = np.random.default_rng([int(top), int(100 * abs(scale))])
    unit = abs(scale) * np.log2(np.e)
    z0 = np.float32(2.0 ** np.floor(np.log2(top / unit / 32))) * (1 + g.integers(0, 64, Bz) / 64.0)          # bf16 holds it
    step = 2.0 ** max(np.floor(np.log2(top / unit)) - 22, 0) / 32                # S of both rows is a multiple of an fp32 step
    z1 = np.maximum(np.round(g.uniform(1.0, 12.0, Bz) / unit / 32 / step), 1) * step
    z1 = np.where(inputs.to_grid(z1.astype(np.float32), "bf16") == z1, z1, 4 * step)
    k = np.zeros((Bz, 1, cap, d), dtype=np.float32)
    k[..., :32] = (np.sign(scale) * z0)[:, None, None, None]
    k[:, :, 16:, 32:] = (np.sign(scale) * z1)[:, None, None, None]
    f = Filled(g, [cap] * Bz, cap, 1, d, 32, k=k)
    assert np.array_equal(f.k, k.astype(np.float64))
    S = 32.0 * np.stack([z0, z0 + z1])
    assert np.array_equal(S.astype(np.float32), S)
    o = binding.str_kv4_attn(ctx, f.cache, dev(np.ones((Bz, 1, 1, d), dtype=np.float32), dtype), _i32(f.lens), scale).float().cpu().numpy()[:, 0, 0]
    ctx.check_status()
    assert np.isfinite(o).all()
    D, half = unit * 32.0 * z1, 2.0 ** -24 * unit * S.sum(0)
    lo, hi = (1.0 / (1.0 + np.exp2(np.clip(-(D * (1 + s * 2.0 ** -22) + s * half), -1000, 1000))) for s in (-1, 1))
    v = f.v[:, 0].reshape(Bz, 2, 16, d)
    a, b = v.mean(2)[:, 0], v.mean(2)[:, 1]
    ends = np.stack([a + (b - a) * lo[:, None], a + (b - a) * hi[:, None]])
    # beside the weights' range: their roundings and sum, the factor of the matrix product, the output's own
    tol = (64 + cap) * E * np.abs(f.v).max() + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) * 15.0 * f.v_scale.max() + HALF[dtype] * np.abs(ends).max(0)
    assert np.all((o >= ends.min(0) - tol) & (o <= ends.max(0) + tol))


def _values_of_many_sizes(kind, g, n, cap, d, R):
    """(q [R, d], k [cap, d], v [cap, d]) of one key head; score units are natural."""
    q, k, v = g.standard_normal((R, d)), 0.3 * g.standard_normal((cap, d)), g.standard_normal((cap, d))
    q[:, 0], k[:, 0] = np.sqrt(d), 0.0                                           # k[:, 0] is what it adds to the scores
    t = np.arange(cap)
    if kind == "unseen":                                                        # huge values that draw no weight, between others
        k[[3, 100, 101], 0], v[[3, 100, 101]] = -300.0, v[[3, 100, 101]] * 2.0 ** 45
    elif kind == "outweighed":                                                  # huge values first, all weight on what follows
        k[16:, 0], v[:16] = 300.0, v[:16] * 2.0 ** 45
    elif kind == "heads":                                                       # every other head sees the huge values, the rest do not
        q[1::2, 0] *= -1.0
        k[[3, 100], 0], v[[3, 100]] = -300.0, v[[3, 100]] * 2.0 ** 40
    elif kind == "groups":
        v *= np.exp2(np.repeat([0.0, -45.0, 30.0, -80.0], 32)[:d])
    elif kind == "falling":                                                     # weights grow as the values shrink
        k[:, 0], v = 1.1 * t, v * np.exp2(-t)[:, None]
    elif kind == "rising":                                                      # and the other way round
        k[:, 0], v = -0.6 * t, v * np.exp2(t / 2.0 + t % 3)[:, None]
    elif kind == "constant":                                                    # rows of equal elements: scale 0, with rising scores
        k[20:, 0], v[20:] = 2.5 * (t[20:, None] - 19)[:, 0], np.float32(0.5)
    elif kind == "tiny":
        v *= 2.0 ** -115
    elif kind == "largest":
        v *= 2.0 ** 122
    return q, k, v


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d,group,R", [(64, 32, 4), (128, 32, 4), (128, 64, 8), (64, 64, 2), (128, 128, 1), (128, 32, 12)])
@pytest.mark.parametrize("kind", ["unseen", "outweighed", "heads", "groups", "falling", "rising", "constant", "tiny", "largest"])
def test_attention_of_values_of_many_sizes(ctx, dtype, d, group, R, kind):
    """The bound holds for each query row and group by itself: what draws no weight, and what other groups and other heads see, adds
    nothing to it.  With S = sum p scale and G = sum p max |v| of the row's softmax and the group: rel (as above, of every weight) of
    the two sums that make up the output, |zero + 8 scale| and |scale (c - 8)| <= 2.2 max |v|; half a step of the fp16 factors (2^-11,
    or 2^-22 for two) times at most 8; and for factors so small that fp16 holds them with fewer bits half its smallest
    step, 2^-25, each.  The largest p scale met is 2^11 of a unit when that is set, less a window of 2^12 (two factors: 2^8) that larger
    scales of other rows have, and the maximum may rise by 2^5 (2^4) before it is set anew: 2^-6 (2^-1) is the least it can be."""
    n, cap = 200, 208
    g = np.random.default_rng([d, group, R, len(kind), ord(kind[0])])
    q, k, v = _values_of_many_sizes(kind, g, n, cap, d, R)
    f = Filled(g, [n], cap, 1, d, group, k=k.astype(np.float32)[None, None], v=v.astype(np.float32)[None, None])
    q = inputs.to_grid(q.astype(np.float32)[None, None], dtype)
    scale = d ** -0.5
    w_out = torch.zeros(1, 1, cap, device="cuda")
    o = binding.str_kv4_attn(ctx, f.cache, dev(q, dtype), _i32([n]), scale, weight_out=w_out).float().cpu().numpy()[0, 0]
    o2 = binding.str_kv4_attn(ctx, f.cache, dev(q, dtype), _i32([n]), scale).float().cpu().numpy()[0, 0]
    ctx.check_status()
    assert np.array_equal(o, o2)
    K, V, sc = f.k[0, 0, :n], f.v[0, 0, :n], f.v_scale[0, 0, :n].astype(np.float64)
    gmax = np.abs(V).reshape(n, -1, group).max(2)
    for r in range(R):
        s = K @ q[0, 0, r].astype(np.float64) * scale
        p = np.exp(s - s.max())
        p /= p.sum()
        rel = 2 * (d + 64) * E * scale * (np.abs(K) @ np.abs(q[0, 0, r]).astype(np.float64)).max() + (32 + n) * E
        bound = 2.2 * rel * (p @ gmax) + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -22) * 8 * (p @ sc) + n * 2.0 ** (-19 if dtype == "bf16" else -24) * 8 * (p[:, None] * sc).max(0)
        ref = p @ V
        bound = np.repeat(bound, group) + HALF[dtype] * np.abs(ref) + 2.0 ** -133                      # bf16 holds multiples of that
        assert np.all(np.abs(o[r] - ref) <= bound), (r, float((np.abs(o[r] - ref) / bound).max()))


def test_attention_scores_that_grow_along_the_row(ctx):
    """Every later row beats all before it: the running maximum moves all the way."""
    d, n, Hkv, Hq = 128, 1000, 1, 4
    g = np.random.default_rng(10)
    k = np.broadcast_to(np.linspace(0, 6, 1008)[:, None], (1, Hkv, 1008, d)) + 0.01 * g.standard_normal((1, Hkv, 1008, d))
    f = Filled(g, [n], 1008, Hkv, d, 32, k=k.astype(np.float32))
    for sign in (1.0, -1.0):
        q = inputs.to_grid(np.full((1, 1, Hq, d), 0.5 * sign), "bf16")
        check_attention(ctx, f, q, "bf16", d ** -0.5, True)


def test_attention_passes_nan_and_infinity_on(ctx):
    g = np.random.default_rng(11)
    k, v = _rows(g, (3, 2, 80, 64), "f32", True), _rows(g, (3, 2, 80, 64), "f32", False)
    k[0, 0, 5, 3] = np.nan                                          # one head of one sequence
    v[1, 1, 70, 40] = np.inf                                        # one group of one value row
    f = Filled(g, [80, 80, 70], 80, 2, 64, 32, k=k, v=v)
    q = g.standard_normal((3, 1, 4, 64)).astype(np.float32)
    q[2, 0, 3, 9] = np.inf
    o = binding.str_kv4_attn(ctx, f.cache, dev(q), _i32(f.lens), 0.125).cpu().numpy()
    nan = np.isnan(o[:, 0])
    assert nan[0, :2].all() and not nan[0, 2:].any()
    assert nan[1, 2:, 32:].all() and not nan[1, :, :32].any() and not nan[1, :2].any()
    assert nan[2, 3].all() and not nan[2, :3].any()
    ctx.check_status()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Hq,Hkv,d,group", [(2, 2, 64, 64), (4, 1, 128, 32), (8, 1, 128, 128), (24, 2, 64, 32)])
def test_attention_rows_that_only_later_tokens_see_do_not_reach_the_earlier_ones(ctx, dtype, Hq, Hkv, d, group):
    """NaN in the keys or values of the newest rows: a token that does not see such a row is as if it were not there."""
    g = np.random.default_rng([Hq, d])
    n_q, lens = 4, [70, 67, 64, 5]
    k, v = _rows(g, (4, Hkv, 80, d), "f32", True), _rows(g, (4, Hkv, 80, d), "f32", False)
    bad_k, bad_v = k.copy(), v.copy()
    bad_k[0, 0, 69, 0], bad_v[1, Hkv - 1, 66, d - 1], bad_v[2, 0, 62, 1], bad_k[3, 0, 4, 3] = np.nan, np.inf, np.nan, -np.inf
    q = inputs.to_grid(g.standard_normal((4, n_q, Hq, d)), dtype)
    f, bad = Filled(g, lens, 80, Hkv, d, group, k=k, v=v), Filled(g, lens, 80, Hkv, d, group, k=bad_k, v=bad_v)
    got = binding.str_kv4_attn(ctx, bad.cache, dev(q, dtype), _i32(lens), d ** -0.5).float().cpu().numpy()
    good = binding.str_kv4_attn(ctx, f.cache, dev(q, dtype), _i32(lens), d ** -0.5).float().cpu().numpy()
    R = Hq // Hkv
    want = np.zeros(got.shape, dtype=bool)
    want[0, 3, :R] = True                                           # row 69 of 70: the last token only, all elements
    want[1, 3, (Hkv - 1) * R:, d - group:] = True                   # row 66 of 67, one group
    want[2, 2:, :R, :group] = True                                  # row 62 of 64: the last two tokens
    want[3, 3, :R] = True
    assert np.array_equal(np.isnan(got), want)
    assert np.array_equal(got[~want], good[~want])
    ctx.check_status()


@pytest.mark.parametrize("Bz,weights", [(33, True), (100, False), (257, True)])
def test_attention_of_many_sequences(ctx, Bz, weights):
    """More sequences than a warp has lanes, many of them empty, some long: the line of work is cut at odd places."""
    g = np.random.default_rng(Bz)
    lens = [int(n) for n in np.where(g.random(Bz) < 0.4, 0, g.integers(1, 400, Bz))]
    lens[0], lens[-1], lens[Bz // 2] = 0, 3, 2000
    f = Filled(g, lens, 2000, 1, 64, 32)
    q = inputs.to_grid(g.standard_normal((Bz, 1, 4, 64)), "bf16")
    check_attention(ctx, f, q, "bf16", 0.125, weights)


@pytest.mark.parametrize("n_q,R", [(512, 8), (1365, 3), (4096, 1)])
def test_attention_of_as_many_query_rows_as_a_key_head_may_have(ctx, n_q, R):
    g = np.random.default_rng([n_q, R])
    f = Filled(g, [n_q + 100, 33, 0], (n_q + 127) // 16 * 16, 1, 64, 32)
    q = g.standard_normal((3, n_q, R, 64)).astype(np.float32)
    check_attention(ctx, f, q, "f32", 0.125, True)
    with pytest.raises(binding.StrError) as e:
        binding.str_kv4_attn(ctx, f.cache, dev(np.zeros((3, 4097, 1, 64), dtype=np.float32)), _i32(f.lens), 0.125)
    assert e.value.code == -2


def test_decode_calls_on_as_many_sequences_as_a_grid_holds(ctx):
    """65535 sequences of up to 16 rows."""
    Bz, d = 65535, 64
    g = torch.Generator(device="cuda").manual_seed(8)
    lens = torch.randint(0, 17, (Bz,), generator=g, device="cuda", dtype=torch.int32)
    cache, out = binding.Kv4Cache.empty(ctx, Bz, 16, 1, d), binding.Kv4Cache.empty(ctx, Bz, 16, 1, d)
    k, v, q = (torch.randn(Bz, n, 1, d, generator=g, device="cuda") for n in (16, 16, 1))
    zero = torch.zeros_like(lens)
    binding.str_kv4_append(ctx, cache, k, v, zero, n_new=lens)
    kr, vr = binding.str_kv4_read(ctx, cache, zero, 16, torch.float32, n_rows=lens)
    o = binding.str_kv4_attn(ctx, cache, q, lens, 0.125, weight_out=cache.weight)
    n, kept = binding.str_kv4_evict(ctx, cache, lens, 4, 1, out)
    ctx.check_status()
    pick = np.random.default_rng(8).integers(0, Bz, 300)
    pick[:2] = 0, Bz - 1
    w, kept, host = cache.weight.cpu().numpy(), kept.cpu().numpy(), lens.cpu().numpy()
    for b in pick:
        m = host[b]
        qb, kb, vb = (t.cpu().numpy() for t in (q[b], kr[b, :m, 0], vr[b, :m, 0]))
        ref, drawn = decode.kv4_attention(qb, kb[None], vb[None], 0.125)
        if m:                                                       # as at the top of the file; read-back rows are off by 2 e, a scale is span / 15
            rel = 2 * (d + 64) * E * 0.125 * (np.abs(kb) @ np.abs(qb[0, 0])).max() + (32 + m) * E
            assert np.all(np.abs(o[b].cpu().numpy() - ref) <= (rel + 2 * E) * np.abs(vb).max() + 2.0 ** -22 * 1.1 * np.ptp(vb) + E * np.abs(ref))
            assert np.all(np.abs(w[b, 0, :m] - drawn[0]) <= (rel + 2 * E) * drawn[0])
        else:
            assert not o[b].any()
        idx = decode.kv4_evict(w[b], m, 4, 1)
        assert int(n[b]) == len(idx) and np.array_equal(kept[b, :len(idx)], idx) and np.all(kept[b, len(idx):] == -1)


def test_attention_weights_in_place_and_the_same_bits_every_time(ctx):
    g = np.random.default_rng(12)
    f = Filled(g, [2000, 0, 517], 2016, 4, 128, 32)
    q, lens = dev(inputs.to_grid(g.standard_normal((3, 2, 16, 128)), "bf16"), "bf16"), _i32(f.lens)
    w1 = f.cache.weight.clone()
    o1 = binding.str_kv4_attn(ctx, f.cache, q, lens, 0.09, weight_out=w1)
    for _ in range(3):
        w2 = f.cache.weight.clone()
        o2 = binding.str_kv4_attn(ctx, f.cache, q, lens, 0.09, weight_out=w2)
        assert torch.equal(o1, o2) and torch.equal(w1, w2)
    binding.str_kv4_attn(ctx, f.cache, q, lens, 0.09, weight_out=f.cache.weight)
    assert torch.equal(f.cache.weight, w1)
    assert torch.equal(binding.str_kv4_attn(ctx, f.cache, q, lens, 0.09), o1)       # with and without the weights


def test_attention_lengths_outside_the_capacity_are_held_to_it_and_reported(ctx):
    g = np.random.default_rng(13)
    f = Filled(g, [48, 0], 48, 1, 64, 32)
    q = g.standard_normal((2, 1, 2, 64)).astype(np.float32)
    got = binding.str_kv4_attn(ctx, f.cache, dev(q), _i32([1000, -3]), 0.125)
    with pytest.raises(binding.StrError) as e:
        ctx.check_status()
    assert e.value.code == -1
    check_attention(ctx, f, q, "f32", 0.125, False, got=got)


def test_rows_beyond_four_gigabytes(ctx):
    """Codes of more than 2^32 bytes: the last head of the last sequence, whose rows start behind that."""
    Bz, Hkv, cap, d = 3, 8, 3000016, 128
    cache = binding.Kv4Cache.empty(ctx, Bz, cap, Hkv, d, 32)
    assert cache.k_codes.numel() > 1 << 32
    g = np.random.default_rng(14)
    k, v = (_rows(g, (Bz, 40, Hkv, d), "f32", False) for _ in range(2))
    lens = _i32([0, 17, cap - 5])
    binding.str_kv4_append(ctx, cache, dev(k), dev(v), _i32([0, 0, cap - 45]), n_new=_i32([0, 17, 40]))
    kr, vr = binding.str_kv4_read(ctx, cache, _i32([0, 0, cap - 45]), 40, torch.float32)
    code, zero, scale = decode.kv4_quantise(v[2], 32)
    assert np.all(np.abs(vr[2].cpu().numpy() - decode.kv4_values(code, zero, scale, 32)) <= 4 * E * 16)
    q = 30.0 * kr[2, 39].repeat_interleave(2, 0).expand(Bz, 1, 2 * Hkv, d).contiguous()    # finds its own row: a score of thousands
    o = binding.str_kv4_attn(ctx, cache, q, lens, 1.0, weight_out=cache.weight)
    ctx.check_status()
    assert not o[0].any()
    want = vr[2, 39].repeat_interleave(2, 0)
    assert float((o[2, 0] - want).abs().max()) <= 2.0 ** -20 * float(want.abs().max())
    assert float((cache.weight[2, :, cap - 6] - 2.0).abs().max()) <= 1e-5 and not cache.weight[2, :, :cap - 45].any()
    out = binding.Kv4Cache.empty(ctx, Bz, 16, Hkv, d, 32)
    n, kept = binding.str_kv4_evict(ctx, cache, lens, 16, 3, out)
    assert n.tolist() == [0, 16, 16] and kept[2].tolist() == [*range(13), cap - 8, cap - 7, cap - 6] and kept[0].tolist() == [-1] * 16
    assert torch.equal(out.v_codes[2, 7, 15], cache.v_codes[2, 7, cap - 6])
    ctx.check_status()


# ---------------------------------------------------------------- eviction
@pytest.mark.parametrize("d,group", SHAPES)
@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "odd"])
def test_evict_matches_the_definition_bit_for_bit(ctx, d, group, kind):
    g = np.random.default_rng([d, group, len(kind)])
    lens, cap, Hkv = [0, 1, 30, 500, 777, 1008], 1008, 3
    f = Filled(g, lens, cap, Hkv, d, group)
    w = np.abs(g.standard_normal(f.weight.shape)).astype(np.float32)
    if kind == "ties":
        w = g.integers(0, 4, w.shape).astype(np.float32)
    if kind == "equal":
        w[:] = 0.25
    if kind == "odd":
        w[:, 0, ::7], w[:, 1, ::11], w[:, 2, ::13] = np.nan, np.inf, -np.inf
    f.cache.weight.copy_(torch.from_numpy(w))
    src = {n: getattr(f.cache, n).cpu().numpy() for n in ("k_codes", "v_codes", "k_scales", "v_scales", "pos", "weight")}
    for keep, recent, evictable, cap_out in [(256, 32, None, 256), (1, 0, None, 16), (1008, 1008, None, 1024), (31, 31, None, 64),
                                             (300, 5, [0, 0, 9, 400, 777, 1000], 304), (200, 0, [5, 5, 5, 5, -3, 5000], 208), (0, 0, None, 16)]:
        out = binding.Kv4Cache.empty(ctx, len(lens), cap_out, Hkv, d, group)
        for n in ("k_codes", "v_codes"):
            getattr(out, n).fill_(0x3C)
        for n in ("k_scales", "v_scales", "pos"):
            getattr(out, n).fill_(-9)
        out.weight.fill_(-9.0)
        n_out, kept = binding.str_kv4_evict(ctx, f.cache, _i32(lens), keep, recent, out, n_evictable=None if evictable is None else _i32(evictable))
        ctx.check_status()
        kept = kept.cpu().numpy()
        for b, n in enumerate(lens):
            idx = decode.kv4_evict(w[b], n, keep, recent, None if evictable is None else evictable[b])
            m = len(idx)
            assert int(n_out[b]) == m == min(n, keep)
            assert np.array_equal(kept[b, :m], idx) and np.all(kept[b, m:] == -1)
            for name, a in src.items():
                o = getattr(out, name)[b].cpu().numpy()
                rows = (lambda x: x) if name == "pos" else (lambda x: np.moveaxis(x, 1, 0))
                assert np.array_equal(rows(o)[:m], rows(a[b])[idx], equal_nan=name == "weight"), name
                assert np.all(rows(o)[m:] == {"k_codes": 0x3C, "v_codes": 0x3C}.get(name, -9)), name


@pytest.mark.parametrize("cap,keep", [(16, 7), (4096, 1000), (40000, 39999), (140000, 30000)])
def test_evict_long_and_short_rows(ctx, cap, keep):
    g = np.random.default_rng(cap)
    lens = [cap, cap - 3, cap // 2]
    cache = binding.Kv4Cache.empty(ctx, 3, cap, 1, 64, 64)
    w = g.choice(np.array([0.5, 1.0, 1.5, 2.0], dtype=np.float32), (3, 1, cap)) if cap == 4096 else g.random((3, 1, cap)).astype(np.float32)
    cache.weight.copy_(torch.from_numpy(w))
    cache.pos.copy_(torch.arange(cap, dtype=torch.int32).expand(3, cap))
    out = binding.Kv4Cache.empty(ctx, 3, (keep + 15) // 16 * 16, 1, 64, 64)
    n_out, kept = binding.str_kv4_evict(ctx, cache, _i32(lens), keep, 5, out)
    ctx.check_status()
    for b, n in enumerate(lens):
        m, idx = min(n, keep), decode.kv4_evict(w[b], n, keep, 5)
        assert np.array_equal(kept[b, :m].cpu().numpy(), idx) and np.array_equal(out.pos[b, :m].cpu().numpy(), idx)


def test_evict_without_ids_or_weights_to_copy(ctx):
    cache = binding.Kv4Cache.empty(ctx, 1, 32, 1, 64, 32)
    cache.weight.copy_(torch.arange(32.0).view(1, 1, 32))
    out = binding.Kv4Cache.empty(ctx, 1, 16, 1, 64, 32, pos=False, weight=False)
    n, kept = binding.str_kv4_evict(ctx, cache, _i32([20]), 3, 0, out)
    assert kept.tolist() == [[17, 18, 19]] and n.tolist() == [3]


# ---------------------------------------------------------------- the recurrent step
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("Bz,T,H,p,n,G,skip", [(1, 1, 8, 64, 128, 2, False), (2, 3, 6, 32, 16, 3, True), (1, 1, 1, 1, 1, 1, True), (3, 5, 4, 17, 20, 1, True),
                                               (1, 2, 2, 80, 256, 2, False), (2, 1, 3, 7, 33, 3, True), (1, 4, 2, 5, 512, 1, True), (1, 2, 2, 9, 511, 2, False),
                                               (1, 16, 4, 64, 64, 4, True), (2, 2, 2, 130, 36, 1, True)])
def test_step_matches_the_recurrence(ctx, dtype, Bz, T, H, p, n, G, skip):
    """Bound: with M the recurrence of magnitudes, a state element is off by at most 5 e M per token (decay, its product, the
    token's two products, one sum) and y by (n + 8) e sum M |c| on top, plus the storage type's half step."""
    g = np.random.default_rng([Bz, T, H, p, n])
    x, B, C = (inputs.to_grid(g.standard_normal(s), dtype) for s in ((Bz, T, H, p), (Bz, T, G, n), (Bz, T, G, n)))
    dt = g.uniform(0.001, 0.1, (Bz, T, H)).astype(np.float32)
    A = -np.exp(g.uniform(0, np.log(16), H)).astype(np.float32)
    D = g.standard_normal(H).astype(np.float32) if skip else None
    S0 = g.standard_normal((Bz, H, p, n)).astype(np.float32)
    state = dev(S0)
    out = torch.full_like(state, float("nan"))
    args = [dev(x, dtype), dev(dt), dev(A), dev(B, dtype), dev(C, dtype)]
    Dd = dev(D) if skip else None
    y, S = binding.str_mamba2_step(ctx, *args, state, D=Dd, state_out=out)
    assert S is out and np.array_equal(state.cpu().numpy(), S0)
    y2, S2 = binding.str_mamba2_step(ctx, *args, state, D=Dd)       # in place: the same bits
    assert S2 is state and torch.equal(state, out) and torch.equal(y, y2)
    for b in range(Bz):
        yr, Sr = decode.mamba2_step(x[b], dt[b], A, B[b], C[b], S0[b], D)
        ym, Sm = decode.mamba2_step(np.abs(x[b]), dt[b], A, np.abs(B[b]), np.abs(C[b]), np.abs(S0[b]), None if D is None else np.abs(D))
        assert np.all(np.abs(out[b].cpu().numpy() - Sr) <= 5 * T * E * Sm)
        assert np.all(np.abs(y[b].float().cpu().numpy() - yr) <= (5 * T + n + 8) * E * ym + HALF[dtype] * np.abs(yr))


def test_step_continues_the_chunked_scan(ctx):
    """One token at a time behind str_mamba2_prefill of the rest: the chunked scan of the whole sequence."""
    a = inputs.ssd_inputs(31, 200, 8, 64, 128, 2, "f32")
    x, dt, A, B, C = (dev(a[k]) for k in ("x", "dt", "A", "B", "C"))
    y_all, s_all = binding.str_mamba2_prefill(ctx, x, dt, A, B, C, want_final_state=True)
    cut = 190
    part = [t[:, :cut].contiguous() for t in (x, dt, B, C)]
    _, state = binding.str_mamba2_prefill(ctx, part[0], part[1], A, part[2], part[3], want_final_state=True)
    for t in range(cut, 200):
        x1, dt1, B1, C1 = (v[:, t:t + 1].contiguous() for v in (x, dt, B, C))
        y1, _ = binding.str_mamba2_step(ctx, x1, dt1, A, B1, C1, state)
        assert float((y1[:, 0] - y_all[:, t]).abs().max()) <= 1e-4 * float(y_all.abs().max())
    assert float((state - s_all).abs().max()) <= 1e-4 * float(s_all.abs().max())


# ---------------------------------------------------------------- as they are used together
def test_decode_of_a_handed_off_attention_layer(ctx):
    """Hand-off of a reducing attention layer -> 4-bit cache -> a few decode steps -> eviction -> more steps, against the oracle
    on the values the cache holds; and the values against the hand-off's."""
    g = np.random.default_rng(41)
    D, Hq, Hkv, d, n_vis, M = 512, 4, 2, 128, 256, 16
    layers = inputs.stack_params(7, "A", None, dict(D=D, Hq=Hq, Hkv=Hkv, d=d, theta=1.0e6), "bf16")
    st = binding.Stack(ctx, layers, "bf16", 2, n_vis, M, [128])
    h0 = inputs.hidden_inputs(7, n_vis + M, D, "bf16", batch=2)
    res = binding.str_stack_prefill_ex(st, dev(h0, "bf16"), want_handoff=True)
    (_, k), (_, v), (_, pos) = res["attn_k"][0], res["attn_v"][0], res["attn_pos"][0]
    cache, n = binding.Kv4Cache.empty(ctx, 2, 176, Hkv, d, 32), k.shape[1]
    binding.str_kv4_append(ctx, cache, k, v, _i32([0, 0]), positions=pos)
    kr, vr = binding.str_kv4_read(ctx, cache, _i32([0, 0]), n, torch.float32)
    for a, r in ((k.float(), kr), (v.float(), vr)):                  # half a step of the group's scale, as the definition has it
        span = a.unflatten(-1, (4, 32)).amax(-1) - a.unflatten(-1, (4, 32)).amin(-1)
        assert bool(((a - r).abs().unflatten(-1, (4, 32)).amax(-1) <= 0.56 * span / 15).all())
    assert torch.equal(cache.pos[:, :n], pos) and not cache.weight.any()
    lens, total = n, 0
    for step in range(12):
        kn, vn = (inputs.to_grid(g.standard_normal((2, 1, Hkv, d)), "bf16") for _ in range(2))
        q = inputs.to_grid(g.standard_normal((2, 1, Hq, d)), "bf16")
        p1 = _i32([[n_vis + M + step]] * 2)
        binding.str_kv4_append(ctx, cache, dev(kn, "bf16"), dev(vn, "bf16"), _i32([lens] * 2), positions=p1)
        lens += 1
        kr, vr = (t.cpu().numpy() for t in binding.str_kv4_read(ctx, cache, _i32([0, 0]), lens, torch.float32))
        before = cache.weight[:, :, :lens].double().cpu().numpy()
        o = binding.str_kv4_attn(ctx, cache, dev(q, "bf16"), _i32([lens] * 2), d ** -0.5, weight_out=cache.weight).float().cpu().numpy()
        total += 1
        after = cache.weight[:, :, :lens].double().cpu().numpy()
        for b in range(2):
            ro, drawn = decode.kv4_attention(q[b], np.swapaxes(kr[b], 0, 1), np.swapaxes(vr[b], 0, 1), d ** -0.5)
            # 2^-8 for the output's bf16, 2^-11 of a group's 15 steps (at most the span of all values) for the fp16 factor
            assert np.all(np.abs(o[b] - ro) <= 2.0 ** -8 * np.abs(ro) + 2.0 ** -11 * np.ptp(vr[b]) + 1e-4)
            assert np.all(np.abs(after[b] - before[b] - drawn) <= 1e-4 * drawn + 1e-6)
        assert np.allclose(after.sum(2), before.sum(2) + Hq / Hkv, rtol=1e-4)
        if step == 7:                                               # a budget: text and generated rows stay, images compete
            out = binding.Kv4Cache.empty(ctx, 2, 96, Hkv, d, 32)
            _, kept = binding.str_kv4_evict(ctx, cache, _i32([lens] * 2), 90, 8, out, n_evictable=_i32([128, 128]))
            for b in range(2):
                assert np.array_equal(kept[b].cpu().numpy(), decode.kv4_evict(cache.weight[b].cpu().numpy(), lens, 90, 8, 128))
                assert torch.equal(out.pos[b, :90], cache.pos[b][kept[b].long()])
            cache, lens = out, 90
    ctx.check_status()


@pytest.mark.parametrize("d,group", [(64, 32), (128, 64)])
def test_a_second_turn_reads_the_cache_back_for_the_prompt_attention(ctx, d, group):
    """A prompt of 40 tokens behind what two sequences' caches hold: appended, all rows read back, str_attn_prefill_rows for the new
    rows; the same outputs as str_kv4_attn's, within the bound that each keeps from the oracle on the cached values."""
    g = np.random.default_rng([77, d])
    Hq, Hkv, n_new, lens = 6, 2, 40, [203, 203]
    f = Filled(g, lens, 256, Hkv, d, group)
    total = [n + n_new for n in lens]
    k, v = (_rows(g, (2, n_new, Hkv, d), "f32", keys) for keys in (True, False))
    q = g.standard_normal((2, n_new, Hq, d)).astype(np.float32)
    binding.str_kv4_append(ctx, f.cache, dev(k), dev(v), _i32(lens))
    kr, vr = binding.str_kv4_read(ctx, f.cache, _i32([0, 0]), total[0], torch.float32)
    rows = _i32([np.arange(n, n + n_new) for n in lens])
    turn = binding.str_attn_prefill_rows(ctx, dev(q), rows, kr, vr, d ** -0.5).cpu().numpy()
    step = binding.str_kv4_attn(ctx, f.cache, dev(q), _i32(total), d ** -0.5).cpu().numpy()
    ctx.check_status()
    kr, vr = (np.swapaxes(t.double().cpu().numpy(), 1, 2) for t in (kr, vr))
    for b in range(2):
        ref, _ = decode.kv4_attention(q[b], kr[b], vr[b], d ** -0.5)
        ds = (d + 64) * E * d ** -0.5 * max((np.abs(kr[b, h]) @ np.abs(q[b].reshape(n_new, Hkv, -1, d)[:, h]).reshape(-1, d).T.astype(np.float64)).max() for h in range(Hkv))
        bound = (2 * ds + (32 + total[b]) * E + 2 * E) * np.abs(vr[b]).max() + 2.0 ** -22 * 15 * np.ptp(vr[b]) / 15 + E * np.abs(ref)
        assert np.all(np.abs(turn[b] - ref) <= bound) and np.all(np.abs(step[b] - ref) <= bound)


def _decode_args(g, Bz=2, cap=512, Hq=8, Hkv=2, d=64):
    f = Filled(g, [400, 77], cap, Hkv, d, 32)
    mk = lambda *s: dev(inputs.to_grid(g.standard_normal(s), "bf16"), "bf16")  # noqa: E731
    step = [mk(Bz, 1, 4, 16), dev(g.uniform(0.001, 0.1, (Bz, 1, 4)).astype(np.float32)), dev(-np.ones(4, dtype=np.float32)), mk(Bz, 1, 2, 32), mk(Bz, 1, 2, 32)]
    return f, mk(Bz, 1, Hq, d), mk(Bz, 1, Hkv, d), mk(Bz, 1, Hkv, d), step, dev(g.standard_normal((Bz, 4, 16, 32)).astype(np.float32))


def _decode_pass(ctx, f, q, k, v, step, state, start, lens, out):
    binding.str_kv4_append(ctx, f.cache, k, v, start)
    o = binding.str_kv4_attn(ctx, f.cache, q, lens, 0.125, weight_out=f.cache.weight)
    n, kept = binding.str_kv4_evict(ctx, f.cache, lens, 64, 8, out)
    y, _ = binding.str_mamba2_step(ctx, *step, state)
    return o, n, kept, y


def test_decode_calls_replay_from_two_graphs_and_run_on_other_streams(ctx):
    """The same pass eagerly, from two captured graphs replayed on two streams at once, and eagerly on a side stream."""
    start, lens = _i32([400, 77]), _i32([401, 78])
    runs, graphs = [], []
    for which in range(3):
        args = _decode_args(np.random.default_rng(50))
        out = binding.Kv4Cache.empty(ctx, 2, 64, 2, 64, 32)
        runs.append((args, out))
    eager = _decode_pass(ctx, *runs[0][0], start, lens, runs[0][1])
    for args, out in runs[1:]:
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            res = _decode_pass(ctx, *args, start, lens, out)
        graphs.append((gr, res, torch.cuda.Stream()))
    torch.cuda.synchronize()
    for gr, _, s in graphs:
        with torch.cuda.stream(s):
            gr.replay()
    torch.cuda.synchronize()
    for (gr, res, _), (args, out) in zip(graphs, runs[1:]):
        for a, b in zip(res, eager):
            assert torch.equal(a, b)
        assert torch.equal(args[0].cache.weight, runs[0][0][0].cache.weight) and torch.equal(args[-1], runs[0][0][-1])
        assert torch.equal(out.k_codes, runs[0][1].k_codes) and torch.equal(out.weight, runs[0][1].weight)
    args = _decode_args(np.random.default_rng(50))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        res = _decode_pass(ctx, *args, start, lens, binding.Kv4Cache.empty(ctx, 2, 64, 2, 64, 32))
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(res, eager))
    ctx.check_status()


def test_a_wrong_count_does_not_stop_other_calls(ctx):
    """Recorded for str_check_status, but the tensor-core kernels of the context go on working meanwhile."""
    f = Filled(np.random.default_rng(61), [16, 0], 16, 1, 64, 32)
    q = dev(np.ones((2, 1, 1, 64), dtype=np.float32))
    binding.str_kv4_attn(ctx, f.cache, q, _i32([17, 0]), 0.1)
    a, w = torch.ones(128, 256, device="cuda").bfloat16(), torch.ones(256, 256, device="cuda").bfloat16()
    assert bool((binding.str_gemm(ctx, a, w) == 256).all())
    with pytest.raises(binding.StrError) as e:
        ctx.check_status()
    assert e.value.code == -1
    ctx.check_status()


_FIRST_CALLS = """
import sys, torch
sys.path.insert(0, ".")
from paper_2603_00198_b200 import binding
ctx = binding.Context(0)
torch.manual_seed(0)
def make():
    cache = binding.Kv4Cache.empty(ctx, 2, 512, 2, 64, 32)
    out = binding.Kv4Cache.empty(ctx, 2, 64, 2, 64, 32)
    k = torch.randn(2, 300, 2, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(1))
    q = torch.randn(2, 2, 6, 64, device="cuda", generator=torch.Generator("cuda").manual_seed(2))
    st = torch.randn(2, 4, 8, 16, device="cuda", generator=torch.Generator("cuda").manual_seed(3))
    x, dt, A, B = torch.ones(2, 1, 4, 8, device="cuda"), torch.ones(2, 1, 4, device="cuda"), -torch.ones(4, device="cuda"), torch.ones(2, 1, 2, 16, device="cuda")
    return cache, out, k, q, st, x, dt, A, B
zero, lens = torch.zeros(2, dtype=torch.int32, device="cuda"), torch.tensor([300, 17], dtype=torch.int32, device="cuda")
def run(cache, out, k, q, st, x, dt, A, B):
    binding.str_kv4_append(ctx, cache, k, -k, zero)
    o = binding.str_kv4_attn(ctx, cache, q, lens, 0.125, weight_out=cache.weight)
    n, kept = binding.str_kv4_evict(ctx, cache, lens, 50, 4, out)
    r = binding.str_kv4_read(ctx, out, zero, 50, torch.float32, n_rows=n)
    y, _ = binding.str_mamba2_step(ctx, x, dt, A, B, B, st)
    return o, n, kept, r[0], r[1], y
graph, args = torch.cuda.CUDAGraph(), make()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    captured = run(*args)
graph.replay()
torch.cuda.synchronize()
eager = run(*make())
assert all(torch.equal(a, b) for a, b in zip(captured, eager))
ctx.check_status()
print("first calls captured")
"""


def test_the_first_calls_of_a_process_may_be_captured():
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    res = subprocess.run([sys.executable, "-c", _FIRST_CALLS], cwd=root, capture_output=True, text=True, timeout=300)
    assert res.returncode == 0 and "first calls captured" in res.stdout, res.stderr[-3000:]


def test_binding_refuses_what_the_kernels_cannot_read(ctx):
    g = np.random.default_rng(60)
    f, q, k, v, step, state = _decode_args(g)
    lens = _i32([400, 77])
    for bad in (lens.long(), lens.cpu(), lens[:1], torch.stack([lens, lens], 1)[:, 0]):
        with pytest.raises((TypeError, ValueError)):
            binding.str_kv4_attn(ctx, f.cache, q, bad, 0.1)
        with pytest.raises((TypeError, ValueError)):
            binding.str_kv4_append(ctx, f.cache, k, v, bad)
    for bad in (q.half(), q[..., :32], q[:1], q.transpose(1, 2), q.cpu()):
        with pytest.raises((TypeError, ValueError, binding.StrError)):
            binding.str_kv4_attn(ctx, f.cache, bad, lens, 0.1)
    with pytest.raises(TypeError):
        binding.str_kv4_append(ctx, f.cache, k, v.float(), lens)
    with pytest.raises(binding.StrError):
        binding.str_kv4_attn(ctx, f.cache, q[:, :, :3].contiguous(), lens, 0.1)                 # 3 heads over 2
    with pytest.raises(ValueError):
        binding.Kv4Cache(f.cache.k_codes, f.cache.v_codes[:, :1], f.cache.k_scales, f.cache.v_scales)
    with pytest.raises(binding.StrError):
        binding.str_kv4_evict(ctx, f.cache, lens, 16, 0, f.cache)                               # onto itself
    for bad in (dict(group=48), dict(group=256), dict(group=16)):
        with pytest.raises(ValueError):
            binding.Kv4Cache.empty(ctx, 1, 16, 1, 128, **bad)
    pool = torch.zeros(2 * 2 * 512 * 2, device="cuda")                                           # weights that half overlap
    half = binding.Kv4Cache(f.cache.k_codes, f.cache.v_codes, f.cache.k_scales, f.cache.v_scales, f.cache.pos, pool[:2048].view(2, 2, 512))
    with pytest.raises(binding.StrError):
        binding.str_kv4_attn(ctx, half, q, lens, 0.1, weight_out=pool[1024:][:2048].view(2, 2, 512))
    states = torch.zeros(3 * 2 * 4 * 16 * 32, device="cuda")
    with pytest.raises(binding.StrError):
        binding.str_mamba2_step(ctx, *step, states[:4096].view(2, 4, 16, 32), state_out=states[2048:6144].view(2, 4, 16, 32))
    with pytest.raises(ValueError):
        binding.str_kv4_evict(ctx, f.cache, lens, 16, 0, binding.Kv4Cache.empty(ctx, 2, 16, 2, 64, 64))
    with pytest.raises((TypeError, ValueError)):
        binding.str_mamba2_step(ctx, *step, state.double())
    with pytest.raises((TypeError, ValueError)):
        binding.str_mamba2_step(ctx, *step, state[:, :, :, :16])
