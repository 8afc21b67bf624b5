"""GPU parity of the operators on packed sequences and continued turns against the plain fp64 oracle, at the sizes, masks and values where they
can go wrong.

Tolerances are bounds worked out from the data of each case, with e = 2^-24 (half a step of fp32) and h the half step of the storage type (bf16
2^-8, fp32 e).
Convolution: u is a sum of W + 1 terms, each a product rounded with the running sum: off by at most (W + 2) e times the sum of the terms'
absolute values; SiLU's slope is at most 1.1, its own evaluation (exponential, quotient) off by 2^-20 relative; h of the output.  dt: the
argument of the exponential is off by 2 e |raw|, which is that much relative in dt, and the functions by 2^-21.
Scan: y is a sum of terms decay * dt x (b . c).  For bf16 storage a term passes through at most two roundings to bf16 (the weights of a
chunk, or the state's copy and its product's operand) and fp32 arithmetic whose exponents are cumulative sums over up to a chunk: 2 h + 2^-12 of the sum
of absolute terms; h of the output.  In fp32 arithmetic a term is multiplied by one rounded decay per token of its way (each off by the
exponential's 2^-22 and its argument's e * 16): (T + 64) 2^-21 at most.  Final states take no rounding to bf16: 2^-16 (two bf16 pieces of a
factor) + (T + 64) 2^-21.
Attention: a score formed in fp32 is off by ds = (d + 64) e * scale * sum |q_c| |k_c|; a weight then by 2 ds + n e + 2^-12 relative (the exponential's
approximation included), for bf16 storage by h more (weights enter the product as bf16); the output by that times sum p |v|, and h of itself.
Rotations: sine and cosine are off by 4 e, the two products and their sum by 2 e: 8 e (|a| + |b|) amplitude, and h of the result.
"""
import math

import numpy as np
import pytest
import torch

from oracle import packed
from paper_2603_00198_b200 import binding, inputs
from util_gpu import dev

pytestmark = [pytest.mark.gpu, pytest.mark.filterwarnings("ignore::RuntimeWarning")]
E = 2.0 ** -24
HALF = {"bf16": 2.0 ** -8, "f32": E}
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
UNTOUCHED = 77.0


@pytest.fixture(scope="module")
def ctx():
    c = binding.Context(0)
    yield c
    c.check_status()
    c.close()


def _i32(a):
    return dev(np.asarray(a, dtype=np.int32))


def _starts(lens, first=0):
    return [first] + [first + int(v) for v in np.cumsum(lens)]


def _f64(t):
    return t.double().cpu().numpy()


def _close(got, want, bound, what):
    """|got - want| <= bound wherever want is a number; elsewhere got has to be untouched."""
    got = _f64(got) if torch.is_tensor(got) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    seen = ~np.isnan(want)
    assert (got[~seen] == UNTOUCHED).all(), what
    with np.errstate(invalid="ignore"):
        bad = seen & ~(np.abs(got - want) <= bound)
    assert not bad.any(), (what, int(bad.sum()), np.argwhere(bad)[0].tolist(), got[bad][:3], want[bad][:3], np.broadcast_to(bound, got.shape)[bad][:3])


# ------------------------------------------------------------------------------------------------ convolution
class Conv:
    def __init__(self, g, lens, dtype, H, p, n, G, W, first=0, tail=0):
        self.dims, self.W, self.dtype, self.lens = (H, p, n, G), W, dtype, lens
        self.starts = _starts(lens, first)
        self.rows, self.ch, self.d_inner = self.starts[-1] + tail, H * p + 2 * G * n, H * p
        self.zx = inputs.to_grid(g.standard_normal((self.rows, 2 * H * p + 2 * G * n + H)), dtype)
        self.w, self.b = g.standard_normal((self.ch, W)).astype(np.float32), g.standard_normal(self.ch).astype(np.float32)
        self.bias = g.uniform(-7, -2, H).astype(np.float32)
        self.window = inputs.to_grid(g.standard_normal((len(lens), W - 1, self.ch)), dtype)
        if self.rows > self.starts[-1]:
            self.zx[self.starts[-1]:] = np.nan
        self.zx[:first] = np.nan
        self.on = [dev(a) for a in (self.w, self.b, self.bias)]

    def check(self, got, window_out, window):
        H, p, n, G = self.dims
        u, mag, dt, out = packed.conv(self.zx, self.d_inner, self.w, self.b, self.bias, self.starts, window)
        bound = 1.1 * (self.W + 2) * E * mag + (2.0 ** -20 + HALF[self.dtype]) * np.abs(u) + 2.0 ** -126
        at = 0
        for name, t, shape in zip("xBC", got, ((H, p), (G, n), (G, n))):
            w = shape[0] * shape[1]
            _close(t.reshape(self.rows, w), u[:, at:at + w], bound[:, at:at + w], name)
            at += w
        raw = np.abs(self.zx[:, self.d_inner + self.ch:] + self.bias)
        _close(got[3].reshape(self.rows, H), dt, dt * (2.0 ** -21 + 4 * E * raw), "dt")
        if window_out is not None:
            assert np.array_equal(_f64(window_out), out)


CONV = [("bf16", 4, (8, 64, 128, 2)), ("bf16", 4, (2, 16, 16, 1)), ("bf16", 3, (3, 20, 12, 3)), ("bf16", 2, (1, 5, 3, 1)), ("f32", 4, (4, 32, 64, 2)),
        ("f32", 3, (24, 32, 20, 3)), ("f32", 2, (1, 7, 5, 1))]
LENS = [[1], [3], [300], [0, 1, 2, 0, 3, 4, 31, 33, 64, 0], [0, 0], [1] * 70]


@pytest.mark.parametrize("windowed", [False, True])
@pytest.mark.parametrize("lens", LENS, ids=str)
@pytest.mark.parametrize("dtype, W, dims", CONV)
def test_convolution_over_ragged_sequences(ctx, dtype, W, dims, lens, windowed):
    g = np.random.default_rng([W, len(lens), sum(lens)])
    H, p, n, G = dims
    for first, tail in ((0, 0), (2, 5)):
        c = Conv(g, lens, dtype, H, p, n, G, W, first, tail)
        if c.rows == 0:
            continue
        out = [torch.full((c.rows, a, b), UNTOUCHED, dtype=TORCH[dtype], device="cuda") for a, b in ((H, p), (G, n), (G, n))]
        out.append(torch.full((c.rows, H), UNTOUCHED, device="cuda"))
        wout = torch.full((len(lens), W - 1, c.ch), UNTOUCHED, dtype=TORCH[dtype], device="cuda")
        window = c.window if windowed else None
        got = binding.str_mamba_conv_packed(ctx, dev(c.zx, dtype), *c.on, _i32(c.starts), *dims, window=dev(window, dtype) if windowed else None,
                                            window_out=wout, out=tuple(out))
        assert all(a is b or a.data_ptr() == b.data_ptr() for a, b in zip(got, out))
        c.check(out, wout, window)


def test_convolution_of_no_rows_hands_the_windows_on(ctx):
    g = np.random.default_rng(3)
    c = Conv(g, [0, 0, 0], "bf16", 2, 16, 16, 1, 4)
    wout = torch.zeros(3, 3, c.ch, dtype=torch.bfloat16, device="cuda")
    x, B, C, dt = binding.str_mamba_conv_packed(ctx, dev(c.zx, "bf16"), *c.on, _i32(c.starts), *c.dims, window=dev(c.window, "bf16"), window_out=wout)
    assert x.shape == (0, 2, 16) and dt.shape == (0, 2) and np.array_equal(_f64(wout), c.window)


@pytest.mark.parametrize("dtype, W, dims", CONV)
@pytest.mark.parametrize("Bz, T", [(1, 1), (3, 1), (5, 2), (2, 7)])
def test_convolution_of_single_tokens(ctx, dtype, W, dims, Bz, T):
    g = np.random.default_rng([W, Bz, T])
    c = Conv(g, [T] * Bz, dtype, *dims, W)
    window = dev(c.window, dtype)
    zx, wout = dev(c.zx, dtype), torch.zeros_like(window)
    got = binding.str_mamba_conv_step(ctx, zx, *c.on, window, Bz, T, *dims, window_out=wout)
    c.check([t.flatten(0, 1) for t in got], wout, c.window)
    assert torch.equal(window, dev(c.window, dtype))
    again = binding.str_mamba_conv_step(ctx, zx, *c.on, window, Bz, T, *dims)                       # in place
    assert torch.equal(window, wout) and all(torch.equal(a, b) for a, b in zip(got, again))
    rows = binding.str_mamba_conv_packed(ctx, zx, *c.on, _i32(c.starts), *dims, window=dev(c.window, dtype), window_out=wout)
    assert torch.equal(window, wout) and all(torch.equal(a.flatten(0, 1), b) for a, b in zip(got, rows))


@pytest.mark.parametrize("off", [1, 2, 4])
def test_convolution_at_addresses_that_allow_no_vectors(ctx, off):
    g = np.random.default_rng(off)
    c = Conv(g, [5, 40], "bf16", 2, 16, 16, 1, 4)
    flat = torch.zeros(c.zx.size + off, dtype=torch.bfloat16, device="cuda")
    flat[off:] = dev(c.zx, "bf16").flatten()
    zx = flat[off:].view(c.zx.shape)
    got = binding.str_mamba_conv_packed(ctx, zx, *c.on, _i32(c.starts), *c.dims, window=dev(c.window, "bf16"))
    want = binding.str_mamba_conv_packed(ctx, dev(c.zx, "bf16"), *c.on, _i32(c.starts), *c.dims, window=dev(c.window, "bf16"))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    c.check(got, None, c.window)


def test_convolution_of_one_prompt_is_that_of_the_unpacked_call(ctx):
    g = np.random.default_rng(5)
    c = Conv(g, [200], "bf16", 8, 64, 128, 2, 4)
    zx = dev(c.zx, "bf16")
    a = binding.str_mamba_conv_packed(ctx, zx, *c.on, _i32(c.starts), *c.dims)
    b = binding.str_mamba_conv_split(ctx, zx, *c.on, 1, 200, *c.dims)
    assert all(torch.equal(x, y[0]) for x, y in zip(a, b))


def test_values_that_are_not_finite_stay_in_their_channel_and_reach(ctx):
    g = np.random.default_rng(6)
    c = Conv(g, [6, 9], "bf16", 2, 16, 16, 1, 4)
    clean = binding.str_mamba_conv_packed(ctx, dev(c.zx, "bf16"), *c.on, _i32(c.starts), *c.dims)
    c.zx[4, c.d_inner + 3] = np.nan                       # rows 4, 5 of channel 3: the next sequence begins at row 6
    dirty = binding.str_mamba_conv_packed(ctx, dev(c.zx, "bf16"), *c.on, _i32(c.starts), *c.dims)
    hit = torch.zeros_like(clean[0], dtype=torch.bool)
    hit[4:6, 0, 3] = True
    assert torch.equal(dirty[0].isnan(), hit) and torch.equal(dirty[0][~hit], clean[0][~hit])
    assert all(torch.equal(a, b) for a, b in zip(clean[1:], dirty[1:]))


# ------------------------------------------------------------------------------------------------ scan
class Scan:
    def __init__(self, g, lens, dtype, H, p, n, G, skip, state, first=0, tail=0, decay=16.0):
        self.lens, self.dtype, self.starts = lens, dtype, _starts(lens, first)
        rows = self.starts[-1] + tail
        self.x, self.B, self.C = (inputs.to_grid(g.standard_normal(s), dtype) for s in ((rows, H, p), (rows, G, n), (rows, G, n)))
        self.dt = (0.001 * 100.0 ** g.random((rows, H))).astype(np.float32)
        self.A = -np.exp(math.log(decay) * g.random(H)).astype(np.float32)
        self.D = g.standard_normal(H).astype(np.float32) if skip else None
        self.state = g.standard_normal((len(lens), H, p, n)).astype(np.float32) if state else None
        for a in (self.x, self.B, self.C, self.dt):
            a[:first] = np.nan
            a[self.starts[-1]:] = np.nan

    def run(self, ctx, final=True, out=True):
        y = torch.full(self.x.shape, UNTOUCHED, dtype=TORCH[self.dtype], device="cuda") if out else None
        fs = torch.full((len(self.lens), *self.x.shape[1:], self.B.shape[2]), UNTOUCHED, device="cuda") if final else None
        opt = lambda a: None if a is None else dev(a)  # noqa: E731
        return binding.str_mamba2_prefill_packed(ctx, dev(self.x, self.dtype), dev(self.dt), dev(self.A), dev(self.B, self.dtype), dev(self.C, self.dtype),
                                                 _i32(self.starts), D=opt(self.D), init_state=opt(self.state), final_state=fs, out=y)

    def check(self, got):
        y, ymag, S, Smag = packed.scan(self.x, self.dt, self.A, self.B, self.C, self.D, self.starts, self.state)
        walk = (max(self.lens) + 64) * 2.0 ** -21
        rel = 2 * HALF["bf16"] + 2.0 ** -12 + walk if self.dtype == "bf16" else walk
        _close(got[0], y, rel * ymag + HALF[self.dtype] * np.abs(y) + 1e-30, "y")
        _close(got[1], S, (2.0 ** -16 + walk if self.dtype == "bf16" else walk) * Smag + 1e-30, "state")


SCAN = [("bf16", (4, 64, 128, 2)), ("bf16", (2, 64, 128, 1)), ("bf16", (3, 32, 64, 3)), ("bf16", (2, 16, 16, 1)), ("bf16", (2, 80, 20, 2)), ("bf16", (1, 64, 200, 1)),
        ("f32", (6, 32, 20, 3)), ("f32", (2, 64, 128, 1)), ("f32", (1, 5, 3, 1))]
SCAN_LENS = [[1], [130], [0, 1, 2, 127, 128, 129, 0, 385], [0, 0], [257, 3]]


@pytest.mark.parametrize("skip, state", [(False, False), (True, True), (False, True), (True, False)])
@pytest.mark.parametrize("lens", SCAN_LENS, ids=str)
@pytest.mark.parametrize("dtype, dims", SCAN)
def test_scan_over_ragged_sequences(ctx, dtype, dims, lens, skip, state):
    g = np.random.default_rng([len(lens), sum(lens), int(skip), int(state)])
    c = Scan(g, lens, dtype, *dims, skip, state, *((0, 0) if skip else (3, 7)))
    if len(c.x):
        c.check(c.run(ctx))


@pytest.mark.parametrize("decay", [1e-3, 1e4])
def test_scan_of_slow_and_fast_decays(ctx, decay):
    g = np.random.default_rng(9)
    c = Scan(g, [300, 77], "bf16", 4, 64, 128, 2, True, True, decay=decay)
    if decay < 1:
        c.A = -(g.random(4) * decay).astype(np.float32)
    c.check(c.run(ctx))


def test_scan_of_many_sequences_and_many_heads(ctx):
    g = np.random.default_rng(10)
    c = Scan(g, [int(v) for v in g.integers(0, 9, 300)], "bf16", 5, 64, 128, 5, False, True)
    c.check(c.run(ctx))
    c = Scan(g, [40], "bf16", 256, 64, 128, 8, True, False)
    c.check(c.run(ctx))


def test_scan_in_place_without_final_states_and_the_same_bits(ctx):
    g = np.random.default_rng(11)
    for dtype, dims in (("bf16", (4, 64, 128, 2)), ("f32", (4, 32, 20, 2))):
        c = Scan(g, [200, 0, 131], dtype, *dims, False, True)
        y, S = c.run(ctx)
        assert torch.equal(c.run(ctx, final=False, out=False)[:331], y)
        state = dev(c.state)
        args = (dev(c.x, dtype), dev(c.dt), dev(c.A), dev(c.B, dtype), dev(c.C, dtype), _i32(c.starts))
        y2, S2 = binding.str_mamba2_prefill_packed(ctx, *args, init_state=state, final_state=state)
        assert S2 is state and torch.equal(S2, S) and torch.equal(y2, y)


def test_scan_in_two_turns_continues_the_first(ctx):
    """The second turn starts from the first one's states: the bounds of the oracle's one run hold for both together."""
    g = np.random.default_rng(12)
    lens, cut = [300, 140], [170, 128]
    c = Scan(g, lens, "bf16", 4, 64, 128, 2, True, False)
    rows = [np.r_[0:170, 300:428], np.r_[170:300, 428:440]]
    fs, ys = None, []
    for turn, ls in zip(rows, (cut, [a - b for a, b in zip(lens, cut)])):
        y, fs = binding.str_mamba2_prefill_packed(ctx, dev(c.x[turn], "bf16"), dev(c.dt[turn]), dev(c.A), dev(c.B[turn], "bf16"), dev(c.C[turn], "bf16"),
                                                  _i32(_starts(ls)), D=dev(c.D), init_state=fs, final_state=torch.zeros(2, 4, 64, 128, device="cuda"))
        ys.append(y)
    whole = torch.empty_like(ys[0][:0].new_empty((440, 4, 64)))
    for turn, y in zip(rows, ys):
        whole[torch.from_numpy(turn).cuda()] = y
    c.check((whole, fs))


def test_final_states_of_sequences_whose_last_tokens_count(ctx):
    """Decays so fast that a state is its last few tokens: every term of it is a product of three bf16 pieces at most 2^-24 off, added up in 24 steps
    of the matrix instruction that may each lose 2^-24 of the sum: 2^-19 of the sum of absolute terms (the factor's two largest pieces alone would be
    2^-16 off)."""
    g = np.random.default_rng(14)
    for lens in ([300, 129, 20], [64]):
        c = Scan(g, lens, "bf16", 4, 64, 128, 2, False, True)
        c.A[:] = -1.0e4
        _, S = c.run(ctx)
        _, _, want, mag = packed.scan(c.x, c.dt, c.A, c.B, c.C, None, c.starts, c.state)
        assert (np.abs(_f64(S) - want) <= 2.0 ** -19 * mag + 1e-30).all()


def test_scan_of_short_and_long_sequences_side_by_side(ctx):
    """Averages on both sides of the length from which the chunked kernel is taken, with and without decay to fade a chunk."""
    g = np.random.default_rng(15)
    for lens in ([16, 16], [17, 16], [32, 32], [33, 32], [1, 40, 2], [500, 0, 1, 3, 2]):
        for decay in (1e-3, 16.0):
            c = Scan(g, lens, "bf16", 3, 64, 128, 1, True, True, decay=max(decay, 1.0))
            if decay < 1:
                c.A[:] = -decay
            c.check(c.run(ctx))


def test_scan_before_a_value_that_is_not_finite(ctx):
    """Tokens before it are as they would be without it; its own and later ones of its column are not finite."""
    g = np.random.default_rng(16)
    for value in (np.nan, np.inf):
        c = Scan(g, [200], "bf16", 2, 64, 128, 1, True, True)
        clean = _f64(c.run(ctx)[0])
        c.x[150, 1, 7] = value
        y, S = (_f64(t) for t in c.run(ctx))
        ref, ymag, _, _ = packed.scan(c.x[:150], c.dt[:150], c.A, c.B[:150], c.C[:150], c.D, [0, 150], c.state)
        rel = 2 * HALF["bf16"] + 2.0 ** -12 + 264 * 2.0 ** -21
        assert (np.abs(y[:150] - ref) <= rel * ymag + HALF["bf16"] * np.abs(ref)).all()
        assert not np.isfinite(y[150:, 1, 7]).any() and np.isfinite(np.delete(y[:, 1], 7, 1)).all() and (y[:, 0] == clean[:, 0]).all()
        assert not np.isfinite(S[0, 1, 7]).any() and np.isfinite(np.delete(S[0, 1], 7, 0)).all()


def test_scan_does_not_carry_what_is_not_finite_into_other_sequences(ctx):
    g = np.random.default_rng(13)
    for dims in ((4, 64, 128, 2), (2, 80, 20, 2)):
        c = Scan(g, [100, 60, 90], "bf16", *dims, True, True)
        y, S = c.run(ctx)
        c.x[130, 0, 3], c.B[131, 0, 5], c.dt[140, 1] = np.nan, np.inf, np.nan
        y2, S2 = c.run(ctx)
        for a, b in ((y[:100], y2[:100]), (y[160:], y2[160:]), (S[[0, 2]], S2[[0, 2]])):
            assert torch.equal(a, b)
        assert S2[1].isnan().any()


def _segmented(c):
    """Does the call cut its sequences into segments (it then asks for a workspace)?"""
    import ctypes
    rows, H, p = c.x.shape
    s = binding.SsdPackedShape(len(c.lens), rows, H, p, c.B.shape[2], c.B.shape[1], 1 if c.dtype == "bf16" else 0)
    return binding.lib().str_mamba2_prefill_packed_workspace_size(ctypes.addressof(s)) > 0


LONG_SCAN = [("bf16", (2, 64, 128, 1), [3000]), ("bf16", (4, 32, 64, 2), [2561, 0, 1, 130, 4000]), ("bf16", (1, 16, 16, 1), [1281]), ("bf16", (2, 80, 20, 2), [700, 0, 1]),
             ("f32", (6, 32, 20, 3), [0, 483, 1, 200]), ("f32", (2, 64, 128, 1), [640]), ("f32", (1, 5, 3, 1), [65, 64, 900, 63]), ("f32", (1, 70, 200, 1), [515])]


@pytest.mark.parametrize("skip, state", [(False, False), (True, True)])
@pytest.mark.parametrize("dtype, dims, lens", LONG_SCAN, ids=str)
def test_scan_of_long_sequences_of_few_heads(ctx, dtype, dims, lens, skip, state):
    """Sequences that are walked in segments: as many rows as a segment, one more, empty ones between, rows of nobody around."""
    g = np.random.default_rng([dims[0], sum(lens), int(skip)])
    c = Scan(g, lens, dtype, *dims, skip, state, *((0, 0) if skip else (3, 7)))
    assert _segmented(c)
    y, S = c.run(ctx)
    c.check((y, S))
    assert torch.equal(c.run(ctx, final=False)[: len(c.x)], y)
    if state:
        at = dev(c.state)
        y2, S2 = binding.str_mamba2_prefill_packed(ctx, dev(c.x, dtype), dev(c.dt), dev(c.A), dev(c.B, dtype), dev(c.C, dtype), _i32(c.starts), D=dev(c.D), init_state=at, final_state=at)
        assert S2 is at and torch.equal(S2, S) and torch.equal(y2, y)


@pytest.mark.parametrize("decay", [1e-4, 1e4])
@pytest.mark.parametrize("dtype, dims, lens", [LONG_SCAN[0], LONG_SCAN[4]], ids=str)
def test_segments_of_slow_and_fast_decays(ctx, dtype, dims, lens, decay):
    """Everything from segment to segment, and nothing."""
    g = np.random.default_rng(17)
    c = Scan(g, lens, dtype, *dims, True, True)
    c.A[:] = -decay
    assert _segmented(c)
    c.check(c.run(ctx))


@pytest.mark.parametrize("dtype, dims, lens, at", [("bf16", (2, 64, 128, 1), [1500], 700), ("f32", (2, 32, 20, 1), [500], 300)], ids=str)
def test_segments_before_a_value_that_is_not_finite(ctx, dtype, dims, lens, at):
    """Tokens of earlier segments, and of the same one before the value, are as they would be without it; later ones of its column are not finite."""
    g = np.random.default_rng(18)
    c = Scan(g, lens, dtype, *dims, True, True)
    assert _segmented(c)
    clean = c.run(ctx)
    c.check(clean)
    for value in (np.nan, np.inf):
        c.x[at, 1, 7] = value
        y, S = (_f64(t) for t in c.run(ctx))
        ref, ymag, _, _ = packed.scan(c.x[:at], c.dt[:at], c.A, c.B[:at], c.C[:at], c.D, [0, at], c.state)
        walk = (lens[0] + 64) * 2.0 ** -21
        rel = 2 * HALF["bf16"] + 2.0 ** -12 + walk if dtype == "bf16" else walk
        assert (np.abs(y[:at] - ref) <= rel * ymag + HALF[dtype] * np.abs(ref)).all()
        assert not np.isfinite(y[at:, 1, 7]).any() and np.isfinite(np.delete(y[:, 1], 7, 1)).all() and (y[:, 0] == _f64(clean[0])[:, 0]).all()
        assert not np.isfinite(S[0, 1, 7]).any() and np.isfinite(np.delete(S[0, 1], 7, 0)).all()


def test_segments_in_two_graphs_at_once_and_the_same_bits(ctx):
    g = np.random.default_rng(19)
    for dtype, dims, lens in (LONG_SCAN[0], LONG_SCAN[4]):
        runs = []
        for _ in range(2):
            c = Scan(g, lens, dtype, *dims, False, True)
            args = (dev(c.x, dtype), dev(c.dt), dev(c.A), dev(c.B, dtype), dev(c.C, dtype), _i32(c.starts))
            init, final = dev(c.state), dev(c.state)
            call = lambda args=args, init=init, final=final: binding.str_mamba2_prefill_packed(ctx, *args, init_state=init, final_state=final)  # noqa: E731
            want = [t.clone() for t in call()]
            final.zero_()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                got = call()
            runs.append((graph, torch.cuda.Stream(), got, want, args, init))
        for _ in range(4):
            for graph, stream, *_ in runs:
                with torch.cuda.stream(stream):
                    graph.replay()
        torch.cuda.synchronize()
        for _, _, got, want, _, _ in runs:
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


@pytest.mark.parametrize("starts", [[0, 900, 200], [-3, 10, 4000000], [0, 2147483647, 2147483647], [1400, 1400, -2147483648], [1500, 0, 1500]], ids=str)
def test_wrong_starts_of_segments(ctx, starts):
    g = np.random.default_rng(20)
    for dtype, dims in (("bf16", (2, 64, 128, 1)), ("f32", (2, 32, 20, 1))):
        c = Scan(g, [1400, 1500], dtype, *dims, False, True)
        assert _segmented(c)
        right, c.starts = c.starts, starts
        c.run(ctx)
        with pytest.raises(binding.StrError):
            ctx.check_status()
        ctx.check_status()
        c.starts = right
        c.check(c.run(ctx))


@pytest.mark.parametrize("dtype, dims, lens", [("f32", (2, 32, 16, 1), [40]), ("f32", (2, 64, 128, 1), [40]), ("bf16", (2, 64, 128, 1), [20]), ("bf16", (2, 80, 32, 1), [150]),
                                               ("bf16", (2, 64, 128, 1), [200])], ids=str)
def test_scan_of_an_infinite_value_with_and_without_skip(ctx, dtype, dims, lens):
    """Positive B and C: the state's row is infinite from the value on, and y with it.  A skip of zero multiplies the value, no skip does not."""
    g = np.random.default_rng(32)
    c = Scan(g, lens, dtype, *dims, False, True)
    c.B, c.C, c.state = np.abs(c.B) + 1.0, np.abs(c.C) + 1.0, np.abs(c.state)
    c.B, c.C = inputs.to_grid(c.B, dtype), inputs.to_grid(c.C, dtype)
    c.x[11, 1, 7] = np.inf
    y, S = (_f64(t) for t in c.run(ctx))
    assert (y[11:, 1, 7] == np.inf).all() and np.isfinite(y[:11]).all() and (S[0, 1, 7] == np.inf).all()
    c.D = np.zeros(dims[0], dtype=np.float32)
    z, _ = (_f64(t) for t in c.run(ctx))
    assert np.isnan(z[11, 1, 7]) and (z[12:, 1, 7] == np.inf).all() and np.array_equal(np.delete(z[:, 1], 7, 1), np.delete(y[:, 1], 7, 1))


@pytest.mark.parametrize("decay", [1e5, 1e6, 1e30])
@pytest.mark.parametrize("dims, lens", [((4, 64, 128, 2), [300, 77]), ((3, 32, 64, 3), [40, 128]), ((2, 64, 128, 1), [3000])], ids=str)
def test_scan_whose_tokens_fade_all_before_them(ctx, dims, lens, decay):
    """Decays beyond what a sum of logarithms in fp32 could keep apart: y is each token's own term, with the bound of any other scan."""
    g = np.random.default_rng(33)
    c = Scan(g, lens, "bf16", *dims, True, True)
    c.A[:] = -decay
    c.check(c.run(ctx))
    c.A[1:] = -0.01                                              # heads side by side, and tokens within one
    c.dt[::5] = 1e-12
    c.check(c.run(ctx))


@pytest.mark.parametrize("dims, lens", [((148, 64, 16, 1), [512, 0, 200]), ((2, 64, 128, 1), [1500])], ids=str)
def test_final_states_that_nothing_fades_take_all_pieces_in_every_chunk(ctx, dims, lens):
    """No decay, and of a chunk's tokens four equal ones that count: rounding errors of a term's pieces add up instead of averaging out, and few products are cut
    off where they meet the sum.  Two pieces alone would be up to 1.4e-5 of the sum off (worked out on the host below).  With the third the terms are right to
    2^-24; a chunk's 12 products and 24 steps of the sum lose 2^-23 of it each at most, the sum over the chunks 2^-24 a chunk."""
    g = np.random.default_rng(36)
    c = Scan(g, lens, "bf16", *dims, False, False)
    assert _segmented(c) == (len(lens) == 1)
    c.x[:], c.B[:], c.A[:] = inputs.to_grid(g.standard_normal(64), "bf16"), 1.0, 0.0
    dt = (0.001 * 100.0 ** g.random(dims[0])).astype(np.float32)
    c.dt[:] = np.where((np.arange(len(c.dt)) % 32 == 5)[:, None], dt, np.float32(1e-30))
    bound = 36 * 2.0 ** -23 + 13 * 2.0 ** -24
    bf = lambda a: inputs.to_grid(np.asarray(a, dtype=np.float64), "bf16").astype(np.float64)  # noqa: E731
    x, w = c.x[0].astype(np.float64), dt.astype(np.float64)[:, None]
    w1 = bf(w)
    high = bf(x * w1)
    two = high + bf(x * bf(w - w1) + (x * w1 - high))
    assert (np.abs(two - x * w) > 2 * bound * np.abs(x * w)).any()
    _, S = c.run(ctx)
    _, _, want, mag = packed.scan(c.x, c.dt, c.A, c.B, c.C, None, c.starts, None)
    assert (np.abs(_f64(S) - want) <= bound * mag).all()


# ------------------------------------------------------------------------------------------------ attention
class Attend:
    def __init__(self, g, lq, lk, dtype, Hq, Hkv, d, first=(0, 0), tail=0, gain=1.0):
        self.dtype, self.d = dtype, d
        self.qs, self.ks = _starts(lq, first[0]), _starts(lk, first[1])
        rq, rk = self.qs[-1] + tail, self.ks[-1] + tail
        self.q = inputs.to_grid(gain * g.standard_normal((rq, Hq, d)), dtype)
        self.k, self.v = (inputs.to_grid(g.standard_normal((rk, Hkv, d)), dtype) for _ in range(2))
        self.scale = d ** -0.5
        self.q[:first[0]] = self.q[self.qs[-1]:] = np.nan
        for a in (self.k, self.v):
            a[:first[1]] = a[self.ks[-1]:] = np.nan

    def run(self, ctx, **kw):
        o = torch.full(self.q.shape, UNTOUCHED, dtype=TORCH[self.dtype], device="cuda")
        return binding.str_attn_prefill_packed(ctx, *(dev(a, self.dtype) for a in (self.q, self.k, self.v)), _i32(self.qs), self.scale, k_start=_i32(self.ks), out=o, **kw)

    def check(self, o):
        want, mag, largest = packed.attention(self.q, self.k, self.v, self.qs, self.ks, self.scale)
        n = max([b - a for a, b in zip(self.ks, self.ks[1:])] + [1])
        rel = 2 * (self.d + 64) * E * largest + n * E + 2.0 ** -12 + (HALF["bf16"] if self.dtype == "bf16" else 0.0)
        if self.dtype == "f32":
            rel += 32 * E - 2.0 ** -12
        _close(o, want, rel * mag + HALF[self.dtype] * np.abs(want) + 1e-30, "o")


TURNS = [([1], [1]), ([5], [3]), ([129], [129]), ([64, 0, 65, 1, 200], [64, 0, 65, 1, 200]), ([3, 1, 70, 2], [300, 129, 70, 0]), ([257], [128]), ([2, 2], [255, 256]),
         ([0], [7]), ([4], [0])]


@pytest.mark.parametrize("lq, lk", TURNS, ids=str)
@pytest.mark.parametrize("dtype, Hq, Hkv, d", [("bf16", 8, 2, 128), ("bf16", 3, 1, 64), ("bf16", 2, 2, 80), ("bf16", 8, 1, 128), ("bf16", 5, 5, 16), ("bf16", 2, 1, 20),
                                                ("f32", 3, 1, 64), ("f32", 4, 2, 128), ("f32", 2, 1, 7)])
def test_attention_over_ragged_sequences(ctx, dtype, Hq, Hkv, d, lq, lk):
    g = np.random.default_rng([Hq, d, sum(lq), sum(lk)])
    for first, tail in (((0, 0), 0), ((2, 3), 5)):
        c = Attend(g, lq, lk, dtype, Hq, Hkv, d, first, tail)
        if len(c.q):
            c.check(c.run(ctx))


def _long_reference(q, k, v, scale):
    """The last lq of lk rows in fp64 on the device: (o, sum p |v|, largest sum |q_c k_c| scale)."""
    lq, Hq, d = q.shape
    lk, Hkv, _ = k.shape
    o, mag, largest = torch.zeros(lq, Hq, d, dtype=torch.float64, device="cuda"), torch.zeros(lq, Hq, d, dtype=torch.float64, device="cuda"), 0.0
    hidden = torch.arange(lk, device="cuda") > lk - lq + torch.arange(lq, device="cuda")[:, None]
    for h in range(Hq):
        K, V, Q = (t[:, i].double() for t, i in ((k, h * Hkv // Hq), (v, h * Hkv // Hq), (q, h)))
        p = torch.softmax((Q @ K.T * scale).masked_fill(hidden, float("-inf")), 1)
        o[:, h], mag[:, h] = p @ V, p @ V.abs()
        largest = max(largest, float((Q.abs() @ K.abs().T).max()) * scale)
    return o, mag, largest


@pytest.mark.parametrize("dtype, lq, lk, Hq, Hkv, d, gain", [("bf16", 1000, 9001, 8, 2, 128, 1.0), ("bf16", 2500, 2500, 4, 4, 128, 3.0), ("bf16", 3, 12345, 8, 2, 64, 1.0),
                                                              ("bf16", 700, 4100, 6, 2, 64, 6.0), ("bf16", 1111, 1111, 16, 1, 96, 1.0), ("f32", 500, 3001, 3, 1, 64, 2.0),
                                                              ("f32", 333, 1000, 4, 1, 128, 1.0)])
def test_attention_over_long_sequences(ctx, dtype, lq, lk, Hq, Hkv, d, gain):
    g = torch.Generator(device="cuda").manual_seed(lq)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda").to(TORCH[dtype])  # noqa: E731
    q, k, v = (gain * rand(lq, Hq, d)).to(TORCH[dtype]), rand(lk, Hkv, d), rand(lk, Hkv, d)
    o = binding.str_attn_prefill_packed(ctx, q, k, v, _i32([0, lq]), d ** -0.5, k_start=_i32([0, lk]))
    want, mag, largest = _long_reference(q, k, v, d ** -0.5)
    rel = 2 * (d + 64) * E * largest + lk * E + (2.0 ** -12 + HALF["bf16"] if dtype == "bf16" else 32 * E)
    bad = (o.double() - want).abs() > rel * mag + HALF[dtype] * want.abs()
    assert not bad.any(), (int(bad.sum()), bad.nonzero()[:3].tolist(), float((o.double() - want).abs().max()))


@pytest.mark.parametrize("dtype, d", [("bf16", 128), ("bf16", 64), ("bf16", 20), ("f32", 64)])
def test_attention_of_scores_that_grow_and_fall_along_the_row(ctx, dtype, d):
    """The running maximum moves at almost every key, by little and by much, and at the last."""
    g = np.random.default_rng(21)
    for step in (0.25, 3.0, -0.5):
        c = Attend(g, [300], [300], dtype, 2, 1, d)
        c.q[:] = 1.0
        c.k[:] = inputs.to_grid((step * np.arange(300) / d)[:, None, None] * np.ones((1, 1, d)), dtype)
        c.scale = 1.0
        c.check(c.run(ctx))


@pytest.mark.parametrize("dtype, Hq, Hkv, d", [("bf16", 8, 2, 128), ("bf16", 2, 1, 64), ("bf16", 2, 1, 20), ("f32", 3, 1, 64)])
def test_attention_hidden_keys_that_are_not_finite_do_not_reach_the_queries_before_them(ctx, dtype, Hq, Hkv, d):
    g = np.random.default_rng(22)
    c = Attend(g, [150, 40], [400, 40], dtype, Hq, Hkv, d)
    clean = c.run(ctx)
    for where, value, at in (("v", np.nan, 330), ("v", np.inf, 399), ("k", np.nan, 300), ("k", np.inf, 380), ("v", -np.inf, 400 + 17)):
        old = getattr(c, where).copy()
        getattr(c, where)[at, 0, d // 2] = value
        o = c.run(ctx)
        s, first = (0, 250) if at < 400 else (1, 400)                  # the key's own query, and those after it, see it
        own = c.qs[s] + at - first
        keep = torch.ones(190, dtype=torch.bool)
        keep[own:c.qs[s + 1]] = False
        heads = slice(0, Hq // Hkv)
        tol = 2 * HALF[dtype] * clean.double().abs() + (2.0 ** -8 if dtype == "bf16" else 2.0 ** -18)
        assert ((o.double() - clean.double()).abs() <= tol)[keep].all(), (where, value, at)
        touched = o[own:c.qs[s + 1], heads].double()
        assert (~torch.isfinite(touched)).any(-1).all() if where == "v" else True
        if where == "k" and np.isnan(value):
            assert touched.isnan().all()
        setattr(c, where, old)


def _shared(c):
    """Does the call share a block's keys out to several CTAs (it then asks for a workspace)?"""
    s = binding.AttnPackedShape(len(c.qs) - 1, len(c.q), len(c.k), c.q.shape[1], c.k.shape[1], c.d, 1)
    import ctypes
    return binding.lib().str_attn_prefill_packed_workspace_size(ctypes.addressof(s)) > 0


@pytest.mark.parametrize("Hq, Hkv, d", [(4, 1, 128), (3, 1, 64), (2, 2, 80), (16, 1, 128)])
@pytest.mark.parametrize("lq, lk", [([3], [2100]), ([40, 1], [1500, 2600]), ([70, 0, 5], [3000, 1200, 2]), ([300], [1100]), ([9, 9], [4000, 6])], ids=str)
def test_attention_whose_keys_are_shared_out(ctx, Hq, Hkv, d, lq, lk):
    """Few queries over many keys: shares that some or all rows of a block see nothing of, sequences with fewer keys than queries or than shares."""
    g = np.random.default_rng([Hq, d, sum(lk)])
    c = Attend(g, lq, lk, "bf16", Hq, Hkv, d, (2, 3), 5, gain=2.0)
    assert _shared(c) or Hq == 16
    c.check(c.run(ctx))


def test_attention_shared_out_with_values_that_are_not_finite(ctx):
    g = np.random.default_rng(26)
    c = Attend(g, [20, 4], [2000, 1500], "bf16", 4, 1, 128)
    assert _shared(c)
    clean = c.run(ctx)
    for where, value, at, seen_by in (("v", np.nan, 1990, range(10, 20)), ("v", np.inf, 100, range(20)), ("k", np.nan, 1985, range(5, 20)), ("v", np.nan, 3499, range(23, 24))):
        old = getattr(c, where).copy()
        getattr(c, where)[at, 0, 5] = value
        o = c.run(ctx)
        hit = torch.zeros(24, dtype=torch.bool)
        hit[list(seen_by)] = True
        assert ((o.double() - clean.double()).abs() <= 2 * HALF["bf16"] * clean.double().abs() + 2.0 ** -8)[~hit].all(), (where, at)
        assert (~torch.isfinite(o[hit].double())).any(-1).all()
        setattr(c, where, old)
    c.q[3, 2, 0] = np.inf
    assert c.run(ctx)[3, 2].isnan().all()


def test_attention_shared_out_in_two_graphs_at_once_and_the_same_bits(ctx):
    g = np.random.default_rng(27)
    c = Attend(g, [30], [3000], "bf16", 8, 2, 128)
    assert _shared(c)
    q, k, v = (dev(a, "bf16") for a in (c.q, c.k, c.v))
    other = [t.flip(0).contiguous() for t in (q, k, v)]
    qs, ks = _i32(c.qs), _i32(c.ks)
    call = lambda t: binding.str_attn_prefill_packed(ctx, *t, qs, c.scale, k_start=ks)  # noqa: E731
    want = [call((q, k, v)).clone(), call(other).clone()]
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for t in ((q, k, v), other):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = call(t)
        graphs.append((graph, out))
    for _ in range(5):
        for (graph, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for (_, out), w in zip(graphs, want):
        assert torch.equal(out, w)


@pytest.mark.parametrize("starts", [[0, 30, 10], [-3, 10, 4000], [40, 40, -2147483648]], ids=str)
def test_wrong_starts_with_keys_shared_out(ctx, starts):
    g = np.random.default_rng(28)
    c = Attend(g, [20, 20], [1500, 1500], "bf16", 4, 1, 128)
    assert _shared(c)
    q, k, v = (dev(a, "bf16") for a in (c.q, c.k, c.v))
    for qs, ks in ((starts, c.ks), (c.qs, starts)):
        binding.str_attn_prefill_packed(ctx, q, k, v, _i32(qs), 0.1, k_start=_i32(ks))
        with pytest.raises(binding.StrError):
            ctx.check_status()
    c.check(c.run(ctx))


def test_attention_rows_that_are_not_finite_stay_by_themselves(ctx):
    g = np.random.default_rng(23)
    for dtype, d in (("bf16", 128), ("f32", 64)):
        c = Attend(g, [90], [90], dtype, 4, 2, d)
        clean = c.run(ctx)
        c.q[50, 1, 3] = np.nan
        o = c.run(ctx)
        hit = torch.zeros(90, 4, dtype=torch.bool, device="cuda")
        hit[50, 1] = True
        assert o[50, 1].isnan().all() and torch.equal(o[~hit], clean[~hit])


def test_attention_without_key_starts_is_that_of_the_unpacked_call(ctx):
    """Equal lengths: the same function as the unpacked call on the same rows, each within its bound of the other."""
    g = torch.Generator(device="cuda").manual_seed(24)
    q, k, v = (torch.randn(3, 200, h, 128, generator=g, device="cuda").bfloat16() for h in (4, 2, 2))
    a = binding.str_attn_prefill(ctx, q, k, v, 0.1)
    b = binding.str_attn_prefill_packed(ctx, *(t.flatten(0, 1) for t in (q, k, v)), _i32([0, 200, 400, 600]), 0.1)
    assert (a.flatten(0, 1).double() - b.double()).abs().max() <= 2.0 ** -6


@pytest.mark.parametrize("Hq, Hkv, d", [(4, 2, 128), (3, 3, 80), (6, 2, 100)])
def test_fp32_attention_of_few_and_of_many_blocks_of_wide_heads(ctx, Hq, Hkv, d):
    """Blocks of 64 rows and of 128."""
    g = np.random.default_rng(26)
    for lens in ([200, 0, 65], [int(v) for v in g.integers(0, 5, 160)] + [70, 300]):
        c = Attend(g, lens, [v + int(w) for v, w in zip(lens, g.integers(0, 90, len(lens)))], "f32", Hq, Hkv, d, (1, 2), 3)
        c.check(c.run(ctx))


def test_attention_of_many_sequences_and_groups_as_large_as_a_block(ctx):
    g = np.random.default_rng(25)
    lens = [int(v) for v in g.integers(0, 6, 500)]
    c = Attend(g, lens, [v + int(w) for v, w in zip(lens, g.integers(0, 3, 500))], "bf16", 2, 1, 64)
    c.check(c.run(ctx))
    for R in (32, 100, 128):
        for dtype in ("bf16", "f32"):
            c = Attend(g, [5, 2], [9, 140], dtype, R, 1, 64)
            c.check(c.run(ctx))


def test_attention_of_no_keys_at_all(ctx):
    q = torch.randn(5, 2, 64, device="cuda")
    for t in (torch.float32, torch.bfloat16):
        o = binding.str_attn_prefill_packed(ctx, q.to(t), *(torch.zeros(0, 1, 64, dtype=t, device="cuda"),) * 2, _i32([0, 5]), 0.1, k_start=_i32([0, 0]))
        assert (o == 0).all()
    assert binding.str_attn_prefill_packed(ctx, q[:0], q[:0], q[:0], _i32([0, 0]), 0.1).shape == (0, 2, 64)


HUGE = {"bf16": 3.3e38, "f32": 3.4e38}


@pytest.mark.parametrize("lq, lk", [([200], [200]), ([150, 40], [400, 40]), ([5, 9], [140, 0]), ([20], [2000]), ([9, 9], [4000, 6])], ids=str)
@pytest.mark.parametrize("dtype, Hq, Hkv, d", [("bf16", 8, 2, 128), ("bf16", 2, 1, 64), ("bf16", 3, 3, 80), ("bf16", 2, 1, 20), ("f32", 3, 1, 64)])
def test_attention_hidden_values_of_the_largest_magnitude_weigh_nothing(ctx, dtype, Hq, Hkv, d, lq, lk):
    """The second half of each sequence's queries see such values, the first half's rows have the bits that they have without them."""
    g = np.random.default_rng([29, Hq, d])
    c = Attend(g, lq, lk, dtype, Hq, Hkv, d)
    assert dtype == "f32" or d == 20 or Hq == 8 or lk[0] < 2000 or _shared(c)
    clean = c.run(ctx)
    keep = torch.zeros(sum(lq), dtype=torch.bool)
    for s, (a, b) in enumerate(zip(lq, lk)):
        keep[c.qs[s]:c.qs[s] + a - a // 2] = True
        c.v[max(c.ks[s], c.ks[s + 1] - a // 2):c.ks[s + 1]] = inputs.to_grid(np.array(HUGE[dtype]), dtype)
    assert torch.equal(c.run(ctx)[keep], clean[keep])
    c.v[:] = np.where(np.abs(c.v) > 1e38, -c.v, c.v)
    assert torch.equal(c.run(ctx)[keep], clean[keep])


@pytest.mark.parametrize("lq, lk", [([200], [200]), ([7], [300]), ([3], [2100])], ids=str)
@pytest.mark.parametrize("dtype, Hq, Hkv, d", [("bf16", 4, 1, 128), ("bf16", 2, 1, 64), ("bf16", 2, 1, 20), ("f32", 3, 1, 64)])
def test_attention_values_whose_weights_underflow_weigh_nothing(ctx, dtype, Hq, Hkv, d, lq, lk):
    """Every second key is seen with a score of -640 or less below the others': exp of that is 2^-923, and times the largest value still zero."""
    g = np.random.default_rng([30, d])
    c = Attend(g, lq, lk, dtype, Hq, Hkv, d)
    c.scale = 1.0
    c.q[:], c.k[::2], c.k[1::2] = 1.0, 0.0, -32.0
    c.v[1::2] = 0.0
    clean = c.run(ctx)
    c.v[1::2] = inputs.to_grid(np.array(HUGE[dtype]), dtype)
    assert torch.equal(c.run(ctx), clean)


@pytest.mark.parametrize("lq, lk", [([150, 30], [150, 30]), ([100], [400]), ([3], [2100])], ids=str)
@pytest.mark.parametrize("dtype, Hq, Hkv, d", [("bf16", 4, 1, 128), ("bf16", 2, 1, 64), ("f32", 3, 1, 64)])
def test_attention_scores_of_minus_infinity(ctx, dtype, Hq, Hkv, d, lq, lk):
    """A row that sees nothing else has no softmax: NaN.  Beside finite scores they weigh nothing."""
    g = np.random.default_rng([31, d])
    c = Attend(g, lq, lk, dtype, Hq, Hkv, d)
    c.q[..., 0] = 1.0
    first = lk[0] // 3                                           # keys of the first sequence from here on are finite
    c.k[:first, :, 0] = -np.inf
    o = c.run(ctx)
    blind = torch.arange(lq[0]) + lk[0] - lq[0] < first
    assert o[:lq[0]][blind].isnan().all()
    c.k[:first, :, 0] = -30000.0
    assert torch.equal(c.run(ctx)[lq[0]:], o[lq[0]:]) and torch.equal(c.run(ctx)[:lq[0]][~blind], o[:lq[0]][~blind])
    c.k[..., 0] = -np.inf
    assert c.run(ctx).isnan().all()


@pytest.mark.parametrize("dtype, blocks", [("f32", 1), ("bf16", 2)])
def test_wrong_starts_that_name_more_blocks_than_an_int_counts(ctx, dtype, blocks):
    """16384 sequences of all rows each, one behind the other, in blocks of one query or two: a count that wrapped would find no block at all, or one before
    the first.  Nothing around the output is touched, and the next call is right."""
    rows, group, d = blocks * ((1 << 17) + 100), 128, 8
    q = torch.zeros(rows, group, d, dtype=TORCH[dtype], device="cuda")
    around = torch.full((rows + 2 * 4096, group, d), UNTOUCHED, dtype=TORCH[dtype], device="cuda")
    k = torch.zeros(3, 1, d, dtype=TORCH[dtype], device="cuda")
    starts = torch.zeros(32769, dtype=torch.int32, device="cuda")
    starts[1::2] = rows
    starts[1] = 1
    assert 16383 * -(-rows // blocks) + 1 > 2 ** 31
    binding.str_attn_prefill_packed(ctx, q, k, k, starts, 0.1, k_start=torch.zeros_like(starts), out=around[4096:-4096])
    with pytest.raises(binding.StrError):
        ctx.check_status()
    assert (around[:4096] == UNTOUCHED).all() and (around[-4096:] == UNTOUCHED).all() and (around[4096:4097] == 0).all()
    del q, around
    c = Attend(np.random.default_rng(35), [40, 3], [40, 90], dtype, group, 1, d)
    c.check(c.run(ctx))


# ------------------------------------------------------------------------------------------------ rotary positions
@pytest.mark.parametrize("scaling", ["none", "linear", "banded"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype, Hq, Hkv, d, rot", [("bf16", 4, 2, 128, 128), ("bf16", 3, 1, 128, 64), ("bf16", 2, 2, 80, 48), ("bf16", 1, 1, 10, 6), ("f32", 3, 1, 64, 64),
                                                     ("f32", 2, 1, 64, 20), ("f32", 1, 1, 6, 2), ("bf16", 2, 1, 256, 256)])
def test_rotary_layouts_parts_and_scalings(ctx, dtype, Hq, Hkv, d, rot, layout, scaling):
    g = np.random.default_rng([d, rot])
    for rows in (1, 7, 300):
        qkv = inputs.to_grid(g.standard_normal((rows, (Hq + 2 * Hkv) * d)), dtype)
        pos = np.concatenate(([0], g.integers(-5000000, 2 ** 31 - 1, rows)))[:rows]
        kw = dict(scaling=scaling, factor=2.5, trained_len=4096, turns=(1.0, 32.0))
        r = binding.Rope(1e4, rot, layout, amplitude=1.25, **kw)
        got = binding.str_rope_split_ex(ctx, r, dev(qkv, dtype), _i32(pos), Hq, Hkv, d)
        f = packed.rope_frequencies(1e4, rot, scaling, 2.5, 4096, (1.0, 32.0))
        want = packed.rope(qkv, pos, Hq, Hkv, d, f, layout, 1.25)
        # a frequency's own 2^-52 grows with the position: up to 2^31 * 2^-51 radians
        angle = 2.0 ** 31 * 2.0 ** -51
        heads = np.abs(qkv.reshape(rows, -1, d))
        mag = 1.25 * 2 * heads.max(-1, keepdims=True)
        for t, w, m in zip(got, want, (mag[:, :Hq], mag[:, Hq:Hq + Hkv], 0)):
            _close(t, w, (8 * E + 2 * angle) * m + HALF[dtype] * np.abs(w) * (np.ndim(m) > 0), "rope")
        assert np.array_equal(_f64(got[2]), want[2])
        if rot < d:
            assert np.array_equal(_f64(got[0])[..., rot:], want[0][..., rot:])


def test_rotary_half_layout_is_that_of_the_plain_call(ctx):
    g = torch.Generator(device="cuda").manual_seed(31)
    qkv = torch.randn(500, 6 * 128, generator=g, device="cuda").bfloat16()
    pos = torch.arange(500, dtype=torch.int32, device="cuda") * 61
    a = binding.str_rope_split(ctx, qkv, pos, 1, 500, 4, 1, 128, 1e6)
    b = binding.str_rope_split_ex(ctx, binding.Rope(1e6, 128), qkv, pos, 4, 1, 128)
    for x, y in zip(a, b):
        assert (x[0].double() - y.double()).abs().max() <= 2.0 ** -8 * 8
    assert torch.equal(a[2][0], b[2])


@pytest.mark.parametrize("off", [1, 2])
def test_rotary_at_addresses_that_allow_no_vectors(ctx, off):
    g = torch.Generator(device="cuda").manual_seed(32)
    for t in (torch.bfloat16, torch.float32):
        flat = torch.randn(9 * 4 * 64 + off, generator=g, device="cuda").to(t)
        pos = torch.arange(9, dtype=torch.int32, device="cuda") * 1000
        for layout in ("half", "interleaved"):
            r = binding.Rope(1e4, 32, layout)
            got = binding.str_rope_split_ex(ctx, r, flat[off:].view(9, 256), pos, 2, 1, 64)
            want = binding.str_rope_split_ex(ctx, r, flat[off:].clone().view(9, 256), pos, 2, 1, 64)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_large_outputs_have_memory_of_their_own(ctx):
    """Keeping the keys of a prompt does not keep its queries."""
    qkv, pos = torch.randn(3000, 8 * 64, device="cuda").bfloat16(), torch.arange(3000, dtype=torch.int32, device="cuda")
    q, k, v = binding.str_rope_split_ex(ctx, binding.Rope(1e4, 64), qkv, pos, 4, 2, 64)
    g = np.random.default_rng(34)
    c = Conv(g, [1] * 5000, "bf16", 8, 16, 32, 2, 4)
    step = binding.str_mamba_conv_step(ctx, dev(c.zx, "bf16"), *c.on, dev(c.window, "bf16"), 5000, 1, *c.dims)
    for t in (q, k, v, *step):
        assert t.untyped_storage().nbytes() == t.numel() * t.element_size() and t.storage_offset() == 0


# ------------------------------------------------------------------------------------------------ together, streams, graphs, wrong starts
def _layer(g, rows):
    H, p, n, G, W = 4, 64, 128, 2, 4
    ch = H * p + 2 * G * n
    return dict(zx=torch.randn(rows, 2 * H * p + 2 * G * n + H, generator=g, device="cuda").bfloat16(), w=torch.randn(ch, W, generator=g, device="cuda") * 0.5,
                b=torch.randn(ch, generator=g, device="cuda") * 0.1, bias=torch.rand(H, generator=g, device="cuda") * 4 - 7, A=-torch.rand(H, generator=g, device="cuda") * 4 - 0.1,
                D=torch.randn(H, generator=g, device="cuda"), dims=(H, p, n, G))


def _mamba(ctx, L, zx, starts, window=None, state=None):
    n_seq, (H, p, n, G) = len(starts) - 1, L["dims"]
    wout = torch.zeros(n_seq, 3, H * p + 2 * G * n, dtype=torch.bfloat16, device="cuda")
    x, B, C, dt = binding.str_mamba_conv_packed(ctx, zx, L["w"], L["b"], L["bias"], _i32(starts), *L["dims"], window=window, window_out=wout)
    y, fs = binding.str_mamba2_prefill_packed(ctx, x, dt, L["A"], B, C, _i32(starts), D=L["D"], init_state=state, final_state=torch.zeros(n_seq, H, p, n, device="cuda"))
    return y, wout, fs


def test_a_mamba_layer_over_a_prompt_a_second_turn_and_single_tokens(ctx):
    """Two sequences of 200 and 90 rows at once, against: a first turn, a second turn, then three tokens one at a time."""
    g = torch.Generator(device="cuda").manual_seed(41)
    L = _layer(g, 290)
    whole, win, fs = _mamba(ctx, L, L["zx"], [0, 200, 290])
    parts = [[], []]
    window = state = None
    cut = [(0, 120, 197), (200, 201, 287)]
    for turn in range(2):
        rows = [L["zx"][c[turn]:c[turn + 1]] for c in cut]
        starts = [0, len(rows[0]), len(rows[0]) + len(rows[1])]
        y, window, state = _mamba(ctx, L, torch.cat(rows), starts, window, state)
        for s in range(2):
            parts[s].append(y[starts[s]:starts[s + 1]])
    for t in range(3):
        zx = torch.stack((L["zx"][197 + t], L["zx"][287 + t]))
        x, B, C, dt = binding.str_mamba_conv_step(ctx, zx, L["w"], L["b"], L["bias"], window, 2, 1, *L["dims"])
        y, state = binding.str_mamba2_step(ctx, x, dt, L["A"], B, C, state, D=L["D"])
        for s in range(2):
            parts[s].append(y[s])
    got = torch.cat([torch.cat(p) for p in parts])
    assert torch.equal(window, win)
    # each side within its bound of the exact recurrence of the same convolution outputs: 2 h + 2^-12 of the terms, h of the result
    x, B, C, dt = binding.str_mamba_conv_packed(ctx, L["zx"], L["w"], L["b"], L["bias"], _i32([0, 200, 290]), *L["dims"])
    y, ymag, S, Smag = packed.scan(*(_f64(t) for t in (x, dt, L["A"], B, C, L["D"])), [0, 200, 290], None)
    walk = 264 * 2.0 ** -21
    for t in (whole, got):
        _close(t, y, (2 * HALF["bf16"] + 2.0 ** -12 + walk) * ymag + HALF["bf16"] * np.abs(y), "y")
    for t in (fs, state):
        _close(t, S, (2.0 ** -15 + walk) * Smag, "state")


def test_an_attention_layer_over_two_turns_and_into_the_cache(ctx):
    """Rotary step, packed attention over both turns' rows, and the keys into the 4-bit cache: two sequences at once against the prompt whole."""
    g = torch.Generator(device="cuda").manual_seed(42)
    Hq, Hkv, d, lens, first = 8, 2, 128, [150, 70], [100, 20]
    rope = binding.Rope(1e6, 64, "interleaved", "banded", 4.0, 32768, amplitude=1.1)
    qkv = torch.randn(220, (Hq + 2 * Hkv) * d, generator=g, device="cuda").bfloat16()
    pos = torch.cat([torch.arange(n, device="cuda") * 7 for n in lens]).int()
    q, k, v = binding.str_rope_split_ex(ctx, rope, qkv, pos, Hq, Hkv, d)
    whole = binding.str_attn_prefill_packed(ctx, q, k, v, _i32([0, 150, 220]), d ** -0.5)
    turn2 = torch.cat((q[100:150], q[170:220]))
    o = binding.str_attn_prefill_packed(ctx, turn2, k, v, _i32([0, 50, 100]), d ** -0.5, k_start=_i32([0, 150, 220]))
    assert (o.double() - torch.cat((whole[100:150], whole[170:220])).double()).abs().max() <= 2.0 ** -6
    q1, k1, v1 = (torch.cat((t[:first[0]], t[150:150 + first[1]])) for t in (q, k, v))
    o1 = binding.str_attn_prefill_packed(ctx, q1, k1, v1, _i32([0, 100, 120]), d ** -0.5)
    assert (o1.double() - torch.cat((whole[:100], whole[150:170])).double()).abs().max() <= 2.0 ** -6
    cache = binding.Kv4Cache.empty(ctx, 2, 160, Hkv, d)
    for b, (s, n) in enumerate(((0, 150), (150, 70))):
        rows = [torch.zeros(2, 150, Hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        rows[0][b, :n], rows[1][b, :n] = k[s:s + n], v[s:s + n]
        binding.str_kv4_append(ctx, cache, *rows, _i32([0, 0]), n_new=_i32([n if i == b else 0 for i in range(2)]))
    kk, vv = binding.str_kv4_read(ctx, cache, _i32([0, 0]), 150, torch.bfloat16, n_rows=_i32([150, 70]))
    span = k[:150].float().unflatten(-1, (-1, 32))
    step = (span.amax(-1) - span.amin(-1)) / 15
    # a value is off by half a step of 1 / 15 of its group's range, scale and zero by their own bf16 roundings
    bound = step * 0.5 + (span.amax(-1).abs() + span.amin(-1).abs()) * 2.0 ** -6
    assert ((kk[0].float() - k[:150].float()).unflatten(-1, (-1, 32)).abs().amax(-1) <= bound).all() and vv.isfinite().all()


def test_calls_replay_from_two_graphs_and_run_on_other_streams(ctx):
    g = torch.Generator(device="cuda").manual_seed(43)
    L = _layer(g, 260)
    q, k, v = (torch.randn(260, h, 128, generator=g, device="cuda").bfloat16() for h in (4, 2, 2))
    qkv, pos = torch.randn(260, 8 * 128, generator=g, device="cuda").bfloat16(), torch.arange(260, dtype=torch.int32, device="cuda")
    rope = binding.Rope(1e4, 128)
    starts, H, p, n, G = _i32([0, 130, 260]), *L["dims"]
    window, token = torch.zeros(2, 3, H * p + 2 * G * n, dtype=torch.bfloat16, device="cuda"), L["zx"][:2].clone()

    def passes():
        x, B, C, dt = binding.str_mamba_conv_packed(ctx, L["zx"], L["w"], L["b"], L["bias"], starts, *L["dims"], window=window)
        y = binding.str_mamba2_prefill_packed(ctx, x, dt, L["A"], B, C, starts, D=L["D"])
        o = binding.str_attn_prefill_packed(ctx, q, k, v, starts, 0.1)
        return [x, B, C, dt, y, o, *binding.str_rope_split_ex(ctx, rope, qkv, pos, 4, 2, 128),
                *binding.str_mamba_conv_step(ctx, token, L["w"], L["b"], L["bias"], window, 2, 1, *L["dims"], window_out=torch.zeros_like(window))]

    want = [t.clone() for t in passes()]
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = passes()
        graphs.append((graph, out))
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(3):
        for (graph, _), st in zip(graphs, streams):
            with torch.cuda.stream(st):
                graph.replay()
    torch.cuda.synchronize()
    for _, out in graphs:
        assert all(torch.equal(a, b) for a, b in zip(out, want))
    results = []
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(st):
            results.append(passes())
    torch.cuda.synchronize()
    for out in results:
        assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("starts", [[0, 50, 20, 100], [-3, 10, 60, 100], [0, 40, 1000000, 2000000], [7, 7, 7, -2147483648], [2147483647] * 4], ids=str)
def test_wrong_starts_are_held_to_the_tensors_and_reported(ctx, starts):
    g = torch.Generator(device="cuda").manual_seed(44)
    L = _layer(g, 100)
    bad = _i32(starts)
    q, k, v = (torch.randn(100, h, 128, generator=g, device="cuda").bfloat16() for h in (4, 2, 2))
    window = torch.zeros(3, 3, 4 * 64 + 2 * 2 * 128, dtype=torch.bfloat16, device="cuda")
    x, B, C, dt = binding.str_mamba_conv_packed(ctx, L["zx"], L["w"], L["b"], L["bias"], _i32([0, 100]), *L["dims"])
    calls = (lambda: binding.str_mamba_conv_packed(ctx, L["zx"], L["w"], L["b"], L["bias"], bad, *L["dims"], window=window, window_out=torch.zeros_like(window)),
             lambda: binding.str_mamba2_prefill_packed(ctx, x, dt, L["A"], B, C, bad, final_state=torch.zeros(3, 4, 64, 128, device="cuda")),
             lambda: binding.str_mamba2_prefill_packed(ctx, x.float(), dt, L["A"], B.float(), C.float(), bad),
             lambda: binding.str_attn_prefill_packed(ctx, q, k, v, bad, 0.1),
             lambda: binding.str_attn_prefill_packed(ctx, q, k, v, _i32([0, 10, 20, 100]), 0.1, k_start=bad),
             lambda: binding.str_attn_prefill_packed(ctx, q.float(), k.float(), v.float(), bad, 0.1))
    for call in calls:
        call()
        with pytest.raises(binding.StrError) as e:
            ctx.check_status()
        assert e.value.code == -1
        ctx.check_status()                                 # said once
    fine = binding.str_attn_prefill_packed(ctx, q, k, v, _i32([0, 30, 100]), 0.1)
    ctx.check_status()
    assert fine.isfinite().all()


def test_rows_beyond_four_gigabytes(ctx):
    """Offsets of the last sequence's elements pass 2^31 in every tensor."""
    rows, H, d = 70000, 256, 128
    big = torch.zeros(rows, H, d, dtype=torch.bfloat16, device="cuda")                              # 4.6 GB
    g = torch.Generator(device="cuda").manual_seed(45)
    big[-64:] = torch.randn(64, H, d, generator=g, device="cuda").bfloat16()
    starts = _i32([rows - 64, rows])
    o = binding.str_attn_prefill_packed(ctx, big, big, big, starts, d ** -0.5)
    want, mag, largest = _long_reference(big[-64:], big[-64:], big[-64:], d ** -0.5)
    rel = 2 * (d + 64) * E * largest + 64 * E + 2.0 ** -12 + HALF["bf16"]
    assert ((o[-64:].double() - want).abs() <= rel * mag + HALF["bf16"] * want.abs()).all()
    del o
    pos = torch.full((rows,), 12345, dtype=torch.int32, device="cuda")
    q, k, v = binding.str_rope_split_ex(ctx, binding.Rope(1e4, 128), big.view(rows, H * d), pos, 128, 64, d)
    qs, ks, vs = binding.str_rope_split_ex(ctx, binding.Rope(1e4, 128), big[-64:].reshape(64, H * d), pos[-64:], 128, 64, d)
    assert torch.equal(q[-64:], qs) and torch.equal(k[-64:], ks) and torch.equal(v[-64:], vs)
