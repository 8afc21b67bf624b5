"""The operators that decode against a reduced context, as cases to measure: the 4-bit key/value cache (append, read back,
attention with accumulated weights, eviction by accumulated weight) and the single-token step of the Mamba-2 recurrence.

``run`` computes a case in plain torch (``own`` false) or through the library's calls (``own`` true); ``exact`` computes
the same results in 64 bits from the definitions.  Shapes are those of the library's 8B-class layers (32 query heads, 8
key/value heads of 128; 128 Mamba heads of 64 with a state of 128) and of its smaller test layers, with ragged lengths.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _append(name, Bz, T, cap, Hkv, d, group, dtype, ragged):
    return dict(name=name, kind="append", Bz=Bz, T=T, cap=cap, Hkv=Hkv, d=d, group=group, dtype=dtype, ragged=ragged)


def _attend(name, Bz, cap, n_q, Hq, Hkv, d, group, dtype, ragged, weights):
    return dict(name=name, kind="attend", Bz=Bz, cap=cap, n_q=n_q, Hq=Hq, Hkv=Hkv, d=d, group=group, dtype=dtype, ragged=ragged,
                weights=weights)


def _evict(name, Bz, cap, keep, recent, Hkv, d, group, ragged):
    return dict(name=name, kind="evict", Bz=Bz, cap=cap, keep=keep, recent=recent, Hkv=Hkv, d=d, group=group, ragged=ragged)


def _step(name, Bz, T, H, p, n, G, dtype, skip):
    return dict(name=name, kind="step", Bz=Bz, T=T, H=H, p=p, n=n, G=G, dtype=dtype, skip=skip)


def listed():
    return [
        # one decode step of a small batch: every sequence's new key and value go into its cache and are read back
        _append("append_step_b16", 16, 1, 8448, 8, 128, 32, "bf16", False),
        # hand-off of the 64-frame attention layer: all its keys and values enter the cache, and come back for a second turn
        _append("append_handoff_16k", 1, 16512, 16640, 8, 128, 32, "bf16", False),
        # one decode step on the survivors of the 128-frame stack (8192 visual + 128 text + a few generated): latency
        _attend("attend_b1_8k", 1, 8448, 1, 32, 8, 128, 32, "bf16", False, False),
        # one decode step on an unreduced two-hundred-frame context of one sequence
        _attend("attend_b1_64k", 1, 65792, 1, 32, 8, 128, 64, "bf16", False, False),
        # one decode step of a ragged batch that also gathers the weights the eviction ranks by
        _attend("attend_b32_16k_weights", 32, 16640, 1, 32, 8, 128, 32, "bf16", True, True),
        # several tokens verified at once, fp32 storage, an odd number of heads per key head, gathering weights
        _attend("attend_f32_verify5", 3, 2064, 5, 21, 7, 64, 64, "f32", True, True),
        # a budget of one sequence's survivors is restored after some generated tokens
        _evict("evict_b1_8k", 1, 8448, 8192, 256, 8, 128, 32, False),
        # a batch's unreduced contexts are cut to a quarter at once
        _evict("evict_b8_32k_quarter", 8, 32896, 8192, 512, 8, 128, 64, True),
        # recurrent step of one 8B-class Mamba layer: one sequence, one token
        _step("step_b1", 1, 1, 128, 64, 128, 8, "bf16", False),
        # the same for a batch of 64 sequences: bound by the state's way through memory
        _step("step_b64", 64, 1, 128, 64, 128, 8, "bf16", True),
        # a few tokens verified at once, fp32 storage, the small test layer's head with an odd state
        _step("step_f32_t5", 9, 5, 24, 32, 20, 3, "f32", True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "attend", "attend", "evict", "step", "step"])
    d = rng.choice([64, 128, 128])
    group = rng.choice([g for g in (32, 64, 128) if g <= d])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    Hkv = rng.choice([1, 2, 4, 5, 8])
    if kind == "append":
        Bz = rng.choice([1, 2, 3, 8, 16])
        T = _log_int(rng, 1, 16512 // Bz // (2 if dtype == "f32" else 1))
        return dict(kind=kind, Bz=Bz, T=T, cap=16 * (-(-T // 16) + rng.randint(1, 9)), Hkv=Hkv, d=d, group=group, dtype=dtype,
                    ragged=rng.random() < 0.6)
    if kind == "attend":
        Bz = rng.choice([1, 1, 2, 3, 7, 16, 32])
        n_q, Hq = rng.choice([1, 1, 1, 2, 5, 8]), Hkv * rng.choice([1, 2, 3, 4, 4, 8])
        cap = 16 * _log_int(rng, 1, min(4112, 32768 // Bz, 32 * 560 * 32 * 128 // (Bz * n_q * Hq * d)))
        return dict(kind=kind, Bz=Bz, cap=cap, n_q=n_q, Hq=Hq, Hkv=Hkv, d=d, group=group, dtype=dtype, ragged=rng.random() < 0.6, weights=rng.random() < 0.5)
    if kind == "evict":
        Bz = rng.choice([1, 2, 5, 8])
        cap = 16 * _log_int(rng, 2, min(4112, 16448 // Bz))
        keep = max(1, min(int(cap * rng.uniform(0.05, 1.0)), 8 * 8192 * 8 * 72 // (Bz * Hkv * (d // 2 + 4 * (d // group)))))
        return dict(kind=kind, Bz=Bz, cap=cap, keep=keep, recent=rng.randint(0, min(keep, 600)), Hkv=Hkv, d=d, group=group,
                    ragged=rng.random() < 0.6)
    G = rng.choice([1, 2, 4, 8])
    H, p, n = G * rng.choice([1, 3, 8, 16]), rng.choice([16, 32, 64, 64, 80]), rng.choice([16, 20, 64, 128, 128, 256])
    return dict(kind=kind, Bz=_log_int(rng, 1, min(64, 64 * 128 * 64 * 128 // (H * p * n))), T=rng.choice([1, 1, 1, 2, 3, 8]), H=H, p=p, n=n,
                G=G, dtype=dtype, skip=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _lens(case):
    """Rows per sequence, the same for every seed: nearly as many as fit, or any number (one of several sequences has none)."""
    Bz, most = case["Bz"], case["T"] if case["kind"] == "append" else case["cap"]
    g = np.random.default_rng([Bz, most])
    if not case["ragged"]:
        return [most] * Bz if case["kind"] == "append" else [max(1, most - int(v)) for v in g.integers(0, 14, Bz)]
    lens = [int(v) for v in g.integers(1, most + 1, Bz)]
    if Bz > 1:
        lens[int(g.integers(0, Bz))] = 0
    return lens


def _floor_bf16(x):
    """Largest bf16 value <= x (x finite fp32), as fp32."""
    bits = x.view(torch.int32)
    kept = bits & -65536
    return torch.where((bits < 0) & (kept != bits), kept + 65536, kept).view(torch.float32)


def _quantise(x, group):
    """(codes uint8 [..., d], zero fp32, scale fp32 [..., d / group]) of fp32 rows: x ~ zero + scale * code."""
    xg = x.unflatten(-1, (x.shape[-1] // group, group))
    zero = _floor_bf16(xg.amin(-1))
    scale = ((xg.amax(-1) - zero) / 15.0).bfloat16().float()
    code = torch.where(scale[..., None] > 0, torch.round((xg - zero[..., None]) / scale[..., None]), 0.0).clamp(0, 15)
    return code.to(torch.uint8).flatten(-2), zero, scale


def _pack(code, keys):
    """Packed rows uint8 [..., d / 2].  Key rows: element 32 g + 8 c + j is nibble j of 32-bit word c * (d / 32) + g; value
    rows: element 32 g + 4 r + i is nibble i of 16-bit word r * (d / 32) + g."""
    d = code.shape[-1]
    c = code.unflatten(-1, (d // 32, 4, 8) if keys else (d // 32, 8, 4)).transpose(-3, -2).flatten(-3)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _unpack(packed, keys):
    """Codes fp32 [..., d] of packed rows: the inverse of _pack."""
    d = packed.shape[-1] * 2
    c = torch.stack((packed & 15, packed >> 4), -1).flatten(-2)
    return c.unflatten(-1, (4, d // 32, 8) if keys else (8, d // 32, 4)).transpose(-3, -2).flatten(-3).float()


def _words(zero, scale):
    """One 32-bit word per group: the bf16 scale in the high half, the bf16 zero in the low half."""
    return (scale.view(torch.int32) & -65536) | ((zero.view(torch.int32) >> 16) & 65535)


def _values(packed, words, group, keys):
    """fp32 values [..., d] of packed rows and their words."""
    scale, zero = (words & -65536).view(torch.float32), (words << 16).view(torch.float32)
    c = _unpack(packed, keys).unflatten(-1, (-1, group))
    return (zero[..., None] + scale[..., None] * c).flatten(-2)


def _rows(g, shape, keys):
    """fp32 rows as a layer's keys or values are: unit normal, keys with a few channels of large offset."""
    x = torch.randn(shape, generator=g, device="cuda")
    if keys:
        d = shape[-1]
        off = torch.where(torch.rand(d, generator=g, device="cuda") < 0.06, 6.0 * torch.randn(d, generator=g, device="cuda"), 0.0)
        x += off
    return x


def _cache(case, g):
    """Logical content of a full cache, head-major: codes, zeros and scales of keys and values."""
    shape = (case["Bz"], case["Hkv"], case["cap"], case["d"])
    return _quantise(_rows(g, shape, True), case["group"]) + _quantise(_rows(g, shape, False), case["group"])


def _inputs(case, seed):
    """Logical inputs of a case: torch tensors on the GPU, before any packing."""
    g = torch.Generator(device="cuda").manual_seed((1000003 * seed + 17) % 2**62)
    dt = _DTYPES.get(case.get("dtype"), torch.float32)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    if case["kind"] == "append":
        Bz, T = case["Bz"], case["T"]
        n_new = _lens(case)
        h = np.random.default_rng([seed, 8])
        start = [int(v) for v in h.integers(0, case["cap"] - T + 1, Bz)]
        shape = (Bz, T, case["Hkv"], case["d"])
        k, v = _rows(g, shape, True).to(dt), _rows(g, shape, False).to(dt)
        return dict(k=k, v=v, start=torch.tensor(start, dtype=torch.int32, device="cuda"),
                    n_new=torch.tensor(n_new, dtype=torch.int32, device="cuda"))
    if case["kind"] == "attend":
        lens = _lens(case)
        x = dict(zip(("kc", "kz", "ks", "vc", "vz", "vs"), _cache(case, g)))
        x.update(q=rand(case["Bz"], case["n_q"], case["Hq"], case["d"]).to(dt), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"))
        if case["weights"]:
            # as after some tens of steps, each of which spreads one unit per query head over the rows
            x["weight"] = rand(case["Bz"], case["Hkv"], case["cap"]).abs() * (32.0 * case["Hq"] / case["Hkv"] / case["cap"])
        return x
    if case["kind"] == "evict":
        lens = _lens(case)
        x = dict(zip(("kc", "kz", "ks", "vc", "vz", "vs"), _cache(case, g)))
        x["weight"] = rand(case["Bz"], case["Hkv"], case["cap"]).pow_(4)          # few tokens carry most of the weight
        x["pos"] = torch.randint(1, 4, (case["Bz"], case["cap"]), generator=g, device="cuda").cumsum(1).int()
        x["lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")
        return x
    Bz, T, H, p, n, G = (case[k] for k in ("Bz", "T", "H", "p", "n", "G"))
    uni = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    return dict(x=rand(Bz, T, H, p).to(dt), B=rand(Bz, T, G, n).to(dt), C=rand(Bz, T, G, n).to(dt), dt=0.001 + 0.099 * uni(Bz, T, H),
                A=-torch.exp(math.log(16.0) * uni(H)), D=rand(H) if case["skip"] else None, state=rand(Bz, H, p, n))


def prepare(case, seed):
    x = _inputs(case, seed)
    st = dict(case=case)
    if case["kind"] == "append":
        Bz, cap, Hkv, d, ng = case["Bz"], case["cap"], case["Hkv"], case["d"], case["d"] // case["group"]
        z = lambda dtp, *s: torch.zeros(s, dtype=dtp, device="cuda")  # noqa: E731
        st.update(x, k_codes=z(torch.uint8, Bz, Hkv, cap, d // 2), v_codes=z(torch.uint8, Bz, Hkv, cap, d // 2),
                  k_scales=z(torch.int32, Bz, Hkv, cap, ng), v_scales=z(torch.int32, Bz, Hkv, cap, ng))
        return st
    if case["kind"] == "step":
        st.update(x, state_out=torch.zeros_like(x["state"]))
        return st
    st.update(k_codes=_pack(x["kc"], True), v_codes=_pack(x["vc"], False), k_scales=_words(x["kz"], x["ks"]), v_scales=_words(x["vz"], x["vs"]))
    if case["kind"] == "attend":
        st.update(q=x["q"], lens=x["lens"], scale=case["d"] ** -0.5)
        if case["weights"]:
            st.update(weight=x["weight"], weight_out=x["weight"].clone())
        return st
    st.update(weight=x["weight"], pos=x["pos"], lens=x["lens"])
    to = -(-case["keep"] // 16) * 16
    st["out"] = {k: torch.zeros((*st[k].shape[:-2], to, st[k].shape[-1]), dtype=st[k].dtype, device="cuda")
                 for k in ("k_codes", "v_codes", "k_scales", "v_scales")}
    st["out"].update(weight=torch.zeros((case["Bz"], case["Hkv"], to), device="cuda"), pos=torch.zeros((case["Bz"], to), dtype=torch.int32, device="cuda"))
    return st


# ------------------------------------------------------------------------------------------------ one pass
_CTX = []
_PARTS = ("k_codes", "v_codes", "k_scales", "v_scales", "pos", "weight")


def _run_own(st):
    from paper_2603_00198_b200 import binding
    if not _CTX:
        _CTX.append(binding.Context(torch.cuda.current_device()))
    ctx, case = _CTX[0], st["case"]
    if case["kind"] == "step":
        return binding.str_mamba2_step(ctx, st["x"], st["dt"], st["A"], st["B"], st["C"], st["state"], D=st["D"], state_out=st["state_out"])
    if "cache" not in st:                                                       # the handles that a program keeps for its caches
        st["cache"] = binding.Kv4Cache(*(st.get(k) for k in _PARTS))
        st["cache_out"] = binding.Kv4Cache(*(st["out"][k] for k in _PARTS)) if case["kind"] == "evict" else None
    cache = st["cache"]
    if case["kind"] == "append":
        binding.str_kv4_append(ctx, cache, st["k"], st["v"], st["start"], n_new=st["n_new"])
        return binding.str_kv4_read(ctx, cache, st["start"], case["T"], st["k"].dtype, n_rows=st["n_new"])
    if case["kind"] == "attend":
        o = binding.str_kv4_attn(ctx, cache, st["q"], st["lens"], st["scale"], weight_out=st.get("weight_out"))
        return (o, st["weight_out"]) if case["weights"] else o
    lens, kept = binding.str_kv4_evict(ctx, cache, st["lens"], case["keep"], case["recent"], st["cache_out"])
    return _evicted(lens, kept, st["out"])


def _evicted(lens, kept, out):
    """The packed rows are copied as they are: returned as the whole numbers of their 32-bit words."""
    return dict(lens=lens, kept=kept, k=out["k_codes"].view(torch.int32), v=out["v_codes"].view(torch.int32), ks=out["k_scales"],
                vs=out["v_scales"], pos=out["pos"], weight=out["weight"])


def run(state):
    if own:
        return _run_own(state)
    return {"append": _plain_append, "attend": _plain_attend, "evict": _plain_evict, "step": _plain_step}[state["case"]["kind"]](state)


def _plain_append(st):
    case = st["case"]
    T, group, dt = case["T"], case["group"], st["k"].dtype
    j = torch.arange(T, device="cuda")
    live = j < st["n_new"][:, None]                                             # [Bz, T]
    b, t = live.nonzero(as_tuple=True)
    row = st["start"].long()[b] + t
    res = []
    for x, codes, words, keys in ((st["k"], st["k_codes"], st["k_scales"], True), (st["v"], st["v_codes"], st["v_scales"], False)):
        c, zero, scale = _quantise(x[b, t].float(), group)                      # [rows, Hkv, d]
        codes[b, :, row] = _pack(c, keys)
        words[b, :, row] = _words(zero, scale)
        out = torch.zeros_like(x)
        out[b, t] = _values(codes[b, :, row], words[b, :, row], group, keys).to(dt)
        res.append(out)
    return tuple(res)


def _plain_attend(st):
    case, q = st["case"], st["q"]
    Bz, n_q, Hq, d = q.shape
    Hkv, cap = case["Hkv"], case["cap"]
    R = Hq // Hkv
    k = _values(st["k_codes"], st["k_scales"], case["group"], True)             # [Bz, Hkv, cap, d]
    qh = q.float().unflatten(2, (Hkv, R)).permute(0, 2, 3, 1, 4).reshape(Bz, Hkv, R * n_q, d)
    s = torch.matmul(qh, k.transpose(-1, -2)) * st["scale"]
    del k
    t = torch.arange(cap, device="cuda")
    last = st["lens"][:, None] - n_q + torch.arange(n_q, device="cuda")          # [Bz, n_q]: the last row each token sees
    seen = (t <= last[..., None])[:, None, None].expand(Bz, 1, R, n_q, cap).reshape(Bz, 1, R * n_q, cap)
    s = s.masked_fill(~seen, float("-inf"))
    top = s.amax(-1, keepdim=True).clamp_min(-3.0e38)
    e = torch.exp(s - top)
    total = e.sum(-1, keepdim=True)
    w = e / torch.where(total > 0, total, 1.0)
    v = _values(st["v_codes"], st["v_scales"], case["group"], False)
    o = torch.matmul(w, v).unflatten(2, (R, n_q)).permute(0, 3, 1, 2, 4).reshape(Bz, n_q, Hq, d).to(q.dtype)
    if not case["weights"]:
        return o
    held = (t < st["lens"][:, None])[:, None]
    st["weight_out"].copy_(torch.where(held, st["weight"] + w.sum(2), st["weight_out"]))
    return o, st["weight_out"]


def _plain_evict(st):
    case, out = st["case"], st["out"]
    keep, cap = case["keep"], case["cap"]
    lens = st["lens"].long()[:, None]
    t = torch.arange(cap, device="cuda")
    score = st["weight"].double().sum(1).float()                                # per row, over the key heads: rounded to fp32 once
    score = torch.where(t >= lens - case["recent"], float("inf"), score)
    score = torch.where(t >= lens, float("-inf"), score)
    order = torch.sort(score, dim=1, descending=True, stable=True).indices[:, :keep].sort(1).values
    n = torch.minimum(lens, torch.full_like(lens, keep))                        # [Bz, 1]
    j = torch.arange(keep, device="cuda")
    live = j < n
    kept = torch.where(live, order, -1).int()
    b, r = live.nonzero(as_tuple=True)
    src = order[b, r]
    for key in ("k_codes", "v_codes", "k_scales", "v_scales", "weight"):
        out[key][b, :, r] = st[key][b, :, src]
    out["pos"][b, r] = st["pos"][b, src]
    return _evicted(n[:, 0].int(), kept, out)


def _plain_step(st):
    case = st["case"]
    per = case["H"] // case["G"]
    B, C = st["B"].float().repeat_interleave(per, 2), st["C"].float().repeat_interleave(per, 2)   # [Bz, T, H, n]
    x, dt = st["x"].float(), st["dt"]
    cum = (dt * st["A"]).cumsum(1)                                              # log-decay from the old state to after token t
    T = case["T"]
    lag = cum[:, :, None] - cum[:, None]                                        # [Bz, t, s, H]
    tri = torch.ones(T, T, device="cuda", dtype=torch.bool).tril()[None, :, :, None]
    w = torch.where(tri, torch.exp(lag.masked_fill(~tri, 0.0)), 0.0) * dt[:, None]
    S = st["state"]
    y = torch.matmul(S, C.permute(0, 2, 3, 1)).permute(0, 3, 1, 2) * torch.exp(cum)[..., None]
    y = y + ((w * (C[:, :, None] * B[:, None]).sum(-1))[..., None] * x[:, None]).sum(2)
    if st["D"] is not None:
        y = y + st["D"][:, None] * x
    xs = (w[:, -1][..., None] * x).permute(0, 2, 3, 1)                          # [Bz, H, p, T]
    torch.add(S * torch.exp(cum[:, -1])[..., None, None], torch.matmul(xs, B.permute(0, 2, 1, 3)), out=st["state_out"])
    return y.to(st["x"].dtype), st["state_out"]


# ------------------------------------------------------------------------------------------------ work and 64-bit results
def work(case):
    es = 2 if case.get("dtype") == "bf16" else 4
    if case["kind"] == "step":
        Bz, T, H, p, n, G = (case[k] for k in ("Bz", "T", "H", "p", "n", "G"))
        small = Bz * T * (2 * H * p * es + 2 * G * n * es + 4 * H)
        return dict(bytes=8 * Bz * H * p * n + small, flops=5 * Bz * T * H * p * n)
    Hkv, d = case["Hkv"], case["d"]
    row = 2 * Hkv * (d // 2 + 4 * (d // case["group"]))                          # one token's keys and values in the cache
    if case["kind"] == "append":
        n = sum(_lens(case))
        return dict(bytes=n * (4 * Hkv * d * es + 2 * row), flops=n * 8 * Hkv * d)
    rows = sum(_lens(case))
    if case["kind"] == "attend":
        Bz, n_q, Hq = case["Bz"], case["n_q"], case["Hq"]
        extra = 8 * rows * Hkv if case["weights"] else 0
        return dict(bytes=rows * row + extra + 2 * Bz * n_q * Hq * d * es, flops=4 * rows * n_q * Hq * d)
    kept = sum(min(v, case["keep"]) for v in _lens(case))
    return dict(bytes=4 * rows * Hkv + kept * (2 * row + 4 * Hkv + 8 + 4), flops=rows * Hkv)


def exact(case, seed):
    """The definitions in 64 bits, sequence by sequence and head by head."""
    x = _inputs(case, seed)
    f8 = lambda t: t.double()  # noqa: E731
    if case["kind"] == "append":
        out = []
        for a in (x["k"], x["v"]):
            rows, r = f8(a), torch.zeros(a.shape, dtype=torch.float64, device="cuda")
            for b, n in enumerate(x["n_new"].tolist()):
                g = rows[b, :n].reshape(n, case["Hkv"], -1, case["group"])
                if n:
                    lo, hi = g.amin(-1, keepdim=True), g.amax(-1, keepdim=True)
                    zero = lo.float().bfloat16()
                    zero = f8(torch.where(f8(zero) > lo, torch.nextafter(zero.cpu(), torch.tensor(-math.inf, dtype=torch.bfloat16)).cuda(), zero))
                    scale = f8(((hi - zero) / 15.0).float().bfloat16())
                    code = ((g - zero) / scale).round().clamp(0, 15).nan_to_num(0.0)
                    r[b, :n] = (zero + scale * code).reshape(n, case["Hkv"], -1)
            out.append(r)
        return tuple(out)
    if case["kind"] == "attend":
        Bz, n_q, Hq, d = x["q"].shape
        R, group = Hq // case["Hkv"], case["group"]
        if Bz * case["cap"] * n_q * Hq * d > 4e9:
            return None
        o = torch.zeros((Bz, n_q, Hq, d), dtype=torch.float64, device="cuda")
        weight = f8(x["weight"]) if case["weights"] else None
        for b, n in enumerate(x["lens"].tolist()):
            for h in range(case["Hkv"]):
                K, V = (f8(x[c][b, h, :n]) * f8(x[s][b, h, :n]).repeat_interleave(group, 1) + f8(x[z][b, h, :n]).repeat_interleave(group, 1)
                        for c, z, s in (("kc", "kz", "ks"), ("vc", "vz", "vs")))
                for i in range(max(0, n_q - n), n_q):
                    m = n - n_q + i + 1
                    p = torch.softmax(f8(x["q"][b, i, h * R:(h + 1) * R]) @ K[:m].T / math.sqrt(d), 1)
                    o[b, i, h * R:(h + 1) * R] = p @ V[:m]
                    if weight is not None:
                        weight[b, h, :m] += p.sum(0)
        return o if weight is None else (o, weight)
    if case["kind"] == "step":
        S, per, ys = f8(x["state"]), case["H"] // case["G"], []
        for t in range(case["T"]):
            dt, xt = f8(x["dt"][:, t]), f8(x["x"][:, t])
            B, C = (f8(x[k][:, t]).repeat_interleave(per, 1) for k in ("B", "C"))
            S = S * torch.exp(dt * f8(x["A"]))[..., None, None] + (dt[..., None] * xt)[..., None] * B[:, :, None]
            y = (S * C[:, :, None]).sum(-1)
            ys.append(y if x["D"] is None else y + f8(x["D"])[:, None] * xt)
        return torch.stack(ys, 1), S
    keep, to = case["keep"], -(-case["keep"] // 16) * 16
    weight, lens_in = x["weight"].cpu().numpy(), x["lens"].tolist()
    full = dict(k=_pack(x["kc"], True).view(torch.int32), v=_pack(x["vc"], False).view(torch.int32), ks=_words(x["kz"], x["ks"]),
                vs=_words(x["vz"], x["vs"]), pos=x["pos"], weight=x["weight"])
    res = {k: torch.zeros((*a.shape[:2], to, a.shape[3]) if a.dim() == 4 else (*a.shape[:-1], to), dtype=a.dtype, device="cuda") for k, a in full.items()}
    kept = np.full((case["Bz"], keep), -1, dtype=np.int32)
    for b, n in enumerate(lens_in):
        score = weight[b, :, :n].astype(np.float64).sum(0).astype(np.float32)
        free = max(0, n - case["recent"])
        room = max(0, min(n, keep) - (n - free))
        best = np.lexsort((np.arange(free), -score[:free]))[:room]
        idx = np.sort(np.concatenate([best, np.arange(free, n)])).astype(np.int64)
        kept[b, :len(idx)] = idx
        at = torch.from_numpy(idx).cuda()
        for k, a in full.items():
            if k == "pos":
                res[k][b, :len(idx)] = a[b, at]
            else:
                res[k][b, :, :len(idx)] = a[b][:, at]
    return dict(lens=torch.tensor([min(n, keep) for n in lens_in], dtype=torch.int32), kept=torch.from_numpy(kept), **res)
