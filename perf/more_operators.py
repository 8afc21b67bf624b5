"""The operators that run the hybrid stack's layers on packed sequences of different lengths and on continued turns, as cases to
measure: the Mamba block's causal convolution with its window (prompts and single tokens), the selective scan from given states,
causal attention with grouped heads over earlier and new keys, and rotary positions in both layouts, on part of the head, scaled for
long contexts.

``run`` computes a case in plain torch (``own`` false) or through the library's calls (``own`` true); ``exact`` computes the
same results in 64 bits from the definitions.  Shapes are those of the library's 8B-class layers (128 Mamba heads of 64 with a
state of 128 in 8 groups; 32 query heads, 8 key/value heads of 128) and of its smaller test layers.  Rows of a packed tensor that
belong to no sequence are left as they were.
"""
import math

import numpy as np
import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------------------------------------ cases
def _conv(name, n_seq, T, tail, H, p, n, G, W, dtype, window):
    return dict(name=name, kind="conv", n_seq=n_seq, T=T, tail=tail, H=H, p=p, n=n, G=G, W=W, dtype=dtype, window=window)


def _conv_step(name, Bz, T, H, p, n, G, W, dtype):
    return dict(name=name, kind="conv_step", Bz=Bz, T=T, H=H, p=p, n=n, G=G, W=W, dtype=dtype)


def _scan(name, n_seq, T, tail, H, p, n, G, dtype, state, skip):
    return dict(name=name, kind="scan", n_seq=n_seq, T=T, tail=tail, H=H, p=p, n=n, G=G, dtype=dtype, state=state, skip=skip)


def _attend(name, n_seq, T, tail, past, blind, Hq, Hkv, d, dtype):
    return dict(name=name, kind="attend", n_seq=n_seq, T=T, tail=tail, past=past, blind=blind, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype)


def _rope(name, rows, Hq, Hkv, d, rot, layout, scaling, factor, reach, dtype):
    return dict(name=name, kind="rope", rows=rows, Hq=Hq, Hkv=Hkv, d=d, rot=rot, layout=layout, scaling=scaling, factor=factor, reach=reach,
                dtype=dtype)


def listed():
    return [
        # one decode step of one 8B-class Mamba layer: the new token through the convolution, its window moved on
        _conv_step("conv_step_b1", 1, 1, 128, 64, 128, 8, 4, "bf16"),
        # the same for a batch of 64 sequences
        _conv_step("conv_step_b64", 64, 1, 128, 64, 128, 8, 4, "bf16"),
        # a batch of short second turns on the small test layer, fp32 storage, three taps, odd state
        _conv("conv_f32_turns", 5, 1237, 3, 24, 32, 20, 3, 3, "f32", True),
        # a batch of prompts of the 8B-class layer, some of them continued
        _conv("conv_b8_24k", 8, 24576, 64, 128, 64, 128, 8, 4, "bf16", True),
        # one short text turn of the 8B-class layer from the state of the turn before: latency
        _scan("scan_turn_300", 1, 300, 0, 128, 64, 128, 8, "bf16", True, True),
        # a batch of prompts of different lengths
        _scan("scan_b8_24k", 8, 24576, 64, 128, 64, 128, 8, "bf16", True, False),
        # a batch of short second turns on the small test layer, fp32 storage, odd state
        _scan("scan_f32_turns", 5, 1237, 3, 24, 32, 20, 3, "f32", True, True),
        # the attention layer of one 64-frame prompt
        _attend("attend_b1_16k", 1, 16512, 0, 0, False, 32, 8, 128, "bf16"),
        # a batch of prompts, some of them second turns over the reduced rows of the first
        _attend("attend_b12_turns", 12, 8200, 40, 4096, True, 32, 8, 128, "bf16"),
        # fp32 storage, an odd number of heads per key head, ragged
        _attend("attend_f32_ragged", 4, 1531, 5, 300, False, 21, 7, 64, "f32"),
        # the rotary step of a long prompt whose positions lie beyond the length that the layer was trained for
        _rope("rope_16k_banded", 16512, 32, 8, 128, 128, "half", "banded", 8.0, 262144, "bf16"),
        # the rotary step of a batch's new tokens, part of the head, interleaved pairs
        _rope("rope_tokens", 16, 32, 8, 128, 64, "interleaved", "none", 1.0, 32768, "bf16"),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["conv", "conv_step", "scan", "scan", "attend", "attend", "rope"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if kind == "rope":
        d = rng.choice([64, 80, 128, 128])
        rot = rng.choice([d, d, d // 2, 16 * rng.randint(1, d // 16)])
        Hkv = rng.choice([1, 2, 4, 5, 8])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 8])
        scaling = rng.choice(["none", "linear", "banded"])
        return dict(kind=kind, rows=_log_int(rng, 1, max(1, 16512 * 48 * 128 // ((Hq + 2 * Hkv) * d * (2 if dtype == "f32" else 1)))), Hq=Hq, Hkv=Hkv, d=d,
                    rot=rot, layout=rng.choice(["half", "interleaved"]), scaling=scaling,
                    factor=1.0 if scaling == "none" else 0.25 * rng.randint(5, 64), reach=_log_int(rng, 1000, 4000000), dtype=dtype)
    n_seq, tail = rng.choice([1, 1, 2, 3, 5, 8, 16, 33]), rng.choice([0, 0, 1, 37])
    if kind == "attend":
        Hkv, d = rng.choice([1, 2, 4, 7, 8]), rng.choice([64, 128, 128, 80])
        Hq = Hkv * rng.choice([1, 2, 3, 4, 4])
        if dtype == "f32":
            Hq, Hkv = min(Hq, 12) // min(Hkv, 4) * min(Hkv, 4), min(Hkv, 4)
        past = rng.choice([0, 0, 0, 129, 1000, 4096])
        # no more products than the largest listed case, a tenth of them in fp32
        most = 16512.0 ** 2 / 2 * 32 * 128 / (Hq * d) * (0.1 if dtype == "f32" else 1.0)
        T = max(n_seq, _log_int(rng, 1, min(16512, int(math.sqrt(past * past + 2 * most)) - past)))
        return dict(kind=kind, n_seq=n_seq, T=T, tail=tail, past=past, blind=rng.random() < 0.3, Hq=Hq, Hkv=Hkv, d=d, dtype=dtype)
    G = rng.choice([1, 2, 4, 8])
    H, p, n = G * rng.choice([1, 3, 8, 16]), rng.choice([16, 32, 64, 64, 80]), rng.choice([16, 20, 64, 128, 128])
    if kind == "conv_step":
        return dict(kind=kind, Bz=_log_int(rng, 1, 64), T=rng.choice([1, 1, 1, 2, 3, 8]), H=H, p=p, n=n, G=G, W=rng.choice([2, 3, 4, 4, 4]), dtype=dtype)
    if kind == "conv":
        most = 24576 * (8192 + 2048) // ((H * p + 2 * G * n) * (2 if dtype == "f32" else 1))
        return dict(kind=kind, n_seq=n_seq, T=max(n_seq, _log_int(rng, 1, min(65536, most))), tail=tail, H=H, p=p, n=n, G=G,
                    W=rng.choice([2, 3, 4, 4, 4]), dtype=dtype, window=rng.random() < 0.6)
    most = 24576 * 128 * 64 * 128 // (H * p * n)
    return dict(kind=kind, n_seq=n_seq, T=max(n_seq, _log_int(rng, 1, min(24576, most) // (8 if dtype == "f32" else 1))), tail=tail, H=H, p=p, n=n, G=G,
                dtype=dtype, state=rng.random() < 0.6, skip=rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs
def _split(T, n_seq, seed):
    """Lengths of n_seq sequences with T rows together, of very different sizes; with four or more, one is empty and one has a single row."""
    g = np.random.default_rng([T, n_seq, seed])
    if n_seq == 1:
        return [T]
    share = g.exponential(size=n_seq) + 0.05
    fixed = {}
    if n_seq >= 4 and T >= n_seq:
        a, b = (int(v) for v in g.permutation(n_seq)[:2])
        fixed = {a: 0, b: 1}
        share[a] = share[b] = 0.0
    lens = np.floor((T - sum(fixed.values())) * share / share.sum()).astype(int)
    for i, v in fixed.items():
        lens[i] = v
    lens[int(np.argmax(share))] += T - int(lens.sum())
    return [int(v) for v in lens]


def _lens(case):
    """(query rows, key rows) of each sequence, the same for every seed; outside attention the two are one."""
    lq = _split(case["T"], case["n_seq"], 1)
    if case["kind"] != "attend" or (not case["past"] and not case["blind"]):
        return lq, lq
    g = np.random.default_rng([case["T"], case["n_seq"], 2])
    lk = [v + int(g.integers(0, case["past"] + 1)) * int(g.integers(0, 3) > 0) for v in lq]
    if case["blind"]:
        lk[0] = lq[0] // 2                                    # more queries than keys: the first half of them see nothing
    return lq, lk


def _starts(lens):
    return torch.tensor([0] + list(np.cumsum(lens)), dtype=torch.int32, device="cuda")


def _conv_dims(case):
    H, p, n, G = (case[k] for k in ("H", "p", "n", "G"))
    return H * p, H * p + 2 * G * n, 2 * H * p + 2 * G * n + H                  # d_inner, conv channels, columns of the projection


def _inputs(case, seed):
    g = torch.Generator(device="cuda").manual_seed((1000003 * seed + 29) % 2**62)
    dt = _DTYPES[case["dtype"]]
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    uni = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    if case["kind"] in ("conv", "conv_step"):
        _, ch, cols = _conv_dims(case)
        rows = case["T"] + case["tail"] if case["kind"] == "conv" else case["Bz"] * case["T"]
        seqs = case["n_seq"] if case["kind"] == "conv" else case["Bz"]
        x = dict(zx=rand(rows, cols).to(dt), conv_w=rand(ch, case["W"]) * case["W"] ** -0.5, conv_b=0.1 * rand(ch),
                 dt_bias=-6.9 + 4.6 * uni(case["H"]))                           # time steps between 0.001 and 0.1
        if case["kind"] == "conv_step" or case["window"]:
            x["window"] = rand(seqs, case["W"] - 1, ch).to(dt)
        return x
    if case["kind"] == "scan":
        rows, H, p, n, G = case["T"] + case["tail"], case["H"], case["p"], case["n"], case["G"]
        return dict(x=rand(rows, H, p).to(dt), B=rand(rows, G, n).to(dt), C=rand(rows, G, n).to(dt), dt=0.001 * 100.0 ** uni(rows, H),
                    A=-torch.exp(math.log(16.0) * uni(H)), D=rand(H) if case["skip"] else None,
                    state=rand(case["n_seq"], H, p, n) if case["state"] else None)
    if case["kind"] == "attend":
        lq, lk = _lens(case)
        rows_k = sum(lk) + case["tail"]
        Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
        offset = torch.where(uni(d) < 0.06, 4.0 * rand(d), 0.0)                 # a few channels of the keys stand out
        return dict(q=(1.5 * rand(case["T"] + case["tail"], Hq, d)).to(dt), k=(rand(rows_k, Hkv, d) + offset).to(dt), v=rand(rows_k, Hkv, d).to(dt))
    rows = case["rows"]
    gaps = uni(rows) * (2.0 * case["reach"] / rows)
    return dict(qkv=rand(rows, (case["Hq"] + 2 * case["Hkv"]) * case["d"]).to(dt), pos=gaps.double().cumsum(0).long().int())


def prepare(case, seed):
    st = dict(_inputs(case, seed), case=case)
    dt = _DTYPES[case["dtype"]]
    new = lambda *s, t=dt: torch.zeros(s, dtype=t, device="cuda")  # noqa: E731
    if case["kind"] == "rope":
        return st
    if case["kind"] == "conv_step":
        st["window_out"] = torch.zeros_like(st["window"])
        return st
    lq, lk = _lens(case)
    st["start"] = _starts(lq)
    rows = case["T"] + case["tail"]
    if case["kind"] == "attend":
        st.update(k_start=st["start"] if lq is lk else _starts(lk), o=new(rows, case["Hq"], case["d"]))
        return st
    H, p, n, G = (case[k] for k in ("H", "p", "n", "G"))
    if case["kind"] == "conv":
        st.update(out=(new(rows, H, p), new(rows, G, n), new(rows, G, n), new(rows, H, t=torch.float32)),
                  window_out=new(case["n_seq"], case["W"] - 1, H * p + 2 * G * n))
        return st
    st.update(y=new(rows, H, p), state_out=new(case["n_seq"], H, p, n, t=torch.float32))
    return st


# ------------------------------------------------------------------------------------------------ one pass
_CTX = []
_THETA, _TRAINED, _TURNS = 1.0e6, 32768, (1.0, 32.0)          # rotary base, trained length, and the turns between which bands blend


def _amplitude(case):
    return 1.0 + 0.1 * math.log(case["factor"]) if case["scaling"] == "banded" else 1.0


def _run_own(st):
    from paper_2603_00198_b200 import binding
    if not _CTX:
        _CTX.append(binding.Context(torch.cuda.current_device()))
    ctx, case = _CTX[0], st["case"]
    if case["kind"] == "rope":
        if "rope" not in st:                                                    # the description that a program keeps for its layers
            st["rope"] = binding.Rope(_THETA, rot_dim=case["rot"], layout=case["layout"], scaling=case["scaling"], factor=case["factor"],
                                      trained_len=_TRAINED, turns=_TURNS, amplitude=_amplitude(case))
        return binding.str_rope_split_ex(ctx, st["rope"], st["qkv"], st["pos"], case["Hq"], case["Hkv"], case["d"])
    if case["kind"] == "attend":
        return binding.str_attn_prefill_packed(ctx, st["q"], st["k"], st["v"], st["start"], case["d"] ** -0.5, k_start=st["k_start"], out=st["o"])
    if case["kind"] == "scan":
        return binding.str_mamba2_prefill_packed(ctx, st["x"], st["dt"], st["A"], st["B"], st["C"], st["start"], D=st["D"], init_state=st["state"],
                                                 final_state=st["state_out"], out=st["y"])
    dims = (case["H"], case["p"], case["n"], case["G"])
    if case["kind"] == "conv":
        out = binding.str_mamba_conv_packed(ctx, st["zx"], st["conv_w"], st["conv_b"], st["dt_bias"], st["start"], *dims, window=st.get("window"),
                                            window_out=st["window_out"], out=st["out"])
    else:
        out = binding.str_mamba_conv_step(ctx, st["zx"], st["conv_w"], st["conv_b"], st["dt_bias"], st["window"], case["Bz"], case["T"], *dims,
                                          window_out=st["window_out"])
    return (*out, st["window_out"])


def run(state):
    if own:
        return _run_own(state)
    return {"conv": _plain_conv, "conv_step": _plain_conv_step, "scan": _plain_scan, "attend": _plain_attend, "rope": _plain_rope}[state["case"]["kind"]](state)


def _taps(rows, w, b):
    """SiLU of the causal convolution of fp32 rows [..., W - 1 + T, channels]: the last T of them."""
    W = w.shape[1]
    T = rows.shape[-2] - (W - 1)
    u = b.expand(*rows.shape[:-2], T, -1)
    for j in range(W):
        u = u + w[:, j] * rows[..., j:j + T, :]
    return u / (1.0 + torch.exp(-u))


def _softplus(v):
    return torch.clamp_min(v, 0.0) + torch.log1p(torch.exp(-v.abs()))


def _plain_conv(st):
    case = st["case"]
    d_inner, ch, _ = _conv_dims(case)
    H, p, n, G, W = (case[k] for k in ("H", "p", "n", "G", "W"))
    x, B, C, dt = st["out"]
    at = 0
    for s, T in enumerate(_lens(case)[0]):
        rows = st["zx"][at:at + T, d_inner:d_inner + ch]
        before = st["window"][s] if case["window"] else torch.zeros_like(st["window_out"][s])
        rows = torch.cat((before, rows))
        st["window_out"][s] = rows[T:]
        if T:
            u = _taps(rows.float(), st["conv_w"], st["conv_b"])
            x[at:at + T] = u[:, :H * p].reshape(T, H, p)
            B[at:at + T] = u[:, H * p:H * p + G * n].reshape(T, G, n)
            C[at:at + T] = u[:, H * p + G * n:].reshape(T, G, n)
            dt[at:at + T] = _softplus(st["zx"][at:at + T, d_inner + ch:].float() + st["dt_bias"])
        at += T
    return x, B, C, dt, st["window_out"]


def _plain_conv_step(st):
    case = st["case"]
    d_inner, ch, cols = _conv_dims(case)
    Bz, T, H, p, n, G = (case[k] for k in ("Bz", "T", "H", "p", "n", "G"))
    zx = st["zx"].view(Bz, T, cols)
    rows = torch.cat((st["window"], zx[..., d_inner:d_inner + ch]), 1)
    st["window_out"].copy_(rows[:, T:])
    u = _taps(rows.float(), st["conv_w"], st["conv_b"]).to(st["zx"].dtype)
    dt = _softplus(zx[..., d_inner + ch:].float() + st["dt_bias"])
    return (u[..., :H * p].reshape(Bz, T, H, p), u[..., H * p:H * p + G * n].reshape(Bz, T, G, n), u[..., H * p + G * n:].reshape(Bz, T, G, n), dt,
            st["window_out"])


_CHUNK = 64


def _plain_scan(st):
    """In chunks: weights exp(l_t - l_j) dt_j (c_t . b_j) within one, states between them; sums of logarithms in 64 bits."""
    case = st["case"]
    H, p, n, G = (case[k] for k in ("H", "p", "n", "G"))
    per, Q = H // G, _CHUNK
    tri = torch.ones(Q, Q, dtype=torch.bool, device="cuda").tril()
    at = 0
    for s, T in enumerate(_lens(case)[0]):
        S = st["state"][s] if case["state"] else torch.zeros((H, p, n), device="cuda")
        for t0 in range(at, at + T, 32 * Q):                                    # 32 chunks at a time
            m = min(32 * Q, at + T - t0)
            nc = -(-m // Q)
            part = lambda t: torch.nn.functional.pad(t[t0:t0 + m].float(), (0, 0) * (t.dim() - 1) + (0, nc * Q - m)).unflatten(0, (nc, Q))  # noqa: E731
            x, dt, B, C = part(st["x"]), part(st["dt"]), part(st["B"]), part(st["C"])
            l = (dt.double() * st["A"].double()).cumsum(1).permute(0, 2, 1)     # [nc, H, Q]
            lag = (l[..., :, None] - l[..., None, :]).float().masked_fill(~tri, float("-inf"))
            CB = torch.matmul(C.permute(0, 2, 1, 3), B.permute(0, 2, 3, 1)).repeat_interleave(per, 1)
            w = CB * torch.exp(lag) * dt.permute(0, 2, 1)[:, :, None]
            xh = x.permute(0, 2, 1, 3)                                          # [nc, H, Q, p]
            y = torch.matmul(w, xh)
            xs = xh * (torch.exp((l[..., -1:] - l).float()) * dt.permute(0, 2, 1))[..., None]
            dS = torch.matmul(xs.transpose(-1, -2), B.permute(0, 2, 1, 3).repeat_interleave(per, 1))
            keep = torch.exp(l[..., -1].float())
            before = []
            for c in range(nc):
                before.append(S)
                S = S * keep[c][:, None, None] + dS[c]
            inter = torch.matmul(C.permute(0, 2, 1, 3).repeat_interleave(per, 1), torch.stack(before).transpose(-1, -2))
            y = y + inter * torch.exp(l.float())[..., None]
            if case["skip"]:
                y = y + st["D"][:, None, None] * xh
            st["y"][t0:t0 + m] = y.permute(0, 2, 1, 3).reshape(nc * Q, H, p)[:m]
        st["state_out"][s] = S
        at += T
    return st["y"], st["state_out"]


def _plain_attend(st):
    case = st["case"]
    Hq, Hkv = case["Hq"], case["Hkv"]
    R, scale = Hq // Hkv, case["d"] ** -0.5
    qa = ka = 0
    for lq, lk in zip(*_lens(case)):
        for r0 in range(0, lq, 4096):
            m = min(4096, lq - r0)
            seen = max(0, lk - lq + r0 + m)
            o = st["o"][qa + r0:qa + r0 + m]
            if seen == 0:
                o.zero_()
                continue
            last = lk - lq + r0 + torch.arange(m, device="cuda")
            hidden = torch.arange(seen, device="cuda") > last[:, None]
            for h in range(Hkv):
                q = st["q"][qa + r0:qa + r0 + m, h * R:(h + 1) * R].float().permute(1, 0, 2)
                K, V = st["k"][ka:ka + seen, h].float(), st["v"][ka:ka + seen, h].float()
                s = (torch.matmul(q, K.T) * scale).masked_fill_(hidden, float("-inf"))
                e = torch.exp(s - s.amax(-1, keepdim=True).clamp_min(-3.0e38))
                total = e.sum(-1, keepdim=True)
                o[:, h * R:(h + 1) * R] = (torch.matmul(e, V) / torch.where(total > 0, total, 1.0)).permute(1, 0, 2)
        qa, ka = qa + lq, ka + lk
    return st["o"]


def _frequencies(case):
    """Angles per position of the pairs, 64 bits."""
    f = _THETA ** (-2.0 * torch.arange(case["rot"] // 2, dtype=torch.float64, device="cuda") / case["rot"])
    if case["scaling"] == "linear":
        return f / case["factor"]
    if case["scaling"] == "banded":                                             # slow pairs stretched, fast ones kept, a ramp over the turns between
        kept = ((_TRAINED * f / (2.0 * math.pi) - _TURNS[0]) / (_TURNS[1] - _TURNS[0])).clamp(0.0, 1.0)
        return f * kept + f / case["factor"] * (1.0 - kept)
    return f


def _plain_rope(st):
    case = st["case"]
    Hq, Hkv, d, rot = (case[k] for k in ("Hq", "Hkv", "d", "rot"))
    rows = st["qkv"].view(case["rows"], Hq + 2 * Hkv, d)
    angle = st["pos"].double()[:, None] * _frequencies(case)
    cos, sin = ((f(angle) * _amplitude(case)).float()[:, None] for f in (torch.cos, torch.sin))
    x = rows[:, :Hq + Hkv].float()
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if case["layout"] == "half" else (x[..., 0:rot:2], x[..., 1:rot:2])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    turned = torch.cat((ra, rb), -1) if case["layout"] == "half" else torch.stack((ra, rb), -1).flatten(-2)
    x = torch.cat((turned, x[..., rot:]), -1).to(st["qkv"].dtype)
    return x[:, :Hq].contiguous(), x[:, Hq:].contiguous(), rows[:, Hq + Hkv:].contiguous()


# ------------------------------------------------------------------------------------------------ work and 64-bit results
def work(case):
    es = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "rope":
        wide = (case["Hq"] + 2 * case["Hkv"]) * case["d"]
        return dict(bytes=case["rows"] * (2 * wide * es + 4), flops=3 * case["rows"] * (case["Hq"] + case["Hkv"]) * case["rot"])
    if case["kind"] == "attend":
        lq, lk = _lens(case)
        pairs = sum(sum(range(max(0, k - q) + 1 if k >= q else 1, k + 1)) for q, k in zip(lq, lk))
        return dict(bytes=es * case["d"] * (2 * sum(lq) * case["Hq"] + 2 * sum(lk) * case["Hkv"]), flops=4 * pairs * case["Hq"] * case["d"])
    H, p, n, G = (case[k] for k in ("H", "p", "n", "G"))
    if case["kind"] == "scan":
        states = (1 + case["state"]) * 4 * case["n_seq"] * H * p * n
        return dict(bytes=case["T"] * (2 * H * p * es + 2 * G * n * es + 4 * H) + states, flops=5 * case["T"] * H * p * n)
    _, ch, _ = _conv_dims(case)
    rows = case["T"] if case["kind"] == "conv" else case["Bz"] * case["T"]
    windows = (2 if case["kind"] == "conv_step" else (1 + case["window"])) * (case["W"] - 1) * ch * es * (case["n_seq"] if case["kind"] == "conv" else case["Bz"])
    return dict(bytes=rows * (2 * ch * es + H * (es + 4)) + windows + 4 * ch * (case["W"] + 1), flops=rows * ch * (2 * case["W"] + 4))


def exact(case, seed):
    """The definitions in 64 bits: the convolution tap by tap over gathered rows, the recurrence token by token, attention head by head with
    a softmax per row, rotations as products of complex numbers."""
    x = _inputs(case, seed)
    f8 = lambda t: None if t is None else t.double()  # noqa: E731
    if case["kind"] == "rope":
        Hq, Hkv, d, rot = (case[k] for k in ("Hq", "Hkv", "d", "rot"))
        f = []
        for i in range(rot // 2):
            v = math.exp(-2.0 * i / rot * math.log(_THETA))
            if case["scaling"] == "linear":
                v /= case["factor"]
            elif case["scaling"] == "banded":
                turns = _TRAINED * v / (2.0 * math.pi)
                g = min(1.0, max(0.0, (turns - _TURNS[0]) / (_TURNS[1] - _TURNS[0])))
                v = g * v + (1.0 - g) * v / case["factor"]
            f.append(v)
        rows = f8(x["qkv"]).view(case["rows"], Hq + 2 * Hkv, d)
        turn = torch.polar(torch.full((case["rows"], rot // 2), _amplitude(case), dtype=torch.float64, device="cuda"),
                           f8(x["pos"])[:, None] * torch.tensor(f, dtype=torch.float64, device="cuda"))[:, None]
        out = rows.clone()
        first = torch.arange(rot // 2, device="cuda") * (1 if case["layout"] == "half" else 2)
        second = first + (rot // 2 if case["layout"] == "half" else 1)
        z = torch.complex(rows[:, :Hq + Hkv, first], rows[:, :Hq + Hkv, second]) * turn
        out[:, :Hq + Hkv, first], out[:, :Hq + Hkv, second] = z.real, z.imag
        return out[:, :Hq], out[:, Hq:Hq + Hkv], out[:, Hq + Hkv:]
    if case["kind"] in ("conv", "conv_step"):
        d_inner, ch, _ = _conv_dims(case)
        H, p, n, G, W = (case[k] for k in ("H", "p", "n", "G", "W"))
        packed = case["kind"] == "conv"
        lens = _lens(case)[0] if packed else [case["T"]] * case["Bz"]
        total = sum(lens)
        zx = x["zx"]
        u = f8(x["conv_b"]).repeat(total, 1)
        window = torch.zeros((len(lens), W - 1, ch), dtype=zx.dtype, device="cuda") if x.get("window") is None else x["window"]
        pool = torch.cat((window.flatten(0, 1), zx[:total, d_inner:d_inner + ch]))              # windows first, then the rows
        src, last, at = [], [], len(lens) * (W - 1)
        for s, T in enumerate(lens):
            line = list(range(s * (W - 1), (s + 1) * (W - 1))) + list(range(at, at + T))
            src += [line[t:t + W] for t in range(T)]
            last += line[T:]
            at += T
        if total:
            src = torch.tensor(src, device="cuda")
            for j in range(W):
                u += f8(x["conv_w"][:, j]) * f8(pool[src[:, j]])
        u = u * torch.special.expit(u)
        raw = f8(zx[:total, d_inner + ch:]) + f8(x["dt_bias"])
        dt = torch.logaddexp(raw, torch.zeros_like(raw))
        res = [u[:, :H * p].reshape(total, H, p), u[:, H * p:H * p + G * n].reshape(total, G, n), u[:, H * p + G * n:].reshape(total, G, n), dt]
        if packed:
            res = [torch.cat((r, torch.zeros((case["tail"], *r.shape[1:]), dtype=torch.float64, device="cuda"))) for r in res]
        else:
            res = [r.unflatten(0, (case["Bz"], case["T"])) for r in res]
        return (*res, f8(pool[torch.tensor(last, device="cuda")]).view(len(lens), W - 1, ch))
    if case["kind"] == "scan":
        H, p, n, G = (case[k] for k in ("H", "p", "n", "G"))
        lens, per = _lens(case)[0], H // G
        y = torch.zeros((case["T"] + case["tail"], H, p), dtype=torch.float64, device="cuda")
        S = torch.zeros((len(lens), H, p, n), dtype=torch.float64, device="cuda") if x["state"] is None else f8(x["state"])
        at = 0
        for s, T in enumerate(lens):
            Ss = S[s].view(G, per, p, n)
            decay = torch.exp(f8(x["dt"][at:at + T]) * f8(x["A"])).view(T, G, per, 1, 1)
            dx = (f8(x["dt"][at:at + T])[..., None] * f8(x["x"][at:at + T])).view(T, G, per * p, 1)
            B, C = f8(x["B"][at:at + T])[:, :, None], f8(x["C"][at:at + T])[..., None]
            for t in range(T):
                Ss.mul_(decay[t])
                Ss.view(G, per * p, n).baddbmm_(dx[t], B[t])
                torch.bmm(Ss.view(G, per * p, n), C[t], out=y[at + t].view(G, per * p, 1))
            at += T
        if case["skip"]:
            y[:at] += f8(x["D"])[:, None] * f8(x["x"][:at])
        return y, S
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    o = torch.zeros((case["T"] + case["tail"], Hq, d), dtype=torch.float64, device="cuda")
    qa = ka = 0
    for lq, lk in zip(*_lens(case)):
        for h in range(Hq):
            K, V = f8(x["k"][ka:ka + lk, h * Hkv // Hq]), f8(x["v"][ka:ka + lk, h * Hkv // Hq])
            for r0 in range(max(0, lq - lk), lq, 2048):
                r1 = min(lq, r0 + 2048)
                s = f8(x["q"][qa + r0:qa + r1, h]) @ K[:lk - lq + r1].T / math.sqrt(d)
                s += torch.full_like(s, float("-inf")).triu(lk - lq + r0 + 1)
                o[qa + r0:qa + r1, h] = torch.softmax(s, 1) @ V[:lk - lq + r1]
        qa, ka = qa + lq, ka + lk
    return o
