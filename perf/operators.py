"""The work of three operators of a decoder layer in training and serving: the gated feed-forward block in FP16 and FP8, activation
checkpoints in 8 bits (alone, and as what the gated block keeps for its backward pass), and the norms and the position rotation of
queries and keys on their way from the fused projection into attention's head layout.

``listed()`` names the cases, ``draw(rng)`` gives others of the same ranges.  ``prepare`` makes what a program has in hand before the
call, ``run`` makes one pass and returns its results: by elementary torch operations, or, where ``own`` is true, by the library's calls.
``exact`` computes the same results in 64 bits, ``work`` counts the bytes and operations that the pass cannot do without.

The operators, every product with the fixed factor that gives its result unit variance:

* gated block: Z = d^-1/2 X Wgu = [Zg | Zu];  H = a f(Zg) Zu;  Y = f^-1/2 H Wd, and backward dH = d^-1/2 G Wd^T;
  dZ = [b f'(Zg) Zu dH | a f(Zg) dH];  dX = (2f)^-1/2 dZ Wgu^T;  dWgu = T^-1/2 X^T dZ;  dWd = T^-1/2 H^T G,
  with a = 1 / rms f(z), b = 1 / rms f'(z) for z ~ N(0, 1).  In FP8 the operands X, Wgu, Wd, H are E4M3 and G, dZ E5M2 codes.
  The backward pass reads Z as it was kept, in FP16 or in 8 bits; nothing else is rounded on the way.
* 8-bit checkpoint of a row: blocks of 32 values share the power of two 2^e, the smallest that keeps the largest magnitude within
  127 steps after rounding; a value is held as round(x / 2^e).  The gated block's backward pass then takes Z and H from the codes.
* heads: x^ = x / sqrt(mean x^2 + eps) over a head, w x^, then every pair of columns turned by position * frequency; K's and V's heads
  are repeated for the query heads that share them, and their gradients added with the factor repeats^-1/2; weights' gradients get rows^-1/2.
"""
import math

import torch

own = False

DEV = "cuda:0"
GATES = ("silu", "gelu", "relu", "sigmoid")
MOST_FLOPS = 18.0 * 16384 * 4096 * 11008


def listed():
    return [
        # the block of a small layer, FP16, forward and backward: latency and launches count
        dict(name="gated_small", kind="gated", tokens=64, d=256, f=688, fp8=False, keep8=False, gate="silu", back=True),
        # serving one token of one user in FP8: three weight matrices are read for one row
        dict(name="gated_one_token", kind="gated", tokens=1, d=4096, f=11008, fp8=True, keep8=False, gate="silu", back=False),
        # serving a handful of users in FP16, a token each
        dict(name="gated_few_tokens", kind="gated", tokens=13, d=2048, f=5632, fp8=False, keep8=False, gate="gelu", back=False),
        # BERT-base widths in FP16 with two thirds of the inner width, which gives the same parameters: the ordinary step
        dict(name="gated_f16_base", kind="gated", tokens=4096, d=768, f=2048, fp8=False, keep8=False, gate="silu", back=True),
        # BERT-large widths in FP8 with its casts; Z is kept in FP16
        dict(name="gated_fp8_large", kind="gated", tokens=8192, d=1024, f=4096, fp8=True, keep8=False, gate="silu", back=True),
        # the same step with Z kept in 8 bits: what the checkpoints cost or gain
        dict(name="gated_fp8_kept8", kind="gated", tokens=8192, d=1024, f=4096, fp8=True, keep8=True, gate="silu", back=True),
        # packed sequences whose token count is odd, FP16 with 8-bit checkpoints, another gate, widths that end inside a tile
        dict(name="gated_f16_kept8_ragged", kind="gated", tokens=1999, d=1552, f=2064, fp8=False, keep8=True, gate="gelu", back=True),
        # LLM-size step in FP8 with 8-bit checkpoints: the largest call
        dict(name="gated_fp8_kept8_llm", kind="gated", tokens=16384, d=4096, f=11008, fp8=True, keep8=True, gate="silu", back=True),
        # checkpoints of a small activation, stored and loaded
        dict(name="keep8_small", kind="keep8", rows=65, n=1040, pitch=1040),
        # checkpoints of a layer's input, a part of wider rows
        dict(name="keep8_large", kind="keep8", rows=16384, n=8192, pitch=12288),
        # a step of generation: one new token of each of 48 sequences, far into them
        dict(name="heads_one_token", kind="heads", batch=48, s=1, heads=16, shared=1, dh=64, rot=64, pairs="halves", start=100000, back=False),
        # a training step with shared key and value heads, forward and backward
        dict(name="heads_train", kind="heads", batch=8, s=2048, heads=32, shared=4, dh=128, rot=128, pairs="halves", start=0, back=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _sixteens(rng, lo, hi):
    """A multiple of 16 in lo .. hi, spread over the logarithm; every other one a multiple of 128 where that fits."""
    v = _log(rng, lo, hi)
    unit = 128 if rng.random() < 0.5 and v >= 128 else 16
    return max(lo, min(hi // unit * unit, v // unit * unit))


def draw(rng):
    kind = rng.choice(["gated", "gated", "gated", "keep8", "heads", "heads"])
    if kind == "gated":
        while True:
            d, back = _sixteens(rng, 128, 4096), rng.random() < 0.6
            f = max(16, int(d * rng.choice([2, 8 / 3, 8 / 3, 3.5, 4])) // 16 * 16)
            case = dict(kind=kind, tokens=_log(rng, 1, 16384) if back else _log(rng, 1, 512), d=d, f=f, fp8=rng.random() < 0.5,
                        keep8=back and rng.random() < 0.5, gate=rng.choice(["silu", "silu", *GATES]), back=back)
            if work(case)["flops"] * (1 if case["fp8"] else 2.2) <= MOST_FLOPS:
                return case
    if kind == "keep8":
        n = _sixteens(rng, 16, 16384)
        pitch = n + rng.choice([0, 0, 8, 64, 4096])
        return dict(kind=kind, rows=_log(rng, 1, min(2 ** 27 // n, 2 ** 28 // pitch)), n=n, pitch=pitch)
    dh = rng.choice([32, 64, 64, 80, 96, 128, 128, 256])
    shared = rng.choice([1, 1, 2, 4, 8])
    s = rng.choice([1, _log(rng, 2, 8192), _log(rng, 2, 8192)])
    heads = shared * _log(rng, 1, 64 // shared)
    batch = _log(rng, 1, max(1, min(64 if s > 1 else 512, 2 ** 26 // (s * heads * dh))))
    return dict(kind=kind, batch=batch, s=s, heads=heads, shared=shared, dh=dh, rot=rng.choice([dh, dh, dh // 32 * 16]),
                pairs=rng.choice(["halves", "neighbours"]), start=rng.choice([0, 1, 5000, 1000000]), back=s > 1 and rng.random() < 0.7)


# ---- what a program has in hand ---------------------------------------------------------------------------------------

def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)

    def normal(*shape, sigma=1.0):
        return torch.empty(shape, dtype=torch.float16, device=DEV).normal_(0.0, sigma, generator=g)

    c, s = case, {"case": dict(case), "kept": {}}
    if c["kind"] == "gated":
        T, d, f = c["tokens"], c["d"], c["f"]
        s["X"], s["Wgu"], s["Wd"] = normal(T, d), normal(d, 2 * f), normal(f, d)
        if c["back"]:
            s["G"] = normal(T, d)
        elif c["fp8"]:            # serving: only the weights' codes are kept
            s["Wgu"], s["Wd"] = _to_e4m3(s["Wgu"]), _to_e4m3(s["Wd"])
    elif c["kind"] == "keep8":
        x = normal(c["rows"], c["pitch"])
        # activations have columns of another size than the rest, and outliers
        x *= torch.empty((c["pitch"],), dtype=torch.float16, device=DEV).log_normal_(0.0, 1.0, generator=g)
        at = torch.randint(0, x.numel(), (max(1, x.numel() // 1000),), generator=g, device=DEV)
        x.view(-1)[at] *= 30.0
        s["X"] = x
    else:
        T, h, k, dh = c["batch"] * c["s"], c["heads"], c["heads"] // c["shared"], c["dh"]
        s["QKV"] = normal(T, (h + 2 * k) * dh, sigma=1.5)
        s["wq"], s["wk"] = normal(dh, sigma=0.2) + 1, normal(dh, sigma=0.2) + 1
        first = torch.randint(0, c["start"] + 1, (c["batch"], 1), generator=g, device=DEV, dtype=torch.int32)
        s["pos"] = (first + torch.arange(c["s"], device=DEV, dtype=torch.int32)).reshape(T).contiguous()
        s["freq"] = 10000.0 ** (-torch.arange(c["rot"] // 2, device=DEV, dtype=torch.float64) / (c["rot"] / 2))
        if c["back"]:
            n = c["batch"] * h
            s["dQ"], s["dK"], s["dV"] = normal(n, c["s"], dh), normal(n, c["s"], dh), normal(n, c["s"], dh)
    return s


def run(state):
    c = state["case"]
    if own:
        return _OWN[c["kind"]](state, c)
    return _PLAIN[c["kind"]](state, c)


# ---- the plain forms ------------------------------------------------------------------------------------------------------

def _to_e4m3(x):
    return x.float().clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _to_e5m2(x):
    return x.float().clamp(-57344.0, 57344.0).to(torch.float8_e5m2)


#: 1 / rms f(z) and 1 / rms f'(z) for z ~ N(0, 1)
FACTORS = {"silu": (1.6765324703310909, 1.6233202579524972), "gelu": (1.5335304411955348, 1.481114412708348),
           "relu": (1.4142135623730951, 1.4142135623730951), "sigmoid": (1.8462285453386054, 4.722646085937973)}


def _plain_gate(gate, z):
    """f(z) and f'(z)."""
    if gate == "relu":
        return z * (z > 0), (z > 0).to(z.dtype)
    if gate == "gelu":
        P = 0.5 * torch.erfc(z * -(0.5 ** 0.5))
        return z * P, P + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    p = 1 / (1 + torch.exp(-z))
    if gate == "sigmoid":
        return p, p * (1 - p)
    return z * p, p * (1 + z * (1 - p))


def _plain_keep8(x):
    """Rows of floats -> the values that their 8-bit checkpoints stand for."""
    rows, n = x.shape
    b = torch.zeros((rows, -(-n // 32) * 32), dtype=x.dtype, device=x.device)
    b[:, :n] = x
    b = b.view(rows, -1, 32)
    big = b.abs().amax(2, keepdim=True)
    m, e = torch.frexp(big)                        # big = m 2^e, 1/2 <= m < 1: 127.5 steps of 2^(e-7) end at m = 255/256
    e = torch.where(m >= 255.0 / 256.0, e - 6, e - 7).clamp(-24, 9)
    step = ((e + 127) << 23).view(torch.float32)   # (torch.ldexp multiplies by a pow() that is not always a power of two)
    return ((b / step).round().clamp(-127, 127) * step).view(rows, -1)[:, :n]


def _run_gated_plain(state, c):
    T, d, f, fp8 = c["tokens"], c["d"], c["f"], c["fp8"]
    a, b = FACTORS[c["gate"]]
    cast = (lambda x: x.float() if "float8" in str(x.dtype) else _to_e4m3(x).float()) if fp8 else (lambda x: x.float())
    X, Wgu, Wd = cast(state["X"]), cast(state["Wgu"]), cast(state["Wd"])
    Z = (X @ Wgu) * d ** -0.5
    H = _plain_gate(c["gate"], Z[:, :f])[0] * Z[:, f:] * a
    H = cast(H)
    Y = (H @ Wd) * f ** -0.5
    if not c["back"]:
        return {"Y": Y.half()}
    if c["keep8"]:
        Z = torch.cat([_plain_keep8(Z[:, :f]), _plain_keep8(Z[:, f:])], 1)
    else:
        Z = Z.half().float()                       # as it is kept for the backward pass
    G = _to_e5m2(state["G"]).float() if fp8 else state["G"].float()
    dH = (G @ Wd.t()) * d ** -0.5
    F, S = _plain_gate(c["gate"], Z[:, :f])
    if c["keep8"]:
        H = cast(F * Z[:, f:] * a)
    dZ = torch.cat([S * Z[:, f:] * dH * b, F * dH * a], 1)
    if fp8:
        dZ = _to_e5m2(dZ).float()
    dX = (dZ @ Wgu.t()) * (2 * f) ** -0.5
    dWgu = (X.t() @ dZ) * T ** -0.5
    dWd = (H.t() @ G) * T ** -0.5
    return {"Y": Y.half(), "dX": dX.half(), "dWgu": dWgu.half(), "dWd": dWd.half()}


def _run_keep8_plain(state, c):
    return {"X": _plain_keep8(state["X"][:, :c["n"]].float()).half()}


def _turn(x, cos, sin, rot, pairs):
    """Every pair of the first `rot` columns of x [tokens, heads, dh] by its angle [tokens, 1, rot / 2]."""
    r, rest = x[..., :rot], x[..., rot:]
    if pairs == "halves":
        u, v = r[..., : rot // 2], r[..., rot // 2:]
        return torch.cat([u * cos - v * sin, v * cos + u * sin, rest], -1)
    u, v = r[..., 0::2], r[..., 1::2]
    return torch.cat([torch.stack([u * cos - v * sin, v * cos + u * sin], -1).flatten(-2), rest], -1)


def _heads_out(x, c, shared):
    """[tokens, heads, dh] -> [batch * query heads, s, dh]"""
    x = x.view(c["batch"], c["s"], -1, 1, c["dh"]).expand(-1, -1, -1, shared, -1)
    return x.permute(0, 2, 3, 1, 4).reshape(c["batch"] * c["heads"], c["s"], c["dh"])


def _heads_in(g, c, shared):
    """... and gradients back, those of shared heads added"""
    g = g.float().view(c["batch"], c["heads"] // shared, shared, c["s"], c["dh"]).sum(2) * shared ** -0.5
    return g.permute(0, 2, 1, 3).reshape(c["batch"] * c["s"], -1, c["dh"])


EPS = 1e-6


def _run_heads_plain(state, c):
    h, k, dh, rot, shared = c["heads"], c["heads"] // c["shared"], c["dh"], c["rot"], c["shared"]
    T = c["batch"] * c["s"]
    x = state["QKV"].float().view(T, h + 2 * k, dh)
    q, kk, v = x[:, :h], x[:, h: h + k], x[:, h + k:]
    angle = state["pos"].double()[:, None, None] * state["freq"]
    cos, sin = angle.cos().float(), angle.sin().float()
    wq, wk = state["wq"].float(), state["wk"].float()
    rq = (q.square().mean(-1, keepdim=True) + EPS).rsqrt()
    rk = (kk.square().mean(-1, keepdim=True) + EPS).rsqrt()
    out = {"Q": _heads_out(_turn(q * rq * wq, cos, sin, rot, c["pairs"]), c, 1).half(),
           "K": _heads_out(_turn(kk * rk * wk, cos, sin, rot, c["pairs"]), c, shared).half(), "V": _heads_out(v, c, shared).half()}
    if not c["back"]:
        return out
    gq = _turn(_heads_in(state["dQ"], c, 1), cos, -sin, rot, c["pairs"])
    gk = _turn(_heads_in(state["dK"], c, shared), cos, -sin, rot, c["pairs"])
    qh, kh = q * rq, kk * rk
    out["dwq"] = ((gq * qh).sum((0, 1)) * (T * h) ** -0.5).half()
    out["dwk"] = ((gk * kh).sum((0, 1)) * (T * k) ** -0.5).half()
    gq, gk = gq * wq, gk * wk
    dq = rq * (gq - qh * (gq * qh).mean(-1, keepdim=True))
    dk = rk * (gk - kh * (gk * kh).mean(-1, keepdim=True))
    out["dQKV"] = torch.cat([dq, dk, _heads_in(state["dV"], c, shared)], 1).reshape(T, -1).half()
    return out


_PLAIN = dict(gated=_run_gated_plain, keep8=_run_keep8_plain, heads=_run_heads_plain)


# ---- the library's calls ------------------------------------------------------------------------------------------------

def _buffer(state, name, shape, dtype=torch.float16):
    """A buffer that a program allocates once and keeps."""
    kept = state["kept"]
    if name not in kept:
        kept[name] = torch.empty(shape, dtype=dtype, device=DEV)
    return kept[name]


def _p(t):
    return None if t is None else t.data_ptr()


def _run_gated_own(state, c):
    import paper_2303_11257_amd as us

    T, d, f, fp8, back = c["tokens"], c["d"], c["f"], c["fp8"], c["back"]
    st = torch.cuda.current_stream().cuda_stream
    X, Wgu, Wd, G = state["X"], state["Wgu"], state["Wd"], state.get("G")
    u8, gate = torch.uint8, getattr(us, "GATE_" + c["gate"].upper())
    mode = (us.FFN_FP8 if fp8 else 0) | (us.FFN_KEEP8 if c["keep8"] else 0)
    if fp8:
        casts = [(X, "X8", us.E4M3)] + ([(Wgu, "Wgu8", us.E4M3), (Wd, "Wd8", us.E4M3), (G, "G8", us.E5M2)] if back else [])
        codes = [_buffer(state, n, x.shape, u8) for x, n, _ in casts]
        us.cast_fp8_batch([_p(x) for x, _, _ in casts], [_p(q) for q in codes], [x.numel() for x, _, _ in casts], [t for _, _, t in casts], st)
        X = codes[0]
        if back:
            Wgu, Wd, G = codes[1:]
    H = _buffer(state, "H", (T, f), u8 if fp8 else torch.float16)
    Y = _buffer(state, "Y", (T, d))
    Z = Zs = None
    if back:
        Z = _buffer(state, "Z", (T, 2 * f), torch.int8 if c["keep8"] else torch.float16)
        if c["keep8"]:
            Zs = _buffer(state, "Zs", (T, 2 * us.keep8_blocks(f)), u8)
    if "ws" not in state["kept"]:
        state["kept"]["ws"] = torch.empty((max(16, us.ffn_gated_workspace_bytes(T, d, f, mode)),), dtype=u8, device=DEV)
    ws = state["kept"]["ws"]
    us.ffn_gated_fwd(_p(X), _p(Wgu), _p(Wd), _p(Z), _p(Zs), _p(H), _p(Y), T, d, f, gate, mode, _p(ws), ws.numel(), st)
    if not back:
        return {"Y": Y}
    dZ = _buffer(state, "dZ", (T, 2 * f), u8 if fp8 else torch.float16)
    dX, dWgu, dWd = _buffer(state, "dX", (T, d)), _buffer(state, "dWgu", (d, 2 * f)), _buffer(state, "dWd", (f, d))
    us.ffn_gated_bwd(_p(X), _p(Wgu), _p(Wd), _p(Z), _p(Zs), _p(H), _p(G), _p(dZ), _p(dX), _p(dWgu), _p(dWd), T, d, f, gate, mode,
                     _p(ws), ws.numel(), st)
    return {"Y": Y, "dX": dX, "dWgu": dWgu, "dWd": dWd}


def _run_keep8_own(state, c):
    import paper_2303_11257_amd as us

    rows, n, st = c["rows"], c["n"], torch.cuda.current_stream().cuda_stream
    codes = _buffer(state, "codes", (rows, n), torch.int8)
    scales = _buffer(state, "scales", (rows, us.keep8_blocks(n)), torch.uint8)
    X = _buffer(state, "X", (rows, n))
    us.keep8_store(_p(state["X"]), c["pitch"], _p(codes), _p(scales), rows, n, st)
    us.keep8_load(_p(codes), _p(scales), _p(X), n, rows, n, st)
    return {"X": X}


def _run_heads_own(state, c):
    import paper_2303_11257_amd as us

    h, k, dh, s, batch = c["heads"], c["heads"] // c["shared"], c["dh"], c["s"], c["batch"]
    T, ld, st = batch * s, (h + 2 * k) * dh, torch.cuda.current_stream().cuda_stream
    pairs = us.ROPE_HALVES if c["pairs"] == "halves" else us.ROPE_NEIGHBOURS
    Q, K, V = (_buffer(state, n, (batch * h, s, dh)) for n in ("Q", "K", "V"))
    x, wq, wk, pos, freq = (_p(state[n]) for n in ("QKV", "wq", "wk", "pos", "freq"))
    us.qk_norm_rope_fwd(x, ld, wq, wk, pos, freq, _p(Q), _p(K), _p(V), batch, s, h, k, dh, c["rot"], pairs, EPS, st)
    out = {"Q": Q, "K": K, "V": V}
    if c["back"]:
        dQKV, dwq, dwk = _buffer(state, "dQKV", (T, ld)), _buffer(state, "dwq", (dh,)), _buffer(state, "dwk", (dh,))
        if "ws" not in state["kept"]:
            state["kept"]["ws"] = torch.empty((max(16, us.qk_norm_rope_workspace_bytes(batch, s, h, k, dh)),), dtype=torch.uint8, device=DEV)
        ws = state["kept"]["ws"]
        us.qk_norm_rope_bwd(x, ld, wq, wk, pos, freq, _p(state["dQ"]), _p(state["dK"]), _p(state["dV"]), _p(dQKV), ld, _p(dwq), _p(dwk),
                            batch, s, h, k, dh, c["rot"], pairs, EPS, 0.0, 0.0, _p(ws), ws.numel(), st)
        out.update(dQKV=dQKV, dwq=dwq, dwk=dwk)
    return out


_OWN = dict(gated=_run_gated_own, keep8=_run_keep8_own, heads=_run_heads_own)


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------

def _exact_fp8(x, bits, least, top):
    """Nearest value with `bits` bits behind the leading one, exponents from `least` on, clipped at `top`."""
    e = torch.frexp(x)[1].long().sub(1).clamp_min(least)
    step = (e - bits + 1023).bitwise_left_shift(52).view(torch.float64)
    return (x / step).round().mul(step).clamp(-top, top)


def _exact_gated(s, c):
    T, d, f = c["tokens"], c["d"], c["f"]
    e4 = (lambda x: _exact_fp8(x, 3, -6, 448.0)) if c["fp8"] else (lambda x: x)
    e5 = (lambda x: _exact_fp8(x, 2, -14, 57344.0)) if c["fp8"] else (lambda x: x)
    X, Wgu, Wd = (e4(s[n].double()) for n in ("X", "Wgu", "Wd"))
    zg = torch.matmul(X, Wgu[:, :f]) / math.sqrt(d)
    zu = torch.matmul(X, Wgu[:, f:]) / math.sqrt(d)
    Phi, phi = torch.special.ndtr, lambda z: torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    fn = {"silu": lambda z: z * torch.sigmoid(z), "gelu": lambda z: z * Phi(z), "relu": torch.relu, "sigmoid": torch.sigmoid}[c["gate"]]
    slope = {"silu": lambda z: torch.sigmoid(z) + z * torch.sigmoid(z) * torch.sigmoid(-z), "gelu": lambda z: Phi(z) + z * phi(z),
             "relu": lambda z: torch.heaviside(z, torch.zeros_like(z)), "sigmoid": lambda z: torch.sigmoid(z) * torch.sigmoid(-z)}[c["gate"]]
    # the factors, by the midpoint rule over the normal density
    t = (torch.arange(48000, dtype=torch.float64, device=X.device) + 0.5) * (24 / 48000) - 12
    a, b = (1 / math.sqrt(float((g(t) ** 2 * phi(t)).sum()) * 24 / 48000) for g in (fn, slope))
    H = e4(a * fn(zg) * zu)
    out = {"Y": torch.matmul(H, Wd) / math.sqrt(f)}
    if not c["back"]:
        return out
    if c["keep8"]:
        zg, zu = _exact_keep8(zg), _exact_keep8(zu)
        H = e4(a * fn(zg) * zu)
    else:
        zg, zu = zg.half().double(), zu.half().double()
    G = e5(s["G"].double())
    dH = torch.matmul(G, Wd.t()) / math.sqrt(d)
    dzg, dzu = e5(b * slope(zg) * zu * dH), e5(a * fn(zg) * dH)
    out["dX"] = (torch.matmul(dzg, Wgu[:, :f].t()) + torch.matmul(dzu, Wgu[:, f:].t())) / math.sqrt(2 * f)
    out["dWgu"] = torch.cat([torch.matmul(X.t(), dzg), torch.matmul(X.t(), dzu)], 1) / math.sqrt(T)
    out["dWd"] = torch.matmul(H.t(), G) / math.sqrt(T)
    return out


def _exact_keep8(x):
    n = x.shape[1]
    parts = []
    for part in torch.nn.functional.pad(x, (0, -n % 32)).split(2 ** 13, dim=1):          # whole blocks at a time
        w = part.reshape(part.shape[0], -1, 32)
        top = w.abs().max(-1, keepdim=True).values
        step = torch.full_like(top, 2.0 ** -24)
        for k in range(-23, 10):                   # the smallest power of two whose 127.5 steps are not reached
            step = torch.where(top >= 127.5 * 2.0 ** (k - 1), 2.0 ** k, step)
        parts.append(((w / step).round().clamp(-127, 127) * step).flatten(1))
    return torch.cat(parts, 1)[:, :n]


def _exact_heads(s, c):
    B, S, h, r, dh, rot = c["batch"], c["s"], c["heads"], c["shared"], c["dh"], c["rot"]
    k = h // r
    x = s["QKV"].double().view(B, S, h + 2 * k, dh).transpose(1, 2)              # batch, head, token, column
    turn = torch.exp(1j * s["pos"].double().view(B, 1, S, 1) * s["freq"])

    def pairs(y):
        y = y[..., :rot]
        return torch.complex(y[..., : rot // 2], y[..., rot // 2:]) if c["pairs"] == "halves" else torch.view_as_complex(y.unflatten(-1, (-1, 2)).contiguous())

    def columns(z, rest):
        z = torch.cat([z.real, z.imag], -1) if c["pairs"] == "halves" else torch.view_as_real(z).flatten(-2)
        return torch.cat([z, rest[..., rot:]], -1)

    out, grads = {}, []
    for name, at, n, rep in (("q", 0, h, 1), ("k", h, k, r)):
        y, w = x[:, at: at + n], s["w" + name].double()
        rms = torch.sqrt((y ** 2).mean(-1, keepdim=True) + EPS)
        u = y / rms
        o = columns(pairs(u * w) * turn, u * w)
        out[name.upper()] = o.repeat_interleave(rep, 1).reshape(B * h, S, dh)
        if c["back"]:
            g = s["d" + name.upper()].double().view(B, n, rep, S, dh).sum(2) / math.sqrt(rep)
            g = columns(pairs(g) * turn.conj(), g)
            out["dw" + name] = (g * u).sum((0, 1, 2)) / math.sqrt(B * S * n)
            g = g * w
            grads.append((g - u * (g * u).mean(-1, keepdim=True)) / rms)
    out["V"] = x[:, h + k:].repeat_interleave(r, 1).reshape(B * h, S, dh)
    if c["back"]:
        grads.append(s["dV"].double().view(B, k, r, S, dh).sum(2) / math.sqrt(r))
        out["dQKV"] = torch.cat(grads, 1).transpose(1, 2).reshape(B * S, -1)
    return out


def exact(case, seed):
    s, c = prepare(case, seed), case
    if c["kind"] == "gated":
        return _exact_gated(s, c)
    if c["kind"] == "keep8":
        return {"X": _exact_keep8(s["X"][:, :c["n"]].double())}
    return _exact_heads(s, c)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------------

def work(case):
    """Inputs read and results written once per direction, what lives from the forward to the backward pass written and read once; a
    product is 2 operations per pair of factors, everything else counts as traffic."""
    c = case
    if c["kind"] == "gated":
        T, d, f, es = c["tokens"], c["d"], c["f"], 1 if c["fp8"] else 2
        operands = es * (T * d + 3 * d * f)
        total = operands + 2 * T * d
        cast = 3 * T * d if c["fp8"] else 0
        if c["back"]:
            kept = (1 + 1 / 32 if c["keep8"] else 2) * 2 * T * f
            total += 2 * kept + operands + es * T * d + 2 * (T * d + 3 * d * f)
            cast += 3 * (T * d + 3 * d * f) if c["fp8"] else 0
        return {"bytes": float(total + cast), "flops": 6.0 * T * d * f * (3 if c["back"] else 1)}
    if c["kind"] == "keep8":
        return {"bytes": c["rows"] * c["n"] * (6 + 2 / 32), "flops": 0.0}
    T, h, k, dh = c["batch"] * c["s"], c["heads"], c["heads"] // c["shared"], c["dh"]
    x, y = 2 * T * (h + 2 * k) * dh, 2 * T * 3 * h * dh
    return {"bytes": float(x + y + (2 * x + y if c["back"] else 0)), "flops": 0.0}
