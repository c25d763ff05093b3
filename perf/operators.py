"""The operators around a transformer's quantized linears, as calls to time and to
compare: the root-mean-square norm with the residual's addition and a quantized
output, the linear with bias, activation and residual in its epilogue, an MLP of
the two, and rotary positions.

A case's ``kind`` says which.  ``run`` computes it with plain torch operations in
32 bits, or (``own``) by the package's calls.  Sizes come from the package's own
workloads (4608 tokens of a 1024 x 1024 image and its prompt, width 3072, MLP 12288,
the translator's 512 tokens and widths 1024 / 2560, batch 4) and from the ragged
shapes of its tests; drawn cases spread over the same ranges.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

HIDDEN, MLP, TOKENS = 3072, 12288, 4608
MAX_MACS = TOKENS * MLP * HIDDEN          # multiply-adds of the largest linear
ACTS = ("none", "relu", "silu", "gelu_tanh", "gelu")
F16 = {"bf16": torch.bfloat16, "fp16": torch.float16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


# ---------------------------------------------------------------- the cases ---

def listed():
    return [
        # the norm before a block's FP8 linears: the residual stream of a 1024 x 1024
        # image's tokens takes the last layer's output, one scale per token
        _case("norm_fp8_rows", "norm", M=TOKENS, K=HIDDEN, dtype="bf16", out="fp8_rows",
              residual=True, weight=True, ld=1),
        # the same for one token, where only latency counts
        _case("norm_fp8_rows_one_token", "norm", M=1, K=HIDDEN, dtype="bf16", out="fp8_rows",
              residual=True, weight=True, ld=1),
        # batch 4 in fp16 without a residual, calibrated scale, x a view of wider rows
        _case("norm_fp8_static_b4", "norm", M=4 * TOKENS, K=HIDDEN, dtype="fp16", out="fp8",
              residual=False, weight=True, ld=3),
        # the MLP's up-projection in FP8: bias, GELU, and only the next layer's FP8
        # input written
        _case("linear_fp8_up_gelu", "linear", fmt="fp8", M=TOKENS, N=MLP, K=HIDDEN, rows=True,
              bias=True, act="gelu_tanh", residual=False, rq=True),
        # the MLP's down-projection in NVFP4, added to the residual stream
        _case("linear_nvfp4_down_residual", "linear", fmt="nvfp4", M=TOKENS, N=HIDDEN, K=MLP,
              rows=False, bias=True, act="none", residual=True, rq=False),
        # one token through a 16-bit linear with SiLU: a step's conditioning vector
        _case("linear_bf16_one_token", "linear", fmt="bf16", M=1, N=MLP, K=HIDDEN, rows=False,
              bias=True, act="silu", residual=False, rq=False),
        # a few tokens against a long K: the down-projection of single-token steps
        _case("linear_fp8_few_tokens", "linear", fmt="fp8", M=8, N=HIDDEN, K=MLP, rows=True,
              bias=True, act="none", residual=True, rq=False),
        # a prompt's odd token count through an fp16 linear of ragged widths
        _case("linear_fp16_ragged", "linear", fmt="fp16", M=1333, N=2112, K=1088, rows=False,
              bias=True, act="gelu", residual=True, rq=False),
        # a block's MLP in NVFP4 as it is used: norm of x + residual, up with GELU
        # re-quantized, down added back
        _case("mlp_nvfp4", "mlp", M=TOKENS, H=HIDDEN, F=MLP, act="gelu_tanh"),
        # q and k of a QKV output, image positions on three axes
        _case("rope_qk_image", "rope", T=TOKENS, H=48, D=128, R=128, axes="16,56,56",
              layout="interleaved", dtype="bf16", inverse=False, scaling="none", factor=1.0,
              span=64, packed=False),
        # one new token far into a long context: half the head rotated, frequencies
        # scaled for the length
        _case("rope_one_token_long", "rope", T=1, H=40, D=128, R=64, axes="", layout="half",
              dtype="bf16", inverse=False, scaling="yarn", factor=32.0, span=1 << 20, packed=True),
        # the gradient's rotation back over an odd number of tokens in fp16
        _case("rope_inverse_ragged", "rope", T=1333, H=24, D=96, R=96, axes="", layout="half",
              dtype="fp16", inverse=True, scaling="ntk", factor=4.0, span=32768, packed=True),
    ]


def _case(name, kind, **kw):
    return {"name": name, "kind": kind, **kw}


def _log_int(rng, lo, hi, multiple=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / multiple)) * multiple
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["norm", "norm", "linear", "linear", "linear", "linear", "mlp", "rope", "rope"])
    if kind == "norm":
        M, K = _log_int(rng, 1, 4 * TOKENS), _log_int(rng, 64, MLP, 64)
        M = max(1, min(M, 4 * TOKENS * HIDDEN // K))
        return {"kind": kind, "M": M, "K": K, "dtype": rng.choice(["bf16", "fp16"]),
                "out": rng.choice(["fp8_rows", "fp8_rows", "fp8", "16"]),
                "residual": rng.random() < 0.6, "weight": rng.random() < 0.8,
                "ld": rng.choice([1, 1, 3])}
    if kind == "linear":
        M, N, K = _log_int(rng, 1, TOKENS), _log_int(rng, 64, MLP, 64), _log_int(rng, 64, MLP, 64)
        M = max(1, min(M, MAX_MACS // (N * K)))
        fmt = rng.choice(["nvfp4", "fp8", "bf16", "fp16"])
        if fmt in F16:
            M = max(1, min(M, MAX_MACS // 4 // (N * K)))
        return {"kind": kind, "fmt": fmt, "M": M, "N": N, "K": K,
                "rows": fmt == "fp8" and rng.random() < 0.6, "bias": rng.random() < 0.7,
                "act": rng.choice(ACTS), "residual": rng.random() < 0.5,
                "rq": fmt == "fp8" and rng.random() < 0.4}
    if kind == "mlp":
        M, H = _log_int(rng, 1, TOKENS), _log_int(rng, 256, HIDDEN, 64)
        F = _log_int(rng, 256, MLP, 64)
        return {"kind": kind, "M": max(1, min(M, MAX_MACS // (2 * H * F))), "H": H, "F": F,
                "act": rng.choice(ACTS[1:])}
    T, H = _log_int(rng, 1, 2 * TOKENS), _log_int(rng, 1, 96)
    D = rng.choice([64, 80, 96, 128, 192, 256])
    T = max(1, min(T, 2 * TOKENS * 48 * 128 // (H * D)))
    axes = rng.choice(["", "", "1,1", "1,2,1"])
    R = rng.choice([D, D, D // 2])
    if axes:
        parts = [int(p) for p in axes.split(",")]
        unit = R // sum(parts) // 2 * 2
        sizes = [unit * p for p in parts]
        R, axes = sum(sizes), ",".join(map(str, sizes))
    scaling = rng.choice(["none", "linear", "ntk", "yarn"])
    return {"kind": kind, "T": T, "H": H, "D": D, "R": R, "axes": axes,
            "layout": rng.choice(["interleaved", "half"]), "dtype": rng.choice(["bf16", "fp16"]),
            "inverse": rng.random() < 0.4, "scaling": scaling,
            "factor": 1.0 if scaling == "none" else rng.choice([2.0, 8.0, 32.0]),
            "span": _log_int(rng, 64, 1 << 20), "packed": rng.random() < 0.5}


# --------------------------------------------------------------- the inputs ---

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + stream * 7919 + 29) % (1 << 62))


def _normal(seed, stream, *shape, sigma=1.0):
    return torch.randn(*shape, generator=_gen(seed, stream), device="cuda").mul_(sigma)


def _stream_values(seed, stream, M, K):
    """A residual stream: N(0, 1) with 1% of the channels x20."""
    x = _normal(seed, stream, M, K)
    ch = torch.randperm(K, generator=_gen(seed, stream + 50), device="cuda")[:max(1, K // 100)]
    x[:, ch] *= 20.0
    return x


def _nvfp4(v):
    """(packed codes, block scales in the 128 x 4 atom layout, tensor scale) of v."""
    rows, K = v.shape
    sdec = (v.abs().amax() / 2688.0).reshape(1)
    b = v.view(rows, K // 16, 16)
    s = (b.abs().amax(2) / sdec / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
    sf = s.float()
    q = torch.where(sf[..., None] > 0, b / sdec / sf[..., None], torch.zeros((), device=v.device))
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=v.device)
    code = torch.bucketize(q.abs(), edges).to(torch.uint8) | (q.signbit().to(torch.uint8) << 3)
    code = code.view(rows, K // 2, 2)
    packed = (code[..., 0] | (code[..., 1] << 4)).contiguous()
    pad = torch.zeros((rows + 127) // 128 * 128, K // 16, dtype=torch.uint8, device=v.device)
    pad[:rows] = s.view(torch.uint8)
    atoms = pad.view(-1, 4, 32, K // 64, 4).permute(0, 3, 2, 1, 4).contiguous()
    return packed, atoms.view(-1), sdec


def _fp8(v, per_row):
    """(codes, scale or scales) of v."""
    amax = v.abs().amax(1) if per_row else v.abs().amax().reshape(1)
    s = torch.where(amax > 0, amax / 448.0, torch.ones((), device=v.device))
    return (v / (s[:, None] if per_row else s)).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8), s


def _weight_like(case, seed, N, K, stream):
    return _normal(seed, stream, N, K, sigma=1.0 / math.sqrt(K))


def _axes(case):
    return [int(a) for a in case["axes"].split(",")] if case["axes"] else [case["R"]]


def _frequencies(R, scaling, factor, base=10000.0, length=4096):
    """(radians per position of each pair, magnitude) in 64 bits."""
    i = np.arange(R // 2, dtype=np.float64)
    if scaling == "ntk" and R > 2:
        return (base * factor ** (R / (R - 2))) ** (-2.0 * i / R), 1.0
    f = base ** (-2.0 * i / R)
    if scaling == "linear" or scaling == "ntk":
        return f / factor, 1.0
    if scaling == "yarn":
        # pairs that turn more than 32 times over the trained length keep their
        # frequency, those that turn less than once take f / factor
        at = lambda turns: R * math.log(length / (turns * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        low, high = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), R - 1)
        ramp = np.clip((i - low) / max(high - low, 1e-3), 0.0, 1.0)
        return f * (1 - ramp) + f / factor * ramp, 0.1 * math.log(factor) + 1.0
    return f, 1.0


def prepare(case, seed):
    kind, st = case["kind"], {"case": case}
    if kind == "norm":
        M, K, dt = case["M"], case["K"], F16[case["dtype"]]
        wide = torch.zeros(M, case["ld"] * K, dtype=dt, device="cuda")
        st["x"] = wide[:, :K].copy_(_stream_values(seed, 1, M, K))
        st["residual"] = _normal(seed, 2, M, K).to(dt) if case["residual"] else None
        st["sum"] = torch.empty(M, K, dtype=dt, device="cuda") if case["residual"] else None
        st["weight"] = (1 + _normal(seed, 3, K, sigma=0.1)).to(dt) if case["weight"] else None
        st["scale"] = torch.full((1,), 16.0 / 448, device="cuda")
        st["y"] = torch.empty(M, K, dtype=dt if case["out"] == "16" else torch.uint8, device="cuda")
        st["row_scales"] = torch.empty(M if case["out"] == "fp8_rows" else 1, device="cuda")
    elif kind == "linear":
        M, N, K, fmt = case["M"], case["N"], case["K"], case["fmt"]
        dt = F16.get(fmt, torch.bfloat16)
        a, w = _stream_values(seed, 1, M, K), _weight_like(case, seed, N, K, 2)
        if fmt == "nvfp4":
            st["a"], st["w"] = _nvfp4(a), _nvfp4(w)
        elif fmt == "fp8":
            st["a"], st["w"] = _fp8(a, case["rows"]), _fp8(w, True)
        else:
            st["a"], st["w"] = a.to(dt), w.to(dt)
        st["bias"] = _normal(seed, 3, N).to(dt) if case["bias"] else None
        st["residual"] = _normal(seed, 4, M, N).to(dt) if case["residual"] else None
        st["next_scale"] = torch.full((1,), 16.0 / 448, device="cuda")
        st["q"] = torch.empty(M, N, dtype=torch.uint8, device="cuda") if case["rq"] else None
        st["q_scale"] = torch.empty(1, device="cuda")
        st["y"] = None if case["rq"] else torch.empty(M, N, dtype=dt, device="cuda")
    elif kind == "mlp":
        M, H, F, dt = case["M"], case["H"], case["F"], torch.bfloat16
        st["x"], st["residual"] = _stream_values(seed, 1, M, H).to(dt), _normal(seed, 2, M, H).to(dt)
        st["sum"], st["y"] = (torch.empty(M, H, dtype=dt, device="cuda") for _ in range(2))
        st["weight"] = (1 + _normal(seed, 3, H, sigma=0.1)).to(dt)
        st["up"], st["down"] = (_nvfp4(_weight_like(case, seed, F, H, 4)),
                                _nvfp4(_weight_like(case, seed, H, F, 5)))
        st["up_bias"], st["down_bias"] = _normal(seed, 6, F, sigma=0.1).to(dt), _normal(seed, 7, H, sigma=0.1).to(dt)
        st["in_scale"], st["h_scale"] = (torch.full((1,), v / 2688, device="cuda") for v in (12.0, 6.0))
        st["qs"] = [(torch.empty(M, w // 2, dtype=torch.uint8, device="cuda"),
                     torch.zeros((M + 127) // 128 * (w // 64) * 512, dtype=torch.uint8, device="cuda"),
                     torch.empty(1, device="cuda")) for w in (H, F)]
    else:
        T, H, D, dt = case["T"], case["H"], case["D"], F16[case["dtype"]]
        wide = torch.zeros(T, H * D if case["packed"] else 3 * H * D // 2, dtype=dt, device="cuda")
        st["x"] = wide[:, :H * D].copy_(_normal(seed, 1, T, H * D)).view(T, H, D)
        A = len(_axes(case))
        pos = torch.randint(0, case["span"], (T, A), generator=_gen(seed, 2), device="cuda")
        st["positions"] = (pos if A > 1 else pos[:, 0].contiguous()).to(torch.int32)
        f = [_frequencies(R, case["scaling"], case["factor"]) for R in _axes(case)]
        # turns per position as 64-bit fractions of a turn
        turns = np.round(np.concatenate([v[0] for v in f]) / (2 * math.pi) * 2.0**64)
        st["turns"] = torch.from_numpy(turns.astype(np.uint64).view(np.int64)).cuda()
        st["magnitude"] = f[0][1]
        st["y"] = torch.empty(T, H, D, dtype=dt, device="cuda")
    return st


# ------------------------------------------------------------ the plain form ---

def _act(v, act):
    if act == "relu":
        return v.clamp(min=0)
    if act == "silu":
        return v / (1 + torch.exp(-v))
    if act == "gelu_tanh":
        return 0.5 * v * (1 + torch.tanh(math.sqrt(2 / math.pi) * (v + 0.044715 * v * v * v)))
    if act == "gelu":
        return 0.5 * v * (1 + torch.erf(v * math.sqrt(0.5)))
    return v


def _decode_nvfp4(q, rows, K):
    """Values of the codes times their block scales; the tensor scale stays apart."""
    packed, scales, _ = q
    grid = torch.tensor(E2M1 + tuple(-v for v in E2M1), device="cuda")
    v = torch.stack([grid[(packed & 15).long()], grid[(packed >> 4).long()]], 2).view(rows, K // 16, 16)
    s = scales.view(-1, K // 64, 32, 4, 4).permute(0, 3, 2, 1, 4).reshape(-1, K // 16)[:rows]
    return (v * s.contiguous().view(torch.float8_e4m3fn).float()[..., None]).view(rows, K)


def _norm_plain(st, M, K):
    s = st["x"].float()
    if st["residual"] is not None:
        s = s + st["residual"].float()
    n = s * torch.rsqrt((s * s).mean(1, keepdim=True) + EPS)
    return s, n if st["weight"] is None else n * st["weight"].float()


def _to_e4m3(v):
    return v.clamp(-448, 448).to(torch.float8_e4m3fn)


def _plain_nvfp4_values(v, sdec):
    """v through NVFP4 with tensor scale sdec: values without it."""
    b = v.view(v.shape[0], -1, 16)
    senc = 1.0 / sdec
    s = _to_e4m3(b.abs().amax(2) * senc / 6.0).float()
    r = torch.where(s > 0, senc / s, torch.zeros((), device=v.device))
    q = b * r[..., None]
    a = q.abs()
    # nearest, ties to the even code
    up = torch.tensor(E2M1, device=v.device)
    code = ((a > 0.25).int() + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    return (torch.copysign(up[code.long()], q) * s[..., None]).view(v.shape)


def _run_plain(st):
    case, kind = st["case"], st["case"]["kind"]
    if kind == "norm":
        s, n = _norm_plain(st, case["M"], case["K"])
        out = {} if st["residual"] is None else {"sum": s.to(st["x"].dtype)}
        if case["out"] == "16":
            return {**out, "y": n.to(st["x"].dtype)}
        if case["out"] == "fp8":
            return {**out, "codes": _to_e4m3(n * (1.0 / st["scale"]))}
        amax = n.abs().amax(1)
        S = torch.where(amax > 0, amax / 448.0, torch.ones((), device="cuda"))
        return {**out, "codes": _to_e4m3(n * (1.0 / S)[:, None]), "scales": S}
    if kind == "linear":
        M, N, K, fmt = case["M"], case["N"], case["K"], case["fmt"]
        if fmt == "nvfp4":
            v = _decode_nvfp4(st["a"], M, K) @ _decode_nvfp4(st["w"], N, K).t()
            v = v * (st["a"][2] * st["w"][2])
        elif fmt == "fp8":
            v = st["a"][0].view(torch.float8_e4m3fn).float() @ st["w"][0].view(torch.float8_e4m3fn).float().t()
            v = v * (st["a"][1][:, None] * st["w"][1])
        else:
            v = st["a"].float() @ st["w"].float().t()
        if st["bias"] is not None:
            v = v + st["bias"].float()
        v = _act(v, case["act"])
        if st["residual"] is not None:
            v = v + st["residual"].float()
        y = v.to(F16.get(fmt, torch.bfloat16))
        return {"codes": _to_e4m3(y.float() * (1.0 / st["next_scale"]))} if case["rq"] else {"y": y}
    if kind == "mlp":
        M, H, F = case["M"], case["H"], case["F"]
        s, n = _norm_plain(st, M, H)
        a = _plain_nvfp4_values(n, st["in_scale"])
        v = a @ _decode_nvfp4(st["up"], F, H).t() * (st["in_scale"] * st["up"][2]) + st["up_bias"].float()
        h = _plain_nvfp4_values(_act(v, case["act"]).to(torch.bfloat16).float(), st["h_scale"])
        y = h @ _decode_nvfp4(st["down"], H, F).t() * (st["h_scale"] * st["down"][2])
        sum16 = s.to(torch.bfloat16)
        return {"sum": sum16, "y": (y + st["down_bias"].float() + sum16.float()).to(torch.bfloat16)}
    # rotary: the top 32 bits of position x turns are the angle as a fraction of a turn
    x, R = st["x"], case["R"]
    pairs = [a // 2 for a in _axes(case)]
    pos = st["positions"].long().view(case["T"], -1)
    p = torch.repeat_interleave(pos, torch.tensor(pairs, device="cuda"), 1, output_size=R // 2)
    angle = ((p * st["turns"]) >> 32).float() * (math.pi * 2.0**-31)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None] * (-1.0 if case["inverse"] else 1.0)
    v = x[..., :R].float()
    a, b = (v[..., 0::2], v[..., 1::2]) if case["layout"] == "interleaved" else (v[..., :R // 2], v[..., R // 2:])
    ra, rb = (a * c - b * s) * st["magnitude"], (a * s + b * c) * st["magnitude"]
    rot = torch.stack([ra, rb], 3).flatten(2) if case["layout"] == "interleaved" else torch.cat([ra, rb], 2)
    return {"y": torch.cat([rot.to(x.dtype), x[..., R:]], 2)}


# ------------------------------------------------------- the package's calls ---

def _run_own(st):
    from paper_2609_21849_gb300 import qlin
    case, kind = st["case"], st["case"]["kind"]
    if kind == "norm":
        M, K = case["M"], case["K"]
        args = (st["x"], st["weight"], st["residual"], EPS, st["sum"])
        out = {} if st["residual"] is None else {"sum": st["sum"]}
        if case["out"] == "16":
            y, _ = qlin.qlin_rmsnorm(*args, y=st["y"])
            return {**out, "y": y}
        rows = case["out"] == "fp8_rows"
        q = qlin.FP8Tensor(st["y"], st["row_scales"], M, K, 1 if rows else 0)
        qlin.qlin_rmsnorm_fp8(*args, static_scale=None if rows else st["scale"], out=q)
        out["codes"] = q.codes.view(torch.float8_e4m3fn)
        return {**out, "scales": q.scale} if rows else out
    if kind == "linear":
        M, N, K, fmt = case["M"], case["N"], case["K"], case["fmt"]
        act = _act_code(qlin, case["act"])
        if fmt == "nvfp4":
            A, W = qlin.NVFP4Tensor(*st["a"], M, K), qlin.NVFP4Tensor(*st["w"], N, K)
            y, _ = qlin.qlin_linear_nvfp4(A, W, st["bias"], act, st["residual"], st["y"])
            return {"y": y}
        if fmt == "fp8":
            A, W = qlin.FP8Tensor(*st["a"], M, K, 1 if case["rows"] else 0), qlin.FP8Tensor(*st["w"], N, K, 1)
            if not case["rq"]:
                y, _ = qlin.qlin_linear_fp8(A, W, st["bias"], act, st["residual"], st["y"])
                return {"y": y}
            q = qlin.FP8Tensor(st["q"], st["q_scale"], M, N, 0)
            qlin.qlin_linear_fp8(A, W, st["bias"], act, st["residual"], None, st["next_scale"], q)
            return {"codes": q.codes.view(torch.float8_e4m3fn)}
        call = qlin.qlin_linear_bf16 if fmt == "bf16" else qlin.qlin_linear_fp16
        return {"y": call(st["a"], st["w"], st["bias"], act, st["residual"], st["y"])}
    if kind == "mlp":
        M, H, F = case["M"], case["H"], case["F"]
        a, h = qlin.NVFP4Tensor(*st["qs"][0], M, H), qlin.NVFP4Tensor(*st["qs"][1], M, F)
        up, down = qlin.NVFP4Tensor(*st["up"], F, H), qlin.NVFP4Tensor(*st["down"], H, F)
        qlin.qlin_rmsnorm_nvfp4(st["x"], st["in_scale"], st["weight"], st["residual"], EPS, st["sum"], out=a)
        qlin.qlin_linear_nvfp4(a, up, st["up_bias"], _act_code(qlin, case["act"]), None, None, st["h_scale"], h)
        qlin.qlin_linear_nvfp4(h, down, st["down_bias"], qlin.QLIN_ACT_NONE, st["sum"], st["y"])
        return {"sum": st["sum"], "y": st["y"]}
    plan = qlin.RopePlan(st["turns"], case["layout"], st["magnitude"], tuple(a // 2 for a in _axes(case)))
    return {"y": qlin.qlin_rope(st["x"], st["positions"], plan, st["y"], inverse=case["inverse"])}


def _act_code(qlin, act):
    return {"none": qlin.QLIN_ACT_NONE, "relu": qlin.QLIN_ACT_RELU, "silu": qlin.QLIN_ACT_SILU,
            "gelu_tanh": qlin.QLIN_ACT_GELU_TANH, "gelu": qlin.QLIN_ACT_GELU}[act]


def run(state):
    return _run_own(state) if own else _run_plain(state)


# --------------------------------------------------------------- what it takes ---

def _linear_work(fmt, M, N, K, written, extra):
    el = {"nvfp4": 0.5625, "fp8": 1.0}.get(fmt, 2.0)
    return {"bytes": (M + N) * K * el + M * N * written + extra, "flops": 2.0 * M * N * K}


def work(case):
    kind = case["kind"]
    if kind == "norm":
        M, K = case["M"], case["K"]
        per = 2 + (4 if case["residual"] else 0) + (2 if case["out"] == "16" else 1)
        return {"bytes": M * K * per + (4 * M if case["out"] == "fp8_rows" else 0) + (2 * K if case["weight"] else 0),
                "flops": 6.0 * M * K}
    if kind == "linear":
        M, N = case["M"], case["N"]
        extra = (2 * N if case["bias"] else 0) + (2 * M * N if case["residual"] else 0)
        extra += 4 * (N + (M if case["rows"] else 1)) if case["fmt"] == "fp8" else 0
        return _linear_work(case["fmt"], M, N, case["K"], 1 if case["rq"] else 2, extra)
    if kind == "mlp":
        M, H, F = case["M"], case["H"], case["F"]
        return {"bytes": M * H * 8 + 2 * F * H * 0.5625 + 2 * F + 4 * H, "flops": 4.0 * M * H * F}
    n = case["T"] * case["H"] * case["D"]
    return {"bytes": 4 * n + 4 * case["T"] * len(_axes(case)) + 4 * case["R"], "flops": 3.0 * n}


# ------------------------------------------------- the definition in 64 bits ---

def _round_grid(v, mantissa, least, most):
    """v (float64) to the nearest value with `mantissa` fraction bits, exponents from
    `least` up, ties to even, saturating at `most`."""
    e = torch.clamp(torch.frexp(v)[1].long() - 1, min=least) - mantissa
    two = lambda n: ((n + 1023) << 52).view(torch.float64)  # noqa: E731  2^n
    return (torch.round(v * two(-e)) * two(e)).clamp(-most, most)


def _e4m3(v):
    return _round_grid(v, 3, -6, 448.0)


def _nvfp4_exact(v, sdec):
    b = v.reshape(v.shape[0], -1, 16)
    s = _e4m3(b.abs().amax(2) / sdec / 6)[..., None]
    q = torch.where(s > 0, b / (sdec * torch.where(s > 0, s, torch.ones_like(s))), torch.zeros_like(b))
    return (_round_grid(q, 1, 0, 6.0) * s).reshape(v.shape) * sdec


def _act_exact(v, act):
    if act == "relu":
        return torch.relu(v)
    if act == "silu":
        return v * torch.sigmoid(v)
    if act == "gelu_tanh":
        u = (2 / math.pi) ** 0.5 * (v + 0.044715 * v**3)
        return v * torch.sigmoid(2 * u)
    if act == "gelu":
        return v * 0.5 * torch.erfc(-v / 2**0.5)
    return v


def _operand(q, rows, K):
    """An operand's values in 64 bits, its scales among them."""
    if isinstance(q, torch.Tensor):
        return q.double()
    if len(q) == 2:
        return q[0].view(torch.float8_e4m3fn).double() * q[1].double()[:, None]
    packed, scales, sdec = q
    grid = torch.tensor(E2M1, dtype=torch.float64, device="cuda")
    out = torch.empty(rows, K, dtype=torch.float64, device="cuda")
    for half in (0, 1):
        c = (packed >> (4 * half)) & 15
        out[:, half::2] = torch.where(c >= 8, -1.0, 1.0) * grid[(c & 7).long()]
    r, k = torch.arange(rows, device="cuda")[:, None], torch.arange(K // 16, device="cuda")[None]
    at = (r // 128 * (K // 64) + k // 4) * 512 + r % 32 * 16 + r // 32 % 4 * 4 + k % 4
    s = scales[at].view(torch.float8_e4m3fn).double() * sdec.double()
    return (out.view(rows, K // 16, 16) * s[..., None]).view(rows, K)


def _norm_exact(st):
    s = st["x"].double() if st["residual"] is None else st["x"].double() + st["residual"].double()
    n = s / torch.sqrt(s.square().mean(1, keepdim=True) + EPS)
    return s, n if st["weight"] is None else n * st["weight"].double()


def exact(case, seed):
    st, kind = prepare(case, seed), case["kind"]
    if kind == "norm":
        s, n = _norm_exact(st)
        out = {} if st["residual"] is None else {"sum": s}
        if case["out"] == "16":
            return {**out, "y": n}
        if case["out"] == "fp8":
            return {**out, "codes": _e4m3(n / st["scale"].double())}
        S = n.abs().amax(1) / 448
        return {**out, "codes": _e4m3(n / S[:, None]), "scales": S}
    if kind == "linear":
        v = _operand(st["a"], case["M"], case["K"]) @ _operand(st["w"], case["N"], case["K"]).t()
        if st["bias"] is not None:
            v += st["bias"].double()
        v = _act_exact(v, case["act"])
        if st["residual"] is not None:
            v += st["residual"].double()
        if not case["rq"]:
            return {"y": v}
        # the next layer's input is the code of the 16-bit output
        return {"codes": _e4m3(_round_grid(v, 7, -126, 3.38e38) / st["next_scale"].double())}
    if kind == "mlp":
        s, n = _norm_exact(st)
        a = _nvfp4_exact(n, st["in_scale"].double())
        v = _act_exact(a @ _operand(st["up"], case["F"], case["H"]).t() + st["up_bias"].double(), case["act"])
        h = _nvfp4_exact(_round_grid(v, 7, -126, 3.38e38), st["h_scale"].double())
        y = h @ _operand(st["down"], case["H"], case["F"]).t() + st["down_bias"].double()
        return {"sum": s, "y": y + _round_grid(s, 7, -126, 3.38e38)}
    x, R, first = st["x"].double(), case["R"], 0
    pos = st["positions"].double().view(case["T"], -1)
    y = x.clone()
    for axis, size in enumerate(_axes(case)):
        f, m = _frequencies(size, case["scaling"], case["factor"])
        angle = (pos[:, axis, None] * torch.from_numpy(f).cuda())[:, None]
        if case["inverse"]:
            angle = -angle
        i = torch.arange(first, first + size // 2, device="cuda")
        j, k = (2 * i, 2 * i + 1) if case["layout"] == "interleaved" else (i, i + R // 2)
        y[..., j] = m * (x[..., j] * torch.cos(angle) - x[..., k] * torch.sin(angle))
        y[..., k] = m * (x[..., j] * torch.sin(angle) + x[..., k] * torch.cos(angle))
        first += size // 2
    return {"y": y}
