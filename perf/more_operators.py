"""The operators of a serving step with block-scaled FP8 linears, as calls to time and to
compare: the quantizer with a scale for each block of 128, the FP8 linear of such operands,
keys and values appended to a paged cache with their rotary positions, and the attention of
new tokens (one per sequence, a causal run or a drafted tree) over that cache.

A case's ``kind`` says which.  ``run`` computes it with plain torch operations in 32 bits,
or (``own``) by the package's calls.  Sizes come from the package's own workloads (4608
tokens of a 1024 x 1024 image and its prompt, width 3072 in 24 heads, MLP 12288) and from
the ragged shapes of its tests; what the package has no sizes for (cache lengths, grouped
heads, batches, drafts) is generic.  Drawn cases spread over the same ranges.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

HIDDEN, MLP, TOKENS, HEADS = 3072, 12288, 4608, 24
MAX_MACS = TOKENS * MLP * HIDDEN          # multiply-adds of the largest linear
MAX_KEYS = 16 * 16384 * 8 * 128           # elements of the largest cache's keys
MAX_SCORES = 16 * 64 * 32 * 16384
ACTS = ("none", "relu", "silu", "gelu_tanh", "gelu")
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}


# ---------------------------------------------------------------- the cases ---

def listed():
    return [
        # the MLP's hidden activations before the down-projection
        _case("quantize_mlp_rows", "quantize", rows=TOKENS, K=MLP, block_rows=1, dtype="bf16", ld=1),
        # one new token's, where only latency counts; x a view of wider rows
        _case("quantize_one_token", "quantize", rows=1, K=HIDDEN, block_rows=1, dtype="fp16", ld=3),
        # a weight, offline: 128 x 128 blocks
        _case("quantize_weight", "quantize", rows=MLP, K=HIDDEN, block_rows=128, dtype="bf16", ld=1),
        # the up-projection of an image's tokens
        _case("linear_up_gelu", "linear", M=TOKENS, N=MLP, K=HIDDEN, bias=True, act="gelu_tanh", residual=False),
        # the down-projection of one new token, added to the residual stream
        _case("linear_one_token", "linear", M=1, N=HIDDEN, K=MLP, bias=True, act="none", residual=True),
        # a prompt's odd token count, widths that end inside a block
        _case("linear_ragged", "linear", M=1333, N=2112, K=1088, bias=True, act="silu", residual=True),
        # an image's tokens into a fresh cache: three position axes, q and k and v in one
        # QKV output
        _case("append_image", "append", B=1, T=TOKENS, ragged=False, Hq=HEADS, Hkv=HEADS, D=128, R=128, L=0,
              spread=0.0, axes="16,56,56", layout="interleaved", dtype="bf16", cache="bf16", page=64,
              scaling="none", factor=1.0, given=True, packed=True),
        # one new token of each of 64 sequences into an FP8 cache, positions those of the cache
        _case("append_one_token_each", "append", B=64, T=1, ragged=False, Hq=32, Hkv=8, D=128, R=128, L=512,
              spread=0.9, axes="", layout="half", dtype="bf16", cache="e4m3", page=32, scaling="yarn",
              factor=8.0, given=False, packed=True),
        # one new token of one sequence over a short cache: latency
        _case("attention_one_token", "attention", B=1, T=1, ragged=False, Hq=32, Hkv=8, D=128, L=1000, spread=0.0,
              page=64, dtype="bf16", cache="bf16", tree=False, lse=False),
        # one new token of each of 64 sequences of very different lengths, FP8 cache
        _case("attention_decode_fp8_cache", "attention", B=64, T=1, ragged=False, Hq=64, Hkv=8, D=128, L=8192,
              spread=0.75, page=32, dtype="bf16", cache="e4m3", tree=False, lse=False),
        # small drafts of a ragged batch: odd heads per group, width and counts, long caches
        _case("attention_tree_ragged", "attention", B=6, T=13, ragged=True, Hq=35, Hkv=7, D=96, L=30001, spread=0.9,
              page=16, dtype="fp16", cache="fp16", tree=True, lse=True),
        # trees of 64 drafted tokens, a batch of long caches
        _case("attention_tree_large", "attention", B=16, T=64, ragged=False, Hq=32, Hkv=8, D=128, L=16384, spread=0.5,
              page=128, dtype="bf16", cache="bf16", tree=True, lse=False),
    ]


def _case(name, kind, **kw):
    return {"name": name, "kind": kind, **kw}


def _log_int(rng, lo, hi, multiple=1):
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi))) / multiple)) * multiple
    return max(lo, min(hi, v))


def draw(rng):
    kind = rng.choice(["quantize", "linear", "linear", "linear", "append", "attention", "attention", "attention"])
    if kind == "quantize":
        rows, K = _log_int(rng, 1, TOKENS), _log_int(rng, 64, MLP, 64)
        return {"kind": kind, "rows": rows, "K": K, "block_rows": rng.choice([1, 1, 128]),
                "dtype": rng.choice(["bf16", "fp16"]), "ld": rng.choice([1, 1, 3])}
    if kind == "linear":
        M, N, K = _log_int(rng, 1, TOKENS), _log_int(rng, 64, MLP, 64), _log_int(rng, 64, MLP, 64)
        return {"kind": kind, "M": max(1, min(M, MAX_MACS // (N * K))), "N": N, "K": K, "bias": rng.random() < 0.7,
                "act": rng.choice(ACTS), "residual": rng.random() < 0.5}
    Hkv, G = rng.choice([1, 2, 3, 4, 7, 8]), rng.choice([1, 2, 4, 5, 7, 8])
    D, B = rng.choice([64, 80, 96, 128, 192, 256]), _log_int(rng, 1, 64)
    dtype = rng.choice(["bf16", "fp16"])
    heads = {"Hq": Hkv * G, "Hkv": Hkv, "D": D, "dtype": dtype, "cache": rng.choice([dtype, dtype, "e4m3"]),
             "page": rng.choice([8, 16, 32, 64, 128, 256]), "ragged": rng.random() < 0.5,
             "spread": rng.choice([0.0, 0.5, 0.9])}
    if kind == "append":
        T = max(1, min(_log_int(rng, 1, TOKENS), TOKENS * 3 * HEADS * 128 // (B * Hkv * (G + 2) * D)))
        axes, R = rng.choice(["", "", "1,1", "1,2,1"]), rng.choice([D, D, D // 2])
        if axes:
            parts = [int(p) for p in axes.split(",")]
            sizes = [R // sum(parts) // 2 * 2 * p for p in parts]
            R, axes = sum(sizes), ",".join(map(str, sizes))
        scaling = rng.choice(["none", "linear", "ntk", "yarn"])
        return {"kind": kind, "B": B, "T": T, **heads, "R": R, "axes": axes, "L": _log_int(rng, 1, 1024),
                "layout": rng.choice(["interleaved", "half"]), "scaling": scaling,
                "factor": 1.0 if scaling == "none" else rng.choice([2.0, 8.0, 32.0]),
                "given": bool(axes) or rng.random() < 0.5, "packed": rng.random() < 0.5}
    T = rng.choice([1, _log_int(rng, 1, 128)])
    L = _log_int(rng, 1, 65536)
    L = max(1, min(L, MAX_KEYS // (B * Hkv * D) - T, MAX_SCORES // (B * T * Hkv * G) - T))
    return {"kind": kind, "B": B, "T": T, **heads, "L": L, "tree": T > 1 and rng.random() < 0.7,
            "lse": rng.random() < 0.3}


def _lengths(case):
    """(tokens in the cache, new tokens) of each sequence: from the whole L and T down."""
    B, L, T = case["B"], case["L"], case["T"]
    cached = [L - int(L * case["spread"] * ((7 * b) % B) / B) for b in range(B)]
    return cached, [T - (T * ((5 * b) % B) // (2 * B)) if case["ragged"] else T for b in range(B)]


# --------------------------------------------------------------- the inputs ---

def _gen(seed, stream):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + stream * 7919 + 31) % (1 << 62))


def _normal(seed, stream, *shape, sigma=1.0):
    return torch.randn(*shape, generator=_gen(seed, stream), device="cuda").mul_(sigma)


def _stream_values(seed, stream, M, K):
    """Activations: N(0, 1) with 1% of the channels x20."""
    x = _normal(seed, stream, M, K)
    ch = torch.randperm(K, generator=_gen(seed, stream + 50), device="cuda")[:max(1, K // 100)]
    x[:, ch] *= 20.0
    return x


def _blocks(v, block_rows):
    """v as [row blocks, block_rows, K blocks, 128], its ends filled with zeros."""
    rows, K = v.shape
    pad = torch.nn.functional.pad(v, (0, -K % 128, 0, -rows % block_rows))
    return pad.view(-1, block_rows, pad.shape[1] // 128, 128)


def _quantized(v, block_rows):
    """(codes, scales [K blocks, row blocks]) of v."""
    b = _blocks(v, block_rows)
    amax = b.abs().amax((1, 3))
    S = torch.where(amax > 0, amax / 448.0, torch.ones((), device=v.device))
    q = (b * (1.0 / S)[:, None, :, None]).view(-1, b.shape[2] * 128)[:v.shape[0], :v.shape[1]]
    return q.clamp(-448, 448).to(torch.float8_e4m3fn), S.t().contiguous()


def _tree_bits(case, new, seed):
    """int64 words [tokens, ceil(T / 64)]: token i sees its ancestors of a random tree and
    itself; each token's parent is a random earlier one, or the cache's last."""
    g = np.random.default_rng([seed & 0x7FFFFFFF, 77])
    words = (max(new) + 63) // 64
    out = []
    for n in new:
        rows = []
        for i in range(n):
            parent = int(g.integers(-1, i)) if i else -1
            rows.append((rows[parent] if parent >= 0 else 0) | (1 << i))
        out += [[(r >> (64 * w)) & (2**64 - 1) for w in range(words)] for r in rows]
    return torch.from_numpy(np.array(out, dtype=np.uint64).view(np.int64)).cuda()


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


def _cache(case, seed, st):
    """Pages in random order, every slot filled, and the sequences' places in them."""
    B, Hkv, D, page = case["B"], case["Hkv"], case["D"], case["page"]
    cached, new = _lengths(case)
    per_seq = [(c + n + page - 1) // page for c, n in zip(cached, new)]
    pages, width = sum(per_seq) + 1, max(per_seq)
    order = torch.randperm(pages, generator=_gen(seed, 60), device="cuda").to(torch.int32)
    table = torch.zeros(B, width, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(per_seq):
        table[b, :n] = order[at:at + n]
        at += n
    st["table"] = table
    ints = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    st["cached"], st["q_start"] = ints(cached), ints([0] + list(np.cumsum(new)))
    fp8 = case["cache"] == "e4m3"
    st["k_scale"], st["v_scale"] = ((torch.full((1,), s / 448, device="cuda") for s in (6.0, 5.0)) if fp8
                                    else (None, None))
    for i, n in enumerate("kv"):
        c = torch.empty(pages, page, Hkv, D, dtype=TYPES[case["cache"]], device="cuda")
        step = max(1, (1 << 27) // (page * Hkv * D))
        g = _gen(seed, 61 + i)
        for p in range(0, pages, step):
            v = torch.randn(c[p:p + step].shape, generator=g, device="cuda")
            c[p:p + step] = ((v / st[n + "_scale"]).clamp(-448, 448) if fp8 else v).to(c.dtype)
        st[n + "_cache"] = c
    st["cached_list"], st["new_list"] = cached, new
    return sum(new)


def prepare(case, seed):
    kind, st = case["kind"], {"case": case}
    if kind == "quantize":
        rows, K = case["rows"], case["K"]
        wide = torch.zeros(rows, case["ld"] * K, dtype=TYPES[case["dtype"]], device="cuda")
        v = _stream_values(seed, 1, rows, K) if case["block_rows"] == 1 else _normal(seed, 1, rows, K, sigma=0.02)
        st["x"] = wide[:, :K].copy_(v)
        st["codes"] = torch.empty(rows, K, dtype=torch.uint8, device="cuda")
        st["scales"] = torch.empty((K + 127) // 128, -(-rows // case["block_rows"]), device="cuda")
    elif kind == "linear":
        M, N, K, dt = case["M"], case["N"], case["K"], torch.bfloat16
        st["a"] = _quantized(_stream_values(seed, 1, M, K), 1)
        st["w"] = _quantized(_normal(seed, 2, N, K, sigma=1.0 / math.sqrt(K)), 128)
        st["bias"] = _normal(seed, 3, N).to(dt) if case["bias"] else None
        st["residual"] = _normal(seed, 4, M, N).to(dt) if case["residual"] else None
        st["y"] = torch.empty(M, N, dtype=dt, device="cuda")
    elif kind == "append":
        n = _cache(case, seed, st)
        Hq, Hkv, D, dt = case["Hq"], case["Hkv"], case["D"], TYPES[case["dtype"]]
        qkv = _normal(seed, 1, n, Hq + 2 * Hkv, D).to(dt)
        parts = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        st["q"], st["k"], st["v"] = parts if case["packed"] else (p.contiguous() for p in parts)
        st["q_out"] = torch.empty(n, Hq, D, dtype=dt, device="cuda")
        A = len(_axes(case))
        if case["given"]:
            pos = torch.randint(0, 1 << 17, (n, A), generator=_gen(seed, 2), device="cuda").to(torch.int32)
            st["positions"] = pos if A > 1 else pos[:, 0].contiguous()
        else:
            st["positions"] = None
        f = [_frequencies(R, case["scaling"], case["factor"]) for R in _axes(case)]
        # turns per position as 64-bit fractions of a turn
        turns = np.round(np.concatenate([v[0] for v in f]) / (2 * math.pi) * 2.0**64)
        st["turns"] = torch.from_numpy(turns.astype(np.uint64).view(np.int64)).cuda()
        st["magnitude"] = f[0][1]
    else:
        n = _cache(case, seed, st)
        st["q"] = _normal(seed, 1, n, case["Hq"], case["D"], sigma=1.5).to(TYPES[case["dtype"]])
        st["mask"] = _tree_bits(case, st["new_list"], seed) if case["tree"] else None
        st["out"] = torch.empty_like(st["q"])
        st["lse"] = torch.empty(n, case["Hq"], device="cuda") if case["lse"] else None
        st["workspace"] = torch.zeros(64 << 20, dtype=torch.uint8, device="cuda")
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


def _dequantized(q, block_rows):
    codes, S = q
    b = _blocks(codes.float(), block_rows) * S.t()[:, None, :, None]
    return b.view(-1, b.shape[2] * 128)[:codes.shape[0], :codes.shape[1]]


def _places(st):
    """(sequence, index among its new tokens) of every new token."""
    starts, n = st["q_start"].long(), st["q"].shape[0]
    t = torch.arange(n, device="cuda")
    b = torch.searchsorted(starts, t, right=True) - 1
    return b, t - starts[b]


def _rotated(x, pos, st):
    case, R = st["case"], st["case"]["R"]
    pairs = [a // 2 for a in _axes(case)]
    # the top 32 bits of position x turns are the angle as a fraction of a turn
    p = torch.repeat_interleave(pos, torch.tensor(pairs, device="cuda"), 1, output_size=R // 2)
    angle = ((p * st["turns"]) >> 32).float() * (math.pi * 2.0**-31)
    c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
    v = x[..., :R].float()
    a, b = (v[..., 0::2], v[..., 1::2]) if case["layout"] == "interleaved" else (v[..., :R // 2], v[..., R // 2:])
    ra, rb = (a * c - b * s) * st["magnitude"], (a * s + b * c) * st["magnitude"]
    rot = torch.stack([ra, rb], 3).flatten(2) if case["layout"] == "interleaved" else torch.cat([ra, rb], 2)
    return torch.cat([rot, x[..., R:].float()], 2)


def _to_cache(v, scale, dtype):
    return v.to(dtype) if scale is None else (v * (1.0 / scale)).clamp(-448, 448).to(dtype)


def _run_plain(st):
    case, kind = st["case"], st["case"]["kind"]
    if kind == "quantize":
        codes, S = _quantized(st["x"].float(), case["block_rows"])
        return {"codes": codes, "scales": S}
    if kind == "linear":
        v = _dequantized(st["a"], 1) @ _dequantized(st["w"], 128).t()
        if st["bias"] is not None:
            v = v + st["bias"].float()
        v = _act(v, case["act"])
        if st["residual"] is not None:
            v = v + st["residual"].float()
        return {"y": v.to(torch.bfloat16)}
    seq, i = _places(st)
    if kind == "append":
        slot = st["cached"].long()[seq] + i
        pos = slot[:, None] if st["positions"] is None else st["positions"].long().view(len(slot), -1)
        page, at = st["table"].long()[seq, slot // case["page"]], slot % case["page"]
        st["k_cache"][page, at] = _to_cache(_rotated(st["k"], pos, st), st["k_scale"], st["k_cache"].dtype)
        st["v_cache"][page, at] = _to_cache(st["v"].float(), st["v_scale"], st["v_cache"].dtype)
        q = _rotated(st["q"], pos, st).to(st["q"].dtype)
        return {"q": q, "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    # attention: the batch as one, padded to its longest
    B, T, Hkv, D, page = case["B"], max(st["new_list"]), case["Hkv"], case["D"], case["page"]
    G = case["Hq"] // Hkv
    L = max(c + n for c, n in zip(st["cached_list"], st["new_list"]))
    key = torch.arange(L, device="cuda")
    cached = st["cached"].long()
    new = st["q_start"][1:].long() - st["q_start"][:-1].long()
    where = st["table"].long()[:, key // page], (key % page).expand(B, L)
    k, v = (st[n + "_cache"][where].float() for n in "kv")
    if st["k_scale"] is not None:
        k, v = k * st["k_scale"], v * st["v_scale"]
    q = torch.zeros(B, T, Hkv * G, D, device="cuda")
    q[seq, i] = st["q"].float()
    q = q.view(B, T, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, T * G, D)
    s = q @ k.permute(0, 2, 3, 1) * (1 / math.sqrt(D))
    j = key - cached[:, None]                                   # index among the new tokens
    if st["mask"] is None:
        seen = j[:, None] <= torch.arange(T, device="cuda")[:, None]
    else:
        bits = torch.zeros(B, T, st["mask"].shape[1], dtype=torch.int64, device="cuda")
        bits[seq, i] = st["mask"]
        inside = j.clamp(0, 64 * bits.shape[2] - 1)[:, None].expand(B, T, L)
        seen = (torch.gather(bits, 2, inside >> 6) >> (inside & 63)) & 1 == 1
        seen |= j[:, None] < 0
    seen = seen & (j < new[:, None])[:, None]
    s = s.view(B, Hkv, T, G, L).masked_fill(~seen[:, None, :, None], -math.inf)
    m = s.amax(4, keepdim=True)
    p = torch.exp(s - torch.where(torch.isinf(m), torch.zeros_like(m), m))
    total = p.sum(4, keepdim=True)
    o = (p.view(B, Hkv, T * G, L) @ v.permute(0, 2, 1, 3)).view(B, Hkv, T, G, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o)).permute(0, 2, 1, 3, 4).reshape(B, T, Hkv * G, D)
    out = {"out": o[seq, i].to(st["q"].dtype)}
    if st["lse"] is not None:
        lse = (m + torch.log(total)).squeeze(4).permute(0, 2, 1, 3).reshape(B, T, Hkv * G)
        out["lse"] = lse[seq, i]
    return out


# ------------------------------------------------------- the package's calls ---

def _run_own(st):
    from paper_2609_21849_gb300 import qlin
    case, kind = st["case"], st["case"]["kind"]
    if kind == "quantize":
        out = qlin.FP8BlockTensor(st["codes"], st["scales"], case["rows"], case["K"], case["block_rows"])
        qlin.qlin_quantize_fp8_block(st["x"], out=out)
        return {"codes": st["codes"].view(torch.float8_e4m3fn), "scales": st["scales"]}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        A = qlin.FP8BlockTensor(st["a"][0].view(torch.uint8), st["a"][1], M, K, 1)
        W = qlin.FP8BlockTensor(st["w"][0].view(torch.uint8), st["w"][1], N, K, 128)
        act = {"none": qlin.QLIN_ACT_NONE, "relu": qlin.QLIN_ACT_RELU, "silu": qlin.QLIN_ACT_SILU,
               "gelu_tanh": qlin.QLIN_ACT_GELU_TANH, "gelu": qlin.QLIN_ACT_GELU}[case["act"]]
        return {"y": qlin.qlin_linear_fp8_block(A, W, st["bias"], act, st["residual"], st["y"])}
    cache = qlin.PagedCache(st["k_cache"], st["v_cache"], st["table"], st["cached"], st["q_start"], st["k_scale"],
                            st["v_scale"])
    if kind == "append":
        plan = qlin.RopePlan(st["turns"], case["layout"], st["magnitude"], tuple(a // 2 for a in _axes(case)))
        qlin.qlin_cache_append(cache, st["k"], st["v"], plan, st["positions"], st["q"], st["q_out"])
        return {"q": st["q_out"], "k_cache": st["k_cache"], "v_cache": st["v_cache"]}
    qlin.qlin_cache_attention(cache, st["q"], 1 / math.sqrt(case["D"]), st["mask"], st["out"], st["lse"],
                              st["workspace"])
    return {"out": st["out"]} if st["lse"] is None else {"out": st["out"], "lse": st["lse"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# --------------------------------------------------------------- what it takes ---

def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n = case["rows"] * case["K"]
        return {"bytes": 3.0 * n + 4.0 * n / (128 * case["block_rows"]), "flops": 2.0 * n}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        extra = (2 * N if case["bias"] else 0) + (2 * M * N if case["residual"] else 0)
        scales = 4 * ((K + 127) // 128) * (M + (N + 127) // 128)
        return {"bytes": (M + N) * K + 2 * M * N + extra + scales, "flops": 2.0 * M * N * K}
    cached, new = _lengths(case)
    es, D, Hq, Hkv = 1 if case["cache"] == "e4m3" else 2, case["D"], case["Hq"], case["Hkv"]
    n = sum(new)
    if kind == "append":
        axes = len(_axes(case)) if case["given"] else 0
        return {"bytes": n * D * (4 * Hq + 2 * Hkv * (2 + es)) + 4 * n * axes, "flops": 3.0 * n * (Hq + Hkv) * D}
    keys = sum(c + t for c, t in zip(cached, new))
    seen = sum(c * t + t * (t + 1) // 2 for c, t in zip(cached, new))
    return {"bytes": 2 * keys * Hkv * D * es + 4 * n * Hq * D + (4 * n * Hq if case["lse"] else 0)
            + 4 * keys // case["page"] + (8 * n * ((max(new) + 63) // 64) if case["tree"] else 0),
            "flops": 4.0 * seen * Hq * D}


# ------------------------------------------------- the definition in 64 bits ---

def _wide(q, block_rows):
    """An operand's values in 64 bits, its scales among them."""
    codes, S = q
    rows, K = codes.shape
    r, k = torch.arange(rows, device="cuda") // block_rows, torch.arange(K, device="cuda") // 128
    return codes.double() * S.double()[k[None], r[:, None]]


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


def _turned(x, pos, case):
    x, R, first = x.double(), case["R"], 0
    y = x.clone()
    for axis, size in enumerate(_axes(case)):
        f, m = _frequencies(size, case["scaling"], case["factor"])
        angle = (pos[:, axis, None].double() * torch.from_numpy(f).cuda())[:, None]
        i = torch.arange(first, first + size // 2, device="cuda")
        j, k = (2 * i, 2 * i + 1) if case["layout"] == "interleaved" else (i, i + R // 2)
        y[..., j] = m * (x[..., j] * torch.cos(angle) - x[..., k] * torch.sin(angle))
        y[..., k] = m * (x[..., j] * torch.sin(angle) + x[..., k] * torch.cos(angle))
        first += size // 2
    return y


def exact(case, seed):
    """What is rounded to 16 or 8 bits is given before that rounding."""
    st, kind = prepare(case, seed), case["kind"]
    if kind == "quantize":
        x, r = st["x"].double(), case["block_rows"]
        S = torch.stack([torch.stack([b.abs().max() for b in c.split(r)]) if r > 1 else c.abs().amax(1)
                         for c in x.split(128, 1)]) / 448
        i, k = torch.arange(case["rows"], device="cuda") // r, torch.arange(case["K"], device="cuda") // 128
        return {"codes": x / S[k[None], i[:, None]], "scales": S}
    if kind == "linear":
        v = _wide(st["a"], 1) @ _wide(st["w"], 128).t()
        if st["bias"] is not None:
            v += st["bias"].double()
        v = _act_exact(v, case["act"])
        return {"y": v if st["residual"] is None else v + st["residual"].double()}
    starts, page = st["q_start"].tolist(), case["page"]
    if kind == "append":
        k_cache, v_cache = st["k_cache"].double(), st["v_cache"].double()
        qs = []
        for b, c in enumerate(st["cached_list"]):
            t = slice(starts[b], starts[b + 1])
            at = c + torch.arange(starts[b + 1] - starts[b], device="cuda")
            pos = at[:, None] if st["positions"] is None else st["positions"][t].view(len(at), -1)
            where = st["table"][b, at // page].long(), at % page
            k, v = _turned(st["k"][t], pos, case), st["v"][t].double()
            if st["k_scale"] is not None:
                k, v = ((x / s.double()).clamp(-448, 448) for x, s in ((k, st["k_scale"]), (v, st["v_scale"])))
            k_cache[where], v_cache[where] = k, v
            qs.append(_turned(st["q"][t], pos, case))
        return {"q": torch.cat(qs), "k_cache": k_cache, "v_cache": v_cache}
    G, outs, lses = case["Hq"] // case["Hkv"], [], []
    for b, c in enumerate(st["cached_list"]):
        n = starts[b + 1] - starts[b]
        at = torch.arange(c + n, device="cuda")
        where = st["table"][b, at // page].long(), at % page
        q = st["q"][starts[b]:starts[b + 1]].double()
        see = torch.ones(n, c + n, dtype=torch.bool, device="cuda")
        for j in range(n):
            if st["mask"] is None:
                see[:j, c + j] = False
            else:
                see[:, c + j] = (st["mask"][starts[b]:starts[b + 1], j // 64] >> (j % 64)) & 1 == 1
        o, l = torch.empty_like(q), torch.empty(n, case["Hq"], dtype=torch.float64, device="cuda")
        for h in range(case["Hkv"]):
            k, v = st["k_cache"][where + (h,)].double(), st["v_cache"][where + (h,)].double()
            if st["k_scale"] is not None:
                k, v = k * st["k_scale"].double(), v * st["v_scale"].double()
            s = torch.einsum("tgd,ld->tgl", q[:, h * G:(h + 1) * G], k) / math.sqrt(case["D"])
            s = s.masked_fill(~see[:, None], -math.inf)
            l[:, h * G:(h + 1) * G] = torch.logsumexp(s, 2)
            o[:, h * G:(h + 1) * G] = torch.einsum("tgl,ld->tgd", torch.softmax(s, 2), v)
        outs.append(o)
        lses.append(l)
    return {"out": torch.cat(outs)} if st["lse"] is None else {"out": torch.cat(outs), "lse": torch.cat(lses)}
