"""The operators of a training step around the shard that this repository snapshots (include/ckpt_train.h), in the calls
whose speed it answers for: the norm of all gradients with the clipping factor, the AdamW step over the whole tensor
list with moments in 32 or in 8 bits, the conversion of matrices to block-scaled 4-bit or 8-bit floating point and back,
and the product of two 4-bit matrices.

A shard's tensors lie in one arena per role, as flattened optimizer buffers do: `pad` 32 starts every tensor at a
multiple of 32 elements (what lies between two tensors is zero), `pad` 0 packs them without gaps, so that most starts
are aligned to the element size only. Tensors that decay come first, then those that do not (norm weights, biases).

Block-scaled formats: 32 consecutive elements of a row share the scale 2^e, e the smallest exponent at which none of
them is above the largest element value (6 for the 4-bit E2M1, 448 for the 8-bit E4M3); an element is rounded to the
nearest value, ties to the even code, or, stochastically, to n steps, n = floor(|x| / step + r / 2^16), from 16 random
bits r that are a hash of the seed and the element's place.
"""
import math
import random

import torch

own = False

G, A1, A2, M64 = 0x9E3779B97F4A7C15, 0xBF58476D1CE4E5B9, 0x94D049BB133111EB, (1 << 64) - 1
DT = {"bf16": torch.bfloat16, "f32": torch.float32, "f16": torch.float16}
SIZE = {"bf16": 2, "f32": 4, "f16": 2}
HYPER = {"lr": 3e-4, "beta1": 0.9, "beta2": 0.95, "eps": 1e-8, "step": 100}
DECAY, MAX_NORM, BLOCK = 0.1, 1.0, 32
FP4 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------ the cases

def listed():
    return [
        # The gradients of a model of 50 thousand parameters, 28 tensors: launches and host work.
        dict(name="norm-tiny", kind="norm", shard="gpt2", layers=2, hidden=24, vocab=503, pad=0, grad="bf16"),
        # The gradients of a 124 M parameter model in f32, as accumulated over micro-batches.
        dict(name="norm-gpt2", kind="norm", shard="gpt2", layers=12, hidden=768, vocab=50257, pad=32, grad="f32"),
        # The update of the smallest model, unaligned tensors.
        dict(name="adamw-tiny", kind="adamw", bits=32, shard="gpt2", layers=2, hidden=24, vocab=503, pad=0, grad="bf16", stochastic=0),
        # The update of a 124 M parameter model: 148 tensors, f32 gradients and moments, the state that a snapshot holds.
        dict(name="adamw-gpt2", kind="adamw", bits=32, shard="gpt2", layers=12, hidden=768, vocab=50257, pad=32, grad="f32", stochastic=0),
        # Two layers of a 7B model with 8-bit moments, stochastically rounded as a long run needs: the largest update.
        dict(name="adamw8-llama", kind="adamw", bits=8, shard="llama", layers=2, hidden=4096, ffn=11008, pad=32, grad="bf16", stochastic=1),
        # A run with 32-bit moments goes on with 8-bit ones: the second moment of an attention matrix as one flat tensor.
        dict(name="quantize8-moment", kind="quantize8", numel=4096 * 4096, nonzero=1, stochastic=0),
        # Serving: the activations of 64 tokens before a product.
        dict(name="quantize4-tokens", kind="quantize4", rows=64, cols=4096, src="bf16", by_col=0, stochastic=0),
        # Training: an MLP matrix from its f32 master weights, in the forms of the forward and of the backward product.
        dict(name="quantize4-weights", kind="quantize4", rows=11008, cols=4096, src="f32", by_col=1, stochastic=0),
        # Serving, a single token through an MLP matrix: the weights are read once.
        dict(name="product-token", kind="product", m=1, n=11008, k=4096, out="bf16", accumulate=0),
        # A small batch of tokens through the attention input of a 768-wide model.
        dict(name="product-1000", kind="product", m=1000, n=2304, k=768, out="bf16", accumulate=0),
        # The gradient of a weight: few tiles, a long ragged axis of tokens, added to the f32 gradient.
        dict(name="product-gradient", kind="product", m=2304, n=768, k=8190, out="f32", accumulate=1),
        # The product of the benchmark's forward and backward passes.
        dict(name="product-8192", kind="product", m=8192, n=8192, k=8192, out="bf16", accumulate=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "adamw", "adamw", "quantize8", "quantize4", "quantize4", "product", "product", "product"))
    if kind in ("norm", "adamw"):
        bits = rng.choice((8, 32))
        shape = _draw_shard(rng, 300_000_000)
        case = dict(kind=kind, **shape, pad=rng.choice((0, 32)), grad=rng.choice(("bf16", "f32", "f16")))
        if kind == "adamw":
            case.update(bits=bits, pad=32 if bits == 8 else case["pad"], stochastic=rng.randint(0, 1) if bits == 8 else 0)
        return case
    if kind == "quantize8":
        return dict(kind=kind, numel=_log(rng, 1, 60_000_000), nonzero=rng.randint(0, 1), stochastic=rng.randint(0, 1))
    if kind == "quantize4":
        rows = _log(rng, 1, 16384)
        return dict(kind=kind, rows=rows, cols=_log(rng, 1, min(16384, 90_000_000 // rows)), src=rng.choice(("bf16", "f32", "f16")),
                    by_col=rng.randint(0, 1), stochastic=rng.randint(0, 1))
    if rng.random() < 0.4:        # a few tokens
        return dict(kind=kind, m=_log(rng, 1, 64), n=_log(rng, 64, 16384), k=_log(rng, 64, 16384), out=rng.choice(("bf16", "f32")), accumulate=0)
    return dict(kind=kind, m=_log(rng, 64, 8192), n=_log(rng, 64, 8192), k=_log(rng, 64, 8192), out=rng.choice(("bf16", "f32")), accumulate=rng.randint(0, 1))


def _draw_shard(rng, most):
    what = rng.choice(("gpt2", "llama", "fragments"))
    target = _log(rng, 30_000, most)
    if what == "fragments":
        hi = _log(rng, 1000, 4_000_000)
        return dict(shard=what, params=max(1, min(4000, int(target / (hi / math.log(hi))))), lo=1, hi=hi)
    layers = rng.randint(1, 12)
    if what == "gpt2":
        hidden = max(24, 8 * int(math.sqrt(target / (12 * layers)) / 8))
        return dict(shard=what, layers=layers, hidden=hidden, vocab=max(1, min(50257, int(target / (4 * hidden)))))
    hidden = max(64, 32 * int(math.sqrt(target / (12 * layers)) / 32))
    return dict(shard=what, layers=layers, hidden=hidden, ffn=max(1, int(8 * hidden / 3)))


def _sizes(case):
    """Element counts of a shard's tensors: those that decay, those that do not."""
    if case["shard"] == "fragments":
        rng = random.Random(17)
        every = [_log(rng, case["lo"], case["hi"]) for _ in range(case["params"])]
        return every[: len(every) // 2], every[len(every) // 2:]
    h, n = case["hidden"], case["layers"]
    if case["shard"] == "gpt2":
        return [case["vocab"] * h, 1024 * h] + n * [3 * h * h, h * h, 4 * h * h, 4 * h * h], n * [h, h, 3 * h, h, h, h, 4 * h, h] + [h, h]
    return n * (4 * [h * h] + 3 * [h * case["ffn"]]), n * [h, h]


def _layout(case):
    """[(offset, elements)] of every tensor in an arena, where those that do not decay begin, the arena's length."""
    decay, other = _sizes(case)
    places, at, cut = [], 0, 0
    for k, n in enumerate(decay + other):
        if k == len(decay):
            cut = at
        places.append((at, n))
        at += -(-n // 32) * 32 if case["pad"] else n
    return places, cut if other else at, at


# ------------------------------------------------------------------ random bits

def _mix(x):
    z = (x + G) & M64
    z = ((z ^ (z >> 30)) * A1) & M64
    z = ((z ^ (z >> 27)) * A2) & M64
    return z ^ (z >> 31)


def _signed(x):
    return x - (1 << 64) if x >> 63 else x


def _bits16(key, groups, device):
    """[groups, 4]: sixteen random bits for each of the four elements of a group."""
    z = torch.arange(groups, device=device, dtype=torch.int64) + _signed((key + G) & M64)
    z = (z ^ ((z >> 30) & ((1 << 34) - 1))) * _signed(A1)
    z = (z ^ ((z >> 27) & ((1 << 37) - 1))) * _signed(A2)
    z = z ^ ((z >> 31) & ((1 << 33) - 1))
    return torch.stack([z & 0xFFFF, (z >> 16) & 0xFFFF, (z >> 32) & 0xFFFF, (z >> 48) & 0xFFFF], 1).to(torch.int32)


def _bits_of_rows(key, rows, cols, device):
    """[rows, cols]: every row begins with a group of its own."""
    groups = -(-cols // 4)
    return _bits16(key, rows * groups, device).view(rows, 4 * groups)[:, :cols]


# ------------------------------------------------------------------ block-scaled formats, plain form

def _scale_byte(blocks, four_bits):
    """The biased exponent that the 32 values of the last axis share."""
    bits = blocks.abs().amax(-1).view(torch.int32)
    most, threshold = (2, 0x400000) if four_bits else (8, 0x600000)
    byte = ((bits >> 23) - most + ((bits & 0x7FFFFF) > threshold).to(torch.int32)).clamp(0, 254)
    return torch.where(bits >= 0x7F800000, 255, byte)


def _unscaled(blocks, byte):
    """The values over their block's scale."""
    inverse = ((254 - byte.clamp(max=253)) << 23).view(torch.float32)
    return blocks * torch.where(byte == 255, math.nan, inverse).unsqueeze(-1)


def _scale(byte):
    return byte.to(torch.uint8).view(torch.float8_e8m0fnu).float()


def _fp4_codes(y, bits16):
    """Codes 0 to 15 of values up to 6."""
    a = y.abs()
    if bits16 is None:
        code = (a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5)
    else:
        halves = (a * 131072).to(torch.int32)          # in units of 0.5 / 2^16
        s = (halves >= 4 << 16).to(torch.int32) + (halves >= 8 << 16).to(torch.int32)
        code = ((halves + (bits16 << s)) >> (16 + s)) + 2 * s
    return torch.where(a.isnan(), 0, code).to(torch.uint8) | (torch.signbit(y).to(torch.uint8) << 3)


def _fp8_codes(y, bits16, nonzero):
    """E4M3 codes of values up to 448."""
    a = y.abs()
    if bits16 is None:
        code = a.to(torch.float8_e4m3fn).view(torch.uint8).to(torch.int32)
    else:
        normal = ((a.view(torch.int32) + (bits16 << 4)) >> 20) - 960
        small = ((a * 33554432).clamp(max=2.0 ** 20).to(torch.int32) + bits16) >> 16
        code = torch.where(a >= 2.0 ** -6, normal, small)
    if nonzero:
        code = torch.where((a > 0) & (code == 0), 1, code)
    code = torch.where(a.isnan(), 0x7F, code)
    return (code | (torch.signbit(y).to(torch.int32) << 7)).to(torch.uint8)


def _blocks(x):
    """The rows of x in blocks of 32, filled up with zeros."""
    rows, cols = x.shape
    return torch.nn.functional.pad(x, (0, -cols % BLOCK)).view(rows, -1, BLOCK)


def _to_fp8(x, bits16=None, nonzero=False):
    """Codes and scales of a flat f32 tensor."""
    blocks = _blocks(x.view(1, -1))
    byte = _scale_byte(blocks, False)
    codes = _fp8_codes(_unscaled(blocks, byte).view(-1)[: x.numel()], bits16, nonzero)
    return codes, byte.view(-1).to(torch.uint8)


def _from_fp8(codes, scales):
    values = _blocks(codes.view(torch.float8_e4m3fn).float().view(1, -1))
    return (values * scales.view(torch.float8_e8m0fnu).float().view(1, -1, 1)).view(-1)[: codes.numel()]


def _to_fp4(x, bits16=None):
    """Codes (one a byte) in blocks and their biased exponents, of the rows of an f32 matrix."""
    blocks = _blocks(x)
    byte = _scale_byte(blocks, True)
    if bits16 is not None:
        bits16 = _blocks(bits16)
    return _fp4_codes(_unscaled(blocks, byte), bits16), byte


def _from_fp4(codes, byte, cols):
    table = torch.tensor(FP4 + tuple(-v for v in FP4), device=codes.device)
    return (table[codes.int()] * _scale(byte).unsqueeze(-1)).view(codes.shape[0], -1)[:, :cols]


# ------------------------------------------------------------------ inputs

def _pitches(rows, cols):
    """Bytes from row to row of 4-bit codes and of their scales."""
    return -(-cols // 256) * 128, -(-cols // 512) * 16


def _packed(x):
    """A matrix in 4 bits as the product takes it: codes two a byte, scales, rows filled up with zeros."""
    codes, byte = _to_fp4(x.float())
    rows, (code_pitch, scale_pitch) = x.shape[0], _pitches(*x.shape)
    flat = torch.nn.functional.pad(codes.view(rows, -1), (0, 2 * code_pitch - codes[0].numel()))
    return (flat[:, 0::2] | (flat[:, 1::2] << 4)).contiguous(), torch.nn.functional.pad(byte.to(torch.uint8), (0, scale_pitch - byte.shape[1])).contiguous()


def _binding():
    from paper_2406_10707_amd import binding
    return binding


def _code(dtype):
    b = _binding()
    return {"bf16": b.CKPT_BF16, "f32": b.CKPT_F32, "f16": b.CKPT_F16}[dtype]


def _arena_values(case, seed, dev):
    """Gradients of a shard: tensors of different scale, stretches without any (rows of an embedding that no token met)."""
    places, cut, total = _layout(case)
    gen = torch.Generator(dev).manual_seed(seed)
    g = torch.randn(total, device=dev, generator=gen)
    rough = torch.rand(-(-total // 1024), device=dev, generator=gen)
    factor = torch.where(rough < 0.05, 0.0, 1e-3 * torch.exp2(6 * rough - 3)).repeat_interleave(1024)[:total]
    g *= factor
    if case["pad"]:
        for at, n in places:
            g[at + n: -(-(at + n) // 32) * 32] = 0
    return gen, factor, g


def prepare(case, seed):
    dev = torch.device("cuda:0")
    kind = case["kind"]
    s = {"case": dict(case), "seed": int(seed)}
    if kind in ("norm", "adamw"):
        places, cut, total = _layout(case)
        gen, factor, g = _arena_values(case, seed, dev)
        s["grad"] = g.to(DT[case["grad"]])
        s["norm"] = torch.zeros(6, device=dev)            # 24 bytes: sum of squares, norm, scale, flags
        if kind == "adamw":
            live = (g != 0).float()
            w = 0.02 * torch.randn(total, device=dev, generator=gen)
            m = 0.3 * factor * torch.randn(total, device=dev, generator=gen)
            v = (0.5 * factor * torch.randn(total, device=dev, generator=gen)) ** 2 + 0.1 * g * g
            w, m, v = w * live, m * live, v * live
            s["master"], s["param"] = w, w.to(torch.bfloat16)
            s["norm"][3] = 0.37
            s["m_scale"] = s["v_scale"] = None
            if case["bits"] == 8:
                s["m"], s["m_scale"] = _to_fp8(m)
                s["v"], s["v_scale"] = _to_fp8(v, nonzero=True)
            else:
                s["m"], s["v"] = m, v
        if own:
            b = _binding()
            size, ptr = SIZE[case["grad"]], {k: s[k].data_ptr() for k in ("grad", "param", "master", "m", "v", "m_scale", "v_scale") if s.get(k) is not None}
            tensors = []
            for at, n in places:
                if kind == "norm":
                    tensors.append(dict(numel=n, grad=ptr["grad"] + size * at))
                    continue
                e = 1 if case["bits"] == 8 else 4
                t = dict(numel=n, grad=ptr["grad"] + size * at, param=ptr["param"] + 2 * at, master=ptr["master"] + 4 * at, m=ptr["m"] + e * at,
                         v=ptr["v"] + e * at, weight_decay=DECAY if at < cut else 0.0)
                if case["bits"] == 8:
                    t.update(m_scale=ptr["m_scale"] + at // 32, v_scale=ptr["v_scale"] + at // 32)
                tensors.append(t)
            s["optimizer"] = b.Optimizer(tensors, grad_dtype=_code(case["grad"]), param_dtype=b.CKPT_BF16, state_bits=case.get("bits", 32))
        return s
    gen = torch.Generator(dev).manual_seed(seed)
    if kind == "quantize8":
        n = case["numel"]
        s["x"] = torch.randn(n, device=dev, generator=gen) * torch.exp2(torch.randint(-12, 1, (-(-n // 64),), device=dev, generator=gen).float()).repeat_interleave(64)[:n]
        if case["nonzero"]:
            s["x"] = s["x"] ** 2 * 1e-6
        s["codes"], s["scales"] = (torch.empty(k, dtype=torch.uint8, device=dev) for k in (n, -(-n // 32)))
        if own:
            s["to"] = _binding().mx_matrix(_binding().CKPT_MXFP8, 1, n, s["codes"].data_ptr(), n, s["scales"].data_ptr(), s["scales"].numel())
    elif kind == "quantize4":
        r, c = case["rows"], case["cols"]
        x = torch.randn(r, c, device=dev, generator=gen) * torch.exp2(torch.randn(c, device=dev, generator=gen))
        s["x"] = (0.02 * x).to(DT[case["src"]])
        s["values"] = [torch.empty(r, c, dtype=torch.bfloat16, device=dev)] + ([torch.empty(c, r, dtype=torch.bfloat16, device=dev)] if case["by_col"] else [])
        if own:
            b, s["to"], s["held"] = _binding(), [], []
            for v in s["values"]:
                cp, sp = _pitches(*v.shape)
                codes, scales = (torch.empty(v.shape[0] * p, dtype=torch.uint8, device=dev) for p in (cp, sp))
                s["held"] += [codes, scales]
                s["to"].append(b.mx_matrix(b.CKPT_MXFP4, v.shape[0], v.shape[1], codes.data_ptr(), cp, scales.data_ptr(), sp))
    else:
        m, n, k = case["m"], case["n"], case["k"]
        s["a"] = _packed(torch.randn(m, k, device=dev, generator=gen))
        s["b"] = _packed(0.02 * torch.randn(n, k, device=dev, generator=gen))
        s["c"] = torch.randn(m, n, device=dev, generator=gen).to(DT[case["out"]])
        if own:
            b = _binding()
            (cp, sp) = _pitches(1, k)
            s["am"], s["bm"] = (b.mx_matrix(b.CKPT_MXFP4, rows, k, x[0].data_ptr(), cp, x[1].data_ptr(), sp) for rows, x in ((m, s["a"]), (n, s["b"])))
            s["workspace"] = torch.empty(max(1, b.mx_gemm_workspace(m, n, k)), dtype=torch.uint8, device=dev)
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    return (_run_own if own else _run_plain)(s, s["case"])


def _norm_outputs(s):
    return {"norm": s["norm"][2:4], "nonfinite": s["norm"].view(torch.int32)[4:5]}


def _state_outputs(s):
    if s["m_scale"] is None:
        return {"param": s["param"], "master": s["master"], "m": s["m"], "v": s["v"]}
    as_value = {"m": torch.float8_e4m3fn, "v": torch.float8_e4m3fn, "m_scale": torch.float8_e8m0fnu, "v_scale": torch.float8_e8m0fnu}
    return {"param": s["param"], "master": s["master"], **{k: s[k].view(t) for k, t in as_value.items()}}


def _run_own(s, case):
    b, stream, kind = _binding(), torch.cuda.current_stream().cuda_stream, case["kind"]
    if kind == "norm":
        s["optimizer"].grad_norm(s["norm"].data_ptr(), stream, max_norm=MAX_NORM)
        return _norm_outputs(s)
    if kind == "adamw":
        s["optimizer"].step(stream, **HYPER, seed=s["seed"], stochastic=bool(case["stochastic"]), norm=s["norm"].data_ptr())
        return _state_outputs(s)
    rounding = (b.CKPT_ROUND_STOCHASTIC if case.get("stochastic") else b.CKPT_ROUND_NEAREST) | (b.CKPT_ROUND_NONZERO if case.get("nonzero") else 0)
    if kind == "quantize8":
        b.mx_quantize(s["x"].data_ptr(), b.CKPT_F32, s["x"].numel(), s["to"], None, stream, rounding=rounding, seed=s["seed"])
        return {"codes": s["codes"].view(torch.float8_e4m3fn), "scales": s["scales"].view(torch.float8_e8m0fnu)}
    if kind == "quantize4":
        to = s["to"]
        b.mx_quantize(s["x"].data_ptr(), _code(case["src"]), case["cols"], to[0], to[1] if len(to) > 1 else None, stream, rounding=rounding, seed=s["seed"])
        for matrix, values in zip(to, s["values"]):
            b.mx_dequantize(matrix, values.data_ptr(), b.CKPT_BF16, values.shape[1], stream)
        return s["values"]
    b.mx_gemm(s["am"], s["bm"], s["c"].data_ptr(), _code(case["out"]), case["n"], stream, accumulate=bool(case["accumulate"]),
              workspace=s["workspace"].data_ptr(), workspace_bytes=s["workspace"].numel())
    return s["c"]


def _run_plain(s, case):
    kind = case["kind"]
    if kind == "norm":
        norm = s["grad"].float().square().sum().sqrt()
        s["norm"][2], s["norm"][3] = norm, (MAX_NORM / norm).clamp(max=1.0)
        s["norm"].view(torch.int32)[4] = (~norm.isfinite()).to(torch.int32)
        return _norm_outputs(s)
    if kind == "adamw":
        return _plain_adamw(s, case)
    if kind == "quantize8":
        bits16 = _bits_of_rows(_mix(s["seed"]), 1, case["numel"], s["x"].device).reshape(-1) if case["stochastic"] else None
        s["codes"], s["scales"] = _to_fp8(s["x"], bits16, bool(case["nonzero"]))
        return {"codes": s["codes"].view(torch.float8_e4m3fn), "scales": s["scales"].view(torch.float8_e8m0fnu)}
    if kind == "quantize4":
        s["values"] = [_plain_fp4(s, s["x"].float(), _mix(s["seed"]))]
        if case["by_col"]:
            s["values"].append(_plain_fp4(s, s["x"].float().t().contiguous(), _mix(~s["seed"] & M64)))
        return s["values"]
    a, b = _unpacked(s["a"], case["k"]), _unpacked(s["b"], case["k"])
    c = a @ b.t()
    s["c"].copy_(s["c"].float() + c if case["accumulate"] else c)
    return s["c"]


def _plain_fp4(s, x, key):
    codes, byte = _to_fp4(x, _bits_of_rows(key, x.shape[0], x.shape[1], x.device) if s["case"]["stochastic"] else None)
    return _from_fp4(codes, byte, x.shape[1]).to(torch.bfloat16)


def _unpacked(packed, k):
    codes, scales = packed
    codes = torch.stack([codes & 15, codes >> 4], -1).view(codes.shape[0], -1, BLOCK)
    return _from_fp4(codes, scales[:, : codes.shape[1]], k)


def _plain_adamw(s, case):
    h, (_, cut, total) = HYPER, _layout(case)
    g = s["grad"].float() * s["norm"][3]
    eight = case["bits"] == 8
    m = _from_fp8(s["m"], s["m_scale"]) if eight else s["m"]
    v = _from_fp8(s["v"], s["v_scale"]) if eight else s["v"]
    m = m * h["beta1"] + g * (1 - h["beta1"])
    v = v * h["beta2"] + (g * g) * (1 - h["beta2"])
    if eight:
        bits_m = bits_v = None
        if case["stochastic"]:
            four = _bits16(_mix((_mix(s["seed"]) + h["step"]) & M64), total // 4, g.device)
            bits_m, bits_v = four.view(-1), four.flip(1).reshape(-1)
        s["m"], s["m_scale"] = _to_fp8(m, bits_m)
        s["v"], s["v_scale"] = _to_fp8(v, bits_v, nonzero=True)
    else:
        s["m"], s["v"] = m, v
    w = s["master"].clone()
    w[:cut] *= 1 - h["lr"] * DECAY
    w -= h["lr"] * (m / (1 - h["beta1"] ** h["step"])) / ((v / (1 - h["beta2"] ** h["step"])).sqrt() + h["eps"])
    s["master"], s["param"] = w, w.to(torch.bfloat16)
    return _state_outputs(s)


# ------------------------------------------------------------------ what a pass cannot do without

def work(case):
    kind = case["kind"]
    if kind in ("norm", "adamw"):
        n, g = sum(sum(x) for x in _sizes(case)), SIZE[case["grad"]]
        if kind == "norm":
            return {"bytes": n * g + 24, "flops": 2 * n}
        moments = 16 if case["bits"] == 32 else 4 + 4 / 32
        return {"bytes": n * (g + 8 + 2 + moments), "flops": 14 * n}
    if kind == "quantize8":
        return {"bytes": case["numel"] * (4 + 1 + 1 / 32), "flops": 2 * case["numel"]}
    if kind == "quantize4":
        n, forms = case["rows"] * case["cols"], 1 + case["by_col"]
        return {"bytes": n * (SIZE[case["src"]] + forms * (2 * (0.5 + 1 / 32) + 2)), "flops": 3 * n * forms}
    m, n, k = case["m"], case["n"], case["k"]
    return {"bytes": (m + n) * k * (0.5 + 1 / 32) + m * n * SIZE[case["out"]] * (1 + case["accumulate"]), "flops": 2 * m * n * k}


# ------------------------------------------------------------------ the definition in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "norm":
        norm = s["grad"].double().pow(2).sum().sqrt()
        both = torch.stack([norm, torch.minimum(torch.ones_like(norm), MAX_NORM / norm)])
        return {"norm": both, "nonfinite": None}
    if kind == "adamw":
        return _exact_adamw(s, case)
    if kind == "quantize8":
        n = case["numel"]
        u = _uniform(_mix(int(seed)), -(-n // 4), s["x"].device).reshape(-1)[:n] if case["stochastic"] else None
        element, scale = _exact_mx(s["x"].double().view(1, n), 8, u, bool(case["nonzero"]))
        return {"codes": element.view(n), "scales": scale.view(-1)}
    if kind == "quantize4":
        out = []
        for x, key in ((s["x"].double(), _mix(int(seed))), (s["x"].double().t(), _mix(~int(seed) & M64)))[: 1 + case["by_col"]]:
            rows, cols = x.shape
            u = _uniform(key, rows * -(-cols // 4), x.device).reshape(rows, -1)[:, :cols] if case["stochastic"] else None
            element, scale = _exact_mx(x, 4, u, False)
            out.append(element * scale.repeat_interleave(32, 1)[:, :cols])
        return out
    a, b = (_exact_matrix(x, case["k"]) for x in (s["a"], s["b"]))
    c = a @ b.t().contiguous()
    return c + s["c"].double() if case["accumulate"] else c


def _uniform(key, groups, dev):
    """The random numbers r / 2^16 of stochastic rounding, four to a group."""
    import numpy as np
    with np.errstate(over="ignore"):
        z = np.arange(groups, dtype=np.uint64) + np.uint64((key + G) & M64)
        z = (z ^ (z >> np.uint64(30))) * np.uint64(A1)
        z = (z ^ (z >> np.uint64(27))) * np.uint64(A2)
        z ^= z >> np.uint64(31)
    fields = z.view(np.uint16).astype(np.int32) if z.size else np.zeros(0, np.int32)
    return torch.from_numpy(fields).to(dev).double().view(groups, 4) / 65536


def _power(exponent):
    """2^exponent, to the bit (the card's pow is not)."""
    return torch.tensor([2.0 ** e for e in range(-160, 160)], dtype=torch.float64, device=exponent.device)[exponent.long() + 160]


def _exact_mx(x, bits, u, nonzero):
    """(element values, scales) of the rows of x in 64 bits."""
    rows, cols = x.shape
    most, lowest, mantissa = (6.0, 0, 1) if bits == 4 else (448.0, -6, 3)
    blocks = torch.nn.functional.pad(x, (0, -cols % 32)).reshape(rows, -1, 32)
    fraction, exponent = torch.frexp(blocks.abs().amax(-1))      # the largest = fraction * 2^exponent, fraction in [0.5, 1)
    most, power = math.frexp(most)
    exponent = exponent - power + (fraction > most)
    exponent = torch.where(fraction == 0, -127, exponent).clamp(-127, 127)
    scale = _power(exponent)
    y = (blocks / scale.unsqueeze(-1)).reshape(rows, -1)[:, :cols]
    a = y.abs()
    step = _power(torch.frexp(a.clamp(min=2.0 ** lowest))[1] - 1 - mantissa)
    n = torch.round(a / step) if u is None else torch.floor(a / step + u.view(rows, -1))      # ties to even steps: even codes
    a = torch.where((n == 0) & (a > 0), step, n * step) if nonzero else n * step
    return torch.where(y < 0, -a, a), scale


def _exact_matrix(packed, k):
    codes, scales = packed
    nibbles = torch.stack([codes & 15, codes >> 4], -1).reshape(codes.shape[0], -1)[:, :k].long()
    e, f = (nibbles >> 1) & 3, (nibbles & 1).double()
    value = torch.where(e == 0, f / 2, (1 + f / 2) * _power(e - 1))
    return torch.where(nibbles > 7, -value, value) * _power(scales.long() - 127).repeat_interleave(32, 1)[:, :k]


def _exact_adamw(s, case):
    _, cut, total = _layout(case)
    g = s["grad"].double() * s["norm"][3].double()
    out, u = {}, None
    if case["bits"] == 8:
        m, v = (s[k].view(torch.float8_e4m3fn).double() * _power(s[k + "_scale"].long() - 127).repeat_interleave(32)[:total] for k in "mv")
        if case["stochastic"]:
            u = _uniform(_mix((_mix(s["seed"]) + HYPER["step"]) & M64), total // 4, g.device)
    else:
        m, v = s["m"].double(), s["v"].double()
    b1, b2 = HYPER["beta1"], HYPER["beta2"]
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g ** 2
    if case["bits"] == 8:
        for k, x, r in (("m", m, u), ("v", v, None if u is None else u.flip(1))):
            element, scale = _exact_mx(x.view(1, total), 8, None if r is None else r.reshape(-1), k == "v")
            out[k], out[k + "_scale"] = element.view(-1), scale.view(-1)
    else:
        out["m"], out["v"] = m, v
    update = (m / (1 - b1 ** HYPER["step"])) / (torch.sqrt(v / (1 - b2 ** HYPER["step"])) + HYPER["eps"])
    decay = torch.full_like(update, 1.0)
    decay[:cut] = 1 - HYPER["lr"] * DECAY
    out["master"] = s["master"].double() * decay - HYPER["lr"] * update
    out["param"] = out["master"]
    return out
