"""Products of a layer with 4-bit microscaled weights and products grouped by expert, as cases that can be timed and compared.

A case is one call (or the pair of calls that a program makes together) on one batch:

    op "quantize"    bf16 activations to 4-bit floating point with one power-of-two scale per 32 values, and back to bf16
                     (what a program does that trains with the rounding in place)
    op "prepare"     a frozen fp32 weight to both 4-bit copies that a layer keeps, with blocks along the input channels
                     (forward) and along the output channels (input gradient), and both back to bf16
    op "mx4_fwd"     forward of such a layer with its LoRA branch, dense (`e` = 0) or with a weight and an adapter per expert
    op "mx4_dx"      its input gradient
    op "fwd"         bf16 products grouped by expert (or by adapter): Y = X W_e for the rows of expert e
    op "dx"          the input gradient dY W_e^T
    op "dw"          the weight gradients X_e^T dY_e

Sizes: t rows in the batch, `e` experts with ragged row counts, c_in x c_out weights, LoRA rank r; `pad` rows at the end of
the batch belong to no expert.  Outputs are fp32, bf16 where `bf16` is true.

With `own` false the same values come from elementary torch operations in fp32.
"""
import itertools
import math

import torch

own = False

DEV = "cuda"
BLOCK, PAD = 32, 256          # values per scale; stored rows are padded to a multiple of PAD values
GRID = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def listed():
    return [
        # the smallest quantizer call: one short prompt through a narrow layer whose width is no multiple of a block
        _case("quantize_37x1040", "quantize", 37, 1040),
        # activations of four 4096-token sequences
        _case("quantize_16384x5120", "quantize", 16384, 5120),
        # loading a model: one frozen 7B-sized MLP projection
        _case("prepare_4096x11008", "prepare", 1, 4096, 11008),
        # one token at a time through an MLP projection with its adapter (generation)
        _case("mx4_fwd_1x4096x11008_r16", "mx4_fwd", 1, 4096, 11008, r=16, bf16=True),
        # the usual batch of four 512-token sequences, hidden -> hidden projection
        _case("mx4_fwd_2048x4096x4096_r16", "mx4_fwd", 2048, 4096, 4096, r=16),
        # long sequences: a 13B-sized gate projection, four 4096-token sequences, backward
        _case("mx4_dx_16384x5120x13824_r16", "mx4_dx", 16384, 5120, 13824, r=16),
        # many small experts, the rows of a 1024-token batch routed to eight of them each
        _case("mx4_fwd_8192x2048x1408_e64", "mx4_fwd", 8192, 2048, 1408, e=64, bf16=True),
        # packed sequences of uneven length, widths that are no multiples of a tile, adapters per expert, a padded batch
        _case("mx4_dx_1003x1040x2064_e5_r32", "mx4_dx", 1003, 1040, 2064, e=5, r=32, pad=21),
        # generation: a few tokens, eight experts each, nearly every expert has no or one row
        _case("fwd_24x2048x1408_e64", "fwd", 24, 2048, 1408, e=64, bf16=True),
        # trainable experts, two per token, input gradient
        _case("dx_8192x4096x4096_e8", "dx", 8192, 4096, 4096, e=8, bf16=True),
        # the weight gradients of sixteen trainable experts
        _case("dw_8192x2048x5632_e16", "dw", 8192, 2048, 5632, e=16),
        # gradient of the first adapter factors of eight experts (or of eight adapters trained together on one base)
        _case("dw_16384x5120x16_e8", "dw", 16384, 5120, 16, e=8),
    ]


def draw(rng):
    """One more case of the same ranges: one to 16384 rows, widths from 208 to 16384 (an adapter's 16 to 64 among the grouped
    products), dense or one to 256 experts, every rank, padded batches."""
    while True:
        op = rng.choice(["quantize", "prepare", "mx4_fwd", "mx4_fwd", "mx4_dx", "mx4_dx", "fwd", "dx", "dw"])
        t = _log(rng, 1, 16384)
        gran = rng.choice([128, 128, 64, 16])
        c_in, c_out = (max(gran, gran * round(_log(rng, 208, 16384) / gran)) for _ in range(2))
        e = 0 if op.startswith("mx4") and rng.random() < 0.5 else _log(rng, 1, 256)
        r = rng.choice([0, 16, 16, 32, 48, 64]) if op.startswith("mx4") else 0
        if op in ("fwd", "dx", "dw") and rng.random() < 0.3:
            narrow = rng.choice([16, 16, 32, 64])
            c_in, c_out = (narrow, c_out) if rng.random() < 0.5 else (c_in, narrow)
        pad = rng.randrange(0, t) if e and t > 1 and rng.random() < 0.3 else 0
        if t * c_in * c_out > 5e11 or max(1, e) * c_in * c_out > 4e8 or max(1, e) * c_in * c_out + t * (c_in + c_out) < 1e5:
            continue
        c = _case("", op, 1 if op == "prepare" else t, c_in, 0 if op == "quantize" else c_out,
                  e=0 if op in ("quantize", "prepare") else e, r=r, pad=0 if op in ("quantize", "prepare") else pad,
                  bf16=op not in ("quantize", "prepare", "dw") and rng.random() < 0.5)
        del c["name"]
        return c


def prepare(case, seed):
    op, t, c_in, c_out, e, r = (case[k] for k in ("op", "t", "c_in", "c_out", "e", "r"))
    gen = torch.Generator(device=DEV).manual_seed(int(seed) * 1000003 + 7 * t + c_in + 3 * c_out + e)
    S = {"case": case}

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32)

    if op == "prepare":
        S["W"] = normal(c_in, c_out).mul_(0.02)
        return S
    if op == "quantize":
        S["X"] = _activations(normal, gen, t, c_in).to(torch.bfloat16)
        return S
    # rows of each expert: uneven shares, so that some experts are several times as busy as others and some idle
    if e:
        share = torch.rand(e, generator=gen, device=DEV).square_()
        of_row = torch.multinomial(share, t - case["pad"], replacement=True, generator=gen)
        S["lens"] = torch.bincount(of_row, minlength=e).tolist()
        S["offsets"] = torch.tensor([0] + S["lens"], device=DEV).cumsum(0)
    else:
        S["lens"], S["offsets"] = [t], None
    n = max(1, e)
    if op.endswith("fwd") or op == "dw":
        S["X"] = _activations(normal, gen, t, c_in).to(torch.bfloat16)
    if op.endswith("dx") or op == "dw":
        S["dY"] = normal(t, c_out).mul_(2.0 ** -6).to(torch.bfloat16)
    if op in ("fwd", "dx"):
        S["W"] = normal(n, c_in, c_out).mul_(0.02).to(torch.bfloat16)
    if op.startswith("mx4"):
        # the weight as a program keeps it: 4-bit codes, two to a byte, and scale bytes, one row per channel of the result
        rows, k = (c_out, c_in) if op == "mx4_fwd" else (c_in, c_out)
        S["codes"], S["scales"] = _pack(normal(n * rows, k).mul_(0.02))
        S["A"] = normal(n, c_in, r).div_(math.sqrt(c_in)).to(torch.bfloat16) if r else None
        S["B"] = normal(n, r, c_out).mul_(0.02).to(torch.bfloat16) if r else None
    out = torch.bfloat16 if case["bf16"] else torch.float32
    shape = (n, c_in, c_out) if op == "dw" else (t, c_out) if op.endswith("fwd") else (t, c_in)
    S["out"] = torch.zeros(shape, dtype=out, device=DEV)
    return S


def run(S):
    if own:
        return _own(S)
    c = S["case"]
    op, c_in, c_out = c["op"], c["c_in"], c["c_out"]
    if op == "quantize":
        return {"X": _rounded(S["X"].float()).to(torch.bfloat16)}
    if op == "prepare":
        W = S["W"]
        return {"fwd": _rounded(W.t().contiguous()).to(torch.bfloat16), "bwd": _rounded(W).to(torch.bfloat16)}
    out = torch.zeros_like(S["out"])
    scale = 0.5
    if op.startswith("mx4"):
        fwd = op == "mx4_fwd"
        rows, k = (c_out, c_in) if fwd else (c_in, c_out)
        busy = torch.tensor([n > 0 for n in S["lens"]])
        W = _unpack(*(S[key].unflatten(0, (-1, rows))[busy].flatten(0, 1) for key in ("codes", "scales")), k)
        X = (S["X"] if fwd else S["dY"]).float()
        Xr = _rounded(X)
    # the experts' rows lie one after the other
    i = -1
    for g, (a, b) in enumerate(_spans(S["lens"])):
        if op == "dw":
            out[g] = scale * (S["X"][a:b].float().t() @ S["dY"][a:b].float())
        elif a == b:
            continue
        elif op == "fwd":
            out[a:b] = (scale * (S["X"][a:b].float() @ S["W"][g].float())).to(out.dtype)
        elif op == "dx":
            out[a:b] = (scale * (S["dY"][a:b].float() @ S["W"][g].float().t())).to(out.dtype)
        else:
            i += 1
            y = Xr[a:b] @ W[i * rows:(i + 1) * rows].t()
            if c["r"]:
                A, B = S["A"][g].float(), S["B"][g].float()
                y += scale * ((X[a:b] @ A) @ B if fwd else (X[a:b] @ B.t()) @ A.t())
            out[a:b] = y.to(out.dtype)
    return {"out": out}


def exact(case, seed):
    S = prepare(case, seed)
    op, c_in, c_out = case["op"], case["c_in"], case["c_out"]
    if op == "quantize":
        return {"X": _exact_values(S["X"])}
    if op == "prepare":
        return {"fwd": _exact_values(S["W"].t()), "bwd": _exact_values(S["W"])}
    out = torch.zeros(S["out"].shape, dtype=torch.float64, device=DEV)
    a = 0
    for g, n in enumerate(S["lens"]):
        rows = slice(a, a + n)
        a += n
        if n == 0:
            continue
        if op == "dw":
            out[g] = torch.matmul(S["X"][rows].double().t(), S["dY"][rows].double()) / 2
        elif op == "fwd":
            out[rows] = torch.matmul(S["X"][rows].double(), S["W"][g].double()) / 2
        elif op == "dx":
            out[rows] = torch.matmul(S["dY"][rows].double(), S["W"][g].double().t()) / 2
        else:
            fwd = op == "mx4_fwd"
            x = (S["X"] if fwd else S["dY"])[rows]
            m, k = (c_out, c_in) if fwd else (c_in, c_out)
            codes, scales = S["codes"][g * m:(g + 1) * m].long(), S["scales"][g * m:(g + 1) * m].double()
            both = torch.stack([codes % 16, codes // 16], -1).flatten(1)
            grid = torch.tensor(GRID, dtype=torch.float64, device=DEV)
            w = grid[both % 8] * (1 - 2 * (both // 8)) * torch.exp2(scales - 127).repeat_interleave(BLOCK, 1)
            out[rows] = torch.matmul(_exact_values(x), w[:, :k].t())
            if case["r"]:
                A, B = S["A"][g].double(), S["B"][g].double()
                out[rows] += torch.matmul(torch.matmul(x.double(), A), B) / 2 if fwd else torch.matmul(torch.matmul(x.double(), B.t()), A.t()) / 2
    return {"out": out}


def work(case):
    """Bytes and operations of a pass: inputs and outputs once each, 17 bytes for 32 values of a 4-bit weight.  An expert
    without rows needs no weight, and no call has more busy experts than rows."""
    op, t, c_in, c_out, r = (case[k] for k in ("op", "t", "c_in", "c_out", "r"))
    if op == "quantize":          # in, codes and scales out, read back, values out
        return {"bytes": t * c_in * (2 + 2 * 17 / 32 + 2), "flops": 0}
    if op == "prepare":
        return {"bytes": c_in * c_out * (4 + 4 * 17 / 32 + 4), "flops": 0}
    t -= case["pad"]
    n = max(1, case["e"])
    busy = min(n, t)
    el = 2 if case["bf16"] else 4
    nbytes = 0
    if op == "dw":
        nbytes = 2 * t * (c_in + c_out) + 4 * n * c_in * c_out
    else:
        x, y = (c_in, c_out) if op.endswith("fwd") else (c_out, c_in)
        nbytes = 2 * t * x + el * t * y + busy * c_in * c_out * (17 / 32 if op.startswith("mx4") else 2)
        nbytes += busy * 2 * r * (c_in + c_out)
    return {"bytes": nbytes, "flops": 2 * t * c_in * c_out + 2 * t * r * (c_in + c_out)}


def _case(name, op, t, c_in, c_out=0, e=0, r=0, pad=0, bf16=False):
    return {"name": name, "op": op, "t": t, "c_in": c_in, "c_out": c_out, "e": e, "r": r, "pad": pad, "bf16": bf16}


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _spans(lens):
    ends = list(itertools.accumulate(lens))
    return [(b - n, b) for n, b in zip(lens, ends)]


def _activations(normal, gen, t, c):
    """Normal values; one channel in a hundred is twenty to a hundred times the others."""
    x = normal(t, c)
    hot = torch.randperm(c, generator=gen, device=DEV)[:max(1, c // 100)]
    x[:, hot] *= 20 * 5 ** torch.rand(hot.numel(), generator=gen, device=DEV)
    return x


def _blocks(x):
    k = x.shape[1]
    return torch.nn.functional.pad(x, (0, -k % BLOCK)).unflatten(1, (-(-k // BLOCK), BLOCK))


def _scale_exponents(blocks):
    """Exponent of the power of two of each block: that of its largest magnitude less 2 (the grid ends at 6 = 1.5 x 2^2)."""
    return (torch.frexp(blocks.abs().amax(-1, keepdim=True)).exponent - 3).clamp(-127, 127)


def _on_grid(v):
    """Nearest value of the grid 0, .5, 1, 1.5, 2, 3, 4, 6 with both signs, ties to the even code, beyond 6 to 6."""
    m = v.abs()
    step = torch.where(m < 2, 0.5, torch.where(m < 4, 1.0, 2.0))
    return torch.copysign((torch.round(m / step) * step).clamp(max=6.0), v)


def _rounded(x):
    """fp32 [rows x k] rounded to 4 bits in blocks of 32 along k, as the values it stands for."""
    b = _blocks(x)
    e = _scale_exponents(b)
    return torch.ldexp(_on_grid(torch.ldexp(b, -e)), e).flatten(1)[:, :x.shape[1]].contiguous()


def _pack(x):
    """fp32 [rows x k] to codes [rows x kp / 2] (even k in the low four bits; bit 3 is the sign) and scales [rows x kp / 32]
    (exponent + 127), kp = k rounded up to 256; the padding holds zeros with scale 1."""
    x = torch.nn.functional.pad(x, (0, -x.shape[1] % BLOCK))
    b = _blocks(x)
    e = _scale_exponents(b)
    v = _on_grid(torch.ldexp(b, -e)).flatten(1)
    code = torch.searchsorted(torch.tensor(GRID, device=DEV), v.abs()).to(torch.uint8) | (torch.signbit(v).to(torch.uint8) << 3)
    code = torch.nn.functional.pad(code, (0, -x.shape[1] % PAD))
    scales = torch.nn.functional.pad((e + 127).flatten(1).to(torch.uint8), (0, -x.shape[1] % PAD // BLOCK), value=127)
    return code[:, 0::2] | (code[:, 1::2] << 4), scales.contiguous()


def _unpack(codes, scales, k):
    table = torch.tensor(GRID + [-v for v in GRID], device=DEV)
    v = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).view(codes.shape[0], scales.shape[1], BLOCK)
    return torch.ldexp(v, scales.int().unsqueeze(-1) - 127).flatten(1)[:, :k]


def _exact_values(x):
    """The same rounding in 64 bits by its definition: the scale from the logarithm, the value from the distances to the grid."""
    rows, k = x.shape
    out = torch.empty(rows, k, dtype=torch.float64, device=DEV)
    grid = torch.tensor(GRID, dtype=torch.float64, device=DEV)
    mid = (grid[1:] + grid[:-1]) / 2
    step = max(1, (1 << 26) // k)
    for a in range(0, rows, step):
        v = torch.nn.functional.pad(x[a:a + step].double(), (0, -k % BLOCK)).unflatten(1, (-(-k // BLOCK), BLOCK))
        top = v.abs().amax(-1, keepdim=True)
        e = torch.floor(torch.log2(torch.where(top > 0, top, 1.0)))
        e = torch.where(torch.exp2(e) > top, e - 1, e)
        s = torch.exp2((e - 2).clamp(-127, 127))
        m = v.abs() / s
        lo = torch.bucketize(m, mid)                # right ends included: a tie goes down, to an odd code half the time
        tie = (lo < 7) & (m == mid[lo.clamp(max=6)]) & (lo % 2 == 1)
        out[a:a + step] = (torch.sign(v) * grid[lo + tie] * s).flatten(1)[:, :k]
    return out


def _own(S):
    from paper_2505_14742_amd import binding as q
    c = S["case"]
    op, t, c_in, c_out, r = (c[k] for k in ("op", "t", "c_in", "c_out", "r"))
    if op == "quantize":
        if "codes" not in S:
            S["codes"], S["scales"] = _room(t, c_in)
            S["values"] = torch.empty_like(S["X"])
        q.mx4_quantize(S["X"], S["codes"], S["scales"])
        q.mx4_dequantize(S["codes"], S["scales"], S["values"])
        return {"X": S["values"]}
    if op == "prepare":
        if "fwd" not in S:
            S["fwd"], S["bwd"] = _room(c_out, c_in), _room(c_in, c_out)
            S["values"] = {"fwd": torch.empty(c_out, c_in, dtype=torch.bfloat16, device=DEV),
                           "bwd": torch.empty(c_in, c_out, dtype=torch.bfloat16, device=DEV)}
        q.mx4_prepare_weight(S["W"], *S["fwd"], *S["bwd"])
        q.mx4_dequantize(*S["fwd"], S["values"]["fwd"])
        q.mx4_dequantize(*S["bwd"], S["values"]["bwd"])
        return S["values"]
    mx4 = op.startswith("mx4")
    if "ws" not in S:
        need = q.mx4_linear_workspace_bytes(t, c_in, c_out, c["e"], r) if mx4 else q.grouped_linear_workspace_bytes(t, c_in, c_out, c["e"])
        S["ws"] = torch.empty(need, dtype=torch.int8, device=DEV)
    out, ws, bf16 = S["out"], S["ws"], c["bf16"]
    if op == "mx4_fwd":
        q.mx4_linear_fwd(S["X"], S["offsets"], S["codes"], S["scales"], c_in, c_out, S["A"], S["B"], r, 0.5, out, ws, bf16_out=bf16)
    elif op == "mx4_dx":
        q.mx4_linear_bwd_dx(S["dY"], S["offsets"], S["codes"], S["scales"], c_in, c_out, S["A"], S["B"], r, 0.5, out, ws, bf16_out=bf16)
    elif op == "fwd":
        q.grouped_linear_fwd(S["X"], S["offsets"], S["W"], 0.5, out, ws, bf16_out=bf16)
    elif op == "dx":
        q.grouped_linear_bwd_dx(S["dY"], S["offsets"], S["W"], 0.5, out, ws, bf16_out=bf16)
    else:
        q.grouped_linear_bwd_dw(S["X"], S["dY"], S["offsets"], 0.5, out, ws)
    return {"out": out}


def _room(rows, k):
    kp = -(-k // PAD) * PAD
    return (torch.empty(rows, kp // 2, dtype=torch.uint8, device=DEV), torch.empty(rows, kp // 32, dtype=torch.uint8, device=DEV))
