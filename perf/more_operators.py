"""Operators of a fine-tuning step in few bits: quantisation to 4-bit floating point and products of such operands, a root-mean-square
norm that takes the residual's addition in and puts 8-bit operands out, log probabilities of given tokens with the entropy and the
likeliest alternatives, and clipping by the norm of all gradients together.

Where `own` is false every operator is written out in elementary torch operations; where it is true the calls go to the library's
entry points, as a training program makes them.
"""
import math

import torch

own = False

_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_F8 = {"e4m3": torch.float8_e4m3fn, "e5m2": torch.float8_e5m2}
_F8_TOP = {"e4m3": 8, "e5m2": 15}       # the largest value of either format is 1.75 * 2^top
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ---- the cases ---------------------------------------------------------------------------------------------------

def listed():
    return [
        # first feed-forward product of the measured 12-layer LM, all of its tokens
        {"name": "f4gemm_8192x8192x2048", "family": "f4gemm", "m": 8192, "n": 8192, "k": 2048, "epilogue": "bias", "out": "bf16"},
        # the weight gradient that goes with it: contraction over the tokens
        {"name": "f4gemm_2048x8192x8192", "family": "f4gemm", "m": 2048, "n": 8192, "k": 8192, "epilogue": "store", "out": "f32"},
        # one token through the same first product: the weights are read once
        {"name": "f4gemm_1x8192x2048", "family": "f4gemm", "m": 1, "n": 8192, "k": 2048, "epilogue": "bias", "out": "bf16"},
        # a projection into the residual stream at sizes that fit no tile
        {"name": "f4gemm_1000x760x1056", "family": "f4gemm", "m": 1000, "n": 760, "k": 1056, "epilogue": "residual", "out": "f32"},
        # activations for the forward product and, transposed, for the weight gradient
        {"name": "f4quant_8192x2048", "family": "f4quant", "rows": 8192, "cols": 2048, "dtype": "bf16", "block": 1, "both": True},
        # a small weight of odd sizes in single precision, the same blocks in both directions
        {"name": "f4quant_333x500", "family": "f4quant", "rows": 333, "cols": 500, "dtype": "f32", "block": 32, "both": True},
        # the norm in front of that product: branch into the residual stream, 8-bit operand out, and its backward pass
        {"name": "rms_8192x2048", "family": "rms", "rows": 8192, "cols": 2048, "dtype": "bf16", "res": True, "format": "e4m3",
         "backward": True},
        # one token of a model that answers
        {"name": "rms_1x2048", "family": "rms", "rows": 1, "cols": 2048, "dtype": "bf16", "res": True, "format": "e4m3",
         "backward": False},
        # every token of the measured LM over its whole vocabulary, with the gradient
        {"name": "logp_8192x32768", "family": "logp", "rows": 8192, "vocab": 32768, "dtype": "bf16", "top": 8, "scale": 1.0,
         "backward": True},
        # the next token of four answers, with the alternatives that a sampler chooses from
        {"name": "logp_4x32768", "family": "logp", "rows": 4, "vocab": 32768, "dtype": "f32", "top": 20, "scale": 1.25,
         "backward": False},
        # gradients of four layers of the measured LM with embedding and head
        {"name": "clip_lm", "family": "clip", "layers": 4, "width": 2048, "vocab": 32768, "dtype": "f32"},
        # a small model of odd sizes
        {"name": "clip_small", "family": "clip", "layers": 2, "width": 61, "vocab": 331, "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    family = rng.choice(["f4gemm", "f4gemm", "f4quant", "rms", "logp", "logp", "clip"])
    if family == "f4gemm":
        m, n, k = _log(rng, 1, 8192), _log(rng, 16, 8192), max(32, _log(rng, 64, 8192) // 32 * 32)
        while m * n * k > 8192 * 8192 * 2048:
            m = m // 2 + 1
        out = rng.choice(["bf16", "f32"])
        epilogues = ["store", "bias", "gelu", "gelu_bwd"] if out == "bf16" else ["store", "bias", "residual", "add"]
        return {"family": family, "m": m, "n": n, "k": k, "epilogue": rng.choice(epilogues), "out": out}
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if family == "f4quant":
        rows = _log(rng, 1, 8192)
        return {"family": family, "rows": rows, "cols": _log(rng, 16, min(8192, (1 << 24) // rows)), "dtype": dtype,
                "block": rng.choice([1, 1, 32]), "both": rng.random() < 0.6}
    if family == "rms":
        rows = _log(rng, 1, 8192)
        return {"family": family, "rows": rows, "cols": _log(rng, 16, min(8192, (1 << 24) // rows)), "dtype": dtype,
                "res": rng.random() < 0.7, "format": rng.choice(["none", "e4m3", "e4m3", "e5m2"]), "backward": rng.random() < 0.6}
    if family == "logp":
        rows = _log(rng, 1, 8192)
        return {"family": family, "rows": rows, "vocab": _log(rng, 64, min(200000, (1 << 28) // rows)), "dtype": dtype,
                "top": rng.choice([0, 1, _log(rng, 2, 32)]), "scale": rng.choice([1.0, round(rng.uniform(0.5, 2.0), 3)]),
                "backward": dtype == "bf16" and rng.random() < 0.6}
    width = _log(rng, 16, 2048)
    return {"family": family, "layers": rng.randint(1, 4), "width": width, "vocab": _log(rng, 64, 32768), "dtype": dtype}


# ---- inputs ------------------------------------------------------------------------------------------------------

class _Draw:
    """Seeded values on the GPU; the order of the calls is part of the recipe."""

    def __init__(self, seed):
        self.g = torch.Generator(device="cuda")
        self.g.manual_seed(int(seed) * 7919 + 17)

    def normal(self, *shape, std=1.0, mean=0.0, dtype=torch.float32):
        t = torch.randn(*shape, generator=self.g, device="cuda", dtype=torch.float32)
        return t.mul_(std).add_(mean).to(dtype)

    def uneven(self, rows, cols, dtype=torch.float32):
        """Rows and columns of different sizes, as activations and gradients have."""
        r = torch.exp(self.normal(rows, 1)) * torch.exp(self.normal(1, cols, std=0.5))
        return (self.normal(rows, cols) * r).to(dtype)

    def integers(self, lo, hi, *shape, dtype=torch.int32):
        return torch.randint(lo, hi, shape, generator=self.g, device="cuda", dtype=dtype)


def _up(n, m):
    return -(-n // m) * m


def _shapes(c):
    """The tensors of an LM: table, positions, and for each layer norms, projections, feed-forward pair and their biases; the head."""
    d, v = c["width"], c["vocab"]
    layer = [(d,), (d, 3 * d), (3 * d,), (d, d), (d,), (d,), (d, 4 * d), (4 * d,), (4 * d, d), (d,)]
    return [(v, d), (128, d)] + layer * c["layers"] + [(d,), (d, v)]


def prepare(case, seed):
    c, r, fam = dict(case), _Draw(seed), case["family"]
    s = {"case": c}
    if fam == "f4gemm":
        m, n, k = c["m"], c["n"], c["k"]
        s["a"], s["a_scale"] = _quantised(r.uneven(m, k), 1)
        s["b"], s["b_scale"] = _quantised(r.uneven(n, k) * 0.02, 32 if c["out"] == "bf16" else 1)   # a weight, or gradients
        ldc = _up(n, 8)                    # rows of outputs start on 16 bytes
        if c["epilogue"] in ("bias", "residual", "gelu"):
            s["bias"] = r.normal(n, std=0.5)
        if c["epilogue"] == "residual":
            s["aux"] = r.normal(m, ldc)
        if c["epilogue"] == "gelu_bwd":
            s["aux"] = r.normal(m, ldc, dtype=torch.bfloat16)
        s["c"] = r.normal(m, ldc, dtype=_TORCH[c["out"]])
        if c["epilogue"] == "add":
            s["c0"] = s["c"].clone()       # a pass adds into what is there: every pass starts from this
    elif fam == "f4quant":
        s["x"] = r.uneven(c["rows"], c["cols"], dtype=_TORCH[c["dtype"]])
        if c["block"] == 32:
            s["x"].mul_(0.02)
    elif fam == "rms":
        n, d, t = c["rows"], c["cols"], _TORCH[c["dtype"]]
        s["x"], s["g"] = r.uneven(n, d), r.normal(d, std=0.2, mean=1.0)
        s["y"] = r.normal(n, d, dtype=t) if c["res"] else None
        if c["backward"]:
            s["dh"], s["dres"] = r.normal(n, d, std=1e-2, dtype=t), r.normal(n, d, std=1e-2) if c["res"] else None
    elif fam == "logp":
        n, v = c["rows"], c["vocab"]
        z = r.normal(n, v, std=2.0)
        z[:, v - v // 32:] = -math.inf     # columns behind the last token of the vocabulary
        s["target"] = r.integers(0, v - v // 32, n)
        z.scatter_add_(1, s["target"].long()[:, None], torch.full((n, 1), 6.0, device="cuda"))
        s["z"] = z.to(_TORCH[c["dtype"]])
        s["target"][r.integers(0, 10, n) == 0] = -1           # positions that are not scored, as prompts are
        if c["backward"]:
            s["dlogp"], s["dent"] = r.normal(n, std=1.0 / n), r.normal(n, std=0.01 / n)
    else:
        s["grads"] = [r.normal(*shape, std=1e-3, dtype=torch.float32 if len(shape) == 1 else _TORCH[c["dtype"]]) for shape in _shapes(c)]
        s["max_norm"] = 0.2
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------------

def _two_to(e):
    """2^e in 64 bits, put together from its bits: pow() and ldexp() are not exact on every device."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _fit(amax, top):
    """Smallest e in [-127, 127] with amax <= top * 2^e, 1 <= top / 2^floor(log2 top) < 2."""
    low = math.floor(math.log2(top))
    m, k = torch.frexp(amax.double())                 # amax = 2 m * 2^(k - 1)
    e = k.long() - 1 - low + (2 * m > top / 2.0 ** low).long()
    return torch.where(amax == 0, torch.full_like(e, -127), e).clamp(-127, 127)


def _f4_index(rows, blocks, device):
    """Where the scale of (row, block of 32) is: 256 bytes for 64 rows and four blocks, one block's 64 after another's, the four rows
    r, r + 16, r + 32, r + 48 side by side."""
    r, b = torch.arange(rows, device=device)[:, None], torch.arange(blocks, device=device)[None, :]
    return (b // 4 * _up(rows, 64) + r // 64 * 64) * 4 + b % 4 * 64 + r % 16 * 4 + r % 64 // 16


def _f4_codes(y):
    """Codes of the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code, and the sign."""
    a = y.abs()
    code = (a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte() + (a > 2.5).byte() + (a >= 3.5).byte() + \
        (a > 5.0).byte()
    return code + torch.signbit(y).byte() * 8


def _quantised(x, block):
    """(two codes to a byte [rows, columns up to a multiple of 32 / 2], scale bytes as the product reads them) of x."""
    rows, cols = x.shape
    nb = _up(cols, 32) // 32
    xp = torch.zeros(_up(rows, block), nb * 32, dtype=torch.float32, device=x.device)
    xp[:rows, :cols] = x
    e = _fit(xp.abs().view(-1, block, nb, 32).amax(dim=(1, 3)), 6.0).repeat_interleave(block, 0)[:rows]
    code = _f4_codes((xp[:rows].view(rows, nb, 32) * _two_to(-e)[:, :, None]).view(rows, -1))
    table = torch.zeros(_up(rows, 64) * 4 * (_up(nb, 4) // 4), dtype=torch.uint8, device=x.device)
    table[_f4_index(rows, nb, x.device).reshape(-1)] = (e + 127).to(torch.uint8).reshape(-1)
    return code[:, ::2] | code[:, 1::2] << 4, table


def _plain_f4quant(s, c):
    """Codes and scales.  The sixteen codes of a byte's halves stand for the sixteen values one for one: returned as they are, they
    have to be equal."""
    x = s["x"].float()
    q, scale = _quantised(x, c["block"])
    out = {"q": q, "scale": scale}
    if c["both"]:
        out["qt"], out["scale_t"] = _quantised(x.T, c["block"])
    return out


def _f4_values(q, table):
    rows, k = q.shape[0], 2 * q.shape[1]
    v = torch.tensor(_E2M1 + tuple(-x for x in _E2M1), device=q.device)
    code = torch.stack([q & 15, q >> 4], -1).view(rows, k)
    scale = _two_to(table[_f4_index(rows, k // 32, q.device)].long() - 127).float()
    return v[code.int()] * scale.repeat_interleave(32, 1)


def _gelu_parts(u):
    return torch.tanh(math.sqrt(2 / math.pi) * (u + 0.044715 * u * u * u)), math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * u * u)


def _plain_f4gemm(s, c):
    n, epi, t = c["n"], c["epilogue"], _TORCH[c["out"]]
    v = _f4_values(s["a"], s["a_scale"]) @ _f4_values(s["b"], s["b_scale"]).T
    if epi in ("bias", "residual", "gelu"):
        v = v + s["bias"]
    if epi == "residual":
        v = v + s["aux"][:, :n]
    elif epi == "gelu":
        th, _ = _gelu_parts(v)
        return {"u": v.to(t), "h": (0.5 * v * (1 + th)).to(t)}
    elif epi == "gelu_bwd":
        u = s["aux"][:, :n].float()
        th, dz = _gelu_parts(u)
        v = v * (0.5 * (1 + th) + 0.5 * u * (1 - th * th) * dz)
    elif epi == "add":
        v = v + s["c0"][:, :n]
    return {"c": v.to(t)}


_EPS = 1e-5


def _plain_rms(s, c):
    t = _TORCH[c["dtype"]]
    x = s["x"] + s["y"].float() if c["res"] else s["x"]
    rstd = torch.rsqrt(x.square().mean(1) + _EPS)
    xh = x * rstd[:, None]
    h = xh * s["g"]
    out = {"h": h.to(t), "rstd": rstd}
    if c["res"]:
        out["x"] = x
    if c["format"] != "none":
        rows, cols = x.shape
        nb = _up(cols, 128) // 128
        hp = torch.zeros(rows, nb * 128, device=x.device)
        hp[:, :cols] = h
        e = _fit(hp.abs().view(rows, nb, 128).amax(2), 1.75 * 2.0 ** _F8_TOP[c["format"]])
        q = (hp.view(rows, nb, 128) * _two_to(-e)[:, :, None]).view(rows, -1).float().to(_F8[c["format"]])
        r, b = torch.arange(rows, device=x.device)[:, None], torch.arange(nb, device=x.device)[None, :]
        table = torch.zeros(_up(rows, 64) * nb, dtype=torch.uint8, device=x.device)
        table[(b * _up(rows, 64) + r // 64 * 64 + r % 16 * 4 + r % 64 // 16).reshape(-1)] = (e + 127).to(torch.uint8).reshape(-1)
        out.update(q=q[:, :_up(cols, 16)].contiguous(), scale=table.view(torch.float8_e8m0fnu))
    if c["backward"]:
        dh = s["dh"].float()
        dg = dh * s["g"]
        dx = rstd[:, None] * (dg - xh * (dg * xh).mean(1, keepdim=True))
        if c["res"]:
            dx = dx + s["dres"]
        out.update(dx=dx, dy=dx.to(t), dg=(dh * xh).sum(0, dtype=torch.float64).float())
    return out


def _plain_logp(s, c):
    z, target, k = s["z"].float() * c["scale"], s["target"].long(), c["top"]
    rows = torch.arange(z.shape[0], device=z.device)
    zero = torch.zeros((), device=z.device)
    d = z - z.amax(1, keepdim=True)
    e = torch.exp(d)
    total = e.sum(1)
    logp = d - torch.log(total)[:, None]
    p = e / total[:, None]
    plogp = torch.where(p > 0, p * logp, zero)
    entropy = -plogp.sum(1)
    given = target >= 0
    out = {"logp": torch.where(given, logp[rows, target.clamp(min=0)], zero), "entropy": entropy}
    if k:
        order = torch.sort(s["z"].float(), dim=1, descending=True, stable=True).indices[:, :k]     # the lowest index first among equals
        best = logp.gather(1, order)
        out.update(top_id=torch.where(best > -math.inf, order, -1).int(), top_logp=best)
    if c["backward"]:
        dz = -(s["dlogp"] * given)[:, None] * p - s["dent"][:, None] * (plogp + p * entropy[:, None])
        dz[rows, target.clamp(min=0)] += s["dlogp"] * given
        out["dz"] = (dz * c["scale"]).to(s["z"].dtype)
    return out


def _plain_clip(s, c):
    norm = torch.stack([g.float().square().sum(dtype=torch.float64) for g in s["grads"]]).sum().sqrt()
    factor = torch.where(norm > s["max_norm"], s["max_norm"] / norm, torch.ones_like(norm)).float()
    return {"norm": norm.float(), "factor": factor, "grads": [(g.float() * factor).to(g.dtype) for g in s["grads"]]}


# ---- the library's calls -----------------------------------------------------------------------------------------

_context = _stream = None


def _ctx():
    """One context per program, as in any program that uses the library, on a stream of the program's that is its current one from
    here on, behind what was under way on the one before: what makes inputs, the operators and what reads their outputs follow one
    another."""
    global _context, _stream
    if _context is None:
        from paper_2203_12533_amd import binding
        _stream = torch.cuda.Stream()
        _context = binding.Context(0, _stream.cuda_stream)
        _stream.wait_stream(torch.cuda.current_stream())
        torch.cuda.set_stream(_stream)
    return _context


def _p(x):
    return x.data_ptr() if x is not None else None


def _buffers(s, c):
    """What a program allocates once per size: outputs and workspaces."""
    from paper_2203_12533_amd import binding as pwb
    new = lambda *shape, dtype=torch.float32: torch.empty(*shape, dtype=dtype, device="cuda")  # noqa: E731
    fam = c["family"]
    dt = {"f32": pwb.PW_F32, "bf16": pwb.PW_BF16}
    if fam == "f4gemm":
        epi = {"store": pwb.PW_EPI_STORE, "add": pwb.PW_EPI_STORE, "bias": pwb.PW_EPI_BIAS, "residual": pwb.PW_EPI_BIAS_RESIDUAL,
               "gelu": pwb.PW_EPI_BIAS_GELU, "gelu_bwd": pwb.PW_EPI_GELU_BWD}[c["epilogue"]]
        c2 = torch.empty_like(s["c"]) if c["epilogue"] == "gelu" else None
        args = pwb.F4GemmArgs(M=c["m"], N=c["n"], K=c["k"], lda=c["k"], ldb=c["k"], ldc=s["c"].shape[1], epilogue=epi, out_dtype=dt[c["out"]],
                              accumulate=int(c["epilogue"] == "add"), A=_p(s["a"]), B=_p(s["b"]), a_scale=_p(s["a_scale"]),
                              b_scale=_p(s["b_scale"]), bias=_p(s.get("bias")), aux=_p(s.get("aux")), C=_p(s["c"]), C2=_p(c2))
        return {"args": args, "c2": c2}
    if fam == "f4quant":
        rows, cols, byte = c["rows"], c["cols"], torch.uint8
        o = {"q": new(rows, _up(cols, 32) // 2, dtype=byte), "scale": new(pwb.f4_scale_bytes(rows, cols), dtype=byte)}
        if c["both"]:
            o.update(qt=new(cols, _up(rows, 32) // 2, dtype=byte), scale_t=new(pwb.f4_scale_bytes(cols, rows), dtype=byte))
        o["args"] = pwb.F4QuantizeArgs(dtype=dt[c["dtype"]], block_rows=c["block"], x=_p(s["x"]), rows=rows, cols=cols, ldx=cols,
                                       q=_p(o["q"]), ldq=_up(cols, 32), q_scale=_p(o["scale"]), qt=_p(o.get("qt")),
                                       ldqt=_up(rows, 32), qt_scale=_p(o.get("scale_t")))
        return o
    if fam == "rms":
        n, d, t = c["rows"], c["cols"], _TORCH[c["dtype"]]
        o = {"h": new(n, d, dtype=t), "rstd": new(n), "x": new(n, d) if c["res"] else None, "f8": None}
        if c["format"] != "none":
            o.update(q=new(n, _up(d, 16), dtype=_F8[c["format"]]), scale=new(pwb.f8_scale_bytes(n, d), dtype=torch.uint8))
            o["f8"] = pwb.F8Out(format={"e4m3": pwb.PW_E4M3, "e5m2": pwb.PW_E5M2}[c["format"]], q=_p(o["q"]), ldq=_up(d, 16),
                                scale=_p(o["scale"]))
        o["args"] = pwb.RmsnormArgs(dtype=dt[c["dtype"]], rows=n, cols=d, ldx=d, ldh=d, eps=_EPS, g=_p(s["g"]))
        if c["backward"]:
            o.update(dx=new(n, d), dy=new(n, d, dtype=t), dg=new(d), ws=new(max(1, pwb.rmsnorm_bwd_ws_floats(n, d))))
        return o
    if fam == "logp":
        n, v, k = c["rows"], c["vocab"], c["top"]
        o = {"logp": new(n), "entropy": new(n), "stats": new(n, 2), "ws": new(max(1, pwb.logprob_ws_floats(n, v, k))),
             "args": pwb.LogprobArgs(dtype=dt[c["dtype"]], z=_p(s["z"]), ldz=v, rows=n, vocab=v, targets=_p(s["target"]), scale=c["scale"])}
        o["top_id"], o["top_logp"] = (new(n, k, dtype=torch.int32), new(n, k)) if k else (None, None)
        if c["backward"]:
            o["dz"] = torch.empty_like(s["z"])
        return o
    o = {"grads": [torch.empty_like(g) for g in s["grads"]], "result": new(2), "ws": new(pwb.grad_clip_ws_floats())}
    o["tensors"] = pwb.grad_tensors([(_p(g), _p(x), g.numel(), dt["f32" if g.dtype == torch.float32 else "bf16"])
                                     for g, x in zip(s["grads"], o["grads"])])
    return o


def _own_run(s, c):
    ctx = _ctx()                           # first: buffers belong to the stream that is current then
    if "own" not in s:
        s["own"] = _buffers(s, c)
    o, fam = s["own"], c["family"]
    if fam == "f4gemm":
        if c["epilogue"] == "add":
            s["c"].copy_(s["c0"])
        ctx.f4_gemm(o["args"])
        out = s["c"][:, :c["n"]]
        return {"u": out, "h": o["c2"][:, :c["n"]]} if c["epilogue"] == "gelu" else {"c": out}
    if fam == "f4quant":
        ctx.f4_quantize(o["args"])
        return {k: o[k] for k in ("q", "scale", "qt", "scale_t") if k in o}
    if fam == "rms":
        ctx.rmsnorm_fwd(o["args"], _p(s["x"]), _p(s["y"]), _p(o["x"]), _p(o["h"]), o["f8"], _p(o["rstd"]))
        out = {k: o[k] for k in ("h", "rstd") + (("x",) if c["res"] else ())}
        if o["f8"] is not None:
            out.update(q=o["q"], scale=o["scale"].view(torch.float8_e8m0fnu))
        if c["backward"]:
            ctx.rmsnorm_bwd(o["args"], _p(s["dh"]), _p(o["x"] if c["res"] else s["x"]), _p(o["rstd"]), _p(s["dres"]), _p(o["dx"]),
                            _p(o["dy"]), _p(o["dg"]), _p(o["ws"]))
            out.update({k: o[k] for k in ("dx", "dy", "dg")})
        return out
    if fam == "logp":
        ctx.logprob_fwd(o["args"], _p(o["logp"]), _p(o["entropy"]), _p(o["stats"]), c["top"], _p(o["top_id"]), _p(o["top_logp"]), _p(o["ws"]))
        out = {k: o[k] for k in ("logp", "entropy") + (("top_id", "top_logp") if c["top"] else ())}
        if c["backward"]:
            ctx.logprob_bwd(o["args"], _p(o["stats"]), _p(o["entropy"]), _p(s["dlogp"]), _p(s["dent"]), _p(o["dz"]), c["vocab"])
            out["dz"] = o["dz"]
        return out
    ctx.grad_clip(o["tensors"], s["max_norm"], _p(o["result"]), _p(o["ws"]))
    return {"norm": o["result"][0], "factor": o["result"][1], "grads": o["grads"]}


_PLAIN = {"f4gemm": _plain_f4gemm, "f4quant": _plain_f4quant, "rms": _plain_rms, "logp": _plain_logp, "clip": _plain_clip}


def run(state):
    c = state["case"]
    if own:
        return _own_run(state, c)
    return _PLAIN[c["family"]](state, c)


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------

_POWERS = [math.ldexp(1.0, i - 300) for i in range(601)]


def _power(e):
    return torch.tensor(_POWERS, dtype=torch.float64, device="cuda")[e.long() + 300]


def _exact_operand(q, table):
    rows, k = q.shape[0], 2 * q.shape[1]
    value = [(-1.0 if i & 8 else 1.0) * (math.ldexp(2 + (i & 1), (i >> 1 & 3) - 2) if i & 6 else (i & 1) / 2) for i in range(16)]
    pair = torch.tensor([[value[b & 15], value[b >> 4]] for b in range(256)], dtype=torch.float64, device="cuda")
    v = pair[q.long()].reshape(rows, k)
    # [four blocks][64 rows][block][row % 16][row / 16] to [row][block]
    t = table.view(-1, _up(rows, 64) // 64, 4, 16, 4).permute(1, 4, 3, 0, 2).reshape(_up(rows, 64), -1)[:rows]
    for b in range(k // 32):
        v[:, 32 * b:32 * b + 32] *= _power(t[:, b:b + 1].long() - 127)
    return v


def _exact_f4gemm(s, c):
    v = torch.matmul(_exact_operand(s["a"], s["a_scale"]), _exact_operand(s["b"], s["b_scale"]).T.contiguous())
    epi, n = c["epilogue"], c["n"]
    sig = lambda u: 1 / (1 + torch.exp(-2 * math.sqrt(2 / math.pi) * (u + 0.044715 * u ** 3)))  # noqa: E731
    if epi == "bias":
        v += s["bias"].double()
    elif epi == "residual":
        v += s["bias"].double() + s["aux"][:, :n].double()
    elif epi == "add":
        v += s["c0"][:, :n].double()
    elif epi == "gelu":
        v += s["bias"].double()
        return {"u": v, "h": v * sig(v)}
    elif epi == "gelu_bwd":
        u = s["aux"][:, :n].double()
        e = sig(u)
        v *= e + u * e * (1 - e) * 2 * math.sqrt(2 / math.pi) * (1 + 0.134145 * u ** 2)
    return {"c": v}


def _exact_rms(s, c):
    x = s["x"].double()
    if c["res"]:
        x = x + s["y"].double()
    d = x.shape[1]
    rms = torch.sqrt((x * x).sum(1) / d + _EPS)
    h = x / rms[:, None] * s["g"].double()
    out = {"h": h, "rstd": 1 / rms, "x": x.float().double() if c["res"] else None}
    if c["format"] != "none":
        top, mant, low = (448.0, 3, -6) if c["format"] == "e4m3" else (57344.0, 2, -14)
        q, scales = [], []
        for j in range(0, d, 128):
            part = h[:, j:j + 128]
            peak = part.abs().amax(1)
            e = torch.ceil(torch.log2(peak / top)).clamp(-127, 127)
            e = torch.where(peak <= top * _power(e - 1), e - 1, torch.where(peak > top * _power(e), e + 1, e)).clamp(-127, 127)
            y = part / _power(e)[:, None]
            step = _power(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** low))) - mant)
            q.append(torch.round(y / step) * step)             # halves to even, as the format's last bit goes
            full = torch.full((_up(x.shape[0], 64),), 2.0 ** -127, dtype=torch.float64, device="cuda")
            full[:x.shape[0]] = _power(e)
            scales.append(full.view(-1, 4, 16).transpose(1, 2).reshape(-1))
        q = torch.cat(q, 1)
        out.update(q=torch.nn.functional.pad(q, (0, _up(d, 16) - d)), scale=torch.cat(scales))
    if c["backward"]:
        dh, g = s["dh"].double(), s["g"].double()
        dot = (dh * g * x).sum(1) / d
        dx = (dh * g) / rms[:, None] - x * (dot / rms ** 3)[:, None]
        if c["res"]:
            dx = dx + s["dres"].double()
        out.update(dx=dx, dy=dx, dg=(dh * x / rms[:, None]).sum(0))
    return out


def _exact_logp(s, c):
    """A few rows at a time."""
    n, v, scale = c["rows"], c["vocab"], c["scale"]
    parts = []
    for i in range(0, n, 1024):
        z = s["z"][i:i + 1024].double() * scale
        t = s["target"][i:i + 1024].long()
        on = t >= 0
        lse = torch.logsumexp(z, 1)
        lp = z - lse[:, None]
        p = torch.exp(lp)
        h = torch.special.entr(p).sum(1)
        o = {"logp": torch.where(on, lp.gather(1, t.clamp(min=0)[:, None])[:, 0], torch.zeros_like(lse)), "entropy": h}
        if c["top"]:
            o["top_logp"] = torch.topk(lp, c["top"]).values
        if c["backward"]:
            dl, de = s["dlogp"][i:i + 1024].double() * on, s["dent"][i:i + 1024].double()
            dz = p * (-dl - de * h)[:, None] + de[:, None] * torch.special.entr(p)
            dz.scatter_add_(1, t.clamp(min=0)[:, None], dl[:, None])
            o["dz"] = (dz * scale).float() if n * v > 1 << 26 else dz * scale       # half the memory, far below a bf16 step
        parts.append(o)
    return {k: torch.cat([o[k] for o in parts]) for k in parts[0]}


def _exact_clip(s, c):
    total = math.sqrt(math.fsum(float((g.double() ** 2).sum()) for g in s["grads"]))
    factor = min(1.0, s["max_norm"] / total) if total > 0 else 1.0
    return {"norm": torch.tensor(total, dtype=torch.float64), "factor": torch.tensor(factor, dtype=torch.float64),
            "grads": [g.double() * factor for g in s["grads"]]}


_EXACT = {"f4gemm": _exact_f4gemm, "rms": _exact_rms, "logp": _exact_logp, "clip": _exact_clip}


def exact(case, seed):
    if case["family"] == "f4quant":
        return None                        # whole numbers only
    return _EXACT[case["family"]](prepare(case, seed), case)


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    c, fam = case, case["family"]
    if fam == "f4gemm":
        m, n, k = c["m"], c["n"], c["k"]
        es = 2 if c["out"] == "bf16" else 4
        out = m * n * es * (2 if c["epilogue"] == "gelu" else 1)
        extra = m * n * {"residual": 4, "add": 4, "gelu_bwd": 2}.get(c["epilogue"], 0)
        return {"bytes": float((m + n) * k * (1 / 2 + 1 / 32) + out + extra + 4 * n), "flops": 2.0 * m * n * k}
    es = 2 if c["dtype"] == "bf16" else 4
    if fam == "f4quant":
        n = c["rows"] * c["cols"]
        return {"bytes": float(n * (es + (2 if c["both"] else 1) * (1 / 2 + 1 / 32))), "flops": 4.0 * n}
    if fam == "rms":
        n = c["rows"] * c["cols"]
        fwd = 4 + (4 + es if c["res"] else 0) + es + (1 + 1 / 128 if c["format"] != "none" else 0)
        bwd = es + 4 + (4 if c["res"] else 0) + 4 + es if c["backward"] else 0
        return {"bytes": float(n * (fwd + bwd) + 8 * c["cols"]), "flops": float(n * (18 if c["backward"] else 8))}
    if fam == "logp":
        n = c["rows"] * c["vocab"]
        return {"bytes": float(n * es * (3 if c["backward"] else 1) + 16 * c["rows"]), "flops": float(n * (14 if c["backward"] else 6))}
    n = [math.prod(shape) * (4 if len(shape) == 1 else es) for shape in _shapes(c)]
    return {"bytes": float(2 * sum(n)), "flops": float(3 * sum(n) // es)}
