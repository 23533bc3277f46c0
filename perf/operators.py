"""Operators of a low-precision LM head and of scoring its logits, as measurable cases.

A case names one call (or the pair that a user needs to see the values) of the
public binding:

  quantize  Model.mx_quantize, and Model.mx_dequantize of its result: blocks of
            32 columns share a power-of-two scale, values in E2M1 (4 bits) or
            E4M3 (8 bits)
  norm      Model.add_norm_mx: residual addition, RMS or layer norm, output in
            E4M3 or E2M1 with block scales (and its values, by mx_dequantize)
  matmul    Model.mx_matmul: A [M, K] in E4M3 or E2M1 times the transpose of
            B [N, K] in E2M1, to fp32 or bf16
  scores    Model.token_scores: log2 probabilities of given tokens, entropies in
            bits and the most probable alternatives, from logit rows

With `own` false, `run` computes the same in elementary torch operations in 32
bits.  A matrix held with block scales is its codes [rows, pitch] (two E2M1 codes
a byte, the even column in the low half) and its scales [groups, slots, 8]: a
group is 256 columns, one byte 2^(s - 127) for each 32 of them; columns are
filled up to whole groups with zeros, the scales' rows up to a multiple of 32.
"""
import math

import torch

own = False

TOP_OF = {"fp4": 6.0, "fp8": 448.0}     # largest value of a format
GROUP = 256
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# the values of the 16 E2M1 codes
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]
E2M1 = E2M1 + [-v for v in E2M1]


def listed():
    return [
        # a head's weights are quantised once, when a model is made: the small
        # vocabulary at the 8B-shaped width
        dict(name="quantize_head", kind="quantize", rows=32768, cols=4096, fmt="fp4", dtype="bf16"),
        # rows of activations of the last, partial chunk of an input
        dict(name="quantize_rows", kind="quantize", rows=777, cols=4096, fmt="fp8", dtype="f32"),
        # a layer's norm at the 8B shape: one 2048-token chunk, the branch's
        # output added to the fp32 residual stream
        dict(name="norm_pass", kind="norm", rows=2048, cols=4096, norm="rmsnorm", fmt="fp8",
             dtype="f32", delta="bf16", gain=True),
        # the same for one position, where the launches count
        dict(name="norm_token", kind="norm", rows=1, cols=4096, norm="rmsnorm", fmt="fp8",
             dtype="f32", delta="bf16", gain=True),
        # the LM head of the 8B shape over a fully masked chunk
        dict(name="matmul_head", kind="matmul", M=2048, N=126464, K=4096, fmt="fp8", out="f32"),
        # the same head for the 16 rows that a pass of a block schedule commits
        dict(name="matmul_committed", kind="matmul", M=16, N=126464, K=4096, fmt="fp8", out="f32"),
        # a wide projection on 4-bit activations
        dict(name="matmul_ffn", kind="matmul", M=2048, N=24576, K=4096, fmt="fp4", out="bf16"),
        # one row through a square projection: latency
        dict(name="matmul_token", kind="matmul", M=1, N=4096, K=4096, fmt="fp4", out="bf16"),
        # odd sizes throughout: a partial chunk, a ragged vocabulary, a width that
        # ends inside a block of 32
        dict(name="matmul_odd", kind="matmul", M=777, N=4099, K=1000, fmt="fp8", out="f32"),
        # every row of a fully masked chunk at the 8B vocabulary, eight alternatives
        dict(name="scores_pass", kind="scores", rows=2048, vocab=126464, top=8, dtype="f32",
             masked=0.0),
        # one row with twenty alternatives: latency
        dict(name="scores_token", kind="scores", rows=1, vocab=126464, top=20, dtype="f32",
             masked=0.0),
        # the small model's batch: 64 chunks, 8 committed symbols each, from bf16
        # logits of which a tenth are ruled out (-inf), without alternatives
        dict(name="scores_batch", kind="scores", rows=512, vocab=32768, top=0, dtype="bf16",
             masked=0.1),
    ]


# --------------------------------------------------------------------------
# drawn cases: the ranges the listed ones stand for
# --------------------------------------------------------------------------
def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(["quantize", "norm", "matmul", "scores"], weights=[2, 2, 4, 3])[0]
    if kind == "quantize":
        cols = rng.choice([128, 768, 1000, 2048, 4096, 8192, _log_int(rng, 33, 8192)])
        return dict(kind=kind, rows=_log_int(rng, 1, 2 ** 26 // cols), cols=cols,
                    fmt=rng.choice(["fp4", "fp8"]), dtype=rng.choice(["f32", "bf16"]))
    if kind == "norm":
        cols = rng.choice([128, 768, 1000, 2048, 4096, 8192, _log_int(rng, 33, 8192)])
        return dict(kind=kind, rows=_log_int(rng, 1, 2 ** 26 // cols), cols=cols,
                    norm=rng.choice(["rmsnorm", "rmsnorm", "layernorm"]),
                    fmt=rng.choice(["fp8", "fp8", "fp4"]), dtype=rng.choice(["f32", "f32", "bf16"]),
                    delta=rng.choice(["", "bf16", "f32"]), gain=rng.random() < 0.5)
    if kind == "matmul":
        K = rng.choice([128, 768, 1000, 2048, 4096, 12288, _log_int(rng, 33, 12288)])
        N = rng.choice([4096, 4099, 12288, 32768, 126464, _log_int(rng, 256, 126464)])
        while N * K > 126464 * 4096:
            N = (N + 1) // 2
        top = min(8192, int(2048 * 126464 * 4096 / (N * K)), int(2 ** 28 // N))
        return dict(kind=kind, M=rng.choice([1, 16, _log_int(rng, 1, max(1, top))]), N=N, K=K,
                    fmt=rng.choice(["fp8", "fp4"]), out=rng.choice(["f32", "bf16"]))
    vocab = rng.choice([126464, 50257, 32768, 32000, 4099, 256, _log_int(rng, 256, 126464)])
    top = rng.choice([0, 1, 5, 8, 20, 64])
    return dict(kind=kind, rows=_log_int(rng, 1, min(65536, 2 ** 28 // vocab)), vocab=vocab, top=top,
                dtype=rng.choice(["f32", "f32", "bf16"]), masked=rng.choice([0.0, 0.1, 0.5]))


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _rows(gen, rows, cols, scale):
    """Activations: normal, with the uneven column sizes of a residual stream."""
    x = torch.randn(rows, cols, generator=gen, device="cuda")
    return x * (scale * torch.exp(torch.randn(cols, generator=gen, device="cuda")))


def _held(x, fmt):
    """Codes and scales of x [rows, cols] (fp32) as a program holds them."""
    rows, cols = x.shape
    groups = -(-cols // GROUP)
    per = 2 if fmt == "fp4" else 1
    codes = torch.empty(rows, groups * GROUP // per, dtype=torch.uint8, device=x.device)
    scales = torch.zeros(groups, rows + -rows % 32, 8, dtype=torch.uint8, device=x.device)
    for r in range(0, rows, 16384):
        part = torch.nn.functional.pad(x[r:r + 16384], (0, groups * GROUP - cols))
        v, s = _scaled(part, fmt)
        if fmt == "fp4":
            a = v.abs()
            code = torch.zeros_like(a, dtype=torch.uint8)
            for t, even in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False),
                            (3.5, True), (5.0, False)):
                code += ((a >= t) if even else (a > t)).to(torch.uint8)
            code += 8 * (v < 0).to(torch.uint8)
            codes[r:r + 16384] = code[:, 0::2] + 16 * code[:, 1::2]
        else:
            codes[r:r + 16384] = v.to(torch.float8_e4m3fn).view(torch.uint8)
        scales[:, r:r + len(part)] = s.view(-1, groups, 8).permute(1, 0, 2)
    return codes, scales


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    kind = case["kind"]
    st = dict(case)
    if kind == "quantize":
        st["x"] = _rows(gen, case["rows"], case["cols"], 1.0).to(TYPES[case["dtype"]])
    elif kind == "norm":
        st["x"] = _rows(gen, case["rows"], case["cols"], 2.0).to(TYPES[case["dtype"]])
        st["d"] = (_rows(gen, case["rows"], case["cols"], 0.5).to(TYPES[case["delta"]])
                   if case["delta"] else None)
        st["w"] = (1.0 + 0.1 * torch.randn(case["cols"], generator=gen, device="cuda")
                   if case["gain"] else None)
    elif kind == "matmul":
        a = torch.randn(case["M"], case["K"], generator=gen, device="cuda")
        st["a"] = _held(a, case["fmt"])
        b = torch.empty(case["N"], case["K"], device="cuda")
        b.uniform_(-0.25, 0.25, generator=gen)
        st["b"] = _held(b, "fp4")
    else:
        n, V = case["rows"], case["vocab"]
        lg = torch.empty(n, V, device="cuda", dtype=TYPES[case["dtype"]])
        for r in range(0, n, 4096):
            part = torch.randn(min(4096, n - r), V, generator=gen, device="cuda")
            part *= 1.0 + 5.0 * torch.rand(part.shape[0], 1, generator=gen, device="cuda")
            if case["masked"]:
                out = torch.rand(part.shape, generator=gen, device="cuda") < case["masked"]
                out[:, 0] = False
                part.masked_fill_(out, float("-inf"))
            lg[r:r + 4096] = part
        st["logits"] = lg
        # tokens a row gives some weight: one of a few drawn at random, the best
        pick = torch.randint(0, V, (n, 16), generator=gen, device="cuda")
        best = torch.gather(lg, 1, pick).argmax(1, keepdim=True)
        st["tokens"] = torch.gather(pick, 1, best)[:, 0].to(torch.int32)
    if own:
        st["m"] = _handle(case["vocab"] if kind == "scores" else 256)
    return st


def _handle(vocab):
    """The model that a program has open: the operators run on its GPU and stream."""
    import paper_2608_11249_amd as dl
    import workloads as wl
    sh = wl.ModelShape(name="handle", n_layers=0, d_model=128, n_heads=2, d_ffn=128, vocab=vocab,
                       ffn="gelu", norm="layernorm", dtype="bf16", head_exp=3)
    return dl.Model(sh, max_chunk=1, max_batch=1)


# --------------------------------------------------------------------------
# one pass
# --------------------------------------------------------------------------
def run(st):
    kind = st["kind"]
    if own:
        import paper_2608_11249_amd as dl
        m = st["m"]
        if kind == "quantize":
            return m.mx_dequantize(m.mx_quantize(st["x"], st["fmt"]))
        if kind == "norm":
            r, q = m.add_norm_mx(st["x"], st["d"], gain=st["w"], norm=st["norm"], eps=1e-5,
                                 fmt=st["fmt"])
            return r, m.mx_dequantize(q)
        if kind == "matmul":
            a = dl.MXMatrix(*st["a"], st["fmt"], st["M"], st["K"])
            b = dl.MXMatrix(*st["b"], "fp4", st["N"], st["K"])
            return m.mx_matmul(a, b, out_dtype=TYPES[st["out"]])
        return m.token_scores(st["logits"], st["tokens"], top=st["top"])
    if kind == "quantize":
        return _values(st["x"].float(), st["fmt"])
    if kind == "norm":
        return _norm(st)
    if kind == "matmul":
        a = _decode(*st["a"], st["fmt"], st["K"])
        b = _decode(*st["b"], "fp4", st["K"])
        return (a @ b.t()).to(TYPES[st["out"]])
    return _scores(st)


def _scaled(x, fmt):
    """x over its blocks' scales, and the scales' bytes [rows, blocks]; x [rows, 32 n]."""
    blocks = x.view(x.shape[0], -1, 32)
    # the least power of two that brings the largest value within the format's range
    top = blocks.abs().amax(2)
    frac, e = torch.frexp(top)
    fmax, emax = math.frexp(TOP_OF[fmt])
    e = e - emax + (frac > fmax).to(e.dtype)
    e = torch.where(top > 0, e, torch.full_like(e, -127)).clamp(-127, 127)
    v = torch.ldexp(blocks, -e.unsqueeze(2)).view(x.shape)
    return v, (e + 127).to(torch.uint8)


def _values(x, fmt):
    """The values that x [rows, cols] stands for once it is held in fmt."""
    cols = x.shape[1]
    v, s = _scaled(torch.nn.functional.pad(x, (0, -cols % 32)), fmt)
    if fmt == "fp8":
        r = v.to(torch.float8_e4m3fn).float()
    else:
        a = v.abs()
        # steps of 1/2 up to 2, of 1 up to 4, of 2 above; halves go to the even step
        r = torch.where(a < 2, torch.round(2 * a) / 2,
                        torch.where(a < 4, torch.round(a), 2 * torch.round(a / 2)))
        r = torch.copysign(r, v)
    r = torch.ldexp(r.view(x.shape[0], -1, 32), s.int().unsqueeze(2) - 127)
    return r.view(x.shape[0], -1)[:, :cols].to(torch.bfloat16)


def _norm(st):
    x, d = st["x"], st["d"]
    r = x.float() if d is None else (x.float() + d.float()).to(x.dtype).float()
    y = r
    if st["norm"] == "layernorm":
        y = y - y.mean(1, keepdim=True)
    y = y * torch.rsqrt((y * y).mean(1, keepdim=True) + 1e-5)
    if st["w"] is not None:
        y = y * st["w"]
    return r.to(x.dtype), _values(y, st["fmt"])


def _decode(codes, scales, fmt, cols):
    """The matrix [rows, cols] that codes and scales stand for, in fp32."""
    if fmt == "fp4":
        table = torch.tensor(E2M1, device=codes.device)
        v = torch.stack((table[(codes & 15).int()], table[(codes >> 4).int()]), 2)
    else:
        v = codes.view(torch.float8_e4m3fn).float()
    rows = codes.shape[0]
    s = scales[:, :rows].permute(1, 0, 2).reshape(rows, -1, 1).int() - 127
    return torch.ldexp(v.view(rows, -1, 32), s).view(rows, -1)[:, :cols].contiguous()


def _scores(st):
    lg, k = st["logits"].float(), st["top"]
    t = lg - lg.amax(1, keepdim=True)
    e = torch.exp(t)
    z = e.sum(1)
    log2z = torch.log2(z)
    h = log2z - (e * t.clamp_min(-1e30)).sum(1) / z / math.log(2.0)
    lp = torch.gather(t, 1, st["tokens"].long()[:, None])[:, 0] / math.log(2.0) - log2z
    # a stable sort leaves equal logits in the order of their ids
    ids = torch.sort(lg, dim=1, descending=True, stable=True)[1][:, :k]
    return lp, h, ids.int(), torch.gather(t, 1, ids) / math.log(2.0) - log2z[:, None]


# --------------------------------------------------------------------------
# what a pass cannot do without
# --------------------------------------------------------------------------
def _bytes(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    kind = case["kind"]
    if kind == "quantize":
        n = case["rows"] * case["cols"]
        return dict(bytes=n * (_bytes(case["dtype"]) + 2), flops=4 * n)
    if kind == "norm":
        n = case["rows"] * case["cols"]
        per = 2 * _bytes(case["dtype"]) + (_bytes(case["delta"]) if case["delta"] else 0) + 2
        return dict(bytes=n * per + (4 * case["cols"] if case["gain"] else 0), flops=9 * n)
    if kind == "matmul":
        M, N, K = case["M"], case["N"], case["K"]
        held = lambda rows, fmt: rows * (K // (2 if fmt == "fp4" else 1) + -(-K // 32))  # noqa: E731
        return dict(bytes=held(M, case["fmt"]) + held(N, "fp4") + M * N * _bytes(case["out"]),
                    flops=2 * M * N * K)
    n, V, k = case["rows"], case["vocab"], case["top"]
    return dict(bytes=n * V * _bytes(case["dtype"]) + n * (12 + 8 * k), flops=6 * n * V)


# --------------------------------------------------------------------------
# the definitions in 64 bits
# --------------------------------------------------------------------------
def _held64(x, fmt):
    """Nearest values of the format, block by block, of x [rows, cols] in 64 bits."""
    rows, cols = x.shape
    least, digits = (1.0, 2) if fmt == "fp4" else (2.0 ** -6, 4)
    out = torch.zeros_like(x)
    pad = -cols % 32
    x = torch.cat((x, x.new_zeros(rows, pad)), 1).view(rows, -1, 32)
    big = x.abs().max(2)[0]
    e = torch.ceil(torch.log2(big / TOP_OF[fmt]))
    # log2 is off by a rounding at most: put the border right
    e = torch.where(big > TOP_OF[fmt] * 2.0 ** e, e + 1, e)
    e = torch.where(big <= TOP_OF[fmt] * 2.0 ** (e - 1), e - 1, e)
    s = 2.0 ** e.clamp(-127, 127).nan_to_num(nan=-127.0, neginf=-127.0)
    u = x / s[:, :, None]
    # a value's step: its binade's, or the smallest normal binade's below that
    step = 2.0 ** (torch.floor(torch.log2(u.abs().clamp_min(least))) - (digits - 1))
    out = torch.round(u / step) * step * s[:, :, None]
    return out.view(rows, -1)[:, :cols]


def exact(case, seed):
    st = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        return _held64(st["x"].double(), case["fmt"])
    if kind == "norm":
        r = st["x"].double()
        if st["d"] is not None:
            r = (r + st["d"].double()).to(st["x"].dtype).double()
        c = r - r.sum(1, keepdim=True) / r.shape[1] if case["norm"] == "layernorm" else r
        y = c / torch.sqrt((c ** 2).sum(1, keepdim=True) / r.shape[1] + 1e-5)
        if st["w"] is not None:
            y = y * st["w"].double()
        return r, _held64(y, case["fmt"])
    if kind == "matmul":
        def of(held, fmt):
            codes, scales = held
            c = codes.to(torch.int16)
            if fmt == "fp4":
                c = torch.stack((c % 16, c // 16), 2).view(c.shape[0], -1)
                sign, ex, man, bias, digits = c // 8, c // 2 % 4, c % 2, 1, 1
            else:
                sign, ex, man, bias, digits = c // 128, c // 8 % 16, c % 8, 7, 3
            man = man.double() / 2 ** digits
            v = torch.where(ex == 0, man * 2.0 ** (1 - bias), (1 + man) * 2.0 ** (ex - bias).double())
            v = v * (1 - 2 * sign.double())
            s = scales[:, :len(c)].permute(1, 0, 2).reshape(len(c), -1)
            s = 2.0 ** (s.double() - 127)
            return (v.view(c.shape[0], -1, 32) * s[:, :, None]).view(c.shape[0], -1)[:, :case["K"]]
        a = of(st["a"], case["fmt"])
        codes, scales = st["b"]
        out = torch.empty(case["M"], case["N"], dtype=torch.float64, device=a.device)
        for n in range(0, case["N"], 8192):
            out[:, n:n + 8192] = a @ of((codes[n:n + 8192], scales[:, n:n + 8192]), "fp4").t()
        return out
    n, k = case["rows"], case["top"]
    lp, h, ids, tlp = [], [], [], []
    for r in range(0, n, 256):
        p = st["logits"][r:r + 256].double()
        logp = p - torch.logsumexp(p, 1, keepdim=True)
        lp.append(logp.gather(1, st["tokens"][r:r + 256].long()[:, None])[:, 0] / math.log(2.0))
        h.append(-torch.where(logp.isinf(), torch.zeros_like(logp), logp.exp() * logp).sum(1) / math.log(2.0))
        # the largest k, equal ones by their ids: all values above the k-th, then
        # the first of those equal to it
        if k:
            kth = torch.topk(p, k, 1)[0][:, -1:]
            rank = torch.where(p > kth, 2, torch.where(p == kth, 1, 0))
            first = (rank == 1).long().cumsum(1) <= (k - (rank == 2).sum(1, keepdim=True))
            keep = (rank == 2) | ((rank == 1) & first)
            id_ = keep.nonzero()[:, 1].view(-1, k)
            val = p.gather(1, id_)
            order = torch.argsort(val, dim=1, descending=True, stable=True)
            ids.append(id_.gather(1, order).int())
            tlp.append(logp.gather(1, id_).gather(1, order) / math.log(2.0))
        else:
            ids.append(torch.zeros(len(p), 0, dtype=torch.int32, device=p.device))
            tlp.append(torch.zeros(len(p), 0, dtype=torch.float64, device=p.device))
    return torch.cat(lp), torch.cat(h), torch.cat(ids), torch.cat(tlp)
