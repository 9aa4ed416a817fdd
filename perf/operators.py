"""The two ends of a quantized encoder, and the training of its token table, as timed cases: products of few tokens with
4-bit weights that have a step per group (the head over the vocabulary, single linears), the lookup of token rows from a
float table and from the same 4-bit table, the table's gradient by sorted tokens, and the gradient norm with clipping over
the tensors of a model.

A case is a dict of plain values.  ``listed()`` names the ones that are always measured, ``draw(rng)`` gives more of the
same ranges; ``prepare`` makes what a program holds before the call, ``run`` is one pass: where ``own`` is false in plain
torch operations, else through the package's entry points.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
VOCABULARY = 30522  # BERT's


def listed():
    return [
        # one sentence through the FFN-up linear of the 4-layer student: the smallest products, K no multiple of a group
        dict(name="linear_student_sentence", kind="linear", M=37, K=312, N=1200, group=32, x="f32", out="f32", act="gelu"),
        # scores over the vocabulary for one position: latency, and a stream of 12 MB
        dict(name="head_one_token", kind="linear", M=1, K=768, N=VOCABULARY, group=64, x="f16", out="f32", act="none"),
        # scores for the masked positions of a few sentences
        dict(name="head_masked_positions", kind="linear", M=120, K=1024, N=VOCABULARY, group=128, x="f16", out="f16", act="none"),
        # a few tokens against weights of a hundred megabytes
        dict(name="linear_few_rows_large", kind="linear", M=16, K=8192, N=28672, group=128, x="bf16", out="bf16", act="none"),
        # a padding-free batch of short sentences enters the encoder: binary32 table, binary16 hidden states
        dict(name="lookup_ragged_440", kind="lookup", M=440, V=VOCABULARY, D=768, table="f32", out="f16", bits=64, scaled=False),
        # offline scoring of long documents
        dict(name="lookup_large", kind="lookup", M=65536, V=VOCABULARY, D=1024, table="f16", out="f16", bits=32, scaled=True),
        # one sentence from the student's 4-bit table
        dict(name="lookup4_sentence", kind="lookup4", M=128, V=VOCABULARY, D=312, group=32, out="f32", bits=32, scaled=False),
        # a large padded batch from the 4-bit table
        dict(name="lookup4_large", kind="lookup4", M=32768, V=VOCABULARY, D=768, group=64, out="f16", bits=64, scaled=True),
        # the table's gradient of a usual training batch of 32 x 128 tokens
        dict(name="gradient_base", kind="gradient", M=4096, V=VOCABULARY, D=768, dy="f16", grad="f32", bits=64, padded=True, scaled=False),
        # ... of 128 x 512 tokens of a large model, no padding: the most frequent token has a twentieth of the rows
        dict(name="gradient_large", kind="gradient", M=65536, V=VOCABULARY, D=1024, dy="bf16", grad="f32", bits=64, padded=False, scaled=True),
        # all gradients of the 4-layer student, clipped
        dict(name="clip_student", kind="clip", layers=4, hidden=312, ffn=1200, V=VOCABULARY, grad="f32", clipped=True),
        # those of four layers and the table of a large model
        dict(name="clip_large", kind="clip", layers=4, hidden=1024, ffn=4096, V=VOCABULARY, grad="f32", clipped=True),
    ]


def _spread(rng, lo, hi):
    """An integer between lo and hi, uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["linear", "linear", "lookup", "lookup4", "gradient", "gradient", "clip"])
    if kind == "linear":
        K = rng.choice([312, 768, 1024, 1200, 4096, 8192, _spread(rng, 32, 8192)])
        N = rng.choice([312, 768, 1024, 4096, VOCABULARY, _spread(rng, 16, 28672), _spread(rng, 16, 28672)])
        M = _spread(rng, 1, 128 if K * N <= 1 << 25 else 16)
        x = rng.choice(["f32", "f16", "f16", "bf16"])
        return dict(kind=kind, M=M, K=K, N=N, group=rng.choice([32, 64, 128]), x=x, out=rng.choice([x, "f32"]),
                    act=rng.choice(["none", "none", "gelu"]))
    if kind == "clip":
        hidden, ffn = rng.choice([(312, 1200), (768, 2048), (1024, 4096), (_spread(rng, 16, 768), _spread(rng, 16, 2048))])
        return dict(kind=kind, layers=rng.randint(1, 4), hidden=hidden, ffn=ffn, V=_spread(rng, 32, VOCABULARY),
                    grad=rng.choice(["f32", "f16", "bf16"]), clipped=rng.random() < 0.75)
    D = rng.choice([312, 768, 1024, _spread(rng, 32, 1024), _spread(rng, 32, 1024)])
    V = rng.choice([VOCABULARY, _spread(rng, 100, VOCABULARY)])
    bits, scaled = rng.choice([32, 64]), rng.random() < 0.5
    out = rng.choice(["f32", "f16", "bf16"])
    if kind == "lookup":
        return dict(kind=kind, M=_spread(rng, 1, 32768), V=V, D=D, table=rng.choice(["f32", "f16", "bf16"]), out=out, bits=bits, scaled=scaled)
    if kind == "lookup4":
        return dict(kind=kind, M=_spread(rng, 1, 32768), V=V, D=D, group=rng.choice([32, 64, 128]), out=out, bits=bits, scaled=scaled)
    return dict(kind=kind, M=_spread(rng, 1, 65536), V=V, D=D, dy=out, grad=rng.choice(["f32", "f32", out]), bits=bits,
                padded=rng.random() < 0.5, scaled=scaled)


# ------------------------------------------------------------------------------------------------
def _cdiv(a, b):
    return -(-a // b)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _packed(g, rows, K, group):
    """Group-scaled 4-bit rows as a program holds them: nibbles, element 2i low, rows of ceil(K / 32) * 16 bytes with zero
    codes past K, and a step per group.  Codes as weights of a Gaussian have them."""
    codes = torch.zeros(rows, _cdiv(K, 32) * 32, dtype=torch.uint8, device="cuda")
    codes[:, :K] = torch.randn(rows, K, generator=g, device="cuda").mul_(2.6).round_().clamp_(-8, 7).to(torch.int8).view(torch.uint8) & 15
    Wq = codes[:, 0::2] | (codes[:, 1::2] << 4)
    s_w = torch.rand(rows, _cdiv(K, group), generator=g, device="cuda") * 0.006 + 0.004
    return Wq.contiguous(), s_w


def _tokens(g, M, V, bits):
    """Token ids with the frequencies of a text: the r-th most frequent about 1 / r as often as the first."""
    t = torch.rand(M, generator=g, device="cuda", dtype=torch.float64).mul_(math.log(V)).exp_().long().sub_(1).clamp_(0, V - 1)
    order = torch.randperm(V, generator=g, device="cuda")
    return order[t].to(torch.int64 if bits == 64 else torch.int32)


def _tensors_of_model(c):
    """Shapes of the parameters of c["layers"] encoder layers, the table and the head's bias."""
    h, f = c["hidden"], c["ffn"]
    layer = [(3 * h, h), (3 * h,), (h, h), (h,), (f, h), (f,), (h, f), (h,), (h,), (h,), (h,), (h,)]
    return [(c["V"], h), (c["V"],)] + c["layers"] * layer


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = dict(case=c)
    if c["kind"] == "linear":
        st["Wq"], st["s_w"] = _packed(g, c["N"], c["K"], c["group"])
        st["x"] = _randn(g, (c["M"], c["K"]), TORCH[c["x"]])
        st["bias"] = _randn(g, c["N"], torch.float32, 0.1)
    elif c["kind"] in ("lookup", "lookup4"):
        st["tokens"] = _tokens(g, c["M"], c["V"], c["bits"])
        st["scale"] = math.sqrt(c["D"]) if c["scaled"] else 1.0
        if c["kind"] == "lookup":
            st["table"] = _randn(g, (c["V"], c["D"]), TORCH[c["table"]], 0.02)
        else:
            st["Wq"], st["s_w"] = _packed(g, c["V"], c["D"], c["group"])
    elif c["kind"] == "gradient":
        st["tokens"] = _tokens(g, c["M"], c["V"], c["bits"])
        st["padding"] = -1
        if c["padded"]:  # a third of the places lies behind a sentence's end
            st["padding"] = 0
            st["tokens"][torch.rand(c["M"], generator=g, device="cuda") < 1 / 3] = 0
        st["scale"] = math.sqrt(c["D"]) if c["scaled"] else 1.0
        st["dy"] = _randn(g, (c["M"], c["D"]), TORCH[c["dy"]])
    else:
        shapes = _tensors_of_model(c)
        st["grads"] = [_randn(g, s, TORCH[c["grad"]], 0.01) for s in shapes]
        st["outs"] = [torch.empty_like(t) for t in st["grads"]]
        norm = 0.01 * math.sqrt(sum(math.prod(s) for s in shapes))
        st["max_norm"] = norm * (0.3 if c["clipped"] else 3.0)
    return st


# ------------------------------------------------------------------------------------------------
def _unpack(Wq, K):
    """Codes of rows of nibbles, binary32."""
    codes = torch.stack((Wq & 15, Wq >> 4), dim=-1).flatten(1)[:, :K]
    return ((codes ^ 8).to(torch.int8) - 8).float()


def _unpack_scaled(Wq, s_w, K, group):
    return _unpack(Wq, K) * s_w.repeat_interleave(group, dim=1)[:, :K]


def _plain(c, st):
    if c["kind"] == "linear":
        y = st["x"].float() @ _unpack_scaled(st["Wq"], st["s_w"], c["K"], c["group"]).T + st["bias"]
        if c["act"] == "gelu":
            y = 0.5 * y * (1.0 + torch.erf(y * math.sqrt(0.5)))
        return y.to(TORCH[c["out"]])
    if c["kind"] == "clip":
        norm = torch.stack([t.float().square().sum(dtype=torch.float64) for t in st["grads"]]).sum().sqrt()
        coef = (st["max_norm"] / (norm + 1e-6)).clamp(max=1.0).float()
        return [norm.float().reshape(1)] + [(t.float() * coef).to(t.dtype) for t in st["grads"]]
    t = st["tokens"].long()
    valid = (t >= 0) & (t < c["V"])
    if c["kind"] == "gradient":
        valid &= t != st["padding"]
        total = torch.zeros(c["V"] + 1, c["D"], device=t.device)
        total.index_add_(0, torch.where(valid, t, c["V"]), st["dy"].float())
        return (total[:c["V"]] * st["scale"]).to(TORCH[c["grad"]])
    t = torch.where(valid, t, 0)
    rows = st["table"][t].float() if c["kind"] == "lookup" else _unpack_scaled(st["Wq"][t], st["s_w"][t], c["D"], c["group"])
    return torch.where(valid[:, None], rows * st["scale"], 0.0).to(TORCH[c["out"]])


def run(state):
    c, st = state["case"], state
    if not own:
        return _plain(c, st)
    import paper_2203_13483_amd as mkq
    code = {"f32": mkq.MKQ_F32, "f16": mkq.MKQ_F16, "bf16": mkq.MKQ_BF16}
    if c["kind"] == "linear":
        return mkq.mkq_linear_int4_group(st["x"], st["Wq"], st["s_w"], st["bias"], c["N"], c["K"], c["group"], code[c["out"]],
                                         act=mkq.MKQ_ACT_GELU if c["act"] == "gelu" else mkq.MKQ_ACT_NONE)
    if c["kind"] == "lookup":
        return mkq.mkq_embedding(st["tokens"], st["table"], st["scale"], code[c["out"]])
    if c["kind"] == "lookup4":
        return mkq.mkq_embedding_int4_group(st["tokens"], st["Wq"], st["s_w"], c["V"], c["D"], c["group"], st["scale"], code[c["out"]])
    if c["kind"] == "gradient":
        return mkq.mkq_embedding_gradient(st["tokens"], st["dy"], c["V"], st["scale"], code[c["grad"]], padding_token=st["padding"])
    return [mkq.mkq_clip_gradients(st["grads"], st["max_norm"], outs=st["outs"])] + st["outs"]


def work(case):
    c = case
    if c["kind"] == "linear":
        M, K, N = c["M"], c["K"], c["N"]
        moved = N * (_cdiv(K, 32) * 16 + 4 * _cdiv(K, c["group"]) + 4) + M * K * BYTES[c["x"]] + M * N * BYTES[c["out"]]
        return {"bytes": moved, "flops": 2 * M * K * N}
    if c["kind"] == "clip":
        n = sum(math.prod(s) for s in _tensors_of_model(c))
        return {"bytes": 3 * n * BYTES[c["grad"]], "flops": 3 * n}  # the norm needs every value before the first is scaled
    M, D = c["M"], c["D"]
    if c["kind"] == "gradient":
        return {"bytes": M * c["bits"] // 8 + M * D * BYTES[c["dy"]] + c["V"] * D * BYTES[c["grad"]], "flops": M * D}
    # distinct rows among the tokens, by their frequencies: the table's rows are read once
    H = math.log(c["V"])
    distinct = sum(1 - (1 - math.log1p(1 / (r + 1)) / H) ** M for r in range(c["V"] - 1))
    row = D * BYTES[c["table"]] if c["kind"] == "lookup" else _cdiv(D, 32) * 16 + 4 * _cdiv(D, c["group"])
    return {"bytes": M * c["bits"] // 8 + int(distinct * row) + M * D * BYTES[c["out"]], "flops": M * D}


# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    """What run() returns, in 64 bits."""
    c, st = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] in ("linear", "lookup4"):
        K = c["K"] if c["kind"] == "linear" else c["D"]
        at = torch.arange(K, device="cuda")

        def values(rows):  # the values that some packed rows stand for
            code = (st["Wq"][rows][:, at // 2].int() >> (4 * (at % 2))) % 16
            return torch.where(code < 8, code, code - 16).to(f64) * st["s_w"][rows][:, at // c["group"]].to(f64)

    if c["kind"] == "linear":
        out = torch.empty(c["M"], c["N"], dtype=f64, device="cuda")
        x = st["x"].to(f64)
        for n in range(0, c["N"], 4096):
            rows = torch.arange(n, min(c["N"], n + 4096), device="cuda")
            out[:, rows] = torch.mm(x, values(rows).T.contiguous()) + st["bias"][rows].to(f64)
        if c["act"] == "gelu":
            out = out * torch.special.ndtr(out)
        return out
    if c["kind"] == "clip":
        norm = math.sqrt(math.fsum(float(torch.dot(t.flatten().to(f64), t.flatten().to(f64))) for t in st["grads"]))
        coef = min(1.0, st["max_norm"] / (norm + 1e-6))
        return [torch.tensor([norm], dtype=f64)] + [t.to(f64) * coef for t in st["grads"]]
    tokens = st["tokens"].long()
    if c["kind"] == "gradient":
        out = torch.zeros(c["V"], c["D"], dtype=f64, device="cuda")
        kept = torch.nonzero(tokens != st["padding"]).flatten()
        for part in kept.split(8192):
            out.index_put_((tokens[part],), st["dy"][part].to(f64) * st["scale"], accumulate=True)
        return out
    out = torch.empty(c["M"], c["D"], dtype=f64, device="cuda")
    for i in range(0, c["M"], 8192):
        t = tokens[i:i + 8192]
        out[i:i + 8192] = st["scale"] * (st["table"][t].to(f64) if c["kind"] == "lookup" else values(t))
    return out
