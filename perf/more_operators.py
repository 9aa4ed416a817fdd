"""Adapters on a shared quantized model, and what their answers and their training need, as timed cases: low-rank adapters of many
requests beside one projection with their gradients, log probabilities of given tokens with entropies and top alternatives and
the gradient of both, activations kept in 8 bits from the forward pass to the backward.

A case is a dict of plain values.  ``listed()`` names the ones that are always measured, ``draw(rng)`` gives more of the
same ranges; ``prepare`` makes what a program holds before the call, ``run`` is one pass: where ``own`` is false in plain
torch operations, else through the package's entry points.
"""
import math

import torch

own = False

TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2, "i8": 1}
VOCABULARY = 30522  # BERT's


def listed():
    return [
        # scores of one position: latency, over a vocabulary that does not fill a workgroup's share evenly
        dict(name="answers_one_position", kind="answers", M=1, V=VOCABULARY, x="f32", top=5, scale=1.0, bits=64, banned=False),
        # a corpus scored: every position of 8192 tokens, some of the vocabulary not to be answered with
        dict(name="answers_corpus", kind="answers", M=8192, V=VOCABULARY, x="f16", top=20, scale=1.0, bits=32, banned=True),
        # the masked positions of 32 sentences of 128 tokens, a step of fine-tuning
        dict(name="loss_masked_positions", kind="loss", M=614, V=VOCABULARY, x="f16", grad="f16", scale=1.0, bits=64, entropy=False),
        # every position of a batch of a model with a large vocabulary, with a weight on the entropy and a temperature
        dict(name="loss_every_position", kind="loss", M=2048, V=131072, x="bf16", grad="bf16", scale=0.7, bits=64, entropy=True),
        # a token each of 16 requests, no two with the same adapter: the smallest linears of a base model
        dict(name="adapt_tokens", kind="adapt", M=16, requests=16, R=16, rank=8, K=768, N=768, x="f16", w="f16", out="f16", base=True),
        # ragged prompts of requests that share 8 adapters through the FFN-up linear of a large model
        dict(name="adapt_prompts", kind="adapt", M=8192, requests=40, R=8, rank=16, K=1024, N=4096, x="bf16", w="bf16", out="bf16", base=True),
        # one adapter tuned on a few sentences by the 4-layer student, all in binary32
        dict(name="tune_student", kind="tune", M=437, requests=12, R=1, rank=4, K=312, N=1200, x="f32", group=0, dy="f32", w="f32", grad="f32"),
        # four adapters at once through the FFN-up linear of a large model, whose inputs were kept in 8 bits
        dict(name="tune_large", kind="tune", M=8192, requests=64, R=4, rank=16, K=1024, N=4096, x="i8", group=128, dy="bf16", w="bf16", grad="f32"),
        # hidden states of a padding-free batch of short sentences, kept and read back
        dict(name="keep_ragged_440", kind="keep", M=440, K=768, x="f16", group=64, out="f16", act="none"),
        # FFN activations of a large batch kept before the GELU, and made again behind it
        dict(name="keep_large", kind="keep", M=16384, K=4096, x="bf16", group=128, out="bf16", act="gelu"),
        # the GELU's backward pass of the student from 8 bits
        dict(name="gelu_student", kind="gelu", M=437, K=1200, group=32, dy="f32", dx="f32"),
        # ... of a large batch
        dict(name="gelu_large", kind="gelu", M=16384, K=4096, group=128, dy="bf16", dx="bf16"),
    ]


def _spread(rng, lo, hi):
    """An integer between lo and hi, uniform in its logarithm."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["answers", "answers", "loss", "adapt", "adapt", "tune", "tune", "keep", "gelu"])
    x = rng.choice(["f32", "f16", "bf16"])
    if kind in ("answers", "loss"):
        V = rng.choice([VOCABULARY, 131072, _spread(rng, 50, 200000)])
        M = _spread(rng, 1, min(8192, (1 << 27) // V))
        scale, bits = rng.choice([1.0, 1.0, 0.7, 1.3]), rng.choice([32, 64])
        if kind == "answers":
            return dict(kind=kind, M=M, V=V, x=x, top=rng.choice([0, 1, 5, 20, 50]), scale=scale, bits=bits, banned=rng.random() < 0.5)
        return dict(kind=kind, M=M, V=V, x=x, grad=rng.choice([x, x, "f32"]), scale=scale, bits=bits, entropy=rng.random() < 0.5)
    if kind in ("adapt", "tune"):
        K = rng.choice([312, 768, 1024, 4096, _spread(rng, 24, 4096)])
        N = rng.choice([312, 768, 1024, 4096, _spread(rng, 24, 4096)])
        M = _spread(rng, 1, 8192 if K + N <= 5120 else 4096)
        R = _spread(rng, 1, 32)
        c = dict(kind=kind, M=M, requests=_spread(rng, 1, M), R=R, rank=rng.choice([4, 8, 16, 16, 32, 64, rng.randint(1, 64)]) if M <= 2048 else rng.choice([4, 8, 16]),
                 K=K, N=N, x=x, w=rng.choice([x, x, "f32"]))
        if kind == "adapt":
            return dict(c, out=rng.choice([x, x, "f32"]), base=rng.random() < 0.7)
        group = rng.choice([0, 32, 64, 128])
        return dict(c, x="i8" if group else x, group=group, dy=x, grad=rng.choice(["f32", "f32", x]))
    K = rng.choice([312, 768, 1200, 4096, _spread(rng, 24, 8192)])
    M = _spread(rng, 1, min(16384, (1 << 26) // K))
    group = rng.choice([32, 64, 128])
    if kind == "keep":
        return dict(kind=kind, M=M, K=K, x=x, group=group, out=x, act=rng.choice(["none", "none", "gelu"]))
    return dict(kind=kind, M=M, K=K, group=group, dy=x, dx=rng.choice([x, x, "f32"]))


# ------------------------------------------------------------------------------------------------
def _cdiv(a, b):
    return -(-a // b)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _randn(g, shape, dtype, std=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * std).to(dtype)


def _logits(g, c):
    """Scores over a vocabulary: broad ones, and in half of the rows one token far ahead, as a model that has learned gives them;
    the given token is the one ahead in most of these rows."""
    M, V = c["M"], c["V"]
    z = torch.randn(M, V, generator=g, device="cuda").mul_(2.0)
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda")
    sure = torch.rand(M, generator=g, device="cuda") < 0.5
    ahead = torch.where(torch.rand(M, generator=g, device="cuda") < 0.8, tokens, torch.randint(0, V, (M,), generator=g, device="cuda"))
    z[torch.arange(M, device="cuda"), ahead] += torch.where(sure, 14.0, 0.0)
    if c.get("banned"):  # one token in a hundred, but not the given ones
        off = torch.rand(V, generator=g, device="cuda") < 0.01
        off[tokens] = False
        z[:, off] = -math.inf
    return z.to(TORCH[c["x"]]), tokens.to(torch.int64 if c["bits"] == 64 else torch.int32)


def _rows_of_requests(g, M, requests, R):
    """The adapter of every row: ragged requests one after the other, one in ten without an adapter (-1)."""
    cuts = torch.randperm(M - 1, generator=g, device="cuda")[:requests - 1].add_(1).sort().values if M > 1 else torch.zeros(0, dtype=torch.int64, device="cuda")
    request = torch.bucketize(torch.arange(M, device="cuda"), cuts, right=True)
    ids = torch.randperm(max(requests, R), generator=g, device="cuda")[:requests] % R
    ids = torch.where(torch.rand(requests, generator=g, device="cuda") < 0.1, -1, ids) if requests > 1 else ids
    return ids[request].to(torch.int32)


def _kept(x, group):
    """Rows in 8 bits as a program keeps them: codes in rows of ceil(K / 32) * 32 bytes, zeros past K, a step per group."""
    M, K = x.shape
    groups = _cdiv(K, group)
    padded = torch.zeros(M, groups * group, device=x.device)
    padded[:, :K] = x
    steps = padded.view(M, groups, group).abs().amax(-1) / 127
    steps = torch.where(steps > 0, steps, 1.0)
    codes = (padded.view(M, groups, group).double() / steps.double()[:, :, None]).round().to(torch.int8).view(M, -1)
    pitch = _cdiv(K, 32) * 32
    return codes[:, :pitch].contiguous(), steps


def prepare(case, seed):
    c, g = case, _gen(seed)
    st = dict(case=c)
    if c["kind"] in ("answers", "loss"):
        st["logits"], st["tokens"] = _logits(g, c)
        if c["kind"] == "loss":  # the mean over the rows, weighted as by rewards
            st["d_log_probs"] = -(torch.rand(c["M"], generator=g, device="cuda") + 0.5) / c["M"]
            st["d_entropies"] = torch.full((c["M"],), -0.01 / c["M"], device="cuda") if c["entropy"] else None
    elif c["kind"] in ("adapt", "tune"):
        M, K, N, R, rank = (c[k] for k in ("M", "K", "N", "R", "rank"))
        st["adapter"] = _rows_of_requests(g, M, c["requests"], R)
        st["down"] = _randn(g, (R, rank, K), TORCH[c["w"]], K ** -0.5)
        st["up"] = _randn(g, (R, rank, N), TORCH[c["w"]], 0.05)
        st["scales"] = torch.rand(R, generator=g, device="cuda") + 0.5
        x = _randn(g, (M, K), TORCH["f32" if c["x"] == "i8" else c["x"]])
        if c["kind"] == "adapt":
            st["x"] = x
            st["base"] = _randn(g, (M, N), TORCH[c["out"]]) if c["base"] else None
        else:
            st["dy"] = _randn(g, (M, N), TORCH[c["dy"]])
            st["hidden"] = _hidden(x.float(), st["down"], st["adapter"])
            st["x"], st["steps"] = _kept(x, c["group"]) if c["x"] == "i8" else (x, None)
    elif c["kind"] == "keep":
        st["x"] = _randn(g, (c["M"], c["K"]), TORCH[c["x"]])
    else:
        st["codes"], st["steps"] = _kept(_randn(g, (c["M"], c["K"]), torch.float32), c["group"])
        st["dy"] = _randn(g, (c["M"], c["K"]), TORCH[c["dy"]])
    return st


# ------------------------------------------------------------------------------------------------
def _own_rows(t, adapter, R):
    """[M, R, rank] products with all adapters -> those with a row's own, zeros in the place of the others."""
    mine = adapter.long()[:, None] == torch.arange(R, device=t.device)
    return torch.where(mine[:, :, None], t, 0.0)


def _hidden(x, down, adapter):
    """What a row's own adapter makes of it, [M, rank]: products with all adapters, its own chosen."""
    R, rank, K = down.shape
    t = (x @ down.float().view(R * rank, K).T).view(-1, R, rank)
    return _own_rows(t, adapter, R).sum(1)


def _spread_out(t, adapter, R):
    """[M, rank] -> [M, R * rank], a row's values in the place of its adapter."""
    return _own_rows(t[:, None, :].expand(-1, R, -1), adapter, R).flatten(1)


def _restored(codes, steps, K, group):
    return codes[:, :K].float() * steps.repeat_interleave(group, dim=1)[:, :K]


def _gelu(x):
    return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))


def _log_softmax(c, st):
    """Scaled scores relative to their largest, the logarithm of the sum of their exponentials, probabilities, entropy."""
    z = st["logits"].float() * c["scale"]
    z = z - z.amax(1, keepdim=True)
    e = z.exp()
    total = e.sum(1)
    log_total = total.log()
    p = e / total[:, None]
    entropy = log_total - torch.where(e > 0, p * z, 0.0).sum(1)
    return z, log_total, p, entropy


def _plain(c, st):
    if c["kind"] in ("answers", "loss"):
        z, log_total, p, entropy = _log_softmax(c, st)
        tokens = st["tokens"].long()[:, None]
        log_probs = z.gather(1, tokens)[:, 0] - log_total
        if c["kind"] == "answers":
            # whole numbers in the order of the scores, the lowest token first among equal ones
            at = torch.arange(c["V"], device=z.device)
            bits = (st["logits"].float() + 0.0).view(torch.int32)
            order = ((bits ^ ((bits >> 31) & 0x7FFFFFFF)).long() << 32) | (c["V"] - 1 - at)
            top = c["V"] - 1 - (order.topk(c["top"], dim=1).values & 0xFFFFFFFF)
            return [log_probs, entropy, top.to(torch.int32), z.gather(1, top) - log_total[:, None]]
        grad = -p * st["d_log_probs"][:, None]
        grad.scatter_add_(1, tokens, st["d_log_probs"][:, None])
        if c["entropy"]:
            log_p = torch.where(p > 0, z - log_total[:, None], 0.0)
            grad -= st["d_entropies"][:, None] * p * (log_p + entropy[:, None])
        return [log_probs, entropy, (grad * c["scale"]).to(TORCH[c["grad"]])]
    if c["kind"] in ("adapt", "tune"):
        R, rank = c["R"], c["rank"]
        down, up = st["down"].float().view(R * rank, c["K"]), st["up"].float().view(R * rank, c["N"])
        scale = torch.where(st["adapter"] >= 0, st["scales"][st["adapter"].clamp(min=0).long()], 0.0)[:, None]
        if c["kind"] == "adapt":
            t = _hidden(st["x"].float(), st["down"], st["adapter"])
            y = _spread_out(t * scale, st["adapter"], R) @ up
            return (y + st["base"].float() if c["base"] else y).to(TORCH[c["out"]])
        x = _restored(st["x"], st["steps"], c["K"], c["group"]) if c["x"] == "i8" else st["x"].float()
        dy = st["dy"].float()
        u = _spread_out(_hidden(dy, st["up"], st["adapter"]) * scale, st["adapter"], R)
        t = _spread_out(st["hidden"] * scale, st["adapter"], R)
        grad = TORCH[c["grad"]]
        return [(u @ down).to(TORCH[c["dy"]]), (u.T @ x).view(R, rank, -1).to(grad), (t.T @ dy).view(R, rank, -1).to(grad)]
    if c["kind"] == "keep":
        codes, steps = _kept(st["x"].float(), c["group"])
        x = _restored(codes, steps, c["K"], c["group"])
        return [steps, (_gelu(x) if c["act"] == "gelu" else x).to(TORCH[c["out"]])]
    x = _restored(st["codes"], st["steps"], c["K"], c["group"])
    slope = 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))
    return (st["dy"].float() * slope).to(TORCH[c["dx"]])


def run(state):
    c, st = state["case"], state
    if not own:
        return _plain(c, st)
    import paper_2203_13483_amd as mkq

    code = {"f32": mkq.MKQ_F32, "f16": mkq.MKQ_F16, "bf16": mkq.MKQ_BF16}
    act = {"none": mkq.MKQ_ACT_NONE, "gelu": mkq.MKQ_ACT_GELU}
    if c["kind"] == "answers":
        a = mkq.mkq_token_log_probs(st["logits"], st["tokens"], c["scale"], c["top"])
        return [a.log_probs, a.entropies, a.top_tokens, a.top_log_probs]
    if c["kind"] == "loss":
        a = mkq.mkq_token_log_probs(st["logits"], st["tokens"], c["scale"])
        grad = mkq.mkq_token_log_probs_gradient(st["logits"], st["tokens"], a, st["d_log_probs"], c["scale"], code[c["grad"]],
                                                d_entropies=st["d_entropies"])
        return [a.log_probs, a.entropies, grad]
    if c["kind"] == "adapt":
        return mkq.mkq_low_rank_adapters(st["x"], st["adapter"], st["down"], st["up"], st["scales"], code[c["out"]], base=st["base"])
    if c["kind"] == "tune":
        return list(mkq.mkq_low_rank_adapters_gradient(st["dy"], st["x"], st["adapter"], st["hidden"], st["down"], st["up"], st["scales"],
                                                       code[c["dy"]], code[c["grad"]], steps=st["steps"], group=c["group"]))
    if c["kind"] == "keep":
        codes, steps = mkq.mkq_checkpoint_int8(st["x"], c["group"])
        return [steps, mkq.mkq_checkpoint_restore(codes, steps, c["K"], c["group"], code[c["out"]], act=act[c["act"]])]
    return mkq.mkq_checkpoint_gelu_gradient(st["codes"], st["steps"], st["dy"], c["group"], code[c["dx"]])


# ------------------------------------------------------------------------------------------------
def work(case):
    c, M = case, case["M"]
    if c["kind"] in ("answers", "loss"):
        rows = M * c["V"]
        if c["kind"] == "answers":
            return {"bytes": rows * BYTES[c["x"]] + M * (c["bits"] // 8 + 8 + 8 * c["top"]), "flops": 4 * rows}
        return {"bytes": rows * (BYTES[c["x"]] + BYTES[c["grad"]]) + M * (c["bits"] // 8 + 16), "flops": 8 * rows}
    if c["kind"] in ("adapt", "tune"):
        K, N, rank = c["K"], c["N"], c["rank"]
        weights = min(c["R"], c["requests"]) * rank * (K + N)
        if c["kind"] == "adapt":
            rows = M * (K * BYTES[c["x"]] + N * BYTES[c["out"]] * (2 if c["base"] else 1) + 4)
            return {"bytes": rows + weights * BYTES[c["w"]], "flops": 2 * M * rank * (K + N)}
        rows = M * ((N + K) * BYTES[c["dy"]] + K * BYTES[c["x"]] + 4 * rank + 4) + (4 * M * _cdiv(K, c["group"]) if c["group"] else 0)
        return {"bytes": rows + weights * BYTES[c["w"]] + c["R"] * rank * (K + N) * BYTES[c["grad"]], "flops": 4 * M * rank * (K + N)}
    K = c["K"]
    kept = M * (_cdiv(K, 32) * 32 + 4 * _cdiv(K, c["group"]))
    if c["kind"] == "keep":  # written, and read in the backward pass
        return {"bytes": M * K * (BYTES[c["x"]] + BYTES[c["out"]]) + 2 * kept, "flops": 4 * M * K}
    return {"bytes": kept + M * K * (BYTES[c["dy"]] + BYTES[c["dx"]]), "flops": 12 * M * K}


# ------------------------------------------------------------------------------------------------
def exact(case, seed):
    """What run() returns, in 64 bits."""
    c, st = case, prepare(case, seed)
    f64 = torch.float64
    if c["kind"] in ("answers", "loss"):
        outs = []
        for r in range(0, c["M"], 512):  # a few rows at a time
            raw = st["logits"][r:r + 512]
            z = raw.to(f64) * c["scale"]
            log_p = z - torch.logsumexp(z, 1, keepdim=True)
            p, at = log_p.exp(), st["tokens"][r:r + 512].long().unsqueeze(1)
            entropy = -torch.special.xlogy(p, p).sum(1)
            out = [log_p.gather(1, at).squeeze(1), entropy]
            if c["kind"] == "answers":
                top = torch.sort(raw.float(), dim=1, descending=True, stable=True).indices[:, :c["top"]]
                out += [top.to(torch.int32), log_p.gather(1, top)]
            else:
                g = st["d_log_probs"][r:r + 512].to(f64).unsqueeze(1)
                one = torch.zeros_like(p).scatter_(1, at, 1.0)
                d = g * (one - p)
                if c["entropy"]:
                    h = st["d_entropies"][r:r + 512].to(f64).unsqueeze(1)
                    d = d - h * (torch.special.xlogy(p, p) + p * entropy.unsqueeze(1))
                out.append(d * c["scale"])
            outs.append(out)
        return [torch.cat(parts) for parts in zip(*outs)]
    if c["kind"] in ("adapt", "tune"):
        M, K, N = c["M"], c["K"], c["N"]
        if c["kind"] == "adapt":
            y = st["base"].to(f64) if c["base"] else torch.zeros(M, N, dtype=f64, device="cuda")
        else:
            dx = torch.zeros(M, K, dtype=f64, device="cuda")
            d_down, d_up = (torch.zeros(c["R"], c["rank"], n, dtype=f64, device="cuda") for n in (K, N))
        for a in range(c["R"]):
            rows = torch.nonzero(st["adapter"] == a).flatten()
            A, B, s = st["down"][a].to(f64), st["up"][a].to(f64), float(st["scales"][a])
            x = st["x"][rows]
            if c["kind"] == "adapt":
                y[rows] += s * torch.mm(torch.mm(x.to(f64), A.T.contiguous()), B)
                continue
            if c["x"] == "i8":
                at = torch.arange(K, device="cuda")
                x = x[:, :K].to(f64) * st["steps"][rows].to(f64)[:, at // c["group"]]
            dy, t = st["dy"][rows].to(f64), st["hidden"][rows].to(f64)
            u = s * torch.mm(dy, B.T.contiguous())
            dx[rows] = torch.mm(u, A)
            d_down[a] = torch.mm(u.T.contiguous(), x.to(f64))
            d_up[a] = s * torch.mm(t.T.contiguous(), dy)
        return y if c["kind"] == "adapt" else [dx, d_down, d_up]
    K, group, at = c["K"], c["group"], torch.arange(c["K"], device="cuda")
    if c["kind"] == "keep":
        # the step is a number of 32 bits and the code is decided from it exactly
        x = st["x"].to(f64)
        largest = torch.stack([x[:, k:k + group].abs().amax(1) for k in range(0, K, group)], 1)
        steps = (largest / 127).to(torch.float32).to(f64)
        steps = torch.where(steps > 0, steps, torch.ones_like(steps))[:, at // group]
        x = torch.round(x / steps) * steps
        return [torch.where(largest > 0, largest / 127, 1.0), x * torch.special.ndtr(x) if c["act"] == "gelu" else x]
    x = st["codes"][:, :K].to(f64) * st["steps"].to(f64)[:, at // group]
    return st["dy"].to(f64) * (torch.special.ndtr(x) + x * torch.exp(-x * x / 2) / math.sqrt(2 * math.pi))
