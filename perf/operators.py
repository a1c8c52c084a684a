"""The operators beside the watermark, as a decode step and a training step call them.

``head_logits``         next-token logits from hidden states by a head with 4-bit weights
``top_candidates``      the k largest logits of every row, in order
``token_logprobs``      log probabilities of given tokens, log sum, entropy, top alternatives
``token_logprobs_grad`` the gradient of those with respect to the logits

Each case is a dict of plain values.  The cases on logits have ``B`` rows of ``V`` tokens;
the head has ``V`` rows of ``K`` 4-bit weights, with one scale for every ``group`` of them.
"""
from __future__ import annotations

import math

import torch

own = False   # whether run() calls the framework's operators; else their plain form

INV_TEMPERATURE = 1.0 / 0.8


def _logprobs(name, B, V, dtype, n=1, top=0, masked=False):
    return dict(name=name, op="logprobs", B=B, V=V, dtype=dtype, n=n, top=top, masked=masked)


def _grad(name, B, V, dtype, n=1, entropy=False):
    return dict(name=name, op="grad", B=B, V=V, dtype=dtype, n=n, entropy=entropy)


def _top(name, B, V, dtype, k):
    return dict(name=name, op="top", B=B, V=V, dtype=dtype, k=k)


def _head(name, B, V, K, group, scales, dtype):
    return dict(name=name, op="head", B=B, V=V, K=K, group=group, scales=scales, dtype=dtype)


def listed():
    return [
        # One interactive request that asks for its token's log probability and five others.
        _logprobs("logprob_one_request", 1, 32000, "f32", top=5),
        # A serving batch whose requests ask for the 20 alternatives.
        _logprobs("logprob_batch64_bf16", 64, 128256, "bf16", top=20),
        # Scoring a prompt's 512 positions (perplexity, entropy): the largest pass over logits.
        _logprobs("logprob_prompt512", 512, 152064, "f32"),
        # Constrained decoding on an odd vocabulary: most tokens masked, four choices compared.
        _logprobs("logprob_masked_choices", 48, 128259, "f32", n=4, top=8, masked=True),
        # Loss gradient of a micro-batch in fp32.
        _grad("grad_f32", 256, 152064, "f32"),
        # Policy gradient with an entropy term over 1024 positions of bf16 logits.
        _grad("grad_entropy_bf16", 1024, 128256, "bf16", entropy=True),
        # A teacher's 32 most likely tokens per position, odd vocabulary.
        _grad("grad_teacher32", 33, 32001, "f32", n=32),
        # Candidates of one request.
        _top("top50_one_request", 1, 32000, "f32", 50),
        # The top-40 scheme's candidates of a large batch.
        _top("top40_batch256_bf16", 256, 152064, "bf16", 40),
        # As many candidates as the candidate watermark takes.
        _top("top1024", 16, 151936, "f32", 1024),
        # One request through the head of a small model.
        _head("head_one_request", 1, 32000, 2048, 128, "bf16", "f32"),
        # A decode batch through the head of a large vocabulary.
        _head("head_batch16", 16, 128256, 4096, 64, "f32", "bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["logprobs", "grad", "top", "head"])
    dtype = rng.choice(["f32", "bf16"])
    V = _log_uniform(rng, 16000, 152064)
    if rng.random() < 0.5:
        V -= V % 64                                        # a padded vocabulary
    if op == "logprobs":
        B = max(1, min(_log_uniform(rng, 1, 512), 512 * 152064 // V))
        n = rng.choice([1, 1, 1, 2, 4, 16])
        top = rng.choice([0, 0, 1, 5, 10, 20, 50])
        if top:
            B = min(B, 256)
        c = _logprobs("", B, V, dtype, n, top, rng.random() < 0.25)
    elif op == "grad":
        B = max(1, min(_log_uniform(rng, 1, 1024), (250 if dtype == "f32" else 860) * 152064 // V))
        c = _grad("", B, V, dtype, rng.choice([1, 1, 1, 8, 32, 64]), rng.random() < 0.5)
    elif op == "top":
        B = max(1, min(_log_uniform(rng, 1, 256), 256 * 152064 // V))
        c = _top("", B, V, dtype, _log_uniform(rng, 1, 1024))
    else:
        K = 128 * _log_uniform(rng, 8, 64)                 # hidden sizes of 1024 to 8192
        V = min(V, 128256 * 4096 // K)
        c = _head("", rng.choice([1, 1, 2, 3, 4, 8, 11, 16]), V, K, rng.choice([32, 64, 128]),
                  rng.choice(["f32", "bf16"]), dtype)
    del c["name"]
    return c


# --- inputs -----------------------------------------------------------------------------

_TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    B, V, dtype = case["B"], case["V"], _TYPES[case["dtype"]]

    if case["op"] == "head":
        K, groups = case["K"], case["K"] // case["group"]
        # two weights a byte; scales such that a unit hidden state gives logits of a few units
        codes = torch.randint(0, 256, (V, K // 2), generator=g, device="cuda", dtype=torch.uint8)
        scales = torch.empty((V, groups), device="cuda").uniform_(0.5, 1.5, generator=g)
        scales = (scales * (0.65 / math.sqrt(K))).to(_TYPES[case["scales"]])
        hidden = torch.empty((B, K), device="cuda").normal_(generator=g).to(torch.bfloat16)
        return dict(case=case, codes=codes, scales=scales, hidden=hidden)

    # a broad spread with a twentieth of the vocabulary raised, as next-token logits have
    logits = torch.empty((B, V), device="cuda").normal_(0.0, 3.0, generator=g)
    logits.add_(torch.empty((B, V), device="cuda").uniform_(generator=g) < 0.05, alpha=8.0)
    if case.get("masked"):
        # nine tokens of ten are barred; rows say so by -inf or by the type's lowest value, and
        # one row in sixteen has nothing left
        barred = torch.empty((B, V), device="cuda").uniform_(generator=g) < 0.9
        row = torch.arange(B, device="cuda")
        barred |= (row % 16 == 15)[:, None]
        lowest = torch.where(row % 4 == 1, torch.finfo(dtype).min, -math.inf)
        logits = torch.where(barred, lowest[:, None], logits)
    logits = logits.to(dtype)
    state = dict(case=case, logits=logits)
    if case["op"] == "top":
        return state

    # the tokens: a drawn one, then any others, a few of them padding
    n = case["n"]
    tokens = torch.randint(0, V, (B, n), generator=g, device="cuda")
    uniform = torch.empty((B, V), device="cuda").uniform_(1e-12, 1.0, generator=g)
    noise = uniform.log_().neg_().log_().neg_()
    tokens[:, 0] = noise.add_(logits, alpha=INV_TEMPERATURE).argmax(dim=1)
    del uniform, noise
    padding = torch.empty((B, n), device="cuda").uniform_(generator=g) < 0.03
    tokens = tokens.masked_fill(padding, -100).to(torch.int32)
    state["tokens"] = tokens[:, 0].contiguous() if n == 1 else tokens
    if case["op"] == "grad":
        # what the forward pass left: each row's largest logit and log sum relative to it
        _, lse, entropy = _row_statistics(logits)
        highest = logits.float().amax(dim=1)
        state["stats"] = torch.stack([highest, lse - highest * INV_TEMPERATURE], dim=1)
        state["entropy"] = entropy
        state["grad_logprobs"] = torch.empty_like(state["tokens"], dtype=torch.float32).normal_(
            0.0, 1.0 / n, generator=g)
        if case["entropy"]:
            state["grad_entropy"] = torch.empty(B, device="cuda").uniform_(-0.02, 0.0, generator=g)
            state["grad_lse"] = 2e-4 * lse                 # of a penalty on the squared log sum
    return state


# --- one pass ---------------------------------------------------------------------------

def _row_statistics(logits):
    """Shifted scores, log sum and entropy of every row, in 32 bits."""
    x = logits.float()
    highest = x.amax(dim=1, keepdim=True)
    highest = highest.masked_fill(highest == -math.inf, 0.0)   # a row with nothing left
    y = (x - highest) * INV_TEMPERATURE
    e = y.exp()
    total = e.sum(dim=1)
    mean = torch.where(e > 0, y * e, 0.0).sum(dim=1) / total
    lse = highest[:, 0] * INV_TEMPERATURE + total.log()
    entropy = torch.where(total > 0, total.log() - mean, 0.0)
    return y - total.log()[:, None], lse, entropy


def _largest(logits, k):
    """Values and ids of the k largest logits, equal ones by their ids: one integer holds both."""
    x = logits.float() + 0.0
    bits = x.view(torch.int32).long()
    order = torch.where(bits < 0, -(bits & 0x7FFFFFFF) - 1, bits)
    ids = torch.arange(x.shape[1], device=x.device)
    keys = order * (1 << 32) + (0x7FFFFFFF - ids)
    ids = 0x7FFFFFFF - (keys.topk(k, dim=1).values & 0xFFFFFFFF)
    return x.gather(1, ids), ids


def _plain(s):
    c = s["case"]
    if c["op"] == "head":
        codes = torch.stack([s["codes"] & 15, s["codes"] >> 4], dim=2).view(c["V"], c["K"])
        weights = (codes.float() - 8.0) * s["scales"].float().repeat_interleave(c["group"], dim=1)
        return torch.matmul(s["hidden"].float(), weights.t()).to(_TYPES[c["dtype"]])
    if c["op"] == "top":
        values, ids = _largest(s["logits"], c["k"])
        return {"ids": ids.to(torch.int32), "values": values}
    B, V = c["B"], c["V"]
    tokens = s["tokens"].view(B, c["n"]).long()
    real = (tokens >= 0) & (tokens < V)
    tokens = tokens.masked_fill(~real, 0)
    if c["op"] == "logprobs":
        logp, lse, entropy = _row_statistics(s["logits"])
        given = torch.where(real, logp.gather(1, tokens), 0.0)
        out = {"logprobs": given.view(s["tokens"].shape), "lse": lse, "entropy": entropy}
        empty = lse == -math.inf
        out["logprobs"] = torch.where(real & empty[:, None], -math.inf, given).view(s["tokens"].shape)
        if c["top"]:
            _, ids = _largest(s["logits"], c["top"])
            best = logp.gather(1, ids)
            out["top_ids"] = ids.to(torch.int32)
            out["top_logprobs"] = torch.where(empty[:, None], -math.inf, best)
        return out
    g = torch.where(real, s["grad_logprobs"].view(B, c["n"]), 0.0)
    logp = (s["logits"].float() - s["stats"][:, :1]) * INV_TEMPERATURE - s["stats"][:, 1:]
    share = -g.sum(dim=1, keepdim=True)
    if c["entropy"]:
        share = share + s["grad_lse"][:, None] - s["grad_entropy"][:, None] * (logp + s["entropy"][:, None])
    grad = (logp.exp() * share).scatter_add_(1, tokens, g)
    return (grad * INV_TEMPERATURE).to(s["logits"].dtype)


def run(state):
    if not own:
        return _plain(state)
    import paper_2609_03844_amd as sbw
    c = state["case"]
    if c["op"] == "head":
        return sbw.head_logits(state["hidden"], state["codes"], state["scales"],
                               dtype=_TYPES[c["dtype"]])
    if c["op"] == "top":
        ids, values = sbw.top_candidates(state["logits"], c["k"])
        return {"ids": ids, "values": values}
    if c["op"] == "logprobs":
        r = sbw.token_logprobs(state["logits"], state["tokens"], INV_TEMPERATURE, top=c["top"])
        out = {"logprobs": r.logprobs, "lse": r.lse, "entropy": r.entropy}
        if c["top"]:
            out["top_ids"], out["top_logprobs"] = r.top_ids, r.top_logprobs
        return out
    return sbw.token_logprobs_grad(state["logits"], state["tokens"], state["stats"],
                                   state["entropy"], state["grad_logprobs"], state.get("grad_lse"),
                                   state.get("grad_entropy"), INV_TEMPERATURE)


# --- what a pass cannot do without --------------------------------------------------------

def work(case):
    B, V, op = case["B"], case["V"], case["op"]
    size = 4 if case["dtype"] == "f32" else 2
    if op == "head":
        K = case["K"]
        scales = V * (K // case["group"]) * (4 if case["scales"] == "f32" else 2)
        return {"bytes": V * K // 2 + scales + 2 * B * K + size * B * V, "flops": 2 * B * V * K}
    if op == "top":
        return {"bytes": size * B * V + 8 * B * case["k"], "flops": B * V}
    if op == "logprobs":
        # shift, scale, exponential, sum, weighted sum (a multiply and an add)
        return {"bytes": size * B * V + B * (8 * case["n"] + 8 + 8 * case["top"]), "flops": 6 * B * V}
    rows = B * (8 * case["n"] + (20 if case["entropy"] else 8))
    return {"bytes": 2 * size * B * V + rows, "flops": (6 if case["entropy"] else 4) * B * V}


# --- the definitions in 64 bits -----------------------------------------------------------

def _head_exact(s):
    c = s["case"]
    hidden = s["hidden"].double().view(c["B"], -1, c["group"])
    out = []
    for v in range(0, c["V"], 8192):
        q = s["codes"][v:v + 8192].to(torch.int16)
        even = (q % 16 - 8).double()
        odd = (q // 16 - 8).double()
        half = c["group"] // 2
        even, odd = (t.view(q.shape[0], -1, half) for t in (even, odd))
        partial = torch.matmul(hidden[:, :, 0::2].transpose(0, 1).contiguous(),
                               even.permute(1, 2, 0).contiguous())
        partial += torch.matmul(hidden[:, :, 1::2].transpose(0, 1).contiguous(),
                                odd.permute(1, 2, 0).contiguous())          # [groups, B, rows]
        out.append((partial * s["scales"][v:v + 8192].double().t()[:, None, :]).sum(dim=0))
    return torch.cat(out, dim=1)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "head":
        return _head_exact(s)
    if case["op"] == "top":
        rows = [torch.sort(r.double(), descending=True).values[:case["k"]] for r in s["logits"]]
        return {"ids": None, "values": torch.stack(rows)}
    B, n = case["B"], case["n"]
    parts = []
    for b in range(B):
        x = s["logits"][b].double()
        z = x * INV_TEMPERATURE
        ids = s["tokens"].view(B, n)[b].long()
        real = ids >= 0
        at = ids.clamp(min=0)
        if case["op"] == "grad":
            g = torch.where(real, s["grad_logprobs"].view(B, n)[b].double(), 0.0)
            logp = (x - s["stats"][b, 0].double()) * INV_TEMPERATURE - s["stats"][b, 1].double()
            p = torch.exp(logp)
            d = p * -g.sum()
            if case["entropy"]:
                d += p * s["grad_lse"][b].double()
                d -= p * s["grad_entropy"][b].double() * (logp + s["entropy"][b].double())
            parts.append((INV_TEMPERATURE * d.index_add(0, at, g),))
            continue
        lse = torch.logsumexp(z, 0)
        logp = z - lse if lse > -math.inf else torch.full_like(z, -math.inf)
        some = logp[logp > -math.inf]
        part = [torch.where(real, logp[at], 0.0), lse, -(some.exp() * some).sum()]
        if case["top"]:
            part.append(torch.sort(logp, descending=True).values[:case["top"]])
        parts.append(part)
    rows = [torch.stack(r) for r in zip(*parts)]
    if case["op"] == "grad":
        return rows[0]
    out = {"logprobs": rows[0].view(s["tokens"].shape), "lse": rows[1], "entropy": rows[2]}
    if case["top"]:
        out["top_ids"], out["top_logprobs"] = None, rows[3]
    return out
