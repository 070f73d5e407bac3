"""The operators around a frozen, compressed model, as cases that can be timed and checked.

A case is a dict of plain values:

  op      "logprobs"       log probability, rank and entropy for one given token a row and the
                           row's `top` best alternatives (a serving step, a scored prompt)
          "logprobs_train" the log probability and entropy with the logits' gradient for both
          "distill"        divergence from a teacher's `top` best log probabilities and the
                           logits' gradient (a training step)
          "lora"           low-rank adapters of many requests beside a shared projection's result
          "lora_train"     the adapters' and the activations' gradients
  rows, vocab, top   for the first three; `pad` more values lie between two rows of the logits,
                     `masked` is the share of rows in which a grammar leaves about 50 tokens
  tail, temperature  distillation with the rest of the vocabulary as one more outcome, or without
  tokens, k, n, rank, adapters, requests   for the last two: activation rows, the projection's
                     columns and rows, the adapters' rank, adapters that are loaded and requests
                     (runs of rows with one adapter; one in ten has none)
  dtype   of the logits, of the projection's result or of its gradient

Sizes: the LM head has 128,256 rows over 4,096 columns, the matrices of the two blocks 1,024 to
28,672 rows over 4,096, 8,192 or 14,336 columns.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
BYTES = {"f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # one request's decoding step that returns 20 alternatives: latency
        {"name": "logprobs_step_1", "op": "logprobs", "rows": 1, "vocab": 128256, "pad": 0, "top": 20, "masked": 0.0,
         "temperature": 1.0, "dtype": "f32"},
        # a full batch of requests, fp32 logits as the products give them, some rows held to a grammar
        {"name": "logprobs_step_64", "op": "logprobs", "rows": 64, "vocab": 128256, "pad": 0, "top": 8, "masked": 0.3,
         "temperature": 0.7, "dtype": "f32"},
        # a teacher scores its prompts and keeps 64 alternatives for each position
        {"name": "logprobs_prompts_4096", "op": "logprobs", "rows": 4096, "vocab": 128256, "pad": 0, "top": 64,
         "masked": 0.0, "temperature": 1.0, "dtype": "bf16"},
        # a policy's update on a small vocabulary of odd size in a padded tensor, entropy in the loss
        {"name": "logprobs_train_1023", "op": "logprobs_train", "rows": 1023, "vocab": 32001, "pad": 63, "top": 0,
         "masked": 0.0, "temperature": 1.0, "dtype": "bf16"},
        # the last rows of an epoch
        {"name": "distill_rows_7", "op": "distill", "rows": 7, "vocab": 32000, "pad": 0, "top": 16, "tail": True,
         "temperature": 1.0, "dtype": "f32"},
        # odd sizes, half precision, softened, without the tail
        {"name": "distill_odd_777", "op": "distill", "rows": 777, "vocab": 50001, "pad": 0, "top": 20, "tail": False,
         "temperature": 2.0, "dtype": "f16"},
        # a training step over long sequences with the large vocabulary
        {"name": "distill_rows_4096", "op": "distill", "rows": 4096, "vocab": 128256, "pad": 0, "top": 64, "tail": True,
         "temperature": 1.0, "dtype": "bf16"},
        # one token of one request beside a square projection: latency
        {"name": "lora_step_1", "op": "lora", "tokens": 1, "k": 4096, "n": 4096, "rank": 16, "adapters": 4,
         "requests": 1, "dtype": "f32"},
        # a full batch of single tokens, each with an adapter of its own choice, beside the gate projection
        {"name": "lora_step_64", "op": "lora", "tokens": 64, "k": 4096, "n": 14336, "rank": 16, "adapters": 32,
         "requests": 64, "dtype": "f32"},
        # ragged prompts of some requests
        {"name": "lora_prompts_6001", "op": "lora", "tokens": 6001, "k": 4096, "n": 14336, "rank": 16, "adapters": 8,
         "requests": 13, "dtype": "bf16"},
        # four tenants' adapters trained together
        {"name": "lora_train_8192", "op": "lora_train", "tokens": 8192, "k": 4096, "n": 4096, "rank": 64, "adapters": 4,
         "requests": 16, "dtype": "bf16"},
        # an adapter of the LM head, from the fp32 gradient that a loss gives
        {"name": "lora_train_head_1024", "op": "lora_train", "tokens": 1024, "k": 4096, "n": 128256, "rank": 16,
         "adapters": 1, "requests": 1, "dtype": "f32"},
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["logprobs", "logprobs_train", "distill", "lora", "lora_train"])
    if op.startswith("lora"):
        k = rng.choice([4096, 8192, 14336])
        n = rng.choice([1024, 4096, 8192, 14336, 28672])
        rank = rng.choice([8, 16, 24, 32, 64])
        adapters = rng.randint(1, 32 if op == "lora" else 4)
        tokens = _log(rng, 1, 4096) if op == "lora" else _log(rng, 64, 4096)
        return {"op": op, "tokens": tokens, "k": k, "n": n, "rank": rank, "adapters": adapters,
                "requests": min(tokens, _log(rng, 1, 64)), "dtype": rng.choice(["f32", "bf16"])}
    rows, vocab = _log(rng, 1, 2048), _log(rng, 8000, 131072)
    case = {"op": op, "rows": rows, "vocab": vocab, "pad": rng.choice([0, 0, 1, 64]), "top": 0, "temperature": 1.0,
            "dtype": rng.choice(["f32", "bf16", "f16"])}
    if op == "logprobs":
        return {**case, "top": rng.choice([0, 1, 5, 20, 64]), "masked": rng.choice([0.0, 0.5]),
                "temperature": rng.choice([1.0, 0.7])}
    if op == "distill":
        return {**case, "top": rng.choice([1, 16, 50, 64]), "tail": rng.random() < 0.5,
                "temperature": rng.choice([1.0, 2.0])}
    return {**case, "masked": 0.0}


def _logits(case, rows, g):
    """Rows of a padded tensor: a broad Gaussian with a few likely tokens far above it."""
    vocab = case["vocab"]
    z = torch.randn((rows, vocab + case["pad"]), generator=g, device="cuda")[:, :vocab].mul_(1.6)
    return z


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def uniform(*shape):
        return torch.rand(shape, generator=g, device="cuda")

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    if case["op"].startswith("lora"):
        t, k, n, r, m = case["tokens"], case["k"], case["n"], case["rank"], case["adapters"]
        # requests: ragged runs of rows, each with a loaded adapter or none
        single = case["requests"] == t
        cuts = torch.arange(1, t, device="cuda") if single else (uniform(case["requests"] - 1) * t).long().sort().values
        which = (uniform(case["requests"]) * m).int()
        if case["requests"] > 1:
            which = torch.where(uniform(case["requests"]) < 0.1, torch.full_like(which, -1), which)
        adapter = which[torch.searchsorted(cuts, torch.arange(t, device="cuda"), right=True)].contiguous()
        state = {"x": normal(t, k).bfloat16(), "a": normal(m, r, k).mul_(k ** -0.5).bfloat16(),
                 "b": normal(m, n, r).mul_(0.05).bfloat16(), "scale": 0.5 + 2.0 * uniform(m), "adapter": adapter}
        if case["op"] == "lora":
            state["base"] = normal(t, n).to(dt)
            state["out"] = torch.empty_like(state["base"])
        else:
            state["dy"] = normal(t, n).mul_(0.1).to(dt)
            state["dx_base"] = normal(t, k).bfloat16()
        return {"op": case["op"], **state}

    rows, vocab, top = case["rows"], case["vocab"], case["top"]
    z = _logits(case, rows, g)
    state = {"op": case["op"], "temperature": case["temperature"], "top": top}
    if case["op"] == "distill":
        # the teacher's alternatives: distinct places, most of the probability, the student near it;
        # some rows have fewer alternatives and some none
        start = (uniform(rows, 1) * vocab).long()
        step = 1 + (uniform(rows, 1) * (vocab // top)).long().clamp_(max=vocab // top - 1)
        index = (start + step * torch.arange(top, device="cuda")) % vocab
        raw = normal(rows, top).mul_(2.5).sort(dim=1, descending=True).values
        logp = raw - raw.exp().sum(1, keepdim=True).log() + (0.6 + 0.38 * uniform(rows, 1)).log()
        z.scatter_(1, index, logp + 0.7 * normal(rows, top) + math.log(vocab) + 4.0)
        few = uniform(rows, 1)
        many = torch.where(few < 0.05, 0, torch.where(few < 0.1, (top + 1) // 2, top))
        keep = torch.arange(top, device="cuda") < many
        keep[0] = True
        scale = 1024.0 if case["dtype"] == "f16" else 1.0  # half precision trains with a loss scale
        state |= {"tail": case["tail"], "index": torch.where(keep, index, -1), "logp": logp,
                  "weight": uniform(rows) * (scale / rows)}
    else:
        likely = (uniform(rows, 8) * vocab).long()
        z.scatter_(1, likely, math.log(vocab) + 3.0 * normal(rows, 8))
        tokens = torch.where(uniform(rows) < 0.7, likely[:, 0], (uniform(rows) * vocab).long())
        if case["masked"]:
            held = uniform(rows) < case["masked"]
            allowed = torch.zeros((rows, vocab), dtype=torch.bool, device="cuda")
            allowed.scatter_(1, (uniform(rows, 50) * vocab).long(), True).scatter_(1, tokens[:, None], True)
            z.masked_fill_(held[:, None] & ~allowed, -math.inf)
        state["tokens"] = tokens
        if case["op"] == "logprobs_train":
            scale = 1024.0 if case["dtype"] == "f16" else 1.0  # half precision trains with a loss scale
            state |= {"grad_logprob": normal(rows) * (scale / rows),
                      "grad_entropy": normal(rows) * (0.01 * scale / rows)}
        state["out"] = tuple(torch.empty(s, dtype=d, device="cuda") for s, d in (
            ((rows,), torch.float32), ((rows,), torch.int64), ((rows,), torch.float32),
            ((rows, top), torch.float32), ((rows, top), torch.int64), ((rows, 4), torch.float32)))
    whole = torch.empty((rows, vocab + case["pad"]), dtype=dt, device="cuda")
    whole[:, :vocab] = z
    whole[:, vocab:] = math.nan  # what lies between two rows is no logit
    state["logits"] = whole[:, :vocab]
    return state


def _plain_logprobs(s):
    z = s["logits"].float() + 0.0  # one zero
    tokens, top = s["tokens"], s["top"]
    zs = (z - z.amax(1, keepdim=True)) / s["temperature"]
    e = zs.exp()
    total = e.sum(1, keepdim=True)
    logs = zs - total.log()
    p = e / total
    logprob = logs.gather(1, tokens[:, None])[:, 0]
    entropy = -torch.where(p > 0, p * logs, 0.0).sum(1)
    zt = z.gather(1, tokens[:, None])
    place = torch.arange(z.shape[1], device=z.device)
    rank = ((z > zt) | ((z == zt) & (place < tokens[:, None]))).sum(1)
    if not top:
        return p, logs, (logprob, rank, entropy, logs[:, :0], rank[:, None][:, :0])
    # values in order, equal ones by their index: one whole number for each
    bits = z.view(torch.int32)
    bits = bits ^ ((bits >> 31) & 0x7FFFFFFF)
    best = (bits.long() * 2 ** 32 + (z.shape[1] - 1 - place)).topk(top, dim=1).indices
    top_logprob = logs.gather(1, best)
    return p, logs, (logprob, rank, entropy, top_logprob, torch.where(top_logprob > -math.inf, best, -1))


def _plain_distill(s):
    z, index, logp, tau = s["logits"].float(), s["index"], s["logp"], s["temperature"]
    there = index >= 0
    at = index.clamp(min=0)
    zs = (z - z.amax(1, keepdim=True)) / tau
    e = zs.exp()
    total = e.sum(1, keepdim=True)
    q = e / total
    logq = (zs - total.log()).gather(1, at)
    p = torch.where(there, logp.exp(), 0.0)
    mass = p.sum(1, keepdim=True)
    # an entry that is not there marks nothing: its place is one past the vocabulary
    inside = torch.zeros((z.shape[0], z.shape[1] + 1), dtype=torch.bool, device=z.device)
    inside = inside.scatter_(1, torch.where(there, index, z.shape[1]), True)[:, :-1]
    if s["tail"]:
        rest = (1.0 - mass).clamp(min=0.0)
        left = (e * ~inside).sum(1, keepdim=True) / total
        loss = torch.where(p > 0, p * (logp - logq), 0.0).sum(1)
        loss = loss + torch.where(rest > 0, rest * (rest.log() - left.log()), 0.0)[:, 0]
        grad = torch.where(inside, q, q * (1.0 - torch.where(rest > 0, rest / left, 0.0)))
    else:
        p = torch.where(mass > 0, p / mass, 0.0)
        loss = torch.where(p > 0, p * (logp - mass.log() - logq), 0.0).sum(1)
        grad = torch.where(mass > 0, q, 0.0)
    grad = grad.scatter_add_(1, at, -p)
    grad = grad * (s["weight"][:, None] / tau)
    return {"loss": loss, "grad": grad.to(s["logits"].dtype)}


def _plain_low(x, a, adapter, scale):
    """scale * A x for every row, in the columns of the row's adapter and zero elsewhere."""
    m, r, k = a.shape
    low = (x @ a.reshape(m * r, k).T).reshape(-1, m, r)
    return (low * ((adapter[:, None] == torch.arange(m, device=x.device)) * scale)[:, :, None]).reshape(-1, m * r)


def _plain(s):
    if s["op"] == "logprobs":
        return dict(zip(("logprob", "rank", "entropy", "top_logprob", "top_index"), _plain_logprobs(s)[2]))
    if s["op"] == "logprobs_train":
        p, logs, (logprob, _, entropy, _, _) = _plain_logprobs(s)
        gl, ge = s["grad_logprob"][:, None], s["grad_entropy"][:, None]
        grad = -p * (gl + ge * (logs + entropy[:, None]))
        grad = grad.scatter_add_(1, s["tokens"][:, None], gl) / s["temperature"]
        return {"logprob": logprob, "entropy": entropy, "grad": grad.to(s["logits"].dtype)}
    if s["op"] == "distill":
        return _plain_distill(s)
    x, a, b, scale, adapter = s["x"].float(), s["a"].float(), s["b"].float(), s["scale"], s["adapter"]
    m, r, k = a.shape
    n = b.shape[1]
    wide = b.permute(0, 2, 1).reshape(m * r, n)
    low = _plain_low(x, a, adapter, scale)
    if s["op"] == "lora":
        return {"out": (s["base"].float() + low @ wide).to(s["base"].dtype)}
    dy = s["dy"].float()
    back = _plain_low(dy, b.permute(0, 2, 1), adapter, scale)
    dx = s["dx_base"].float() + back @ a.reshape(m * r, k)
    return {"dx": dx.to(s["x"].dtype), "da": (back.T @ x).reshape(m, r, k),
            "db": (dy.T @ low).reshape(n, m, r).permute(1, 0, 2).contiguous()}


def run(s):
    if not own:
        return _plain(s)
    from paper_2504_11651_amd import ops
    if s["op"] == "logprobs":
        r = ops.logprobs(s["logits"], s["tokens"], top=s["top"], temperature=s["temperature"], out=s["out"])
        return {"logprob": r.logprob, "rank": r.rank, "entropy": r.entropy, "top_logprob": r.top_logprob,
                "top_index": r.top_index}
    if s["op"] == "logprobs_train":
        r = ops.logprobs(s["logits"], s["tokens"], temperature=s["temperature"], out=s["out"])
        grad = ops.logprobs_backward(s["logits"], s["tokens"], r.stats, s["grad_logprob"], s["grad_entropy"],
                                     temperature=s["temperature"])
        return {"logprob": r.logprob, "entropy": r.entropy, "grad": grad}
    if s["op"] == "distill":
        r = ops.distill(s["logits"], s["index"], s["logp"], tail=s["tail"], temperature=s["temperature"],
                        weight=s["weight"])
        return {"loss": r.loss, "grad": r.grad}
    if s["op"] == "lora":
        return {"out": ops.lora(s["x"], s["a"], s["b"], s["scale"], s["adapter"], base=s["base"], out=s["out"])}
    r = ops.lora_backward(s["x"], s["a"], s["b"], s["scale"], s["adapter"], s["dy"], dx_base=s["dx_base"])
    return {"dx": r.dx, "da": r.da, "db": r.db}


def work(case):
    if case["op"].startswith("lora"):
        t, k, n, r = case["tokens"], case["k"], case["n"], case["rank"]
        m, e = min(case["adapters"], case["requests"]), BYTES[case["dtype"]]
        moved = 2 * t * k + 2 * m * r * (k + n) + 4 * t
        if case["op"] == "lora":
            return {"bytes": moved + 2 * e * t * n, "flops": 2 * t * r * (k + n)}
        return {"bytes": moved + e * t * n + 4 * t * k + 4 * case["adapters"] * r * (k + n),
                "flops": 2 * t * r * (3 * k + 2 * n)}
    rows, size = case["rows"], case["rows"] * case["vocab"]
    e = BYTES[case["dtype"]]
    if case["op"] == "logprobs":
        return {"bytes": e * size + rows * (24 + 12 * case["top"]), "flops": 4 * size}
    return {"bytes": 2 * e * size + rows * (20 + 12 * case["top"]), "flops": 8 * size}


def _exact_rows(s, rows):
    """The definition in 64 bits for some rows; gradients by differentiating it."""
    z = s["logits"][rows].double()
    train = s["op"] != "logprobs"
    z.requires_grad_(train)
    logs = torch.log_softmax(z / s["temperature"], dim=1)
    if s["op"] == "distill":
        index, logp = s["index"][rows], s["logp"][rows].double()
        there = index >= 0
        p = torch.where(there, logp.exp(), 0.0)
        mass = p.sum(1)
        safe = torch.where(mass > 0, mass, 1.0)
        aim = p if s["tail"] else p / safe[:, None]
        at = torch.where(there, index, 0)
        want = torch.where(there, torch.where(aim > 0, aim, 1.0).log() * aim, 0.0).sum(1)
        loss = want - torch.where(there, aim * logs.gather(1, at), 0.0).sum(1)
        if s["tail"]:
            # the rest's log probability: what remains where the entries that are there are taken away
            wide = torch.cat((logs, torch.zeros_like(logs[:, :1])), dim=1)
            wide = wide.scatter(1, torch.where(there, index, logs.shape[1]), -math.inf)
            rest = 1.0 - mass
            loss = loss + rest * (rest.log() - torch.logsumexp(wide[:, :-1], dim=1))
        (loss * s["weight"][rows].double()).sum().backward()
        return {"loss": loss.detach(), "grad": z.grad}
    tokens = s["tokens"][rows]
    logprob = logs.gather(1, tokens[:, None])[:, 0]
    p = logs.exp()
    entropy = -(p * logs.clamp(min=-1e4)).sum(1)
    if train:
        gl, ge = s["grad_logprob"][rows].double(), s["grad_entropy"][rows].double()
        (logprob * gl + entropy * ge).sum().backward()
        return {"logprob": logprob.detach(), "entropy": entropy.detach(), "grad": z.grad}
    got = {"logprob": logprob, "entropy": entropy}
    got["top_logprob"] = logs.topk(s["top"], dim=1).values if s["top"] else logs[:, :0]
    return got


def exact(case, seed):
    s = prepare(case, seed)
    if not s["op"].startswith("lora"):
        rows, step = s["logits"].shape[0], max(1, (1 << 26) // s["logits"].shape[1])
        parts = [_exact_rows(s, slice(i, min(rows, i + step))) for i in range(0, rows, step)]
        got = {k: torch.cat([p[k] for p in parts]) for k in parts[0]}
        return {**got, "rank": None, "top_index": None} if s["op"] == "logprobs" else got
    x, a, b, scale = s["x"].double(), s["a"].double(), s["b"].double(), s["scale"].double()
    out = s["base"].double() if s["op"] == "lora" else s["dx_base"].double()
    da, db = torch.zeros_like(a), torch.zeros_like(b)
    for i in range(a.shape[0]):
        mine = (s["adapter"] == i).nonzero()[:, 0]
        low = x[mine] @ a[i].T
        if s["op"] == "lora":
            out[mine] += scale[i] * (low @ b[i].T)
            continue
        dy = s["dy"][mine].double()
        back = scale[i] * (dy @ b[i])
        out[mine] += back @ a[i]
        da[i] = back.T @ x[mine]
        db[i] = scale[i] * (dy.T @ low)
    return {"out": out} if s["op"] == "lora" else {"dx": out, "da": da, "db": db}
