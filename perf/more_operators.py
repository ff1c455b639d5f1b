"""The operators that follow a model's logits, as cases that can be timed, each in a plain form (elementary torch operations in 32 bits; 64 for the
masses that a draw compares with its random number, and for the difference of two distributions that may be all but the same) and, where `own` is set, through the entry points of the binding:

  draw     twist_draw_raw: a token for every row of logits from a given uniform random number, after temperature, top-k, top-p and min-p
  top      twist_top_logits_raw: the k largest logits of every row in order, and what the others weigh together: what a teacher leaves of its distribution
  distill  twist_distill_raw: the loss of a student's logits against a teacher's top logits and the targets, and its gradient

A case is a dict of plain values.  T rows of V columns in `dtype`.  `draw`: top_k k (0: none), top_p p (1: none), min_p m (0: none), every row its own
temperature between lo and hi; mixed: every row has each rule with an even chance, and one in eight takes the largest logit (temperature 0); a grammar's mask left the share
`allow` of the columns.  `top`: k, temperature tau.  `distill`: k entries a row, temperature tau, the share `weight` of the loss that is the teacher's,
rest: the teacher's other logits count together as one more; pad: rows at the end that belong to no sequence (no target, no entries).
"""
from __future__ import annotations

import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    """Vocabularies are those of the repository's workloads (GPT-2-small, Llama-shaped), an odd small one, and one of 2^17; rows those of its batches."""
    return [
        # one request, one token: latency alone
        {"name": "draw_gpt_one", "kind": "draw", "dtype": "f32", "T": 1, "V": 50257, "k": 50, "p": 1.0, "m": 0.0, "lo": 0.8, "hi": 0.8, "mixed": False, "allow": 1.0},
        # a serving step in which every request has settings of its own, straight from the projection
        {"name": "draw_llama_batch", "kind": "draw", "dtype": "bf16", "T": 64, "V": 32000, "k": 50, "p": 0.9, "m": 0.05, "lo": 0.6, "hi": 1.4, "mixed": True, "allow": 1.0},
        # many samples of one prompt, nucleus alone: the masses of whole rows
        {"name": "draw_gpt_many", "kind": "draw", "dtype": "f32", "T": 256, "V": 50257, "k": 0, "p": 0.95, "m": 0.0, "lo": 1.0, "hi": 1.0, "mixed": False, "allow": 1.0},
        # a large vocabulary under a grammar
        {"name": "draw_wide_masked", "kind": "draw", "dtype": "f32", "T": 48, "V": 131072, "k": 0, "p": 0.98, "m": 0.001, "lo": 0.7, "hi": 1.3, "mixed": False, "allow": 0.2},
        # what a serving step reports of one request's distribution
        {"name": "top_gpt_one", "kind": "top", "dtype": "f32", "T": 1, "V": 50257, "k": 20, "tau": 1.0},
        # an fp32 teacher over an odd vocabulary
        {"name": "top_f32_odd", "kind": "top", "dtype": "f32", "T": 301, "V": 1003, "k": 17, "tau": 2.0},
        # a teacher of Llama shape, long lists
        {"name": "top_llama_long", "kind": "top", "dtype": "bf16", "T": 2048, "V": 32000, "k": 256, "tau": 1.0},
        # a GPT-2-small teacher over a training batch of 8 x 1024 tokens
        {"name": "top_gpt_batch", "kind": "top", "dtype": "bf16", "T": 8192, "V": 50257, "k": 64, "tau": 2.0},
        # a few rows of a small fp32 student, two of them padding
        {"name": "distill_f32_odd", "kind": "distill", "dtype": "f32", "T": 77, "V": 1003, "k": 8, "tau": 1.5, "weight": 0.7, "rest": True, "pad": 2},
        # an fp32 GPT student on 2 x 512 tokens
        {"name": "distill_gpt_f32", "kind": "distill", "dtype": "f32", "T": 1024, "V": 50257, "k": 32, "tau": 4.0, "weight": 0.5, "rest": True, "pad": 0},
        # the teacher alone, its list as the whole of its distribution
        {"name": "distill_llama_long", "kind": "distill", "dtype": "bf16", "T": 2048, "V": 32000, "k": 256, "tau": 1.0, "weight": 1.0, "rest": False, "pad": 0},
        # a GPT-2-small subnet's training batch (the largest)
        {"name": "distill_gpt_batch", "kind": "distill", "dtype": "bf16", "T": 8192, "V": 50257, "k": 64, "tau": 2.0, "weight": 0.5, "rest": True, "pad": 128},
    ]


def draw(rng):
    """One more case of the same ranges: one row to a training batch, vocabularies from 64 to 2^17 columns, either type; no more bytes than the largest
    listed case of its kind."""
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    while True:
        c = {"kind": rng.choice(["draw", "draw", "top", "distill"]), "dtype": rng.choice(["bf16", "f32"])}
        c["V"] = rng.choice([1003, 32000, 50257, log(64, 131072), log(64, 131072)])
        if c["kind"] == "draw":
            c.update(T=log(1, 256), k=rng.choice([0, 0, 1, 50, log(1, 5000)]), p=rng.choice([1.0, 0.9, round(rng.uniform(0.05, 0.999), 3)]),
                     m=rng.choice([0.0, 0.0, 0.05, round(10 ** rng.uniform(-5, -0.3), 6)]), lo=rng.choice([1.0, 0.7, 0.1]), hi=rng.choice([1.0, 1.3, 3.0]),
                     mixed=rng.random() < 0.4, allow=rng.choice([1.0, 1.0, 0.3, 0.02]))
        elif c["kind"] == "top":
            c.update(T=log(1, 8192), k=min(c["V"], log(1, 512)), tau=rng.choice([1.0, 2.0, round(rng.uniform(0.5, 8.0), 2)]))
        else:
            c.update(T=log(1, 8192), k=min(c["V"], log(1, 512)), tau=rng.choice([1.0, 2.0, round(rng.uniform(0.5, 8.0), 2)]), weight=rng.choice([1.0, 0.5, round(rng.random(), 2)]),
                     rest=rng.random() < 0.6)
            c["pad"] = min(c["T"] - 1, rng.choice([0, 0, 1, 13]))
        if work(c)["bytes"] <= max(work(x)["bytes"] for x in listed() if x["kind"] == c["kind"]):
            return c


def work(c):
    """Every logit read once (distill: and its gradient written once); the lists, statistics and results of a row.  An exponential and a few comparisons or sums a
    column."""
    es, T, V = 2 if c["dtype"] == "bf16" else 4, c["T"], c["V"]
    if c["kind"] == "draw":
        return {"bytes": T * (V * es + 32), "flops": 4 * T * V}
    if c["kind"] == "top":
        return {"bytes": T * (V * es + 8 * c["k"] + 4), "flops": 4 * T * V}
    return {"bytes": T * (2 * V * es + 8 * c["k"] + 12), "flops": 8 * T * V}


# ---------------------------------------------------------------------------------------------- inputs
def _logits(c, g, T, V):
    """A model's logits: most columns spread around a low level, some dozens of plausible ones well above it."""
    x = 2.0 * torch.randn((T, V), generator=g, device="cuda")
    n = min(V, 48)
    at = torch.randint(0, V // n, (T, n), generator=g, device="cuda") + torch.arange(n, device="cuda") * (V // n)  # (all different)
    return x.scatter_(1, at, 7.0 + 2.5 * torch.randn((T, n), generator=g, device="cuda"))


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    dt, T, V = DTYPES[c["dtype"]], c["T"], c["V"]
    rand = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    x = _logits(c, g, T, V)
    st = {"c": c}
    if c["kind"] == "draw":
        if c["allow"] < 1:
            x = torch.where(rand(T, V) < c["allow"], x, -math.inf)
        st["logits"] = x.to(dt)
        some = lambda: rand(T) < (0.5 if c["mixed"] else 1.0)  # noqa: E731
        st["uniform"] = rand(T)
        st["temperature"] = c["lo"] + (c["hi"] - c["lo"]) * rand(T)
        if c["mixed"]:
            st["temperature"][rand(T) < 0.125] = 0.0
        st["top_k"] = torch.where(some(), c["k"], 0).to(torch.int32) if c["k"] else None
        st["top_p"] = torch.where(some(), c["p"], 1.0).float() if c["p"] < 1 else None
        st["min_p"] = torch.where(some(), c["m"], 0.0).float() if c["m"] > 0 else None
        return st
    st["logits"] = x.to(dt)
    if c["kind"] == "distill":
        k, pad = c["k"], c["pad"]
        z = torch.add(x, torch.randn((T, V), generator=g, device="cuda"), alpha=1.5)  # the teacher: another model of the same text
        del x
        st["values"], ids = torch.topk(z, k, dim=1)
        st["ids"] = ids.to(torch.int32)
        st["rest"] = None
        if c["rest"]:
            st["rest"] = torch.logsumexp(z.scatter_(1, ids, -math.inf) / c["tau"], 1)
        st["targets"] = torch.where(rand(T) < 0.5, ids[:, 0], torch.randint(0, V, (T,), generator=g, device="cuda")).to(torch.int32)
        if pad:
            st["targets"][T - pad:] = -1
            st["ids"][T - pad:] = -1
            if st["rest"] is not None:
                st["rest"][T - pad:] = -math.inf
    return st


# ---------------------------------------------------------------------------------------------- plain forms
def _lse(x):
    """log of the sum of exponentials along rows (-inf for rows of nothing but -inf)."""
    m = x.amax(1, keepdim=True)
    m = torch.where(m > -math.inf, m, 0.0)
    return (m + torch.log(torch.exp(x - m).sum(1, keepdim=True)))[:, 0]


def _plain_draw(st):
    T, V = st["logits"].shape
    x, at = torch.sort(st["logits"].float(), dim=1, descending=True, stable=True)  # equal logits: lowest column first
    temp = st["temperature"].double()[:, None]
    greedy = temp <= 0
    some = x[:, :1] > -math.inf                                                    # (a row may have nothing to draw from)
    w = torch.exp((x.double() - torch.where(some, x[:, :1], 0.0).double()) / torch.where(greedy, 1.0, temp))  # relative to the largest
    rank = torch.arange(V, device="cuda")
    keep = (rank < 1) | ((x > -math.inf) & ~greedy)
    if st["top_k"] is not None:
        k = st["top_k"].long()[:, None]
        keep &= (k < 1) | (rank < k)
    if st["top_p"] is not None:
        p = st["top_p"].double()[:, None]
        mass = torch.cumsum(torch.where(keep, w, 0.0), 1)
        keep &= (rank < 1) | (p >= 1) | (mass - torch.where(keep, w, 0.0) < p * mass[:, -1:])
    if st["min_p"] is not None:
        keep &= (rank < 1) | (w >= st["min_p"].double()[:, None])
    keep &= some
    w = torch.where(keep, w, 0.0)
    mass = torch.cumsum(w, 1)
    kept = keep.sum(1)
    n = (mass <= st["uniform"].double()[:, None] * mass[:, -1:]).sum(1).minimum(kept - 1).clamp(min=0)[:, None]  # the first whose sum exceeds the random number's share
    logprobs = torch.where(some, torch.log(w.gather(1, n) / torch.where(some, mass[:, -1:], 1.0)), -math.inf)
    return {"tokens": torch.where(some, at.gather(1, n), -1)[:, 0].to(torch.int32), "logprobs": logprobs[:, 0].float(), "kept": kept.to(torch.int32)}


def _plain_top(st):
    k, tau = st["c"]["k"], st["c"]["tau"]
    x, at = torch.sort(st["logits"].float(), dim=1, descending=True, stable=True)
    rest = _lse(x[:, k:] / tau) if k < x.shape[1] else torch.full((x.shape[0],), -math.inf, device="cuda")
    return {"ids": at[:, :k].to(torch.int32), "values": x[:, :k].contiguous(), "rest": rest}


def _plain_distill(st):
    c, x = st["c"], st["logits"].float()
    T, V = x.shape
    tau, weight = c["tau"], c["weight"]
    ids, ok = st["ids"].long().clamp(min=0), st["ids"] >= 0
    # the teacher's distribution over its entries, and over the others together
    t = torch.where(ok, st["values"].double() / tau, -math.inf)
    if st["rest"] is not None:
        t = torch.cat([t, st["rest"].double()[:, None]], 1)
    taught = t.amax(1) > -math.inf
    log_q = torch.where(taught[:, None], t - _lse(t)[:, None], -math.inf)
    q = torch.exp(log_q)
    # the student's over the same
    log_p = x.double() / tau
    log_p = log_p - _lse(log_p)[:, None]
    member = torch.zeros((T, V), device="cuda").scatter_add_(1, ids, ok.float()) > 0
    mine = log_p.gather(1, ids)
    if st["rest"] is not None:
        others = _lse(torch.where(member, -math.inf, log_p))
        mine = torch.cat([mine, others[:, None]], 1)
    kl = torch.where(q > 0, q * (log_q - mine), 0.0).sum(1)
    g = torch.exp(log_p)
    if st["rest"] is not None:
        g = torch.where(member, g, g * (1.0 - q[:, -1:] / torch.exp(others)[:, None]))
    g.scatter_add_(1, ids, torch.where(ok, -q[:, : c["k"]], 0.0))
    g = torch.where(taught[:, None], weight * tau * g, 0.0).float()
    row = (weight * tau * tau * kl).float()
    if weight < 1:
        tgt, on = st["targets"].long().clamp(min=0)[:, None], (st["targets"] >= 0)[:, None]
        log_p = x - _lse(x)[:, None]
        row = row - torch.where(on, (1 - weight) * log_p.gather(1, tgt), 0.0)[:, 0]
        p = torch.exp(log_p).scatter_add_(1, tgt, torch.full((T, 1), -1.0, device="cuda"))
        g += torch.where(on, (1 - weight) * p, 0.0)
    return {"loss": row.mean(), "rowloss": row, "grad": (g / T).to(st["logits"].dtype)}


# ---------------------------------------------------------------------------------------------- the library's calls
_contexts = {}


def _context(c):
    """A program keeps one context per model shape."""
    key = (c["dtype"], c["V"])
    if key not in _contexts:
        import paper_2511_03983_amd as tw
        from synth_inputs import ModelCfg
        _contexts[key] = tw.Context(tw.desc_from_cfg(ModelCfg(arch="llama", d_model=64, n_heads=1, d_head=64, d_ff=8, vocab=c["V"], max_seq=1, act="swiglu", norm="rms",
                                                              has_bias=False, tied_head=False, rope=True, rope_theta=10000.0, dtype=c["dtype"])))
    return _contexts[key]


def _handle(st):
    """What a program keeps beside its buffers: the holder of the rules', or of the teacher's, pointers."""
    if "handle" not in st:
        import paper_2511_03983_amd as tw
        c = st["c"]
        st["ctx"] = _context(c)
        if c["kind"] == "draw":
            st["handle"] = tw.DrawRules(temperature=st["temperature"], top_k=st["top_k"], top_p=st["top_p"], min_p=st["min_p"])
        elif c["kind"] == "distill":
            st["handle"] = tw.Teacher(st["ids"], st["values"], rest=st["rest"], temperature=c["tau"], weight=c["weight"])
        else:
            st["handle"] = None
    return st["ctx"], st["handle"]


def run(st):
    c = st["c"]
    if own:
        ctx, handle = _handle(st)
        if c["kind"] == "draw":
            tokens, logprobs, kept = ctx.twist_draw_raw(st["logits"], st["uniform"], handle)
            return {"tokens": tokens, "logprobs": logprobs, "kept": kept}
        if c["kind"] == "top":
            ids, values, rest = ctx.twist_top_logits_raw(st["logits"], c["k"], temperature=c["tau"])
            return {"ids": ids, "values": values, "rest": rest}
        loss, rowloss, grad = ctx.twist_distill_raw(st["logits"], st["targets"] if c["weight"] < 1 else None, handle)
        return {"loss": loss, "rowloss": rowloss, "grad": grad}
    return {"draw": _plain_draw, "top": _plain_top, "distill": _plain_distill}[c["kind"]](st)


# ---------------------------------------------------------------------------------------------- 64 bits
def _order(x):
    """Whole numbers, all different, in the order of a row's logits: larger logits first, equal ones by column."""
    bits = (x.float() + 0.0).view(torch.int32).long()
    value = torch.where(bits < 0, -(bits & 0x7fffffff), bits)
    return value * 2 ** 20 + torch.arange(x.shape[1] - 1, -1, -1, device="cuda")


def exact(c, seed):
    """From the definitions, in 64 bits: a draw row by row; a teacher's list from whole numbers; the gradient of the loss by differentiating it."""
    st = prepare(c, seed)
    T, V, x = c["T"], c["V"], st["logits"]
    if c["kind"] == "draw":
        tokens, kept, logprobs = [], [], []
        setting = lambda name, t, none: none if st[name] is None else st[name][t].item()  # noqa: E731
        for t in range(T):
            at = torch.argsort(_order(x[t:t + 1])[0], descending=True)
            z = x[t, at].double()
            n, temp, k, p, m = int((z > -math.inf).sum()), setting("temperature", t, 1.0), setting("top_k", t, 0), setting("top_p", t, 1.0), setting("min_p", t, 0.0)
            if n == 0:
                tokens.append(-1)
                kept.append(0)
                logprobs.append(-math.inf)
                continue
            if temp <= 0:
                n = 1
            elif k > 0:
                n = min(n, k)
            w = torch.exp((z[:n] - z[0]) / (temp if temp > 0 else 1.0))
            if p < 1:
                below = torch.cumsum(w, 0)
                n = min(n, 1 + int((below[:-1] < p * below[-1]).sum()))
            n = min(n, max(1, int((w[:n] >= m).sum())))
            sums = torch.cumsum(w[:n], 0)
            j = min(n - 1, int(torch.searchsorted(sums, (sums[-1:] * st["uniform"][t].double()), right=True)))
            tokens.append(int(at[j]))
            kept.append(n)
            logprobs.append(math.log(w[j]) - math.log(sums[-1]))
        back = lambda v, dt: torch.tensor(v, dtype=dt, device="cuda")  # noqa: E731
        return {"tokens": back(tokens, torch.int32), "logprobs": back(logprobs, torch.float64), "kept": back(kept, torch.int32)}
    out = {"ids": [], "values": [], "rest": [], "rowloss": [], "grad": []}
    for a in range(0, T, 256):
        z = x[a:a + 256].double()
        if c["kind"] == "top":
            ids = torch.topk(_order(x[a:a + 256]), c["k"], dim=1).indices
            out["ids"].append(ids.to(torch.int32))
            out["values"].append(z.gather(1, ids))
            out["rest"].append(torch.logsumexp((z / c["tau"]).scatter(1, ids, -math.inf), 1))
            continue
        z.requires_grad_()
        tau, share = c["tau"], c["weight"]
        rows = z.shape[0]
        ids, values = st["ids"][a:a + rows].long(), st["values"][a:a + rows].double()
        on = ids[:, 0] >= 0  # (a row has all of its entries or none)
        ids = ids.clamp(min=0)
        mine, theirs = torch.gather(z / tau, 1, ids), values / tau
        if c["rest"]:
            mine = torch.cat([mine, torch.logsumexp((z / tau).scatter(1, ids, -math.inf), 1, keepdim=True)], 1)
            theirs = torch.cat([theirs, st["rest"][a:a + rows, None].double()], 1)
        q = torch.softmax(theirs, 1)
        whole = torch.logsumexp(z / tau, 1, keepdim=True)
        terms = torch.where(q > 0, q * (torch.log_softmax(theirs, 1) - torch.where(q > 0, mine, 0.0) + whole), 0.0)
        row = torch.where(on, share * tau ** 2 * terms.sum(1), 0.0)
        if share < 1:
            y = st["targets"][a:a + rows].long()
            row = row + torch.where(y >= 0, (1 - share) * -torch.log_softmax(z, 1).gather(1, y.clamp(min=0)[:, None])[:, 0], 0.0)
        row.sum().backward()
        out["rowloss"].append(row.detach())
        out["grad"].append(z.grad / T)
    out = {n: torch.cat(v) for n, v in out.items() if v}
    if c["kind"] == "distill":
        out["loss"] = out["rowloss"].mean()
        out = {n: out[n] for n in ("loss", "rowloss", "grad")}
    return out
