"""Generating tokens with a deployed subnet: twist_subnet_decode against the oracle's forward pass, and the steps of generation as they are used
together (prompts, single tokens, rules on logits, pages handed out on the way, captured steps).

Bounds of the logits (relative Frobenius error over all of them): fp32 1e-4, the repository's bound of an fp32 path.  bf16: a logit has 9 rounding points of
rms 2^-9 / sqrt(3) a layer and 2 at the head behind it, 1.13e-3 sqrt(9 L + 2) = 5e-3 for two layers and 6.1e-3 for three at gain 1; a factor of 2 for the
gain of the residual stream above its start gives 1e-2 (1.2e-2 for three layers)."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import synth_inputs as si
from helpers import rel_fro, to_device, to_numpy
from oracle import model as omodel, move as omove
from oracle.sample import sample_plan

pytestmark = pytest.mark.gpu

MODELS = {
    # name: (cfg, heads, units, layer_shared)
    "gpt_f32": (si.ModelCfg(n_layers=2, d_model=96, n_heads=6, d_head=16, d_ff=200, vocab=301, max_seq=80), 3, 100, None),
    "llama_f32_um": (si.ModelCfg(arch="llama", n_layers=2, d_model=64, n_heads=4, d_head=16, d_ff=176, vocab=259, max_seq=80, act="swiglu", norm="rms", has_bias=False,
                                 tied_head=False, rope=True, out_unit_major=True), 2, 88, None),
    "ragged_f32": (si.ModelCfg(n_layers=1, d_model=36, n_heads=5, d_head=6, d_ff=70, ffn_granule=7, vocab=19, max_seq=70, act="relu"), 3, 6, None),
    "gpt_bf16": (replace(si.CFG2, n_layers=2, d_model=256, n_heads=4, d_head=64, d_ff=1024, vocab=1003, max_seq=192), 2, 512, None),
    "llama_bf16": (replace(si.CFG3, n_layers=2, d_model=256, n_heads=4, d_head=128, d_ff=704, vocab=517, max_seq=256), 2, 352, None),
    "llama_bf16_um": (replace(si.CFG3, n_layers=2, d_model=256, n_heads=4, d_head=64, d_ff=704, vocab=512, max_seq=256, out_unit_major=True), 3, 352, None),
    # wide enough for the fp32 products that form a tile anew where one of its results is no number
    "gpt_f32_wide": (si.ModelCfg(n_layers=1, d_model=512, n_heads=8, d_head=64, d_ff=64, vocab=8003, max_seq=192), 6, 64, None),
    # layers of different widths
    "gpt_bf16_blocks": (replace(si.CFG2, n_layers=3, d_model=384, n_heads=6, d_head=64, d_ff=768, ffn_granule=64, vocab=1003, max_seq=128), 4, 8, [1, 0, 1]),
}


def _bound(cfg):
    return 1e-4 if cfg.dtype == "f32" else 1.2e-2 if cfg.n_layers > 2 else 1e-2


class Deployed:
    """A model, its deployed subnet, and a cache of n_seqs sequences of up to `top` tokens whose pages lie anywhere in the pools."""

    def __init__(self, lib, name, n_seqs, top, page=16, spare=3, stream=None, table=None):
        self.cfg, hs, fs, shared = MODELS[name]
        cfg = self.cfg
        full_np = si.make_weights(cfg, 3, std=0.05 if cfg.dtype == "f32" else 0.02, generic=True)
        full_t = to_device(full_np, cfg)
        torch.cuda.synchronize()
        self.ctx = lib.Context(lib.desc_from_cfg(cfg), stream)
        self.plan = self.ctx.twist_sample(1, hs, fs, seed=9, require_coverage=False, layer_shared=shared)
        oplan = sample_plan(cfg.n_layers, cfg.n_heads, cfg.n_ffn_units, 1, hs, fs, 9, 0, (), (), shared, require_coverage=False)
        self.osub = omove.extract(full_np, oplan, 0, cfg.d_head, cfg.ffn_granule)
        self.fw = lib.FullWeights(full_t["layers"], full_t["globals"])
        self.sub = self.ctx.twist_extract(self.plan, self.fw, 0)
        self.page, self.max_pages = page, -(-top // page)
        n_pages = n_seqs * self.max_pages + spare
        if table is None:
            order = np.random.default_rng(4).permutation(n_pages)[: n_seqs * self.max_pages]
            table = torch.tensor(order.reshape(n_seqs, self.max_pages), dtype=torch.int32).cuda()
        self.table = table
        self.pages = lib.Pages(table, n_pages, page)
        self.cache = torch.full((self.ctx.twist_cache_bytes(self.sub, self.pages),), 0xff, dtype=torch.uint8, device="cuda")     # NaN throughout
        self.ws = {}
        torch.cuda.synchronize()

    def step(self, tokens, lens, seq=None, max_len=None, logits=None):
        """Logits of one call; host lists or device tensors."""
        i32 = lambda v: v if v is None or torch.is_tensor(v) else torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
        tokens, lens, seq = i32(tokens), i32(lens), i32(seq)
        max_len = max_len or self.cfg.max_seq
        key = (tokens.shape[0], max_len)
        if key not in self.ws:
            self.ws[key] = torch.full((self.ctx.twist_decode_workspace_bytes(self.sub, self.pages, *key),), 0xff, dtype=torch.uint8, device="cuda")
        return self.ctx.twist_subnet_decode(self.sub, tokens, lens, max_len, self.pages, self.cache, self.ws[key], seq=seq, logits=logits)

    def want(self, ids):
        """The oracle's logits [N, vocab] of one sequence of ids."""
        kept = []

        def hook(tag, a):
            if tag == "logits":
                kept.append(np.array(a))
            return a
        ids = np.asarray(ids, np.int32)[None]
        omodel.forward_backward(self.cfg, self.osub, ids, np.zeros_like(ids), q=hook, need_grads=False)
        return kept[0][0]


@pytest.mark.parametrize("name", list(MODELS))
def test_prompt_then_single_tokens_give_the_oracles_logits(lib, name):
    """Sequences of different lengths: prompts together in one call, then a token each, then a few drafted ones each."""
    cfg = MODELS[name][0]
    top = min(cfg.max_seq, 70)
    d = Deployed(lib, name, 3, top)
    ids = si.tokens_uniform(cfg.vocab, 3, top, 4)[:, :top]
    start = [5, 33, 17]
    got = [[] for _ in ids]
    rows = [(s, p) for s in range(3) for p in range(start[s])]

    def run(rows, max_len):
        out = to_numpy(d.step([int(ids[s][p]) for s, p in rows], [p + 1 for _, p in rows], [s for s, _ in rows], max_len))
        for (s, p), x in zip(rows, out):
            assert p == len(got[s])
            got[s].append(x)
    run(rows, 40)
    for k in range(8):
        run([(s, start[s] + k) for s in range(3)], 64)
    for k in range(4):
        run([(s, start[s] + 8 + 5 * k + j) for s in (2, 0, 1) for j in range(5)], top)
    worst = 0.0
    for s in range(3):
        n = len(got[s])
        want = d.want(ids[s][:n])
        worst = max(worst, rel_fro(np.stack(got[s]), want))
        assert n == start[s] + 28
    print(f"{name}: logits {worst:.2e}")
    assert worst <= _bound(cfg), worst


@pytest.mark.parametrize("name", ["gpt_f32", "llama_f32_um", "gpt_bf16", "llama_bf16"])
def test_decoded_logits_give_the_loss_of_the_evaluation(lib, name):
    cfg = MODELS[name][0]
    N = 50
    d = Deployed(lib, name, 1, N)
    t = si.tokens_uniform(cfg.vocab, 1, N, 8)
    x, y = torch.tensor(t[:, :N].copy()).cuda(), torch.tensor(t[:, 1:N + 1].copy()).cuda()
    loss = torch.zeros(1, device="cuda")
    ws = torch.empty(d.ctx.twist_workspace_bytes(d.sub, 1, N), dtype=torch.uint8, device="cuda")
    d.ctx.twist_subnet_forward(d.sub, x, y, ws, loss)
    logits = torch.cat([d.step(x[0, p:p + 1].contiguous(), [p + 1]) for p in range(N)]).double()
    ce = torch.nn.functional.cross_entropy(logits, y[0].long()).item()
    assert abs(ce - loss.item()) <= (5e-3 if cfg.dtype == "bf16" else 1e-4) * abs(loss.item()), (ce, loss.item())


@pytest.mark.parametrize("name", ["llama_f32_um", "gpt_bf16", "llama_bf16"])
def test_unused_rows_change_nothing(lib, name):
    """Rows without a token, beyond max_len or of no sequence, and ids outside the vocabulary among them: the others' logits and the cache keep their bits."""
    cfg = MODELS[name][0]
    results = []
    for junk in ((0, 0, 0, 0), (7, -1, 2 ** 31 - 1, 11)):
        d = Deployed(lib, name, 4, 64)
        d.step([1, 2, 3, 4, 5, 6], [1, 2, 1, 2, 3, 1], [0, 0, 1, 1, 1, 3])
        before = d.cache.clone()
        out = d.step([5, junk[0], 8, junk[1], junk[2], junk[3]], [3, 0, 4, -5, 41, 2], [0, 2, 1, 0, 2, 4], max_len=40)
        torch.cuda.synchronize()
        results.append((out[0].clone(), out[2].clone(), d.cache.clone()))
        assert torch.isfinite(out[[0, 2]].float()).all()
        es = 2 if cfg.dtype == "bf16" else 4
        hs = MODELS[name][1]
        changed = int((before != d.cache).view(-1, es).any(1).sum())
        # two rows of keys and values of every layer, no more: the cache held NaN there (all bits set), which no key has
        assert changed == 2 * 2 * cfg.n_layers * hs * cfg.d_head
    for a, b in zip(*results):
        assert torch.equal(a, b)


@pytest.mark.parametrize("name", ["gpt_f32_wide", "llama_f32_um", "llama_bf16"])
@pytest.mark.parametrize("listed", [True, False])
def test_what_a_workspace_held_changes_nothing(lib, name, listed):
    """Rows of no sequence, by the list and beyond the table: the others keep their bits whether the workspace held zeros or NaNs."""
    T, good = 192, 189
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    out = []
    for fill in (0, 0xff):
        d = Deployed(lib, name, good, 16)
        ws = torch.full((d.ctx.twist_decode_workspace_bytes(d.sub, d.pages, T, 16),), fill, dtype=torch.uint8, device="cuda")
        seq = i32(list(range(good)) + [-1, good, 2 ** 31 - 1]) if listed else None
        logits = d.ctx.twist_subnet_decode(d.sub, i32(list(range(T))), i32([1] * T), 16, d.pages, d.cache, ws, seq=seq)
        torch.cuda.synchronize()
        out.append(logits[:good].clone())
    assert torch.isfinite(out[0]).all() and torch.equal(*out)


@pytest.mark.parametrize("name", ["llama_f32_um", "gpt_bf16", "llama_bf16_um"])
def test_generation_as_it_is_used(lib, name):
    """Prompts of their own lengths, then 20 captured steps of three sequences: decode, rules on the logits, choice, bookkeeping on the device, with pages
    handed to the sequences as they grow.  What the steps computed is checked against the oracle on the finished sequences."""
    cfg = MODELS[name][0]
    V, S, top, page, steps = cfg.vocab, 3, 64, 8, 20
    start = [4, 30, 15]
    stream = torch.cuda.Stream()
    free = list(np.random.default_rng(1).permutation(S * top // page + 3))
    with torch.cuda.stream(stream):
        table = torch.full((S, top // page), -1, dtype=torch.int32, device="cuda")
        d = Deployed(lib, name, S, top, page=page, stream=stream, table=table)
        held = [0] * S

        def grow(s, n):                                             # pages for n tokens
            while held[s] * page < n:
                table[s, held[s]] = int(free.pop())
                held[s] += 1
        ids = si.tokens_uniform(V, S, top, 6)
        history = torch.zeros((S, top), dtype=torch.int32, device="cuda")
        lens = torch.tensor(start, dtype=torch.int32).cuda()
        for s in range(S):
            grow(s, start[s])
            history[s, :start[s]] = torch.tensor(ids[s][:start[s]]).cuda()
        rows = [(s, p) for s in range(S) for p in range(start[s])]
        # the last of each prompt is decoded by the first step
        rows = [(s, p) for s, p in rows if p < start[s] - 1]
        d.step([int(ids[s][p]) for s, p in rows], [p + 1 for _, p in rows], [s for s, _ in rows], top)
        words = (V + 31) // 32
        allowed = torch.full((S, words), -1, dtype=torch.int32, device="cuda")
        allowed[1, ::2] = 0                                          # a grammar that leaves every second word of ids
        g = torch.Generator(device="cuda").manual_seed(2)
        rules = lib.LogitRules(history=history, n_history=lens, n_prompt=torch.tensor(start, dtype=torch.int32).cuda(),
                               repetition=1.1 + 0.3 * torch.rand(S, generator=g, device="cuda"), frequency=0.1 * torch.rand(S, generator=g, device="cuda"),
                               presence=0.2 * torch.rand(S, generator=g, device="cuda"), bias_ids=torch.tensor([[3, 5], [64, 64], [9, -1]], dtype=torch.int32).cuda(),
                               bias_values=torch.tensor([[-2.0, 1.0], [5.0, 0.5], [0.3, 9.0]]).cuda(), allowed=allowed)
        tok, out = torch.zeros(S, dtype=torch.int32, device="cuda"), torch.zeros((S, V), device="cuda")
        logits = torch.zeros((S, (V + 7) // 8 * 8), dtype=d.ctx.torch_dtype, device="cuda")[:, :V]
        at = torch.arange(S, device="cuda")

        def step():
            tok.copy_(history[at, (lens - 1).long()])
            d.step(tok, lens, max_len=top, logits=logits)
            d.ctx.twist_logits_raw(logits, rules, out)
            history[at, lens.long()] = out.argmax(-1).to(torch.int32)
            lens.add_(1)
        keep = [x.clone() for x in (history, lens, d.cache)]
        step()                                                       # (workspace and the like exist afterwards)
        for x, y in zip((history, lens, d.cache), keep):
            x.copy_(y)
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step()
        seen = []
        for k in range(steps):
            for s in range(S):
                grow(s, start[s] + k)                                # the step writes token start + k - 1
            graph.replay()
            stream.synchronize()
            seen.append((logits.clone(), out.clone()))
            torch.randn(1 << 16, device="cuda").sum().item()         # the program's own eager work between replays
        # the same steps without the graph: the same bits
        for x, y in zip((history, lens, d.cache), keep):
            x.copy_(y)
        for k in range(steps):
            step()
            assert torch.equal(logits, seen[k][0]) and torch.equal(out, seen[k][1]), k
        stream.synchronize()
    hist = history.cpu().numpy()
    U = 2.0 ** -24
    for s in range(S):
        want = d.want(hist[s][:start[s] + steps - 1])
        got = np.stack([to_numpy(seen[k][0][s]) for k in range(steps)])
        assert rel_fro(got, want[start[s] - 1:]) <= _bound(cfg)
        for k in range(steps):                                       # the rules on the logits that the step had
            n, x = start[s] + k, got[k].copy()
            mag = np.abs(x)
            for c in set(hist[s][:n].tolist()):
                x[c] = x[c] / float(rules.keep["repetition"][s]) if x[c] > 0 else x[c] * float(rules.keep["repetition"][s])
                m = int((hist[s][start[s]:n] == c).sum())
                mag[c] = max(mag[c], abs(x[c])) + m + 1
                x[c] -= float(rules.keep["frequency"][s]) * m + (float(rules.keep["presence"][s]) if m else 0.0)
            for c, b in ({3: -2.0, 5: 1.0}, {64: 0.5}, {9: 0.3})[s].items():
                x[c] += b
                mag[c] += abs(b)
            if s == 1:
                x[(np.arange(V) // 32) % 2 == 0] = -np.inf
            o = to_numpy(seen[k][1][s])
            on = np.isfinite(x)
            assert np.array_equal(on, np.isfinite(o)) and (np.abs(o[on] - x[on]) <= 8 * U * mag[on]).all()
            assert hist[s][n] == int(np.argmax(o))


@pytest.mark.parametrize("per", [1, 3])
def test_captured_calls_serve_every_shorter_length(lib, per):
    """Appending and attention recorded once for up to 6000 tokens (a sequence cut into parts, rows of their own and drafted ones), replayed at other lengths with
    other inputs: the bits of calls of their own."""
    stream, g = torch.cuda.Stream(), torch.Generator(device="cuda").manual_seed(5)
    cfg = si.ModelCfg(arch="llama", d_model=64, n_heads=1, d_head=64, d_ff=8, vocab=8, rope=True, dtype="bf16")
    randn = lambda *s: torch.randn(s, generator=g, device="cuda").bfloat16()  # noqa: E731
    with torch.cuda.stream(stream):
        ctx = lib.Context(lib.desc_from_cfg(cfg), stream)
        k, v = randn(800, 2, 16, 64), randn(800, 2, 16, 64)
        cache = lib.PagedCache(k, v, torch.randperm(800, generator=g, device="cuda")[:750].to(torch.int32).view(2, 375))
        seq = (torch.arange(2 * per, device="cuda") // per).to(torch.int32)
        lens, qkv, q = torch.ones(2 * per, dtype=torch.int32, device="cuda"), randn(2 * per, 3 * 128), torch.empty((2 * per, 128), dtype=torch.bfloat16, device="cuda")
        assert ctx.twist_cache_attention_floats(cache, 2 * per, 6000) > 0

        def run():
            ctx.twist_cache_append_raw(cache, qkv, lens, seq=seq, q_out=q)
            return ctx.twist_cache_attention_raw(cache, q, lens, 6000, seq=seq)
        run()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            o, lse = run()
        for n in (6000, 1, 700, 5999, 3, 4096):
            lens.copy_(torch.tensor([max(1, n - per + 1) + i for i in range(per)] * 2, dtype=torch.int32))
            lens[-1] = 0 if n == 700 else lens[-1]
            qkv.copy_(randn(2 * per, 3 * 128))
            graph.replay()
            stream.synchronize()
            got = [x.clone() for x in (o, lse, k, v)]
            torch.randn(1 << 16, device="cuda").sum().item()         # the program's own eager work between replays
            want = run()
            stream.synchronize()
            for a, b in zip(got, (*want, k, v)):
                assert torch.equal(a, b), n


def test_another_stream_than_the_current_one(lib):
    """A context whose stream is not the current one: the calls' own temporaries live until their kernels are done."""
    stream, g = torch.cuda.Stream(), torch.Generator(device="cuda").manual_seed(3)
    cfg = si.ModelCfg(arch="llama", d_model=64, n_heads=1, d_head=128, d_ff=8, vocab=5000, rope=True, dtype="bf16")
    here, there = lib.Context(lib.desc_from_cfg(cfg)), lib.Context(lib.desc_from_cfg(cfg), stream)
    k, v = (torch.randn((130, 2, 64, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    cache = lib.PagedCache(k, v, torch.arange(128, dtype=torch.int32, device="cuda").view(1, -1))
    q = torch.randn((1, 256), generator=g, device="cuda").bfloat16()
    lens = torch.tensor([8000], dtype=torch.int32).cuda()
    assert here.twist_cache_attention_floats(cache, 1, 8192) > 0
    o, lse = here.twist_cache_attention_raw(cache, q, lens, 8192)
    torch.cuda.synchronize()
    for _ in range(20):
        o2, lse2 = there.twist_cache_attention_raw(cache, q, lens, 8192)
        junk = torch.full((2, 130 * 64), float("nan"), device="cuda")          # what a freed scratch would be taken for
        stream.synchronize()
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
        del junk


def test_results_that_are_dropped_on_another_stream(lib):
    """Memory of results that the current stream drops before the context's stream has written them is not handed out again till then."""
    stream, g = torch.cuda.Stream(), torch.Generator(device="cuda").manual_seed(3)
    cfg = si.ModelCfg(arch="llama", d_model=64, n_heads=1, d_head=128, d_ff=8, vocab=5000, rope=True, dtype="bf16")
    ctx = lib.Context(lib.desc_from_cfg(cfg), stream)
    k, v = (torch.randn((130, 8, 64, 128), generator=g, device="cuda").bfloat16() for _ in range(2))
    cache = lib.PagedCache(k, v, torch.arange(128, dtype=torch.int32, device="cuda").view(1, -1))
    q, lens = torch.randn((1, 1024), generator=g, device="cuda").bfloat16(), torch.tensor([8000], dtype=torch.int32).cuda()
    x, big = torch.randn((1, 5000), generator=g, device="cuda").bfloat16(), torch.empty(1 << 28, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(stream):
            for _ in range(8):
                big.fill_(1.0)                                       # the calls wait behind these
        ctx.twist_cache_attention_raw(cache, q, lens, 8192)
        ctx.twist_logits_raw(x, lib.LogitRules())
        mine = [torch.full(s, 3.0, dtype=t, device="cuda") for s, t in (((1, 1024), torch.bfloat16), ((1, 8), torch.float32), ((1, 5000), torch.float32))]
        torch.cuda.synchronize()
        assert all((m == 3).all() for m in mine)


def test_decode_refusals(lib):
    d = Deployed(lib, "gpt_bf16", 2, 64)
    ok = dict(tokens=[1, 2], lens=[1, 1])

    def refused(status, f):
        with pytest.raises(lib.TwistError) as e:
            f()
        assert e.value.status == status and "twist_" in str(e.value)
    refused(3, lambda: d.ctx.twist_decode_workspace_bytes(d.sub, d.pages, 2, 193))             # beyond max_seq
    refused(3, lambda: d.ctx.twist_decode_workspace_bytes(d.sub, d.pages, 2, 0))
    refused(1, lambda: d.ctx.twist_decode_workspace_bytes(d.sub, d.pages, 0, 64))
    ws = torch.empty(d.ctx.twist_decode_workspace_bytes(d.sub, d.pages, 2, 64), dtype=torch.uint8, device="cuda")
    i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
    call = lambda ctx=d.ctx, cache=d.cache, ws=ws, T=2, **kw: ctx.twist_subnet_decode(d.sub, i32([1] * T), i32([1] * T), 64, d.pages, cache, ws, **kw)  # noqa: E731
    call()
    refused(3, lambda: call(ws=ws[:-256]))
    refused(3, lambda: call(T=40))                                                             # a workspace for fewer rows
    refused(3, lambda: call(cache=d.cache[:-256]))
    refused(3, lambda: call(cache=d.cache[1:]))
    refused(1, lambda: call(ctx=lib.Context(lib.desc_from_cfg(d.cfg))))                        # another context's subnet
    with pytest.raises(lib.TwistError):
        call(seq=i32([0]))
    with pytest.raises(lib.TwistError):
        call(logits=torch.empty((2, 1003), device="cuda"))                                     # fp32 logits of a bf16 model
    bad = lib.Pages(d.table, d.pages.n_pages, 24)
    refused(3, lambda: d.ctx.twist_cache_bytes(d.sub, bad))
    assert d.step(**ok).shape == (2, 1003)
    torch.cuda.synchronize()
