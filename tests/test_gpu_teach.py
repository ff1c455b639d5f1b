"""Subnets that learn from a teacher, and tokens that are drawn step by step: the operators behind a model's logits as they are used together (lists of the whole model's top logits,
training passes against them, draws in a generation loop, captured and replayed, on other streams).

The training pass against a teacher is held to the oracle with the bounds of the pass against targets (test_gpu_train.py): the loss's gradient enters the same way."""
import math
from dataclasses import replace

import numpy as np
import pytest
import torch

import synth_inputs as si
from helpers import rel_fro_of_numbers, subnet_to_numpy, to_device
from oracle import model as omodel, move as omove
from test_gpu_distill import _want
from test_gpu_draw import _draw_want
from test_gpu_generate import Deployed, _bound
from test_gpu_train import CASES, GRAD, _check_bf16_grads, _compare_grads, _data, _round_hook, _setup

pytestmark = pytest.mark.gpu


def _loss_of(lists, tau, weight):
    """The oracle's loss against a teacher's lists: mean over rows, and the gradient of the mean."""
    ids, values, rest = (t.double().cpu().numpy() for t in lists)

    def loss(logits, tgt):
        flat, out, total = logits.reshape(-1, logits.shape[-1]), np.zeros((tgt.size, logits.shape[-1])), 0.0
        for t, y in enumerate(tgt.reshape(-1)):
            row, _, g, _ = _want(flat[t], int(y), ids[t].astype(np.int64), values[t], rest[t], tau, weight)
            total += row
            out[t] = g
        return total / tgt.size, (out / tgt.size).reshape(logits.shape)
    return loss


def _whole(lib, ctx, cfg, fw):
    """The central model as a subnet of all blocks: the teacher."""
    plan = ctx.twist_sample(1, cfg.n_heads, cfg.n_ffn_units, seed=1, require_coverage=False)
    return plan, ctx.twist_extract(plan, fw, 0)


@pytest.mark.parametrize("name", ["gpt_f32", "llama_f32", "ragged_f32", "gpt_bf16", "llama_bf16", "gpt_bf16_bigvocab"])
def test_top_logits_of_a_model(lib, name):
    """Against the oracle's logits: every value within the bound of a logit of the id that it names, and no logit outside the list above its smallest by more."""
    cfg, S, B, N, full_np, _, ctx, _, _, fw = _setup(lib, name)
    x_np, _, x, _ = _data(cfg, B, N, 3)
    plan, sub = _whole(lib, ctx, cfg, fw)
    ws = torch.full((ctx.twist_workspace_bytes(sub, B, N),), 0xff, dtype=torch.uint8, device="cuda")
    k, tau = min(13, cfg.vocab - 1), 1.7
    ids, values, rest = ctx.twist_subnet_top_logits(sub, x, k, ws, temperature=tau)
    kept = []

    def hook(tag, a):
        if tag == "logits":
            kept.append(np.array(a))
        return a
    omodel.forward_backward(cfg, full_np, x_np, np.zeros_like(x_np), q=hook, need_grads=False)
    want = kept[0].reshape(B * N, -1)
    off = _bound(cfg) * np.sqrt((want ** 2).mean()) * 8                  # (a root mean square over all; the largest of a million normal errors is 5 of theirs)
    ids, values, rest = ids.cpu().numpy(), values.double().cpu().numpy(), rest.double().cpu().numpy()
    assert (np.diff(values, axis=1) <= 0).all() and (ids >= 0).all() and all(len(set(r)) == k for r in ids)
    assert np.abs(np.take_along_axis(want, ids, 1) - values).max() <= off
    others = want.copy()
    np.put_along_axis(others, ids, -np.inf, 1)
    assert (others.max(1) <= values[:, -1] + off).all()
    m = others.max(1, keepdims=True)
    assert np.abs((m / tau)[:, 0] + np.log(np.exp((others - m) / tau).sum(1)) - rest).max() <= off / tau + 1e-5


@pytest.mark.parametrize("tau,weight", [(1.0, 1.0), (2.0, 0.5)])
@pytest.mark.parametrize("name", ["gpt_f32", "llama_f32", "ragged_f32", "gpt_bf16", "llama_bf16", "gpt_f32_um", "llama_bf16_um"])
def test_training_pass_against_a_teacher_matches_oracle(lib, name, tau, weight):
    cfg, S, B, N, full_np, _, ctx, plan, oplan, fw = _setup(lib, name)
    x_np, y_np, x, y = _data(cfg, B, N, 3)
    whole, teacher_sub = _whole(lib, ctx, cfg, fw)
    ws = torch.full((ctx.twist_workspace_bytes(teacher_sub, B, N),), 0xff, dtype=torch.uint8, device="cuda")
    lists = ctx.twist_subnet_top_logits(teacher_sub, x, min(20, cfg.vocab - 1), ws, temperature=tau)
    lists[1].mul_(3.0)                                                   # (a teacher with opinions: the weights are random)
    teacher = lib.Teacher(*lists, temperature=tau, weight=weight)
    loss = torch.zeros(1, device="cuda")
    bf = cfg.dtype == "bf16"
    for s in range(S):
        sub = ctx.twist_extract(plan, fw, s, store=lib.STORE_GRADS)
        ws = torch.full((ctx.twist_workspace_bytes(sub, B, N),), 0xff, dtype=torch.uint8, device="cuda")
        ctx.twist_subnet_fwd_bwd_distill(sub, x, None if weight == 1.0 else y, teacher, ws, loss)
        torch.cuda.synchronize()
        osub = omove.extract(full_np, oplan, s, cfg.d_head, cfg.ffn_granule)
        got = subnet_to_numpy(sub, cfg, GRAD)
        of = _loss_of(lists, tau, weight)
        oloss, ograds = omodel.forward_backward(cfg, osub, x_np, y_np, loss_of=of)
        assert abs(loss.item() - oloss) <= (5e-3 if bf else 1e-4) * abs(oloss), (loss.item(), oloss)
        if bf:
            _, rgrads = omodel.forward_backward(cfg, osub, x_np, y_np, q=_round_hook, loss_of=of)
            _check_bf16_grads(cfg, got, ograds, rgrads, f"{name} s={s}")
        else:
            _compare_grads(cfg, got, ograds, 1e-4, name)


def test_pass_with_no_weight_on_the_teacher_is_the_pass_against_targets(lib):
    """Loss and gradients of twist_subnet_fwd_bwd, but for the rounding of the logits' gradient, which two kernels form."""
    cfg, S, B, N, full_np, _, ctx, plan, oplan, fw = _setup(lib, "gpt_f32")
    _, _, x, y = _data(cfg, B, N, 3)
    sub = ctx.twist_extract(plan, fw, 0, store=lib.STORE_GRADS)
    ws = torch.empty(ctx.twist_workspace_bytes(sub, B, N), dtype=torch.uint8, device="cuda")
    loss = torch.zeros(2, device="cuda")
    ctx.twist_subnet_fwd_bwd(sub, x, y, ws, loss[:1])
    want = subnet_to_numpy(sub, cfg, GRAD)
    lists = ctx.twist_subnet_top_logits(sub, x, 5, ws)
    ctx.twist_subnet_fwd_bwd_distill(sub, x, y, lib.Teacher(*lists, weight=0.0), ws, loss[1:])
    got = subnet_to_numpy(sub, cfg, GRAD)
    assert abs(loss[0] - loss[1]) <= 1e-6 * loss[0]
    for l in range(cfg.n_layers):
        for k, w in want["layers"][l].items():
            if k != "bk":                                                # (zero but for roundings)
                assert rel_fro_of_numbers(got["layers"][l][k], w) <= 1e-5, (l, k)
    for k, w in want["globals"].items():
        assert rel_fro_of_numbers(got["globals"][k], w) <= 1e-5, k


def test_passes_refuse_what_does_not_fit(lib):
    cfg, S, B, N, full_np, _, ctx, plan, _, fw = _setup(lib, "gpt_f32")
    _, _, x, y = _data(cfg, B, N, 3)
    sub = ctx.twist_extract(plan, fw, 0, store=lib.STORE_GRADS)
    ws = torch.empty(ctx.twist_workspace_bytes(sub, B, N), dtype=torch.uint8, device="cuda")
    loss = torch.zeros(1, device="cuda")
    ids, values, rest = ctx.twist_subnet_top_logits(sub, x, 5, ws)
    ok = lib.Teacher(ids, values, rest, weight=0.5)
    bare = ctx.twist_extract(plan, fw, 0)
    other = lib.Context(lib.desc_from_cfg(cfg))
    for call in (lambda: ctx.twist_subnet_top_logits(sub, x, 0, ws), lambda: ctx.twist_subnet_top_logits(sub, x, 1025, ws), lambda: ctx.twist_subnet_top_logits(sub, x, 5, ws, temperature=0.0),
                 lambda: ctx.twist_subnet_top_logits(sub, x, 5, ws[:256]), lambda: ctx.twist_subnet_top_logits(sub, x, 5, ws[1:]), lambda: ctx.twist_subnet_top_logits(sub, x.long(), 5, ws),
                 lambda: ctx.twist_subnet_top_logits(sub, x.t(), 5, ws), lambda: ctx.twist_subnet_top_logits(sub, torch.zeros((1, cfg.max_seq + 1), dtype=torch.int32, device="cuda"), 5, ws),
                 lambda: other.twist_subnet_top_logits(sub, x, 5, ws),
                 lambda: ctx.twist_subnet_fwd_bwd_distill(sub, x, None, ok, ws, loss), lambda: ctx.twist_subnet_fwd_bwd_distill(sub, x, y[:, :-1].contiguous(), ok, ws, loss),
                 lambda: ctx.twist_subnet_fwd_bwd_distill(sub, x[:1].contiguous(), y[:1].contiguous(), ok, ws, loss), lambda: ctx.twist_subnet_fwd_bwd_distill(sub, x, y, ok, ws[:1024], loss),
                 lambda: ctx.twist_subnet_fwd_bwd_distill(bare, x, y, ok, ws, loss), lambda: ctx.twist_subnet_fwd_bwd_distill(sub, x, y, ok, ws, loss.double()),
                 lambda: ctx.twist_subnet_fwd_bwd_distill(sub, x, y, lib.Teacher(ids, values, rest, weight=-1.0), ws, loss), lambda: other.twist_subnet_fwd_bwd_distill(sub, x, y, ok, ws, loss)):
        with pytest.raises(lib.TwistError):
            call()
    block = replace(si.CFG1, n_layers=1)
    bctx = lib.Context(lib.desc_from_cfg(block))
    full = to_device(si.make_weights(block, 0), block)
    bplan = bctx.twist_sample(1, block.n_heads, block.n_ffn_units, seed=0)
    bsub = bctx.twist_extract(bplan, lib.FullWeights(full["layers"], full["globals"]), 0, store=lib.STORE_GRADS)
    bws = torch.empty(bctx.twist_workspace_bytes(bsub, 1, 8), dtype=torch.uint8, device="cuda")
    tok = torch.zeros((1, 8), dtype=torch.int32, device="cuda")
    with pytest.raises(lib.TwistError):
        bctx.twist_subnet_top_logits(bsub, tok, 5, bws)
    with pytest.raises(lib.TwistError):
        bctx.twist_subnet_fwd_bwd_distill(bsub, tok, tok, lib.Teacher(ids[:8], values[:8], rest[:8], weight=0.5), bws, loss)


@pytest.mark.parametrize("name", ["gpt_f32", "gpt_bf16", "llama_bf16"])
def test_learning_from_a_teacher_captured_and_replayed(lib, name):
    """The teacher's lists, a pass against them and a step, recorded once on a stream of its own and replayed with eager work in between: the losses and weights of the same steps run eagerly."""
    cfg, S, hs, fs, B, N = CASES[name]
    full_np = si.make_weights(cfg, 3, std=0.05, generic=True)
    _, _, x, y = _data(cfg, B, N, 5)
    stream = torch.cuda.Stream()
    results = {}
    for mode in ("eager", "graph"):
        full_t = to_device(full_np, cfg)
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            ctx = lib.Context(lib.desc_from_cfg(cfg))
            fw = lib.FullWeights(full_t["layers"], full_t["globals"])
            plan = ctx.twist_sample(S, hs, fs, seed=4)
            sub = ctx.twist_extract(plan, fw, 0, store=lib.STORE_GRADS)
            whole, teacher_sub = _whole(lib, ctx, cfg, fw)
            ws = torch.empty(ctx.twist_workspace_bytes(teacher_sub, B, N), dtype=torch.uint8, device="cuda")
            loss = torch.zeros(1, device="cuda")

            def step():
                lists = ctx.twist_subnet_top_logits(teacher_sub, x, 10, ws, temperature=2.0)
                ctx.twist_subnet_fwd_bwd_distill(sub, x, y, lib.Teacher(*lists, temperature=2.0, weight=0.5), ws, loss)
                ctx.twist_subnet_step(sub, lib.OPT_SGD, lr=1e-2)
                return lists

            step()
            stream.synchronize()
            losses = [loss.item()]
            if mode == "graph":
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=stream):
                    kept = step()
            for _ in range(4):
                if mode == "graph":
                    g.replay()
                else:
                    kept = step()
                stream.synchronize()
                losses.append(loss.item())
                torch.randn(1 << 20, device="cuda").sum().item()
            results[mode] = (losses, [t.clone() for t in kept], subnet_to_numpy(sub, cfg))
    assert results["eager"][0] == results["graph"][0] and all(math.isfinite(v) for v in results["eager"][0])
    assert all(torch.equal(a, b) for a, b in zip(results["eager"][1], results["graph"][1]))
    for l in range(cfg.n_layers):
        for k, w in results["eager"][2]["layers"][l].items():
            assert rel_fro_of_numbers(results["graph"][2]["layers"][l][k], w) <= 1e-6, (l, k)    # (the token embedding's gradient is summed in any order)


@pytest.mark.parametrize("name", ["gpt_bf16", "llama_f32_um", "gpt_f32_wide"])
@pytest.mark.parametrize("captured", [False, True])
def test_generation_loop(lib, name, captured):
    """Decode, rules on the logits, a draw whose tokens are the next step's, for sequences of one batch with settings of their own, an unused row among them: every token and every log-probability is
    what the step's logits say, captured or not."""
    n, top = 5, 64
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        d = Deployed(lib, name, n, top, stream=stream)
        cfg, ctx, V = d.cfg, d.ctx, d.cfg.vocab
        i32 = lambda v: torch.tensor(v, dtype=torch.int32).cuda()  # noqa: E731
        f32 = lambda v: torch.tensor(v, dtype=torch.float32).cuda()  # noqa: E731
        tokens, lens, more = i32([1, 2, 3, 4, 0]), i32([1, 1, 1, 1, 0]), i32([1, 1, 1, 1, 0])
        history = torch.zeros((n, top), dtype=torch.int32, device="cuda")
        rules = lib.LogitRules(history=history, n_history=lens, repetition=f32([1.2] * n), presence=f32([0.1] * n))
        settings = dict(temperature=f32([0.0, 1.0, 0.7, 2.0, 1.0]), top_k=i32([0, 40, 0, 5, 3]), top_p=f32([1.0, 0.9, 0.8, 1.0, 0.5]), min_p=f32([0.0, 0.0, 0.02, 0.0, 0.0]))
        draw = lib.DrawRules(**settings)
        uniform = torch.zeros(n, device="cuda")
        logits, ruled = torch.zeros((n, V), dtype=ctx.torch_dtype, device="cuda"), torch.zeros((n, V), device="cuda")
        logprobs, kept = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.int32, device="cuda")
        rows = torch.arange(n, device="cuda")

        def step():
            history[rows, (lens.long() - 1).clamp(min=0)] = tokens
            d.step(tokens, lens, logits=logits)
            ctx.twist_logits_raw(logits, rules, out=ruled)
            ctx.twist_draw_raw(ruled, uniform, draw, tokens=tokens, logprobs=logprobs, kept=kept)
            lens.add_(more)

        g = torch.Generator(device="cuda").manual_seed(3)
        for it in range(12):
            torch.rand(n, generator=g, device="cuda", out=uniform)
            if captured and it == 1:
                stream.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    step()
            if captured and it:
                graph.replay()
            else:
                step()
            stream.synchronize()
            x = ruled.double().cpu().numpy()
            for r in range(n - 1):
                want = _draw_want(x[r], float(uniform[r]), *(float(s[r]) if s.dtype == torch.float32 else int(s[r]) for s in (settings["temperature"], settings["top_k"], settings["top_p"],
                                                                                                                      settings["min_p"])))
                assert (int(tokens[r]), int(kept[r])) == (want[0], want[2]) and abs(float(logprobs[r]) - want[1]) <= 1e-6 * (1 + abs(want[1])), (it, r)
        assert lens.tolist() == [13, 13, 13, 13, 0]


def test_calls_at_the_same_time_on_two_streams(lib):
    """Two contexts, a stream each, the current one a third: results are ready behind their own stream, and no call shares memory with another."""
    from test_gpu_draw import _ctx, _gen, _logits
    V, T = 50257, 64
    g = _gen(3)
    xs = [_logits(g, T, V) for _ in range(2)]
    us = [torch.rand(T, generator=g, device="cuda") for _ in range(2)]
    p = torch.full((T,), 0.9, device="cuda")
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    main = _ctx(lib, V)
    want = []
    for x, u in zip(xs, us):
        lists = main.twist_top_logits_raw(x, 40)
        want.append((*main.twist_draw_raw(x, u, lib.DrawRules(top_p=p)), *lists, *main.twist_distill_raw(x, y, lib.Teacher(*lists, weight=0.5))))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    ctxs = [_ctx(lib, V, stream=s) for s in streams]
    for _ in range(3):
        got = [[], []]
        for i in (0, 1):
            lists = ctxs[i].twist_top_logits_raw(xs[i], 40)
            got[i] = (*ctxs[i].twist_draw_raw(xs[i], us[i], lib.DrawRules(top_p=p)), *lists, *ctxs[i].twist_distill_raw(xs[i], y, lib.Teacher(*lists, weight=0.5)))
        for s in streams:
            torch.cuda.current_stream().wait_stream(s)
        for a, b in zip(want, got):
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_results_are_the_same_every_time(lib):
    from test_gpu_draw import _ctx, _gen, _logits, _rules
    from test_gpu_distill import _targets, _teacher
    for V in (1003, 50257, 70000):
        ctx, g = _ctx(lib, V), _gen(V)
        T = 40
        x = _logits(g, T, V)
        u, rules = torch.rand(T, generator=g, device="cuda"), lib.DrawRules(**_rules(g, T, V, "tkpm"))
        ids, values, rest = _teacher(g, x, 30, 2.0)
        y, teacher = _targets(g, ids, V), lib.Teacher(ids, values, rest, temperature=2.0, weight=0.5)
        run = lambda: (*ctx.twist_draw_raw(x, u, rules), *ctx.twist_top_logits_raw(x, 50), *ctx.twist_distill_raw(x, y, teacher))  # noqa: E731
        want = run()
        for _ in range(5):
            assert all(torch.equal(a, b) for a, b in zip(want, run()))
