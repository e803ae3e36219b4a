"""The operators around a rollout's cache and its logits as they are used: one after the other, in graphs, on
other streams, with more sequences than a block has threads, over a cache longer than 32-bit offsets."""
from __future__ import annotations

import importlib.util
import sys
from pathlib import Path

import numpy as np
import pytest

import cache_reference as ref
import decode_reference as dec
from test_gpu_cache import MASS, call_evict, call_mass, check_evict, check_mass, evict_inputs, i32, mass_inputs, outputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch

    import paper_2609_14636_gb300 as stride

    return torch, stride, torch.device("cuda")


def test_a_run(env):
    """Append, attention, weights, eviction, attention over what remained, controls, sampling: each from what the one before left."""
    torch, stride, dev = env
    g = torch.Generator(device="cuda").manual_seed(3)
    B, Hq, Hk, D, page, pages, V = 3, 8, 2, 64, 16, 12, 1000
    bf16 = lambda *n: torch.randn(n, generator=g, device=dev).bfloat16()  # noqa: E731
    pools, spare = [bf16(B * pages, page, Hk, D) for _ in range(2)], [torch.zeros(B * pages, page, Hk, D, dtype=torch.bfloat16, device=dev) for _ in range(2)]
    table = torch.randperm(B * pages, generator=g, device=dev).int().view(B, pages)
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    ctx, mass = torch.zeros(B, dtype=torch.int32, device=dev), torch.full((B, Hk, pages * page), float("nan"), device=dev)
    K, W, M = [np.zeros((B, 0, Hk, D)) for _ in range(2)] + [np.zeros((B, Hk, 0))]

    def step(n, decay):
        """n new tokens of each sequence."""
        nonlocal ctx, K, W, M
        N = B * n
        q, k, v = bf16(N, Hq, D), bf16(N, Hk, D), bf16(N, Hk, D)
        off = torch.arange(0, N + 1, n, dtype=torch.int32, device=dev)
        out, lse = torch.empty_like(q), torch.empty(N, Hq, device=dev)
        ws = torch.empty(stride.stride_tree_attention_workspace_size(N, Hq, Hk, D), dtype=torch.uint8, device=dev)
        stride.stride_kv_append(k, v, *pools, table, ctx, off, dev_status=status)
        stride.stride_tree_attention(q, *pools, table, ctx, off, None, 0.125, out, lse=lse, workspace=ws, dev_status=status)
        stride.stride_attention_mass(q, lse, pools[0], table, ctx, off, None, 0.125, mass, decay=decay, dev_status=status)
        c = K.shape[1]
        K, W = np.concatenate([K, dec.f64(k).reshape(B, n, Hk, D)], 1), np.concatenate([W, dec.f64(v).reshape(B, n, Hk, D)], 1)
        sees = (np.arange(c + n) - c)[None] <= np.arange(n)[:, None]
        now = np.zeros((B, Hk, c + n))
        for b in range(B):
            for h in range(Hk):
                rows, heads = slice(b * n, (b + 1) * n), slice(h * 4, (h + 1) * 4)
                now[b, h], tol = ref.mass(M[b, h], dec.f64(q)[rows, heads], dec.f64(lse)[rows, heads], K[b, :, h], c, sees, 0.125, decay)
                assert (np.abs(dec.f64(mass)[b, h, :c + n] - now[b, h]) <= tol).all()
                o, z, size = dec.attention(dec.f64(q)[b * n, h * 4], K[b, :, h], W[b, :, h], sees[0], 0.125)
                assert (np.abs(dec.f64(out)[b * n, h * 4] - o) <= 2.0 ** -8 * (size + np.abs(o)) + 2e-5 * size).all()
        M = dec.f64(mass)[:, :, :c + n]  # (what is there is what is chosen from)
        ctx = ctx + n

    step(70, 0.0)  # the prompt: the first vote
    for _ in range(3):
        step(1, 0.9)
    new_len, kept, mass_to = torch.empty_like(ctx), torch.empty(B, Hk, 32, dtype=torch.int32, device=dev), torch.full_like(mass, float("nan"))
    stride.stride_kv_evict(*pools, table, ctx, mass, 24, *spare, table, new_len, kept, mass_to=mass_to, sink=2, recent=5, dev_status=status)
    at = np.stack([[ref.remaining(M[b, h].astype(np.float32), 73, 24, 2, 5) for h in range(Hk)] for b in range(B)])
    assert new_len.tolist() == [24] * B and np.array_equal(kept[:, :, :24].cpu().numpy(), at)
    pools[:], mass, ctx = spare, mass_to, new_len
    i = np.arange(Hk)
    K, W = (np.stack([x[b][at[b].T, i] for b in range(B)]) for x in (K, W))
    M = np.take_along_axis(M, at, 2)
    step(1, 0.9)
    step(2, 0.9)
    assert ctx.tolist() == [27] * B and int(status) == 0

    # the same two rows' logits with a token that was said banned by its penalty, the mask leaving three
    x, out = bf16(2, V), torch.empty(2, V, dtype=torch.bfloat16, device=dev)
    allowed = np.zeros((1, V), bool)
    allowed[0, [10, 500, 999]] = True
    words = torch.tensor(np.packbits(np.pad(allowed, ((0, 0), (0, 24))), axis=1, bitorder="little").view(np.int32), device=dev)
    x[:, 10] = 9.0
    history = i32(torch, [[10, 10, 3], [4, 5, 6]])
    stride.stride_logit_controls(x, out, history=history, history_len=i32(torch, [3, 3]), frequency=20.0, allowed=words, dev_status=status)
    token, state = torch.empty(2, dtype=torch.int32, device=dev), stride.new_state(2)
    stride.stride_sample(out, None, token, temperature=0.0, dev_status=status)
    assert int(token[1]) == 10 and int(token[0]) in (500, 999)
    scored = {"logp_s": torch.empty(2, device=dev)}  # the raw logits are there for the scoring step
    stride.stride_score_step(x, x, token, torch.zeros(2, dtype=torch.uint8, device=dev), stride.TURN_MEAN, -1e9, state, out=scored)
    want = x.double().log_softmax(1).gather(1, token.long()[:, None])[:, 0]
    assert (scored["logp_s"].double() - want).abs().max() < 2e-3 and int(status) == 0


@pytest.mark.parametrize("case", [MASS[2], MASS[12], MASS[8]], ids=str)
def test_mass_in_graphs_and_streams(env, case):
    """Two graphs of the call on two streams at once, replayed on new data; the results of the plain call."""
    torch, stride, dev = env
    x, y = mass_inputs(torch, case, 1), mass_inputs(torch, case, 2)
    want = []
    for z in (x, y):
        m = z["mass"].clone()
        call_mass(stride, torch, z, case, mass=m)
        call_mass(stride, torch, z, case, mass=m)
        want.append(m)
    args = [(i32(torch, z["table"]), i32(torch, [c for c, _ in case[0]]), i32(torch, z["off"])) for z in (x, y)]
    graphs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for z, a, s in zip((x, y), args, streams):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            stride.stride_attention_mass(z["q"], z["lse"], z["k"], *a, z["mask"], z["scale"], z["mass"], decay=case[7])
        graphs.append(graph)
    for _ in range(2):
        for graph, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(x["mass"], want[0]) and torch.equal(y["mass"], want[1])


def test_evict_and_controls_in_graphs(env):
    torch, stride, dev = env
    case = ([370, 16, 5000, 0], 64, 2, 64, 16, 16, "rows", 2, 9, "bf16")
    x = evict_inputs(torch, case, "ties")
    before = outputs(x)
    a = i32(torch, x["table"]), i32(torch, case[0])
    to = i32(torch, x["to_table"])
    V = 30_000
    logits, out = torch.randn(3, V, device=dev), torch.zeros(3, V, device=dev)
    history, length = torch.randint(0, V, (3, 600), device=dev, dtype=torch.int32), i32(torch, [600, 0, 17])
    bias = dict(bias_off=i32(torch, [0, 2, 2, 4]), bias_token=i32(torch, [5, 5, 9, 1]), bias=torch.tensor([1.0, 2.0, 3.0, -4.0], device=dev))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        stride.stride_kv_evict(x["k"], x["v"], *a, x["mass"], 64, x["k_to"], x["v_to"], to, x["new_len"], x["kept"], mass_to=x["mass_to"], sink=2, recent=9)
        stride.stride_logit_controls(logits, out, history=history, history_len=length, repetition=1.5, frequency=0.1, **bias)
    for seed in (5, 6):  # replayed on new values
        x["mass"].copy_(evict_inputs(torch, case, "spread", seed)["mass"])
        logits.copy_(torch.randn(3, V, device=dev))
        history.copy_(torch.randint(0, V, (3, 600), device=dev, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        check_evict(torch, x, case, before)
        other = torch.empty_like(out)
        stride.stride_logit_controls(logits, other, history=history, history_len=length, repetition=1.5, frequency=0.1, **bias)
        assert torch.equal(out, other)
        for name, t in before.items():
            x[name].copy_(t)
    # a stream of their own
    with torch.cuda.stream(s):
        call_evict(stride, torch, x, case)
    other = torch.empty_like(out)
    torch.cuda.synchronize()
    stride.stride_logit_controls(logits, other, history=history, history_len=length, repetition=1.5, frequency=0.1, **bias, stream=s)
    s.synchronize()
    check_evict(torch, x, case, before)
    assert torch.equal(out, other)


@pytest.mark.parametrize("case", [
    ([(3 + i % 40, 1) for i in range(1500)], 2, 2, 64, 16, "rows", False, 1.0, "bf16"),
    ([(3 + i % 400, i % 3 * 20) for i in range(1300)], 4, 1, 64, 16, "rows", False, 0.5, "bf16"),
    ([(i % 50, i % 5) for i in range(900)], 24, 1, 64, 16, "rows", True, 0.5, "f16")], ids=lambda c: f"{len(c[0])} sequences, {c[1]}")
def test_many_sequences(env, case):
    torch, stride, dev = env
    x = mass_inputs(torch, case)
    before = x["mass"].double().cpu().numpy()
    call_mass(stride, torch, x, case)
    after = x["mass"].double().cpu().numpy()
    some = np.random.default_rng(0).permutation(len(case[0]))[:60].tolist() + [0, len(case[0]) - 1]
    check_mass(x, case, before, after, skip=set(range(len(case[0]))) - set(some))


def test_offsets_past_32_bits(env):
    """A cache of 6 GB whose last pages are used: elements past 2^31, for both kernels of the weights and the eviction."""
    torch, stride, dev = env
    Hk, D, page = 8, 128, 64
    pages = 2 ** 31 // (page * Hk * D) + 6
    k = torch.zeros(pages, page, Hk, D, dtype=torch.bfloat16, device=dev)
    g = torch.Generator(device="cuda").manual_seed(1)
    k[-4:] = torch.randn(4, page, Hk, D, generator=g, device=dev).bfloat16()
    table, ctx = i32(torch, [[pages - 1, pages - 4, pages - 2]]), i32(torch, [100])
    small = k[-4:].clone()
    near = i32(torch, [[3, 0, 2]])
    for n in (1, 40):
        q = torch.randn(n, 16, D, generator=g, device=dev).bfloat16()
        off, lse = i32(torch, [0, n]), torch.randn(n, 16, generator=g, device=dev) + 3
        got = [torch.zeros(1, Hk, 192, device=dev) for _ in range(2)]
        stride.stride_attention_mass(q, lse, k, table, ctx, off, None, 0.1, got[0])
        stride.stride_attention_mass(q, lse, small, near, ctx, off, None, 0.1, got[1])
        assert torch.equal(got[0], got[1]) and (got[0][0, :, :100 + n] > 0).all()
    to = torch.zeros_like(small)
    new_len, kept = torch.empty(1, dtype=torch.int32, device=dev), torch.empty(1, Hk, 60, dtype=torch.int32, device=dev)
    stride.stride_kv_evict(k, k, table, ctx, got[0], 60, to, torch.empty_like(to), i32(torch, [[1]]), new_len, kept)
    for h in range(Hk):
        at = kept[0, h].long()
        assert torch.equal(to[1, :60, h], small[near[0].long()[at // page], at % page, h])
    stride.stride_kv_evict(small, small, near, ctx, got[0], 60, k, k, i32(torch, [[pages - 3]]), new_len, kept)
    for h in range(Hk):
        at = kept[0, h].long()
        assert torch.equal(k[-3, :60, h], small[near[0].long()[at // page], at % page, h])


def test_the_example_under_a_budget(env, capsys):
    """With a budget that is never reached the cache is whole; with one, rollouts go on, and repeated tokens get rarer with the penalty."""
    torch, stride, dev = env
    path = Path(__file__).resolve().parents[1] / "examples" / "rollout.py"
    spec = importlib.util.spec_from_file_location("rollout_example_budget", path)
    example = importlib.util.module_from_spec(spec)
    sys.modules[spec.name] = example
    spec.loader.exec_module(example)
    prompts = torch.randint(0, 4096, (4, 30), generator=torch.Generator(device="cuda").manual_seed(5), device="cuda").int()
    _, none, cached = example.write_on(example.Model(example.Shape(), 4, 1), prompts, 40, 100, seed=1)
    assert none == 0 and cached.tolist() == [69] * 4
    tokens, some, cached = example.write_on(example.Model(example.Shape(), 4, 1), prompts, 90, 24, seed=1)
    assert some >= 3 and int(cached.max()) <= 48 and int(tokens.min()) >= 0
    allowed = torch.zeros(1, 128, dtype=torch.int32, device=dev)
    allowed[0, 3] = -1  # tokens 96 .. 127
    tokens, _, _ = example.write_on(example.Model(example.Shape(), 4, 1), prompts, 20, 100, seed=2, repetition=1.0, presence=1000.0, allowed=allowed)
    assert int(tokens.min()) >= 96 and int(tokens.max()) < 128
    assert all(len(set(row)) == 20 for row in tokens.tolist())  # no token twice
