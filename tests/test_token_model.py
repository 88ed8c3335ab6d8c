"""The serving operators together: a small decoder against the same model in 64 bits, and against itself by other routes."""
import math

import pytest
import torch

from paper_2302_00282_amd import tokens as T
from workloads import token_model as M

SIZES = M.Sizes(layers=2, width=96, hidden=200, heads=6, kv_heads=2, head_dim=32, vocab=517, page=16)
# the tolerance of the repository's bf16 path for whole networks, relative to the largest value
TOL = 2e-2


def quantized(x):
    a = x.abs().amax(-1, keepdim=True).clamp_min(2.0 ** -100)
    return torch.round(x * 127 / a) * a / 127


def by_definition(weights, tokens):
    """Logits of one sequence in 64 bits: weights, activations and cache rounded as the formulas say, nothing else rounded."""
    s, w = SIZES, {k: v.double().cpu() for k, v in weights.items()}
    product = lambda x, name, norm=None: (quantized(x) if norm is None else quantized(x * w[norm]) / torch.sqrt(x.square().mean(-1, keepdim=True) + s.eps)) @ quantized(w[name]).t()
    x = weights["embed"].bfloat16().double().cpu()[tokens.cpu()]
    n = len(x)
    hidden = torch.ones(n, n, dtype=torch.bool).triu(1)
    for i in range(s.layers):
        qkv = product(x, f"{i}.qkv", f"{i}.norm1").view(n, -1, s.head_dim)
        q, k, v = qkv[:, :s.heads], quantized(qkv[:, s.heads:s.heads + s.kv_heads]), quantized(qkv[:, s.heads + s.kv_heads:])
        k, v = (t.repeat_interleave(s.heads // s.kv_heads, 1).transpose(0, 1) for t in (k, v))
        p = torch.softmax((q.transpose(0, 1) @ k.transpose(1, 2) / math.sqrt(s.head_dim)).masked_fill(hidden, -math.inf), -1)
        x = x + product((p @ v).transpose(0, 1).reshape(n, -1), f"{i}.out")
        x = x + product(product(x, f"{i}.up", f"{i}.norm2").clamp_min(0), f"{i}.down")
    return product(x, "logits", "final.norm")


def near(got, want):
    return ((got.double().cpu() - want.double().cpu()).abs().max() / want.double().abs().max()).item() <= TOL


@pytest.fixture(scope="module")
def case():
    weights = M.draw(SIZES, 3)
    g = torch.Generator().manual_seed(7)
    return weights, torch.randint(0, SIZES.vocab, (53,), generator=g).cuda(), [torch.randint(0, SIZES.vocab, (n,), generator=g).cuda() for n in (9, 1, 30)]


@pytest.mark.gpu
def test_prompts_match_the_model_in_64_bits(case):
    weights, shared, own = case
    model = M.TokenModel(SIZES, weights, len(own), 64, len(shared))
    first = model.begin(shared)
    assert near(first, by_definition(weights, shared))
    logits = model.append(own)
    at = 0
    for t in own:
        assert near(logits[at:at + len(t)], by_definition(weights, torch.cat([shared, t]))[len(shared):])
        at += len(t)


@pytest.mark.gpu
def test_token_by_token_is_the_prompt_at_once(case):
    weights, shared, own = case
    at_once = M.TokenModel(SIZES, weights, 2, 64)
    want = at_once.append([shared, shared])
    steps = M.TokenModel(SIZES, weights, 2, 64)
    got = torch.stack([steps.step(t.repeat(2)) for t in shared])
    assert near(got[:, 0], want[:53]) and near(got[:, 1], want[53:])
    chunks = M.TokenModel(SIZES, weights, 2, 64)
    got = torch.cat([chunks.append([part, part])[:len(part)] for part in shared.split(11)])
    assert near(got, want[:53])


@pytest.mark.gpu
def test_a_shared_beginning_is_everyones_own(case):
    weights, shared, own = case
    together, apart = M.TokenModel(SIZES, weights, 3, 64, len(shared)), M.TokenModel(SIZES, weights, 3, 128)
    together.begin(shared)
    a, b = together.append(own), apart.append([torch.cat([shared, t]) for t in own])
    at, there = 0, 0
    for t in own:
        there += len(shared)
        assert near(a[at:at + len(t)], b[there:there + len(t)])
        at, there = at + len(t), there + len(t)
    # and what is read from the logits is theirs
    given, entropy, best, token = T.logprobs(a, torch.cat(own), top=4)
    lp = torch.log_softmax(a.double(), -1)
    assert torch.allclose(best.double(), lp.topk(4).values, atol=1e-5) and torch.allclose(given.double(), lp.gather(1, torch.cat(own)[:, None])[:, 0], atol=1e-5)


@pytest.mark.gpu
def test_a_captured_step_answers_as_an_eager_one(case):
    weights, shared, own = case
    model = M.TokenModel(SIZES, weights, 3, 64, len(shared))
    model.begin(shared)
    model.append(own)
    token = torch.tensor([5, 6, 7], device="cuda")
    lengths, held = model.lengths.clone(), [[t.clone() for t in (c.k, c.v, c.k_scale, c.v_scale)] for c in model.caches]

    def back():
        model.lengths.copy_(lengths)
        for c, h in zip(model.caches, held):
            for t, x in zip((c.k, c.v, c.k_scale, c.v_scale), h):
                t.copy_(x)

    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        model.step(token)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = model.step(token)
        read = T.logprobs(logits, token, top=3)
    back()
    replayed = []
    for i in range(3):
        token.add_(i)
        graph.replay()
        replayed.append([t.clone() for t in (logits, *read)])
        torch.cuda.synchronize()
        torch.ones(100, device="cuda").sum().item()
    back()
    token.copy_(torch.tensor([5, 6, 7], device="cuda"))
    for i in range(3):
        token.add_(i)
        y = model.step(token)
        for a, b in zip((y, *T.logprobs(y, token, top=3)), replayed[i]):
            assert torch.equal(a, b)


def room_of(device):
    """A model with two sequences in pages for 16 tokens each, without its kernels: what it would ask of them is kept."""
    model = M.TokenModel.__new__(M.TokenModel)
    model.sizes, model.longest, model.room, model.prefix = SIZES, 16, 16, 0
    model.tables, model.prefix_table = torch.tensor([[1], [2]], dtype=torch.int32, device=device), torch.zeros(1, dtype=torch.int32, device=device)
    model.lengths, model.asked = torch.zeros(2, dtype=torch.int32, device=device), []
    model._attend = lambda tokens, slots, starts, most: model.asked.append(slots.tolist())
    return model


def test_tokens_beyond_the_pages_are_refused_or_not_stored():
    """On the CPU: an index beyond a table is an error there, and stops the whole process on a GPU."""
    model = room_of("cpu")
    model.append([torch.zeros(15, dtype=torch.int64), torch.zeros(3, dtype=torch.int64)])
    model.step(torch.zeros(2, dtype=torch.int64))
    assert model.asked == [[*range(16, 31), 32, 33, 34], [31, 35]]
    for call in (lambda: model.append([torch.zeros(1, dtype=torch.int64)] * 2), lambda: model.append([torch.zeros(0, dtype=torch.int64)]),
                 lambda: M.TokenModel.begin(model, torch.zeros(17, dtype=torch.int64))):
        with pytest.raises(ValueError):
            call()
    assert model.lengths.tolist() == [16, 4] and len(model.asked) == 2
    model.step(torch.zeros(2, dtype=torch.int64))
    assert model.asked[-1] == [-1, 36] and model.lengths.tolist() == [17, 5]


@pytest.mark.gpu
def test_a_step_replayed_beyond_its_pages_leaves_the_others_alone(case):
    weights, shared, own = case
    model = M.TokenModel(SIZES, weights, 2, 16)
    model.append([own[0], own[1]])                              # 9 and 1 of 16
    token = torch.tensor([5, 6], device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        model.step(token)
    s.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        logits = model.step(token)
    replayed = []
    for _ in range(10):                                         # lengths 20 and 12
        graph.replay()
        replayed.append(logits.clone())
        torch.cuda.synchronize()
    apart = M.TokenModel(SIZES, weights, 1, 16)
    apart.append([own[1]])
    apart.step(token[1:])
    for y in replayed:
        assert near(y[1:], apart.step(token[1:])) and torch.isfinite(y).all()
