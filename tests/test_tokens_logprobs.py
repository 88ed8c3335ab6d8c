"""Log probabilities, entropy and the likeliest tokens against the definition in 64 bits, and what is refused."""
import math

import pytest
import torch

from paper_2302_00282_amd import tokens as T
from paper_2302_00282_amd import xenos as X

U32 = 2.0 ** -24
INF, NAN = math.inf, math.nan


def drawn(rows, vocab, dtype, seed, std=3.0):
    return (torch.randn(rows, vocab, generator=torch.Generator().manual_seed(seed)) * std).to(dtype).cuda()


def by_definition(x, targets):
    lp = torch.log_softmax(x.double().cpu(), -1)
    t = targets.cpu()
    given = torch.where((t >= 0) & (t < x.shape[1]), lp.gather(1, t.clamp(0, x.shape[1] - 1)[:, None])[:, 0], torch.zeros((), dtype=torch.float64))
    return given, -torch.where(lp == -INF, torch.zeros_like(lp), lp.exp() * lp).sum(-1), lp


def order_of(x, top):
    """Tokens from the largest logit on, NaN before everything, -0 as 0, equal ones by index."""
    v = x.float().cpu() + 0.0
    return torch.stack([torch.tensor(sorted(range(len(r)), key=lambda i: (not math.isnan(r[i]), 0.0 if math.isnan(r[i]) else -r[i], i))[:top], dtype=torch.int32)
                        for r in v.tolist()]) if top else torch.zeros(len(v), 0, dtype=torch.int32)


def check(x, targets, top):
    given, entropy, best, token = T.logprobs(x, targets, top)
    want, want_entropy, lp = by_definition(x, targets)
    assert torch.equal(token.cpu(), order_of(x, top))
    # log s: every term and the sum in fp32 (a lane adds at most vocab / 64 terms, then trees); logits of size |x| lose half a step of x - m and of x - m - log s
    spread = x.float().cpu().masked_fill(x.cpu() == -INF, 0).abs().amax(-1).double()
    bound = (x.shape[1] / 64 + 40) * U32 + 6 * U32 * spread
    pick = lambda a: a.cpu().double()
    assert torch.all((pick(given) - want).nan_to_num(nan=0.0, posinf=0, neginf=0).abs() <= bound + 2 * U32 * want.nan_to_num(neginf=0).abs())
    assert torch.equal(given.cpu() == -INF, want == -INF)
    # the entropy weighs each term by x - m: up to `spread` times as much
    assert torch.all((pick(entropy) - want_entropy).abs() <= bound * (2 + 2 * spread))
    listed = lp.gather(1, token.cpu().long())
    assert torch.equal(best.cpu() == -INF, listed == -INF)
    assert torch.all((pick(best) - listed).nan_to_num(nan=0.0).abs() <= bound[:, None] + 2 * U32 * listed.nan_to_num(neginf=0).abs())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (1, 1, 0), (3, 2, 2), (2, 63, 5), (2, 64, 64), (5, 1000, 1), (1, 32000, 5), (7, 4097, 20), (4, 50001, 64), (130, 8193, 8),
                                            (1100, 300, 3), (1030, 5000, 0), (1, 200003, 32), (2, 16385, 0)])
def test_logprobs(rows, vocab, top, dtype):
    g = torch.Generator().manual_seed(vocab)
    targets = torch.randint(0, vocab, (rows,), generator=g)
    targets[rows // 2] = -1
    check(drawn(rows, vocab, dtype, rows), targets.cuda(), top)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [600, 5003, 40000])
def test_ties_masks_and_steep_rows(vocab, dtype):
    x = drawn(12, vocab, dtype, 1)
    x[0] = 0
    x[1] = -0.0
    x[1, 5::2] = 0.0
    x[2, 3:] = -INF                                            # fewer tokens left than are asked for
    x[3] = -INF
    x[3, vocab - 1] = 7.0                                      # one token left: entropy 0
    x[4] = torch.finfo(dtype).min                              # masked by the type's lowest value: all of them equal
    x[5, ::3] = torch.finfo(dtype).min
    x[6] = torch.arange(vocab) / 8                             # best tokens last, each better than the one before
    x[7] = -torch.arange(vocab).float() / 8
    x[8] = torch.arange(vocab) % 7
    x[9, 100] = 300.0
    x[10] *= 1e-3
    x[11, ::2] = -INF
    targets = torch.tensor([0, 1, 2, vocab - 1, 3, 1, vocab - 1, 0, 6, 100, 7, 2], device="cuda")
    check(x, targets, 20)
    targets[:3] = torch.tensor([vocab, -5, vocab - 1], device="cuda")
    assert T.logprobs(x, targets)[0][:2].tolist() == [0.0, 0.0] and T.logprobs(x, targets)[0][2] == -INF
    assert T.logprobs(x, targets, 1)[1][3] == 0 and abs(T.logprobs(x)[1][0].item() - math.log(vocab)) < 1e-5


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [600, 40000])
def test_rows_without_a_distribution(vocab, dtype):
    x = drawn(6, vocab, dtype, 1)
    x[0] = -INF
    x[1, 17] = NAN
    x[2, 18] = INF
    x[3, 400] = -NAN
    x[3, 19], x[3, 20] = INF, NAN
    targets = torch.tensor([0, 1, 18, 19, 5, 5], device="cuda")
    given, entropy, best, token = T.logprobs(x, targets, 4)
    assert torch.isnan(given[:4]).all() and torch.isnan(entropy[:4]).all() and torch.isfinite(given[4:]).all() and torch.isfinite(entropy[4:]).all()
    assert torch.isnan(best[[0, 1, 3]]).all()
    assert torch.equal(token.cpu(), order_of(x, 4)) and token[3].tolist()[:3] == [20, 400, 19]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1001, 20011])
def test_rows_at_any_address(vocab, dtype):
    wide = drawn(5, vocab + 37, dtype, 2)
    targets = torch.randint(0, vocab, (5,), device="cuda")
    for at in (0, 1, 2, 3, 5, 7, 8, 13):
        check(wide[:, at:at + vocab], targets, 6)
    check(wide[::2, 1:1 + vocab], targets[:3], 6)
    check(wide[:, :vocab].t().contiguous().t(), targets, 6)
    alone = torch.empty(vocab + 1, dtype=dtype, device="cuda")
    alone[1:] = wide[0, :vocab]
    check(alone[None, 1:], targets[:1], 3)


@pytest.mark.gpu
def test_rows_beyond_the_32_bit_offsets():
    vocab, rows = 1 << 20, 2100
    x = torch.zeros(rows, vocab, dtype=torch.bfloat16, device="cuda")           # 4.4 GB
    x[rows - 1, vocab - 2], x[rows - 1, 5] = 20.0, 19.0
    targets = torch.full((rows,), vocab - 2, device="cuda")
    given, entropy, best, token = T.logprobs(x, targets, 3)
    check(x[-1:], targets[-1:], 3)
    assert token[rows - 1].tolist() == [vocab - 2, 5, 0] and token[0].tolist() == [0, 1, 2]
    assert abs(given[0].item() + math.log(vocab)) < 1e-5


@pytest.mark.gpu
def test_logprobs_refuse_and_take_nothing():
    x, t = drawn(4, 100, torch.float32, 1), torch.zeros(4, dtype=torch.int64, device="cuda")
    for call, status in [(lambda: T.logprobs(x.cpu()), X.XENOS_EINVAL), (lambda: T.logprobs(x.half()), X.XENOS_EUNSUPPORTED), (lambda: T.logprobs(x[0]), X.XENOS_ESHAPE),
                         (lambda: T.logprobs(x, t.int()), X.XENOS_EINVAL), (lambda: T.logprobs(x, t[:2]), X.XENOS_ESHAPE), (lambda: T.logprobs(x, t, 65), X.XENOS_EUNSUPPORTED),
                         (lambda: T.logprobs(x[:, :3], t, 4), X.XENOS_ESHAPE), (lambda: T.logprobs(x, t, -1), X.XENOS_EUNSUPPORTED), (lambda: T.logprobs(x[:, :0], t), X.XENOS_ESHAPE)]:
        with pytest.raises(X.XenosError) as e:
            call()
        assert e.value.status == status, str(e.value)
    given, entropy, best, token = T.logprobs(x[:0], t[:0], 3)
    assert given.shape == entropy.shape == (0,) and best.shape == token.shape == (0, 3)
    assert T.logprobs(x)[0] is None


def test_logprobs_entries_refuse_before_any_launch():
    p = 256
    good = dict(d_logits=p, dtype=0, rows=4, vocab=100000, row_stride=100000, d_targets=p, top=5, d_logprob=p, d_entropy=p, d_top_logprob=p, d_top_token=p, d_workspace=p,
                workspace_bytes=1 << 20)
    assert X.xenos_logprobs_workspace(4, 100000, 5) > 0 and X.xenos_logprobs_workspace(4000, 100000, 5) == 0 and X.xenos_logprobs_workspace(0, 10, 0) == 0
    for change, status in [(dict(rows=-1), X.XENOS_EINVAL), (dict(vocab=0), X.XENOS_EINVAL), (dict(dtype=5), X.XENOS_EINVAL), (dict(top=65), X.XENOS_EINVAL), (dict(top=-1), X.XENOS_EINVAL),
                           (dict(vocab=4), X.XENOS_ESHAPE), (dict(vocab=(1 << 30) + 1, row_stride=1 << 31), X.XENOS_EUNSUPPORTED), (dict(d_logits=0), X.XENOS_EINVAL),
                           (dict(d_targets=0), X.XENOS_EINVAL), (dict(d_logprob=0), X.XENOS_EINVAL), (dict(d_top_token=0), X.XENOS_EINVAL), (dict(row_stride=99999), X.XENOS_ESHAPE),
                           (dict(d_logits=p + 2), X.XENOS_EINVAL), (dict(d_targets=p + 4), X.XENOS_EINVAL), (dict(d_workspace=0), X.XENOS_EINVAL), (dict(workspace_bytes=100), X.XENOS_EINVAL),
                           (dict(rows=1 << 30), X.XENOS_EUNSUPPORTED)]:
        with pytest.raises(X.XenosError) as e:
            X.xenos_logprobs(**dict(good, **change))
        assert e.value.status == status, change
    for bad in [(-1, 10, 1), (1, 0, 0), (1, 10, 11), (1, 100, 65)]:
        with pytest.raises(X.XenosError):
            X.xenos_logprobs_workspace(*bad)
    X.xenos_logprobs(**dict(good, rows=0, d_logits=0))


def check_strictly(x, targets, top):
    """As `check`, but what is a number by definition has to be one, and only such numbers are compared."""
    given, entropy, best, token = T.logprobs(x, targets, top)
    want, want_entropy, lp = by_definition(x, targets)
    spread = x.float().cpu().masked_fill(x.cpu() == -INF, 0).abs().amax(-1).double()
    bound = (x.shape[1] / 64 + 40) * U32 + 6 * U32 * spread
    for got, expected, b in ((given, want, bound), (entropy, want_entropy, bound * (2 + 2 * spread)), (best, lp.gather(1, token.cpu().long()), bound[:, None].expand(-1, top))):
        got, finite = got.cpu().double(), torch.isfinite(expected)
        assert torch.equal(torch.isfinite(got), finite) and torch.equal(got == -INF, expected == -INF)
        assert torch.all((got - expected).abs()[finite] <= (b + 2 * U32 * expected.abs())[finite])
    assert torch.equal(token.cpu(), order_of(x, top))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,vocab,top", [(1, 1, 1), (3, 2, 2), (2, 64, 64), (5, 1000, 1), (1, 32000, 5), (7, 4097, 20), (4, 50001, 64), (130, 8193, 8), (1100, 300, 3), (1030, 5000, 0), (1, 200003, 32)])
def test_logprobs_are_numbers_where_they_are_by_definition(rows, vocab, top, dtype):
    targets = torch.randint(0, vocab, (rows,), generator=torch.Generator().manual_seed(vocab))
    targets[rows // 2] = -1
    check_strictly(drawn(rows, vocab, dtype, rows), targets.cuda(), top)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [600, 5003, 40000])
def test_masked_and_steep_rows_have_numbers_too(vocab, dtype):
    x = drawn(10, vocab, dtype, 1)
    x[0] = 0
    x[1, 3:] = -INF
    x[2] = -INF
    x[2, vocab - 1] = 7.0
    x[3] = torch.finfo(dtype).min
    x[4, ::3] = torch.finfo(dtype).min
    x[5] = torch.arange(vocab) / 8
    x[6] = -torch.arange(vocab).float() / 8
    x[7, 100] = 300.0
    x[8, ::2] = -INF
    x[9, 0] = torch.finfo(dtype).max
    targets = torch.tensor([0, 2, vocab - 1, 3, 1, vocab - 1, 0, 100, 1, 0], device="cuda")
    check_strictly(x, targets, 20)
    targets = torch.tensor([1, 5, 0, vocab - 1, 0, 0, 1, 101, 0, 1], device="cuda")
    check_strictly(x, targets, 3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("large", [64, 4096])
def test_many_small_terms_behind_large_ones_are_not_lost(large, dtype):
    """Each term is less than half a step of what its lane has summed by then; together they are what the bound sees.  (So many rows that none is cut in parts.)"""
    vocab, rows = 200000, 1030
    x = torch.full((rows, vocab), -13.9375, dtype=dtype, device="cuda")         # e^x = 8.9e-7
    x[:, :large] = 0
    targets = torch.full((rows,), vocab - 1, device="cuda")
    given, entropy, best, token = T.logprobs(x, targets, 2)
    total = large + (vocab - large) * math.exp(-13.9375)
    # sums of 16 terms, of a wavefront's blocks, of the lanes and wavefronts; an exponential's two steps; the differences and the logarithm of size 14 and 9
    bound = (16 + vocab / 4096 + 12 + 4) * U32 + (14 + 9) * U32
    assert (given.double() + 13.9375 + math.log(total)).abs().max() <= bound
    assert (best.double() + math.log(total)).abs().max() <= bound
    want = math.log(total) + (vocab - large) * math.exp(-13.9375) * 13.9375 / total
    assert (entropy.double() - want).abs().max() <= 3 * bound


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_entropies_are_as_near_as_their_sums(dtype):
    """Rows whose largest logit comes late and is little above the first block's: what was summed before it counts in its steps."""
    rows, vocab = 1030, 20000
    x = drawn(rows, vocab, dtype, 3, 2.5)
    x[:, 15000] = x[:, :4096].amax(-1) + 7.5
    given, entropy, best, token = T.logprobs(x, torch.full((rows,), 15000, device="cuda"), 1)
    want, want_entropy, lp = by_definition(x[:64], torch.full((64,), 15000))
    d = (lp - lp.amax(-1, keepdim=True)).abs()
    weighed = (lp.exp() * d).sum(-1)                            # (of an exponent: a step of its size and two of its exponential)
    sums = (16 + vocab / 4096 + 12 + 4) * U32 + 2 * U32 * weighed
    assert torch.all((given[:64].double().cpu() - want).abs() <= sums + 24 * U32 + 2 * U32 * want.abs())
    second = (lp.exp() * d * d).sum(-1)
    assert torch.all((entropy[:64].double().cpu() - want_entropy).abs() <= 2 * sums * (1 + weighed) + 2 * U32 * second + 24 * U32)
