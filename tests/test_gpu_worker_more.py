"""More of dropout, the embedding with its gradient and the policy loss: what tests/test_gpu_worker.py does not reach."""
import functools
import math

import pytest

import _worker_reference as ref
from _worker_reference import U, close, dropped
from test_gpu_worker import (BF16, DEV, F16, F32, I32, I64, SEED, TYPES, ap, gen, normal, place, policy_inputs, run_policy, same_bits, torch,
                             untouched)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [-1.7, 1.7, 0.0])
@pytest.mark.parametrize("kind,out_kind", [(F32, F32), (BF16, F32), (F16, BF16)])
def test_padding_is_zero_bit_by_bit(kind, out_kind, scale):
    """+0 whatever the factor's sign, in narrow and wide rows of any alignment"""
    g = gen(31)
    for D in (24, 63, 512, 520, 1001):
        T, V = 12, 20
        ids = ref.zipf_tokens(T, V, g, I64, DEV)
        ids[1], ids[5], ids[11] = -1, V, -100
        dead = (ids < 0) | (ids >= V)
        for offset, out_offset, pad in ((0, 0, 0), (1, 0, 0), (0, 3, 0), (3, 3, 5)):
            table = place((V, D), kind, offset, pad)[1]
            table.copy_(normal((V, D), F32, g))
            for drop in (None, ap.Drop(0.3, SEED, 4, 5)):
                out = place((T, D), out_kind, out_offset, pad)[1]
                ap.aspis_embed(table, ids, out, scale=scale, drop=drop)
                assert same_bits(out[dead], torch.zeros_like(out[dead]))


@pytest.mark.parametrize("a", [1.0, 0.7])
@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V", [24, 3000, 20_001, 70_000, 300_000, 1_100_000])
def test_the_only_token_that_is_left(V, kind, a):
    """its log-probability and the row's gradient are exactly 0, whatever its logit"""
    T = 4
    logits = torch.full((T, V), -math.inf, dtype=kind, device=DEV)
    tokens = torch.tensor([0, V - 1, V // 2, 13], device=DEV)
    logits[torch.arange(T, device=DEV), tokens] = torch.tensor([-3.0, 7.125, 0.0, 1e4], device=DEV).to(kind)
    got = run_policy(logits, tokens, None, normal((T,), F32, gen(V)), logit_scale=a, grad_scale=16.0)
    out = torch.empty(T, device=DEV)
    ap.aspis_token_logp(logits, tokens, out, logit_scale=a)
    assert bool((out == 0).all()) and bool((got["logp"] == 0).all())
    assert bool((got["grad"] == 0).all())


@pytest.mark.parametrize("V", [24, 3000, 70_000])
def test_probabilities_next_to_one(V):
    """One other token is d below the maximum: lp = -log1p(e^-d), relative to itself within the exponent's roundings (d may be off
    by 3 u d, its power by 2^-22), the quotient, the logarithm and the sum that the rest is taken out of (u of the whole, each)."""
    d = torch.linspace(0.5, 14.0, 28, device=DEV)
    T = len(d)
    logits = torch.full((T, V), -math.inf, device=DEV)
    tokens = torch.full((T,), V // 2, device=DEV)
    logits[:, V // 2] = 3.0
    logits[:, 1] = 3.0 - d
    out = torch.empty(T, device=DEV)
    ap.aspis_token_logp(logits, tokens, out)
    gap = logits[:, V // 2].double() - logits[:, 1].double()
    rest = torch.exp(-gap)
    want = -torch.log1p(rest)
    close(out, want, rest * (3 * U * gap + 2.0 ** -21 + 8 * U) + 4 * U)


# ------------------------------------------------------------------ gradients of many tokens
# Pieces of 32 positions a warp and the kernel that joins runs between blocks: from 304 blocks of 256 tokens and 248 columns on.


@functools.lru_cache(maxsize=4)
def mask(p, first, T, D):
    return ref.factors(ap.Drop(p, SEED, 6, first), T, D).to(DEV) if p else None


def long_sums(grad, ids, V, scale, f, old):
    """The gradient in 64 bits, and a bound of its error that long runs do not widen: a summand goes through at most 32
    additions in its piece, 8 in its block, n / 512 + 2 in its half of the run's n / 256 + 2 parts and one of the halves, of n summands
    no more than n; then the factor, itself rounded, the product and the addition to what was there: four roundings."""
    live = (ids >= 0) & (ids < V)
    at, x = ids.long()[live], grad.double() if f is None else dropped(grad.double(), f)
    zero = torch.zeros(V, x.shape[1], dtype=torch.float64, device=DEV)
    total = zero.index_add(0, at, x[live]) * scale
    size = zero.index_add(0, at, x[live].abs()) * abs(scale)
    n = torch.bincount(at, minlength=V).double()[:, None]
    tol = (torch.minimum(n, 43 + n / 512) + 4) * U * size + ref.TINY * (n > 0)
    if old is not None:
        total = total + old.double()
        tol = torch.where(n > 0, tol + 2 * U * total.abs(), 0.0)
    return total, tol


def check_long(ids, grad, V, out_kind, p=0.0, first=16, accumulate=False, scale=1.0, offset=0, pad=0):
    T, D = grad.shape
    assert -(-T // 256) * -(-D // 248) >= 304
    store, out = place((V, D), out_kind, offset, pad)
    old = None
    if accumulate:
        out.copy_(normal((V, D), F32, gen(99)))
        old = out.clone()
    else:
        out.fill_(math.nan)
    buf = ap.EmbedBuffers(T, V, D, DEV)
    buf.work.fill_(0xFF)
    ap.aspis_embed_grad(grad, ids, out, buf.work, scale=scale, drop=ap.Drop(p, SEED, 6, first) if p else None, accumulate=accumulate)
    close(out, *long_sums(grad, ids, V, float(torch.tensor(scale, dtype=F32)), mask(p, first, T, D), old))
    untouched(store, out)
    if accumulate:
        named = torch.zeros(V, dtype=torch.bool, device=DEV)
        named[ids.long()[(ids >= 0) & (ids < V)]] = True
        assert same_bits(out[~named], old[~named])


@pytest.mark.parametrize("T,V,D", [(78_001, 300, 24), (20_001, 997, 999), (40_000, 50_000, 264), (30_000, 60, 600), (77_900, 80_000, 33)])
@pytest.mark.parametrize("p", [0.0, 0.2])
@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("kind,out_kind", [(F32, F32), (BF16, F32), (F16, F32), (BF16, BF16), (F16, F16), (F32, BF16), (BF16, F16), (F16, BF16),
                                           (F32, F16)])
def test_long_batches(T, V, D, p, accumulate, kind, out_kind):
    """types, masks, sums and additions; rows that begin anywhere and rows at multiples of 16 bytes"""
    g = gen(T + V)
    for ids_kind, offset, pad in ((I64, 0, 0), (I32, 1, 3), (I32, 0, 8)):
        ids = ref.zipf_tokens(T, V, g, ids_kind, DEV)
        grad = place((T, D), kind, offset, pad)[1]
        grad.copy_(normal((T, D), F32, g))
        check_long(ids, grad, V, out_kind, p, 16, accumulate, 1.3, offset, pad)


@pytest.mark.parametrize("T,D", [(78_001, 24), (40_100, 264), (40_100, 261)])
@pytest.mark.parametrize("p,accumulate", [(0.0, False), (0.3, True), (0.3, False)])
@pytest.mark.parametrize("name", ["one", "two", "distinct", "padding", "mostly_padding", "last", "runs_96", "runs_256", "runs_700", "runs_10000", "one_after_many"])
def test_long_batches_of_uneven_tokens(name, T, D, p, accumulate):
    """runs inside a block, from block to block and over many blocks, from their first position on and within"""
    V, at = 80_000, torch.arange(T, device=DEV)
    if name.startswith("runs"):
        ids = at // int(name[5:])
    else:
        ids = {"one": lambda: torch.full_like(at, 7), "two": lambda: at % 2 * 900, "padding": lambda: torch.full_like(at, -1),
               "distinct": lambda: torch.randperm(V, device=DEV, generator=gen(1))[:T], "last": lambda: torch.full_like(at, V - 1),
               "mostly_padding": lambda: torch.where(at % 50 == 49, 3, -1),
               "one_after_many": lambda: torch.where(at < 1000, at, 1000)}[name]()
    ids = ids[torch.randperm(T, device=DEV, generator=gen(2))]
    check_long(ids, normal((T, D), BF16, gen(T)), V, F32, p, 16, accumulate)


@pytest.mark.parametrize("first", [2 ** 64 - 16, 2 ** 64 - 5, 2 ** 35])
@pytest.mark.parametrize("D", [24, 27])
def test_long_masks_beyond_the_last_number(D, first):
    T, V = 78_001, 3000
    check_long(ref.zipf_tokens(T, V, gen(3), I64, DEV), normal((T, D), F32, gen(4)), V, F32, 0.4, first)


@pytest.mark.parametrize("T,V,D", [(40_000, 3000, 264), (78_001, 100_000, 24)])
def test_bits_of_long_batches_depend_on_tokens_alone(T, V, D):
    g = gen(9)
    ids, grad = ref.zipf_tokens(T, V, g, I32, DEV), normal((T, D), BF16, g)
    drop, buf = ap.Drop(0.1, SEED, 6), ap.EmbedBuffers(T, V, D, DEV)
    want = torch.empty(V, D, device=DEV)
    ap.aspis_embed_grad(grad, ids, want, buf.work, drop=drop)
    for offset, pad in ((0, 0), (1, 0), (5, 3), (0, 8)):
        moved, out = place((T, D), BF16, offset, pad)[1], place((V, D), F32, offset, pad)[1]
        moved.copy_(grad)
        buf.work.fill_(offset)
        ap.aspis_embed_grad(moved, ids.long(), out, buf.work, drop=drop)
        assert same_bits(out, want)
        out.zero_()
        ap.aspis_embed_grad(moved, ids, out, buf.work, drop=drop, accumulate=True)
        assert torch.equal(out, want)


def test_long_batches_in_a_graph_and_on_two_streams():
    """the bits of calls one after the other, with new tokens at each replay"""
    T, V, D = 78_001, 5000, 40
    jobs = []
    for seed in (1, 2):
        g = gen(seed)
        jobs.append(dict(ids=ref.zipf_tokens(T, V, g, I32, DEV), dy=normal((T, D), BF16, g), dW=torch.zeros(V, D, device=DEV),
                         work=ap.EmbedBuffers(T, V, D, DEV).work, s=torch.cuda.Stream()))
    drop = ap.Drop(0.1, SEED)

    def call(j, stream=None, accumulate=False):
        ap.aspis_embed_grad(j["dy"], j["ids"], j["dW"], j["work"], drop=drop, accumulate=accumulate, stream=stream)

    def twice(j, stream=None):
        call(j, stream)
        call(j, stream, True)
    want = []
    for j in jobs:
        twice(j)
        want.append(j["dW"].clone())
    torch.cuda.synchronize()
    for _ in range(10):
        for j in jobs:
            twice(j, j["s"])
    torch.cuda.synchronize()
    assert all(same_bits(j["dW"], w) for j, w in zip(jobs, want))
    j, graph = jobs[0], torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=j["s"]):
        twice(j)
    for ids in (j["ids"].flip(0).clone(), jobs[1]["ids"].clone()):
        j["ids"].copy_(ids)
        j["dW"].fill_(7.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = j["dW"].clone()
        twice(j)
        assert same_bits(j["dW"], replayed)


# ------------------------------------------------------------------ the loss


@pytest.mark.parametrize("kind", TYPES)
@pytest.mark.parametrize("V", [1001, 2049, 4097, 8193, 10_241, 20_481, 32_769, 65_537, 100_003, 131_080, 262_153, 300_007, 530_000])
def test_long_rows_in_place(V, kind):
    """the gradient's bits where it takes the logits' place, at any alignment and distance; what lies around it stays"""
    T = 5
    for offset, pad in ((0, 0), (1, 6), (3, 0), (8, 8)):
        logits, tokens, old, adv, prior, weights = policy_inputs(T, V, kind, gen(V), offset, pad, level=4.0)
        tokens[0] = 0
        k = dict(clip=(0.2, 0.3), grad_scale=256.0, ref_logp=prior, weights=weights, kl_coef=0.1)
        want = run_policy(logits, tokens, old, adv, **k)
        buffer, inside = place((T, V), kind, offset, pad)
        inside.copy_(logits)
        got = run_policy(inside, tokens, old, adv, grad=inside, **k)
        assert all(same_bits(got[n], want[n]) for n in want)
        untouched(buffer, inside)


# ------------------------------------------------------------------ the largest sizes


@pytest.mark.parametrize("V", [2 ** 27 + 5, 2 ** 31 - 1])
@pytest.mark.parametrize("T", [500, 9000, 20_001])
def test_rows_of_a_table_up_to_the_last_number(V, T):
    """four passes of the sort; zeros to all rows but those that are named"""
    ids = torch.randint(0, V, (T,), device=DEV, generator=gen(T))
    ids[:6] = torch.tensor([0, V - 1, V, -1, 2 ** 31, 2 ** 32], device=DEV)
    ids[T // 2:] = ids[: T - T // 2].clone()             # each twice
    grad = normal((T, 1), F32, gen(1))
    grad[grad == 0] = 1.0
    real = (ids >= 0) & (ids < V)
    rows, at = torch.unique(ids[real], return_inverse=True)
    x = grad[:, 0].double()[real]
    want = torch.zeros(len(rows), dtype=torch.float64, device=DEV).index_add(0, at, x)
    size = torch.zeros(len(rows), dtype=torch.float64, device=DEV).index_add(0, at, x.abs())
    n = torch.bincount(at).double()
    out = torch.full((V, 1), 7.0, dtype=BF16, device=DEV)
    buf = ap.EmbedBuffers(T, V, 1, DEV)
    ap.aspis_embed_grad(grad, ids, out, buf.work)
    close(out[rows, 0], want, (n + 4) * U * size + ref.TINY)
    assert sum(int(torch.count_nonzero(p)) for p in out.view(-1).split(2 ** 28)) == int(torch.count_nonzero(out[rows]))
    out.fill_(0.5)
    ap.aspis_embed_grad(grad, ids, out, buf.work, accumulate=True)
    close(out[rows, 0], 0.5 + want, (n + 6) * U * (size + 0.5))
    out[rows] = 0.5
    assert all(bool((p == 0.5).all()) for p in out.view(-1).split(2 ** 28))


@pytest.mark.parametrize("T,V,D", [(3_000_001, 1000, 1), (1_000_000, 1, 7)])
def test_millions_of_tokens(T, V, D):
    check_long(ref.zipf_tokens(T, V, gen(T), I32, DEV), normal((T, D), BF16, gen(1)), V, F32)


@pytest.mark.parametrize("D,offset", [(3_000_008, 0), (3_000_001, 1)])
def test_rows_of_millions_of_columns(D, offset):
    T, V = 5, 3
    ids = torch.tensor([1, -1, 0, 1, 3], device=DEV)
    table = place((V, D), BF16, offset)[1]
    table.copy_(normal((V, D), F32, gen(1)))
    drop = ap.Drop(0.2, SEED, 6, 8)
    f = ref.factors(drop, T, D).to(DEV)
    buffer, out = place((T, D), F32, offset)
    ap.aspis_embed(table, ids, out, drop=drop)
    real = ((ids >= 0) & (ids < V))[:, None]
    want = dropped(torch.where(real, table[ids.clamp(0, V - 1)].double(), 0.0), f)
    close(out, want, 3 * U * want.abs() + ref.TINY)
    untouched(buffer, out)
    grad = torch.empty(V, D, device=DEV)
    ap.aspis_embed_grad(out, ids, grad, ap.EmbedBuffers(T, V, D, DEV).work, drop=drop)
    close(grad, *ref.embed_grad(out, ids, V, 1.0, f))
    logits, tokens = table[:2].clone(), torch.tensor([D - 1, 0], device=DEV)
    adv = normal((2,), F32, gen(2))
    want, tol = ref.policy(logits, tokens, None, adv, grad_scale=1024.0)
    got = run_policy(logits, tokens, None, adv, grad_scale=1024.0)
    for name in ("sums", "logp", "grad"):
        close(got[name], want[name], tol[name])
