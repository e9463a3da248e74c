"""More of dropout, the embedding with its gradient and the policy loss: what tests/test_gpu_worker.py does not reach."""
import math

import pytest

import _worker_reference as ref
from _worker_reference import U, close
from test_gpu_worker import (BF16, DEV, F16, F32, I64, SEED, TYPES, ap, gen, normal, place, run_policy, same_bits, torch)

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
