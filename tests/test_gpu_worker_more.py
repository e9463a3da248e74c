"""More of dropout, the embedding with its gradient and the policy loss: what tests/test_gpu_worker.py does not reach."""
import math

import pytest

import _worker_reference as ref
from test_gpu_worker import (BF16, DEV, F16, F32, I64, SEED, ap, gen, normal, place, same_bits, torch)

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
