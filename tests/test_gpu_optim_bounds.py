"""An infinite bound clips nothing, whatever the norm is: gradients, parameters and moments come out bit for bit
as without clipping."""
import math

import pytest

ap = pytest.importorskip("paper_2108_02416_gb300")
torch = pytest.importorskip("torch")

from test_gpu_optim import DEV, F16, F32, HYPER, LENGTHS, MIXES, TYPES, clip, generator, make_state, param_list, views  # noqa: E402


def same_bits(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def gradients(n, dtype, kind):
    """a list whose norm is no finite fp32 number"""
    x = torch.randn(n, device=DEV, generator=generator(50)).to(dtype)
    if kind == "sum":                                    # finite values, a norm beyond fp32
        x.fill_(3e38)
    else:
        x[n // 2] = {"inf": math.inf, "-inf": -math.inf, "nan": math.nan}[kind]
    return [x, torch.ones(5, device=DEV, dtype=dtype)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kind", ["inf", "-inf", "nan", "sum"])
@pytest.mark.parametrize("n", [100, 50_000, 17_000_000])     # in one kernel, and (68 MB of fp32) in two
def test_clip(n, kind, dtype):
    if kind == "sum" and dtype == F16:
        pytest.skip("fp16 ends at 65,504")
    ts = gradients(n, dtype, kind)
    before = [t.clone() for t in ts]
    norm = clip(ts, None, math.inf)
    assert math.isnan(norm) if kind == "nan" else math.isinf(norm)
    assert all(same_bits(a, b) for a, b in zip(ts, before))
    outs = [torch.zeros_like(t) for t in ts]
    clip(ts, outs, math.inf)
    clear = [~t.isnan() for t in before]
    assert all(same_bits(a[k], b[k]) and bool(a[~k].isnan().all()) for a, b, k in zip(outs, before, clear))
    clip(ts, None, math.inf, scale=0.5)
    assert all(same_bits(a[k], (b * 0.5)[k]) for a, b, k in zip(ts, before, clear))


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
@pytest.mark.parametrize("ptype,gtype,master", MIXES[::3])
def test_adamw(ptype, gtype, master, value):
    runs = []
    for bound in (None, math.inf):
        s = make_state(LENGTHS["mixed"], ptype, gtype, master)
        s["g"][1][4][1234] = value
        buf = ap.NormBuffers(DEV)
        clipping = {} if bound is None else dict(max_norm=bound, norm=buf.norm, work=buf.work)
        ap.aspis_adamw(param_list(s), 3, **clipping, **HYPER)
        runs.append(s)
    for k in ("p", "m", "v", "w"):
        if runs[0][k]:
            assert same_bits(runs[0][k][0], runs[1][k][0]), k
    assert int((~torch.cat([t.float() for t in runs[1]["p"][1]]).isfinite()).sum()) <= 1


@pytest.mark.gpu
def test_adamw_of_a_norm_beyond_fp32():
    g = torch.full((100,), 3e38, device=DEV)
    p, m, v = (torch.zeros_like(g) for _ in range(3))
    buf = ap.NormBuffers(DEV)
    ap.aspis_adamw(ap.ParamList([p], [g], [m], [v]), 1, 0.1, max_norm=math.inf, norm=buf.norm, work=buf.work)
    assert math.isinf(float(buf.norm)) and bool((m > 2.9e37).all()) and not bool(p.isnan().any())


@pytest.mark.gpu
def test_a_given_infinite_norm():
    x = views([1000], F32, 1, generator(51))[1]
    before = x[0].clone()
    clip(x, None, math.inf, given=math.inf)
    assert same_bits(x[0], before)
    clip(x, None, 1.0, given=math.inf)                   # a finite bound: c = 0
    assert not bool(x[0].any())
