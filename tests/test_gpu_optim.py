"""The norm, clipping and AdamW over many tensors against plain 64-bit arithmetic.

Tolerances.  With u = 2^-24: a norm's partial sums hold at most 64 squares in
32 bits before they are added in 64, so the sum of squares is off by at most 65 u and the norm by
33 u, plus its own rounding: NORM = 34 u.  The factor s * c adds a quotient, a sum and a
product: FACTOR = NORM + 4 u.  What follows is propagated through the formulas.  A 16-bit
output is the rounding of a value within such bounds: rounding is monotone, so it lies between
the roundings of the two ends."""
import math

import pytest

ap = pytest.importorskip("paper_2108_02416_gb300")
torch = pytest.importorskip("torch")

U = 2.0 ** -24
NORM, FACTOR = 34 * U, 38 * U
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
TINY = 2.0 ** -149                 # the smallest fp32 subnormal
DEV = "cuda:0"

LENGTHS = {
    "none": [],
    "empty": [0],
    "one": [1],
    "few": [3, 0, 1, 8, 17],
    "units": [1023, 1024, 1025, 2047, 2048, 2049, 4096, 0, 4095],
    "one_long": [1_300_001],
    "mixed": [70_001, 5, 0, 1, 333_333, 2, 16, 100_000, 7],
    "table": [i % 23 for i in range(121)],
}
MANY = [(i * 37) % 101 for i in range(2300)]             # more than one launch's table holds


def views(lengths, dtype, offset, gen=None, level=1.0, pad=64, fill=None):
    """Tensors in one buffer, each `offset` elements after a 256-byte boundary, with what lies
    between them; returns (buffer, tensors)."""
    at, places = 0, []
    for n in lengths:
        places.append((at + offset, n))
        at += -(-(offset + n + pad) // 128) * 128
    buffer = torch.full((max(at, 128),), 7.0, dtype=dtype, device=DEV)
    ts = [buffer[o: o + n] for o, n in places]
    for t in ts:
        if fill is not None:
            t.fill_(fill)
        else:
            t.copy_(torch.randn(t.shape, device=DEV, generator=gen) * level)
    return buffer, ts


def outside(buffer, ts):
    """bool mask of the buffer's elements that belong to no tensor"""
    mask = torch.ones(buffer.numel(), dtype=torch.bool, device=DEV)
    for t in ts:
        o = (t.data_ptr() - buffer.data_ptr()) // buffer.element_size()
        mask[o: o + t.numel()] = False
    return mask


def generator(seed):
    return torch.Generator(DEV).manual_seed(seed)


def norms(ts, scale=1.0):
    squares = [float(t.double().square().sum()) for t in ts]
    return [scale * math.sqrt(x) for x in squares], scale * math.sqrt(math.fsum(squares))


def take_norm(ts, scale=1.0, each=True):
    buf = ap.NormBuffers(DEV)
    out = torch.full((len(ts),), -1.0, device=DEV) if each else None
    ap.aspis_grad_norm(ap.TensorList(ts), buf.norm, buf.work, tensor_norms=out, scale=scale)
    return float(buf.norm), None if out is None else out.tolist()


def coef(norm, max_norm):
    return min(1.0, max_norm / (norm + 1e-6))


def close(got, want, tol):
    """got is the rounding to its type of a value within tol of want"""
    low, high = (want - tol).to(got.dtype), (want + tol).to(got.dtype)
    bad = ~((low <= got) & (got <= high))
    assert not bool(bad.any()), (got[bad][:4], want[bad][:4])


# ---------------------------------------------------------------- the norm


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset", [0, 1, 2, 3, 4, 5, 7, 8])
@pytest.mark.parametrize("name", LENGTHS)
def test_norm(name, offset, dtype):
    _, ts = views(LENGTHS[name], dtype, offset, generator(1), level=3.0)
    got, each = take_norm(ts)
    want_each, want = norms(ts)
    assert abs(got - want) <= NORM * want
    assert all(abs(x - y) <= NORM * y for x, y in zip(each, want_each))
    assert abs(take_norm(ts, each=False)[0] - want) <= NORM * want


@pytest.mark.gpu
def test_norm_of_thousands_of_tensors():
    for dtype, offset in ((F32, 1), (BF16, 0)):
        _, ts = views(MANY, dtype, offset, generator(1))
        got, each = take_norm(ts)
        want_each, want = norms(ts)
        assert abs(got - want) <= NORM * want
        assert all(abs(x - y) <= NORM * y for x, y in zip(each, want_each))


@pytest.mark.gpu
def test_norm_of_mixed_types_and_scale():
    gen = generator(2)
    ts = [views([n], d, o, gen, level=0.01)[1][0]
          for n, d, o in [(1000, F32, 1), (70_003, BF16, 3), (0, F16, 0), (12_345, F16, 5), (1, F32, 0), (300_000, F32, 2)]]
    got, each = take_norm(ts, scale=1 / 1024)
    want_each, want = norms(ts, 1 / 1024)
    assert abs(got - want) <= NORM * want
    assert all(abs(x - y) <= NORM * y for x, y in zip(each, want_each))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("level", [1e-42, 1e-38, 1e-30, 1e-22, 1e-18, 1e-15, 1e15, 1e18, 1e22, 1e30, 1e36])
@pytest.mark.parametrize("n", [1, 7, 40_000])
def test_norm_over_the_whole_range(n, level, dtype):
    """squares that would overflow or vanish in 32 bits"""
    x = (torch.rand(n, device=DEV, generator=generator(3)) + 0.5).double().mul_(level).to(dtype)
    y = torch.full((5,), level / 100, device=DEV).to(dtype)
    got, each = take_norm([x, y])
    want_each, want = norms([x, y])
    tol = 2.0 ** -149                                    # a subnormal norm's own rounding
    assert abs(got - want) <= NORM * want + tol
    assert all(abs(a - b) <= NORM * b + tol for a, b in zip(each, want_each))


@pytest.mark.gpu
def test_norm_of_one_large_value_among_small_ones():
    for big in (1e19, 1e30, 3e38):
        x = torch.full((100_000,), 1e-3, device=DEV)
        x[54_321] = big
        assert take_norm([x], each=False)[0] == pytest.approx(big, rel=NORM)
    x = torch.zeros(100_000, device=DEV)
    x[99_999] = 1e-30
    assert take_norm([x], each=False)[0] == pytest.approx(1e-30, rel=NORM)
    assert take_norm([torch.zeros(100_000, device=DEV)]) == (0.0, [0.0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("where", [0, 1, 4_999, 9_999])
def test_norm_not_finite(where, dtype):
    for value, check in ((math.inf, math.isinf), (-math.inf, math.isinf), (math.nan, math.isnan)):
        x = torch.ones(10_000, device=DEV, dtype=dtype)
        y = torch.ones(33, device=DEV, dtype=dtype)
        x[where] = value
        got, each = take_norm([y, x, y])
        assert check(got) and check(each[1]) and each[0] == each[2] == pytest.approx(math.sqrt(33), rel=NORM)
    assert math.isinf(take_norm([torch.full((100,), 3e38, device=DEV)])[0])     # beyond fp32


@pytest.mark.gpu
def test_norm_past_32_bit_offsets():
    n = (1 << 31) + 12_345
    x = torch.zeros(n, dtype=BF16, device=DEV)
    x[n - 1], x[1 << 31], x[(1 << 31) - 1], x[0] = 3.0, 4.0, 12.0, 84.0
    assert take_norm([x]) == (pytest.approx(math.sqrt(9 + 16 + 144 + 84 ** 2), rel=NORM),) * 1 + \
        ([pytest.approx(math.sqrt(9 + 16 + 144 + 84 ** 2), rel=NORM)],)


@pytest.mark.gpu
def test_norm_repeats_its_bits():
    _, ts = views(LENGTHS["mixed"], F32, 3, generator(4))
    buf, lst = ap.NormBuffers(DEV), ap.TensorList(ts)
    seen = set()
    for _ in range(20):
        ap.aspis_grad_norm(lst, buf.norm, buf.work)
        seen.add(float(buf.norm))
    assert len(seen) == 1


@pytest.mark.gpu
def test_norm_of_any_order_of_dimensions():
    x = torch.randn(3, 5, 7, 11, device=DEV, generator=generator(5))
    for t in (x.permute(2, 0, 3, 1), x.transpose(0, 3), x.to(memory_format=torch.channels_last)):
        assert take_norm([t], each=False)[0] == pytest.approx(float(x.double().norm()), rel=NORM)


# ---------------------------------------------------------------- clipping


def clip(ts, outs, max_norm, scale=1.0, given=None):
    buf, lst = ap.NormBuffers(DEV), ap.TensorList(ts, outs)
    if given is not None:
        buf.norm.fill_(given)
    ap.aspis_clip_grads(lst, max_norm, buf.norm, None if given is not None else buf.work, scale=scale)
    return float(buf.norm)


def check_clip(before, after, factor):
    for x, y in zip(before, after):
        want = x.double() * factor
        close(y, want, want.abs() * FACTOR + TINY)


@pytest.mark.gpu
@pytest.mark.parametrize("out", [None] + TYPES)
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offsets", [(0, 0), (1, 0), (0, 3), (5, 6), (4, 4)])
@pytest.mark.parametrize("name", LENGTHS)
def test_clip(name, offsets, dtype, out):
    gen = generator(6)
    buffer, ts = views(LENGTHS[name], dtype, offsets[0], gen)
    target, outs = (buffer, ts) if out is None else views(LENGTHS[name], out, offsets[1], gen)
    before, mask = [t.clone() for t in ts], outside(target, outs)
    edges, source = target[mask].clone(), buffer.clone()
    want = norms(before)[1]
    got = clip(ts, None if out is None else outs, 0.75)
    assert abs(got - want) <= NORM * want
    check_clip(before, outs, coef(want, 0.75))
    assert torch.equal(target[mask], edges)              # nothing beside the tensors is written
    if out is not None:
        assert torch.equal(buffer, source)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [(F32, None), (BF16, F32)])
def test_clip_of_thousands_of_tensors(dtype, out):
    _, ts = views(MANY, dtype, 3, generator(6))
    outs = ts if out is None else views(MANY, out, 0, generator(6))[1]
    before = [t.clone() for t in ts]
    clip(ts, None if out is None else outs, 0.75)
    check_clip(before, outs, coef(norms(before)[1], 0.75))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_clip_below_the_bound_changes_no_bit(dtype):
    _, ts = views(LENGTHS["mixed"], dtype, 3, generator(7))
    before = [t.clone() for t in ts]
    for bound in (1e6, math.inf):
        clip(ts, None, bound)
        assert all(torch.equal(a, b) for a, b in zip(ts, before))
        outs = [torch.empty_like(t) for t in ts]
        clip(ts, outs, bound)
        assert all(torch.equal(a, b) for a, b in zip(outs, before))


@pytest.mark.gpu
def test_clip_with_a_scale_a_given_norm_and_the_bound_zero():
    _, ts = views(LENGTHS["mixed"], F32, 1, generator(8))
    before = [t.clone() for t in ts]
    want = norms(before, 0.125)[1]
    got = clip(ts, None, 2.0, scale=0.125)
    assert abs(got - want) <= NORM * want
    check_clip(before, ts, 0.125 * coef(want, 2.0))
    outs = [torch.empty_like(t) for t in before]
    assert clip(before, outs, 2.0, scale=0.5, given=16.0) == 16.0
    check_clip(before, outs, 0.5 * coef(16.0, 2.0))
    clip(before, outs, 0.0)
    assert all(not bool(o.any()) for o in outs)
    below = [t.clone() for t in before]                  # below the bound a scale is still applied
    clip(below, None, 1e9, scale=0.25)
    assert all(torch.equal(a, b * 0.25) for a, b in zip(below, before))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_clip_not_finite(dtype):
    x = torch.ones(5_000, device=DEV, dtype=dtype)
    x[7] = math.inf
    x[8] = -1.0
    y = torch.ones(3, device=DEV, dtype=dtype)
    assert math.isinf(clip([x, y], None, 1.0))           # c = 0: finite values vanish, infinite ones are NaN
    assert bool(x[7].isnan()) and int(x.isnan().sum()) == 1 and not bool(y.any()) and float(x.nan_to_num(0).abs().sum()) == 0
    assert math.copysign(1.0, float(x[8])) == -1.0
    z = torch.ones(5_000, device=DEV, dtype=dtype)
    z[4_321] = math.nan
    assert math.isnan(clip([z, y], None, 1.0))
    assert bool(z.isnan().all()) and bool(y.isnan().all())


@pytest.mark.gpu
def test_clip_saturates_to_infinity_where_the_type_ends():
    x = torch.tensor([70_000.0, -70_000.0, 65_519.0, 1.0], device=DEV)
    out = torch.zeros(4, dtype=F16, device=DEV)
    clip([x], [out], math.inf)
    assert out.tolist() == [math.inf, -math.inf, 65_504.0, 1.0]


@pytest.mark.gpu
def test_clip_past_32_bit_offsets():
    n = (1 << 31) + 777
    x = torch.zeros(n, dtype=BF16, device=DEV)
    x[n - 1], x[1 << 31], x[5] = 3.0, 4.0, 12.0
    assert clip([x], None, 6.5) == 13.0
    assert [float(x[i]) for i in (n - 1, 1 << 31, 5)] == [1.5, 2.0, 6.0] and int((x != 0).sum()) == 3


@pytest.mark.gpu
def test_overlapping_tensors_are_clipped_by_no_call():
    x = torch.ones(100, device=DEV)
    lst, buf = ap.TensorList([x[:60], x[50:]]), ap.NormBuffers(DEV)
    ap.aspis_grad_norm(lst, buf.norm, buf.work)
    assert float(buf.norm) == pytest.approx(math.sqrt(110), rel=NORM)
    with pytest.raises(ap.AspisError) as e:
        ap.aspis_clip_grads(lst, 1.0, buf.norm, buf.work)
    assert e.value.status == ap.E_INVAL and bool((x == 1).all())


# ---------------------------------------------------------------- AdamW


HYPER = dict(lr=1e-2, betas=(0.9, 0.95), eps=1e-8)


def make_state(lengths, ptype, gtype, master, offsets=(0, 0), seed=9, level=0.05):
    gen = generator(seed)
    s = {"p": views(lengths, ptype, offsets[0], gen), "g": views(lengths, gtype, offsets[1], gen, level),
         "m": views(lengths, F32, offsets[0], gen, 0.1 * level), "v": views(lengths, F32, offsets[0], gen, level)}
    for t in s["v"][1]:
        t.square_()
    s["w"] = views(lengths, F32, offsets[0], gen) if master else None
    s["decay"] = [0.1 if i % 2 else 0.0 for i in range(len(lengths))]
    return s


def param_list(s):
    return ap.ParamList(s["p"][1], s["g"][1], s["m"][1], s["v"][1], masters=s["w"] and s["w"][1], weight_decay=s["decay"])


def copy_of(s):
    return {k: [t.double() for t in s[k][1]] if s[k] else None for k in ("p", "g", "m", "v", "w")}


def check_adamw(s, old, factor, step, lr, betas, eps, factor_tol=FACTOR):
    """the state after one step from `old`, with every error propagated"""
    b1, b2 = betas
    for i in range(len(old["p"])):
        h = old["g"][i] * factor
        m = b1 * old["m"][i] + (1 - b1) * h
        v = b2 * old["v"][i] + (1 - b2) * h * h
        tm = 4 * U * b1 * old["m"][i].abs() + (factor_tol + 4 * U) * (1 - b1) * h.abs() + TINY
        tv = 4 * U * b2 * old["v"][i] + (2 * factor_tol + 5 * U) * (1 - b2) * h * h + 2 * TINY
        c1, c2 = 1 - b1 ** step, 1 - b2 ** step
        root = (v / c2).sqrt()
        den = root + eps
        tden = ((v + tv) / c2).sqrt() - root + 5 * U * den
        tden = torch.maximum(tden, root - ((v - tv).clamp(min=0) / c2).sqrt() + 5 * U * den)
        x = (old["w"] or old["p"])[i]
        q = m / den
        move = lr / c1 * q
        tx = lr / c1 * (tm / (den - tden) + q.abs() * tden / (den - tden) + 4 * U * q.abs())
        decay = lr * s["decay"][i] * x
        tx = tx + 4 * U * (decay.abs() + move.abs())
        x = x - decay - move
        close(s["m"][1][i], m, tm)
        close(s["v"][1][i], v, tv)
        if old["w"]:
            close(s["w"][1][i], x, tx + 2 * U * x.abs())
            assert torch.equal(s["p"][1][i], s["w"][1][i].to(s["p"][1][i].dtype))     # the rounding of the master
        else:
            close(s["p"][1][i], x, tx + 2 * U * x.abs())


MIXES = [(F32, F32, False), (F32, BF16, False), (F32, F16, False), (BF16, BF16, True), (BF16, F32, True),
         (F16, F16, True), (F16, F32, True), (BF16, F16, True), (F16, BF16, True), (BF16, BF16, False), (F16, F16, False), (BF16, F32, False)]


@pytest.mark.gpu
@pytest.mark.parametrize("ptype,gtype,master", MIXES)
@pytest.mark.parametrize("offsets", [(0, 0), (0, 1), (0, 3), (1, 1), (8, 5), (7, 2)])
@pytest.mark.parametrize("name", LENGTHS)
def test_adamw(name, offsets, ptype, gtype, master):
    s = make_state(LENGTHS[name], ptype, gtype, master, offsets)
    old = copy_of(s)
    masks = {k: outside(*s[k]) for k in ("p", "m", "v", "w") if s[k]}
    edges = {k: s[k][0][masks[k]].clone() for k in masks}
    grads = s["g"][0].clone()
    buf = ap.NormBuffers(DEV)
    ap.aspis_adamw(param_list(s), 3, max_norm=0.5, norm=buf.norm, work=buf.work, **HYPER)
    want = norms(old["g"])[1]
    assert abs(float(buf.norm) - want) <= NORM * want
    check_adamw(s, old, coef(want, 0.5), 3, **HYPER)
    for k in masks:
        assert torch.equal(s[k][0][masks[k]], edges[k]), k
    assert torch.equal(s["g"][0], grads)


@pytest.mark.gpu
@pytest.mark.parametrize("ptype,gtype,master", [MIXES[0], MIXES[3]])
def test_adamw_of_thousands_of_tensors(ptype, gtype, master):
    s = make_state(MANY, ptype, gtype, master, (0, 1))
    old, buf = copy_of(s), ap.NormBuffers(DEV)
    ap.aspis_adamw(param_list(s), 3, max_norm=0.5, norm=buf.norm, work=buf.work, **HYPER)
    check_adamw(s, old, coef(norms(old["g"])[1], 0.5), 3, **HYPER)


@pytest.mark.gpu
@pytest.mark.parametrize("step", [1, 2, 10, 100_000])
def test_adamw_without_clipping(step):
    s = make_state(LENGTHS["mixed"], F32, F32, False)
    old = copy_of(s)
    ap.aspis_adamw(param_list(s), step, scale=0.5, **HYPER)
    check_adamw(s, old, 0.5, step, factor_tol=U, **HYPER)


@pytest.mark.gpu
def test_adamw_with_a_given_norm_over_two_lists():
    a, b = make_state(LENGTHS["mixed"], F32, F32, False, seed=10), make_state(LENGTHS["units"], BF16, BF16, True, seed=11)
    olds, buf = [copy_of(a), copy_of(b)], ap.NormBuffers(DEV)
    ap.aspis_grad_norm(ap.TensorList(a["g"][1] + b["g"][1]), buf.norm, buf.work)
    for s, lr in ((a, 1e-2), (b, 1e-3)):
        ap.aspis_adamw(param_list(s), 7, lr, HYPER["betas"], HYPER["eps"], max_norm=1.0, norm=buf.norm)
    want = norms(olds[0]["g"] + olds[1]["g"])[1]
    for s, old, lr in ((a, olds[0], 1e-2), (b, olds[1], 1e-3)):
        check_adamw(s, old, coef(want, 1.0), 7, lr, HYPER["betas"], HYPER["eps"])


@pytest.mark.gpu
def test_adamw_of_mixed_types_in_one_list():
    parts = [make_state([n, 9], p, g, w, seed=20 + i) for i, (n, (p, g, w)) in enumerate(zip((5_000, 1, 77_777, 2_048, 31, 1_000), MIXES[::2]))]
    olds = [copy_of(s) for s in parts]
    cat = lambda k: [t for s in parts for t in (s[k][1] if s[k] else [None, None])]  # noqa: E731
    lst = ap.ParamList(cat("p"), cat("g"), cat("m"), cat("v"), masters=cat("w"), weight_decay=[0.0, 0.1] * len(parts))
    buf = ap.NormBuffers(DEV)
    ap.aspis_adamw(lst, 5, max_norm=0.3, norm=buf.norm, work=buf.work, **HYPER)
    want = norms([g for o in olds for g in o["g"]])[1]
    for s, old in zip(parts, olds):
        check_adamw(s, old, coef(want, 0.3), 5, **HYPER)


@pytest.mark.gpu
def test_adamw_of_zeros():
    """a row that has never had a gradient stays where it is; with eps = 0 its quotient is 0 / 0"""
    p = torch.randn(5_000, device=DEV, generator=generator(12))
    m, v, g = torch.zeros_like(p), torch.zeros_like(p), torch.zeros_like(p)
    old = p.clone()
    ap.aspis_adamw(ap.ParamList([p], [g], [m], [v]), 1, 0.1)
    assert torch.equal(p, old) and not bool(m.any()) and not bool(v.any())
    ap.aspis_adamw(ap.ParamList([p], [g], [m], [v]), 1, 0.1, eps=0.0)
    assert bool(p.isnan().all())


@pytest.mark.gpu
@pytest.mark.parametrize("value", [math.inf, math.nan])
@pytest.mark.parametrize("ptype,gtype,master", MIXES[::3])
def test_adamw_skips_a_step_that_is_not_finite(value, ptype, gtype, master):
    s = make_state(LENGTHS["mixed"], ptype, gtype, master)
    s["g"][1][4][1234] = value
    kept = {k: s[k][0].clone() for k in ("p", "m", "v", "w") if s[k]}
    buf, lst = ap.NormBuffers(DEV), param_list(s)
    for bound in (1.0, math.inf):
        ap.aspis_adamw(lst, 3, max_norm=bound, norm=buf.norm, work=buf.work, skip_nonfinite=True, **HYPER)
        assert not math.isfinite(float(buf.norm))
        assert all(torch.equal(s[k][0], kept[k]) for k in kept)
    s["g"][1][4][1234] = 0.5                             # the next step goes through
    old = copy_of(s)
    ap.aspis_adamw(lst, 3, max_norm=1.0, norm=buf.norm, work=buf.work, skip_nonfinite=True, **HYPER)
    check_adamw(s, old, coef(norms(old["g"])[1], 1.0), 3, **HYPER)


@pytest.mark.gpu
def test_adamw_not_finite_without_skipping():
    s = make_state([1000], F32, F32, False)
    s["g"][1][0][10] = math.nan
    buf = ap.NormBuffers(DEV)
    ap.aspis_adamw(param_list(s), 3, max_norm=1.0, norm=buf.norm, work=buf.work, **HYPER)
    assert bool(s["p"][1][0].isnan().all())
    s = make_state([1000], F32, F32, False)
    s["g"][1][0][10] = math.nan
    ap.aspis_adamw(param_list(s), 3, **HYPER)
    assert int(s["p"][1][0].isnan().sum()) == 1


@pytest.mark.gpu
def test_adamw_of_any_order_of_dimensions():
    gen = generator(13)
    make = lambda: torch.randn(6, 5, 33, device=DEV, generator=gen).permute(2, 0, 1)  # noqa: E731
    s = {k: (None, [make()]) for k in ("p", "g", "m", "v")}
    s["v"][1][0].square_()
    s["w"], s["decay"] = None, [0.1]
    old = copy_of(s)
    ap.aspis_adamw(param_list(s), 3, **HYPER)
    check_adamw(s, old, 1.0, 3, factor_tol=U, **HYPER)


@pytest.mark.gpu
def test_adamw_past_32_bit_offsets():
    n = (1 << 31) + 555
    p, m, v = (torch.zeros(n, device=DEV) for _ in range(3))
    g = torch.zeros(n, dtype=BF16, device=DEV)
    at = [0, (1 << 31) - 1, 1 << 31, n - 1]
    g[at] = 1.0
    ap.aspis_adamw(ap.ParamList([p], [g], [m], [v]), 1, 0.25, eps=0.5)
    want = -0.25 / 1.5                                   # m^ = 1, v^ = 1
    assert p[at].tolist() == pytest.approx([want] * 4, rel=1e-6) and int((p != 0).sum()) == 4


@pytest.mark.gpu
def test_many_steps_follow_the_formula():
    """100 steps in 64 bits beside the kernel's: errors of a step are near u, and stay so"""
    s = make_state([4_000, 123], F32, F32, False, offsets=(0, 1))
    x, m, v = ([t.double() for t in s[k][1]] for k in ("p", "m", "v"))
    buf, lst, gen = ap.NormBuffers(DEV), param_list(s), generator(14)
    for step in range(1, 101):
        for t in s["g"][1]:
            t.copy_(torch.randn(t.shape, device=DEV, generator=gen))
        ap.aspis_adamw(lst, step, 1e-3, (0.9, 0.95), 1e-8, max_norm=1.0, norm=buf.norm, work=buf.work)
        f = coef(norms(s["g"][1])[1], 1.0)
        for i, g in enumerate(s["g"][1]):
            h = g.double() * f
            m[i] = 0.9 * m[i] + 0.1 * h
            v[i] = 0.95 * v[i] + 0.05 * h * h
            x[i] = x[i] * (1 - 1e-3 * s["decay"][i]) - 1e-3 * (m[i] / (1 - 0.9 ** step)) / ((v[i] / (1 - 0.95 ** step)).sqrt() + 1e-8)
    for i in range(2):
        # each step rounds x once and its move (at most 1e-3 * ~5) to about FACTOR
        close(s["p"][1][i], x[i], 100 * (U * 5 + 5e-3 * FACTOR) + 0 * x[i])


# ---------------------------------------------------------------- streams, graphs, refusals


@pytest.mark.gpu
def test_calls_follow_their_stream():
    gen = generator(15)
    ts = [torch.randn(n, device=DEV, generator=gen) for n in (3_000_000, 17, 250_000)]
    want = norms(ts)[1] * 2
    side = torch.cuda.Stream()
    buf, lst = ap.NormBuffers(DEV), ap.TensorList(ts)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        for t in ts:
            t.mul_(2.0)
        ap.aspis_clip_grads(lst, 1.0, buf.norm, buf.work)               # the current stream: side
        result = buf.norm.clone()
    side.synchronize()
    assert abs(float(result) - want) <= NORM * want
    assert norms(ts)[1] == pytest.approx(1.0, rel=1e-5)
    ap.aspis_grad_norm(lst, buf.norm, buf.work, stream=side)
    side.synchronize()
    assert float(buf.norm) == pytest.approx(1.0, rel=1e-5)


@pytest.mark.gpu
def test_a_captured_step_replays():
    s = make_state(LENGTHS["mixed"], BF16, BF16, True)
    buf, lst, glist = ap.NormBuffers(DEV), param_list(s), ap.TensorList(s["g"][1])
    graph = torch.cuda.CUDAGraph()
    start = {k: s[k][0].clone() for k in ("p", "g", "m", "v", "w")}
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        ap.aspis_clip_grads(glist, 1.0, buf.norm, buf.work)
        ap.aspis_adamw(lst, 3, max_norm=0.5, norm=buf.norm, work=buf.work, **HYPER)
    for _ in range(2):
        for k in start:
            s[k][0].copy_(start[k])
        graph.replay()
        torch.cuda.synchronize()
    got = {k: s[k][0].clone() for k in start}
    for k in start:
        s[k][0].copy_(start[k])
    ap.aspis_clip_grads(glist, 1.0, buf.norm, buf.work)
    ap.aspis_adamw(lst, 3, max_norm=0.5, norm=buf.norm, work=buf.work, **HYPER)
    assert all(torch.equal(got[k], s[k][0]) for k in start)


@pytest.mark.gpu
def test_a_list_keeps_its_memory():
    x = torch.full((1000,), 2.0, device=DEV)
    lst, buf = ap.TensorList([x]), ap.NormBuffers(DEV)
    del x
    y = torch.full((1000,), 5.0, device=DEV)             # would take x's place
    ap.aspis_grad_norm(lst, buf.norm, buf.work)
    assert float(buf.norm) == pytest.approx(2 * math.sqrt(1000), rel=NORM) and float(y[0]) == 5.0


@pytest.mark.gpu
def test_python_refusals():
    x, h = torch.ones(4, 6, device=DEV), torch.ones(4, 6, device=DEV, dtype=F16)
    for bad in ([x[:, :5]], [x[::2]], [x[:1].expand(4, 6)], [x.double()], [x.long()], [x.to_sparse()]):
        with pytest.raises(ValueError):
            ap.TensorList(bad)
    for out in ([x[:3]], [torch.ones(6, 4, device=DEV).t()], [], [x, x], [x.double()]):
        with pytest.raises(ValueError):
            ap.TensorList([x], out=out)
    a, b, c = (torch.ones(4, 6, device=DEV) for _ in range(3))
    for bad in (([x], [a], [b], [h]), ([x], [a[:3].contiguous()], [b], [c]), ([x], [a], [b], []), ([x], [a], [torch.ones(6, 4, device=DEV).t()], [c])):
        with pytest.raises(ValueError):
            ap.ParamList(*bad)
    with pytest.raises(ValueError):
        ap.ParamList([h], [a], [b], [c], masters=[h.clone()])
    with pytest.raises(ap.AspisError):
        ap.ParamList([x], [a], [b], [c], masters=[torch.ones(4, 6, device=DEV)])
    with pytest.raises(ap.AspisError):
        ap.ParamList([x], [a], [x], [c])
    lst, buf = ap.TensorList([x]), ap.NormBuffers(DEV)
    with pytest.raises(ValueError):
        ap.aspis_grad_norm(lst, buf.norm, buf.work[:100])
    with pytest.raises(ValueError):
        ap.aspis_grad_norm(lst, buf.norm.double(), buf.work)
    with pytest.raises(ValueError):
        ap.aspis_grad_norm(lst, buf.norm, buf.work, tensor_norms=torch.zeros(0, device=DEV))
    for kw in ({"scale": 0.0}, {"scale": math.nan}):
        with pytest.raises(ap.AspisError):
            ap.aspis_grad_norm(lst, buf.norm, buf.work, **kw)
    with pytest.raises(ap.AspisError):
        ap.aspis_clip_grads(lst, -1.0, buf.norm, buf.work)
    with pytest.raises(ap.AspisError):
        ap.aspis_adamw(ap.ParamList([x], [a], [b], [c]), 0, 0.1)
    assert bool((x == 1).all())


# ---------------------------------------------------------------- both sides of the rules on sizes


def random_lengths(rng, most, count):
    return [rng.choice([0, 1, 2, 7, 8, 9, 255, 256, 257]) if rng.random() < 0.4 else int(math.exp(rng.uniform(0, math.log(most))))
            for _ in range(count)]


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(12))
def test_random_lists(seed):
    """lists of random numbers, lengths, types and addresses, through every call with one workspace"""
    import random
    rng = random.Random(seed)
    gen, buf = generator(100 + seed), ap.NormBuffers(DEV)
    count = rng.choice([1, 5, 40, 130, 520, 1010])
    lengths = random_lengths(rng, rng.choice([300, 20_000, 400_000]), count)
    types = [rng.choice(TYPES) for _ in lengths]
    grads = [views([n], d, rng.randrange(9), gen, 10.0 ** rng.uniform(-4, 1))[1][0] for n, d in zip(lengths, types)]
    each = torch.zeros(count, device=DEV)
    ap.aspis_grad_norm(ap.TensorList(grads), buf.norm, buf.work, tensor_norms=each)
    want_each, want = norms(grads)
    assert abs(float(buf.norm) - want) <= NORM * want
    assert all(abs(x - y) <= NORM * y for x, y in zip(each.tolist(), want_each))
    outs = [views([n], rng.choice(TYPES), rng.randrange(9), gen)[1][0] for n in lengths]
    bound = want / 3
    ap.aspis_clip_grads(ap.TensorList(grads, outs), bound, buf.norm, buf.work)
    check_clip(grads, outs, coef(want, bound))
    parts = []
    for n, g in zip(lengths, grads):
        p, off = rng.choice(TYPES), rng.randrange(9)
        s = make_state([n], p, F32, p != F32 and rng.random() < 0.5, (off, 0), seed=rng.randrange(1 << 20))
        s["g"], s["decay"] = (None, [g]), [rng.choice([0.0, 0.1])]
        if rng.random() < 0.2:                           # a moment at another address than the rest
            s["v"] = views([n], F32, (off + 3) % 9, gen, 1.0)
            s["v"][1][0].square_()
        parts.append(s)
    olds = [copy_of(s) for s in parts]
    cat = lambda k: [s[k][1][0] if s[k] else None for s in parts]  # noqa: E731
    lst = ap.ParamList(cat("p"), grads, cat("m"), cat("v"), masters=cat("w"), weight_decay=[s["decay"][0] for s in parts])
    ap.aspis_adamw(lst, 11, max_norm=bound, norm=buf.norm, work=buf.work, **HYPER)
    assert abs(float(buf.norm) - want) <= NORM * want
    for s, old in zip(parts, olds):
        check_adamw(s, old, coef(want, bound), 11, **HYPER)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [(F32, None), (F32, F32), (BF16, F32), (F16, F16), (F32, BF16)])
@pytest.mark.parametrize("offset", [0, 3])
def test_clip_of_more_than_one_kernel_takes(dtype, out, offset):
    """a list too long for the cooperative kernel (64 MB of gradients), short tensors between long ones"""
    lengths = [9_000_001, 3, 0, 1000, 1, 17_000_000 if dtype == F32 else 40_000_000, 77, 5]
    _, ts = views(lengths, dtype, offset, generator(30))
    before = [t.clone() for t in ts]
    outs = ts if out is None else views(lengths, out, 0, generator(31))[1]
    want = norms(before)[1]
    got = clip(ts, None if out is None else outs, 0.25 * want)
    assert abs(got - want) <= NORM * want
    check_clip(before, outs, coef(want, 0.25 * want))


@pytest.mark.gpu
@pytest.mark.parametrize("n", [8, 256, 257, 2_048, 600_000, 655_000, 656_000, 3_000_000])
@pytest.mark.parametrize("ptype,gtype,master", [MIXES[0], MIXES[3], MIXES[9]])
def test_adamw_on_both_sides_of_the_cooperative_kernel(n, ptype, gtype, master):
    s = make_state([n, 5], ptype, gtype, master, (0, 1))
    old, buf = copy_of(s), ap.NormBuffers(DEV)
    ap.aspis_adamw(param_list(s), 3, max_norm=0.5, norm=buf.norm, work=buf.work, **HYPER)
    check_adamw(s, old, coef(norms(old["g"])[1], 0.5), 3, **HYPER)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [5, 3_000, 20_000_000])
@pytest.mark.parametrize("level", [1e-36, 1e-25, 1e22, 1e30])
def test_clip_and_adamw_outside_the_range_of_fp32_squares(n, level):
    x = (torch.rand(n, device=DEV, generator=generator(32)) + 0.5) * level
    want, out, buf = norms([x])[1], torch.empty_like(x), ap.NormBuffers(DEV)
    assert abs(clip([x], [out], want / 8) - want) <= NORM * want
    check_clip([x], [out], coef(want, want / 8))
    if level > 1:
        p, m, v = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(x)
        ap.aspis_adamw(ap.ParamList([p], [x], [m], [v]), 1, 0.1, max_norm=1.0, norm=buf.norm, work=buf.work)
        close(m, 0.1 * x.double() / want, 0.1 * x.double() / want * (FACTOR + 4 * U) + TINY)


@pytest.mark.gpu
def test_two_streams_with_buffers_of_their_own():
    gen = generator(33)
    lists = [[torch.randn(n, device=DEV, generator=gen) for n in (200_000 + i, 33, 1_000_000)] for i in range(2)]
    handles, bufs = [ap.TensorList(x) for x in lists], [ap.NormBuffers(DEV) for _ in lists]
    streams = [torch.cuda.Stream() for _ in lists]
    want = [norms(x)[1] for x in lists]
    torch.cuda.synchronize()
    for _ in range(50):                                  # below the bound: the gradients stay as they are
        for h, b, st in zip(handles, bufs, streams):
            ap.aspis_clip_grads(h, 1e9, b.norm, b.work, stream=st)
            ap.aspis_grad_norm(h, b.norm, b.work, stream=st)
    torch.cuda.synchronize()
    assert all(abs(float(b.norm) - w) <= NORM * w for b, w in zip(bufs, want))


@pytest.mark.gpu
def test_an_empty_list():
    buf = ap.NormBuffers(DEV)
    buf.norm.fill_(7.0)
    ap.aspis_clip_grads(ap.TensorList([]), 1.0, buf.norm, buf.work)
    assert float(buf.norm) == 0.0
    buf.norm.fill_(7.0)
    ap.aspis_adamw(ap.ParamList([], [], [], []), 1, 0.1, max_norm=1.0, norm=buf.norm, work=buf.work)
    assert float(buf.norm) == 0.0
    ap.aspis_adamw(ap.ParamList([], [], [], []), 1, 0.1)


@pytest.mark.gpu
def test_training_example():
    import importlib.util
    import os
    from conftest import ROOT
    spec = importlib.util.spec_from_file_location("train_step", os.path.join(ROOT, "examples", "train_step.py"))
    mod = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(mod)
    history = mod.train(steps=40, quiet=True)
    assert all(math.isfinite(h["loss"]) and math.isfinite(h["norm"]) for h in history)
    assert history[-1]["loss"] < 0.5 * history[0]["loss"]
    assert all(h["clique"] == 5 for h in history)        # both adversaries found every time
