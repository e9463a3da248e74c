"""Calls of include/aspis_worker.h that have no right answer, or none in fp32, are refused before anything is enqueued (CPU:
addresses are fake and never read)."""
import ctypes

import pytest

from test_worker_abi import AT, STEP, Stream, ap, calls, calls_on, embed, embed_grad, policy  # noqa: F401


def drop(p, step=None):
    return ctypes.byref(ap._Drop(p, 1, 2, 0, step))


@pytest.mark.parametrize("call", [embed, embed_grad])
@pytest.mark.parametrize("scale,p,status", [
    (2e38, 0.5, ap.E_RANGE), (-2e38, 0.5, ap.E_RANGE), (3.4028234e38, 2.0 ** -16, ap.E_RANGE), (6e33, 1 - 2.0 ** -16, ap.E_RANGE),
    (1e-40, 0.5, ap.E_RANGE),                                    # a factor that few bits are left of
    (2e38, 0.25, ap.OK), (5e33, 1 - 2.0 ** -16, ap.OK), (2e38, 0.0, ap.OK), (2e38, 1.0, ap.OK),
    (1e-40, 0.0, ap.OK), (0.0, 0.5, ap.OK), (-1.5, 0.5, ap.OK)])
def test_factors_beyond_the_range(call, scale, p, status):
    """scale times what stays is multiplied by is one fp32 number; with no columns nothing is enqueued where it is allowed"""
    assert call(scale=scale, drop=drop(p), width=0) == status
    if status != ap.OK:
        assert call(scale=scale, drop=drop(p)) == status


@pytest.mark.parametrize("change,status", [
    (dict(scale=1e30, grad_scale=1e30), ap.E_RANGE), (dict(scale=-1e30, grad_scale=1e30), ap.E_RANGE),
    (dict(scale=1e30, logit_scale=1e10), ap.E_RANGE), (dict(scale=1e-30, grad_scale=1e-12), ap.E_RANGE),
    (dict(scale=1e30, grad_scale=1e30, grad=None), ap.E_ALIGN),  # nothing is multiplied by it
    (dict(scale=1e30, grad_scale=0.0), ap.E_ALIGN), (dict(scale=1e-20, grad_scale=2.0 ** 60), ap.E_ALIGN),
    (dict(scale=1e30, grad_scale=1e30, logit_scale=1e-25), ap.E_ALIGN)])
def test_factors_of_the_loss(change, status):
    """grad_scale * scale * logit_scale is one fp32 number; work's address stops the calls that are allowed"""
    assert policy(work=AT + 9 * STEP + 8, **change) == status


@pytest.mark.parametrize("step,p,status", [
    (AT, 0.1, ap.E_INVAL), (AT + 64, 0.1, ap.E_INVAL), (AT + 3 * 320 + 248, 0.1, ap.E_INVAL),
    (AT + 256, 0.1, ap.E_ALIGN), (AT + 312, 0.1, ap.E_ALIGN),   # between the rows
    (AT + 4 * 320, 0.1, ap.E_ALIGN), (AT - 8, 0.1, ap.E_ALIGN), (AT, 0.0, ap.E_ALIGN)])   # (without a mask it is not read)
def test_step_of_a_mask_that_is_written(step, p, status):
    """What a call writes must not be what it reads; an address that comes after this check stops the calls that are allowed."""
    from test_worker_abi import dropout
    k = dict(drop=drop(p, step))
    if status != ap.E_ALIGN:
        assert dropout(x=AT + STEP, out=AT, ldo=80, **k) == status
    assert embed(out=AT, out_type=0, T=4, ld_out=80, tokens=AT + STEP + (2 if status == ap.E_ALIGN else 0), table=AT + 2 * STEP, **k) == status
    assert embed_grad(table_grad=AT, V=4, ld_table=80, grad=AT + 2 * STEP, work=AT + 3 * STEP + (8 if status == ap.E_ALIGN else 0), **k) == status


def test_step_in_the_workspace():
    assert embed_grad(drop=drop(0.1, AT + 3 * STEP + 64)) == ap.E_INVAL


@pytest.mark.parametrize("name,value", [("p", 0.5), ("seed", 2), ("stream", 3), ("first", 8), ("step", None)])
def test_a_mask_does_not_change(name, value):
    """its numbers are in the structure that the calls get: another value would not be seen there"""
    d = ap.Drop(0.1, 1, 2, 0)
    with pytest.raises(AttributeError):
        setattr(d, name, value)
    assert (d.p, d.seed, d.stream, d.first, d.step) == (0.1, 1, 2, 0, None)


def test_a_stream_of_another_device_is_refused_by_what_it_is(calls):
    """(these calls have no list)"""
    for call in calls_on(0, Stream(1)):
        with pytest.raises(ValueError, match="^stream must be on device 0, got 1$"):
            call()
    assert calls == []
