"""The per-bird encoder's entry points reject bad arguments on the host before
touching any device, and empty calls are no-ops (no GPU needed)."""

import ctypes
import math

import pytest
import torch

from paper_2512_07009_amd import binding

FAKE = ctypes.c_void_p(0x100000)       # never dereferenced on these paths
FAKE2 = ctypes.c_void_p(0x100002)
FAKE4 = ctypes.c_void_p(0x100004)
FAKE8 = ctypes.c_void_p(0x100008)
F32, F16, BF16 = 0, 1, 2


def refused(status, needle):
    assert status == binding.FLOCK_EINVAL
    assert needle in binding.lib().flock_last_error().decode()


def norm(dtype=BF16, x=FAKE, xs=64, r=None, rs=0, rows=4, width=64, w=FAKE, b=FAKE, eps=1e-5, y=FAKE, ys=64, s=None,
         ss=0, mean=FAKE, rstd=FAKE):
    return binding.lib().layer_norm_rows(dtype, x, xs, r, rs, rows, width, w, b, eps, y, ys, s, ss, mean, rstd, None)


@pytest.mark.parametrize("kwargs,needle", [
    (dict(dtype=3), "dtype"), (dict(dtype=-1), "dtype"), (dict(rows=-1), "rows"), (dict(width=0), "width"),
    (dict(width=(1 << 20) + 1), "width"), (dict(eps=-1.0), "eps"), (dict(eps=math.nan), "eps"), (dict(xs=-1), "strides"),
    (dict(ys=63), "hold a row"), (dict(x=None), "non-NULL"), (dict(y=None), "non-NULL"),
    (dict(r=FAKE, rs=64, ss=64), "sum"), (dict(r=FAKE, rs=64, s=FAKE, ss=1), "hold a row"),
    (dict(dtype=F32, x=FAKE2), "aligned"), (dict(w=FAKE2), "aligned"), (dict(mean=FAKE2), "aligned"),
])
def test_layer_norm_rejects(kwargs, needle):
    refused(norm(**kwargs), needle)


def norm_back(dtype=BF16, gy=FAKE, gys=64, gs=None, gss=0, x=FAKE, xs=64, rows=4, width=64, w=FAKE, mean=FAKE, rstd=FAKE,
              dx=FAKE, dxs=64, dw=FAKE, db=FAKE, ws=None, n=0):
    return binding.lib().layer_norm_rows_backward(dtype, gy, gys, gs, gss, x, xs, rows, width, w, mean, rstd, dx, dxs, dw,
                                                  db, ws, n, None)


@pytest.mark.parametrize("kwargs,needle", [
    (dict(dtype=9), "dtype"), (dict(rows=-2), "rows"), (dict(width=-1), "width"), (dict(gys=-1), "strides"),
    (dict(gs=FAKE, gss=-8), "strides"), (dict(dxs=8), "hold a row"), (dict(gy=None), "non-NULL"),
    (dict(mean=None), "non-NULL"), (dict(dx=None), "non-NULL"), (dict(dw=FAKE2), "aligned"),
    (dict(dtype=F32, x=FAKE2), "aligned"),
])
def test_layer_norm_backward_rejects(kwargs, needle):
    refused(norm_back(**kwargs), needle)


FREQ = (ctypes.c_double * 3)(1.0, 2.0, 3.0)
NAN = (ctypes.c_double * 3)(1.0, math.nan, 3.0)


def rotary(dtype=BF16, q=FAKE, qs=128, k=FAKE, ks=64, total=4, hq=2, hk=1, dim=64, xy=FAKE, time=FAKE, freq=FREQ, nt=1,
           ny=1, nx=1, il=0, inv=0, qo=FAKE8, qos=128, ko=FAKE8, kos=64):
    return binding.lib().rotary_frames(dtype, q, qs, k, ks, total, hq, hk, dim, xy, time, freq, nt, ny, nx, il, inv, qo,
                                       qos, ko, kos, None)


@pytest.mark.parametrize("kwargs,needle", [
    (dict(dtype=7), "dtype"), (dict(total=-1), "total"), (dict(hq=0, hk=0), "heads"), (dict(hq=257), "heads"),
    (dict(dim=0), "head_dim"), (dict(dim=258), "head_dim"), (dict(nt=-1), "pairs"), (dict(nt=0, ny=0, nx=0), "pairs"),
    (dict(nx=31, dim=64), "pairs"), (dict(freq=None), "freq"), (dict(freq=NAN), "finite"), (dict(qs=-1), "strides"),
    (dict(qos=100), "strides"), (dict(q=FAKE, qo=FAKE, qos=136), "in place"), (dict(q=None), "non-NULL"),
    (dict(ko=None), "non-NULL"), (dict(xy=None), "xy"), (dict(time=None), "time"), (dict(xy=FAKE4), "aligned"),
    (dict(dtype=F32, q=FAKE2), "aligned"),
])
def test_rotary_rejects(kwargs, needle):
    refused(rotary(**kwargs), needle)


def attention(dtype=BF16, q=FAKE, qs=128, k=FAKE, ks=64, v=FAKE, vs=64, qo=FAKE, ko=FAKE, frames=2, tq=8, tk=8, hq=2, hk=1,
              dim=64, qxy=None, kxy=None, slopes=None, keep=None, causal=0, prefix=None, scale=0.125, cap=0.0, out=FAKE,
              os=128, lse=FAKE, ws=None, n=0):
    return binding.lib().attention_frames(dtype, q, qs, k, ks, v, vs, qo, ko, frames, tq, tk, hq, hk, dim, qxy, kxy, slopes,
                                          keep, causal, prefix, scale, cap, out, os, lse, ws, n, None)


SHARED = [
    (dict(dtype=F32), "dtype"), (dict(dtype=5), "dtype"), (dict(frames=-1), "n_frames"), (dict(tq=-1), "total_q"),
    (dict(tk=-1), "total_k"), (dict(hq=0), "heads"), (dict(hk=300, hq=300), "heads"), (dict(hq=3, hk=2), "multiple"),
    (dict(dim=0), "head_dim"), (dict(dim=60), "head_dim"), (dict(dim=136), "head_dim"), (dict(causal=2), "causal"),
    (dict(scale=0.0), "scale"), (dict(scale=math.inf), "scale"), (dict(cap=-1.0), "cap"), (dict(cap=math.nan), "cap"),
    (dict(qs=-8), "strides"), (dict(ks=60), "strides"), (dict(os=64), "stride"), (dict(qo=None), "offsets"),
    (dict(ko=None), "offsets"), (dict(q=None), "non-NULL"), (dict(v=None), "non-NULL"), (dict(slopes=FAKE), "q_xy"),
    (dict(q=FAKE8), "16-byte"), (dict(out=FAKE8), "16-byte"), (dict(slopes=FAKE, qxy=FAKE4, kxy=FAKE), "8-byte"),
    (dict(qo=FAKE2), "4-byte"), (dict(lse=FAKE4), "8-byte"),
]


@pytest.mark.parametrize("kwargs,needle", SHARED)
def test_attention_rejects(kwargs, needle):
    refused(attention(**kwargs), needle)


def test_attention_rejects_batches_beyond_its_grid():
    st = attention(tq=2 ** 31 - 1, hq=256, hk=256, dim=8, qs=2048, os=2048)
    assert st == binding.FLOCK_EUNSUPPORTED


def attention_back(dtype=BF16, go=FAKE, gos=128, q=FAKE, qs=128, k=FAKE, ks=64, v=FAKE, vs=64, out=FAKE, os=128, lse=FAKE,
                   qo=FAKE, ko=FAKE, frames=2, tq=8, tk=8, hq=2, hk=1, dim=64, qxy=None, kxy=None, slopes=None, keep=None,
                   causal=0, prefix=None, scale=0.125, cap=0.0, dq=FAKE, dqs=128, dk=FAKE, dks=64, dv=FAKE, dvs=64, ds=None,
                   ws=None, n=0):
    return binding.lib().attention_frames_backward(dtype, go, gos, q, qs, k, ks, v, vs, out, os, lse, qo, ko, frames, tq, tk,
                                                   hq, hk, dim, qxy, kxy, slopes, keep, causal, prefix, scale, cap, dq, dqs,
                                                   dk, dks, dv, dvs, ds, ws, n, None)


@pytest.mark.parametrize("kwargs,needle", SHARED + [
    (dict(gos=-8), "grad_out"), (dict(gos=4), "grad_out"), (dict(dqs=64), "hold a row"), (dict(dks=8), "hold a row"),
    (dict(dvs=68), "multiples of 8"), (dict(ds=FAKE), "without slopes"), (dict(go=None), "non-NULL"),
    (dict(lse=None), "non-NULL"), (dict(dk=None), "non-NULL"), (dict(dq=FAKE8), "16-byte"),
    (dict(slopes=FAKE, qxy=FAKE, kxy=FAKE, ds=FAKE2), "4-byte"),
])
def test_attention_backward_rejects(kwargs, needle):
    refused(attention_back(**kwargs), needle)


def test_empty_calls_without_a_device():
    lib = binding.lib()
    assert norm(rows=0, x=None, y=None, w=None, b=None, mean=None, rstd=None) == 0
    assert norm_back(rows=0, gy=None, x=None, mean=None, rstd=None, dx=None, dw=None, db=None) == 0
    assert rotary(total=0, q=None, k=None, xy=None, time=None, qo=None, ko=None) == 0
    assert attention(frames=0, tq=0, tk=0, q=None, k=None, v=None, qo=None, ko=None, out=None, lse=None) == 0
    assert attention(tq=0, q=None, out=None, lse=None) == 0
    assert attention_back(frames=0, tq=0, tk=0) == 0
    assert lib.flock_last_error().decode() == ""


def test_workspace_queries():
    lib = binding.lib()
    assert lib.layer_norm_rows_backward_workspace(0, 512) == 0
    assert lib.layer_norm_rows_backward_workspace(500, 512) >= 125 * 2 * 512 * 4
    assert lib.attention_frames_workspace(0, 0, 0, 8, 8, 64) == 0
    assert lib.attention_frames_workspace(64, 128000, 128000, 8, 8, 64) == 0
    # one query over a long history: shares of its keys are joined from the workspace
    assert lib.attention_frames_workspace(1, 1, 9000, 8, 2, 64) > 0
    assert lib.attention_frames_backward_workspace(64, 128000, 128000, 8, 8, 64) >= 128000 * 8 * 4
    assert lib.attention_frames_backward_workspace(0, 0, 0, 8, 8, 64) == 0


# Threads of a launch are numbered in 32 bits: 2^24 - 1 workgroups of 256.
@pytest.mark.parametrize("kwargs", [
    dict(frames=2 ** 21, tq=2 ** 21, tk=2 ** 21, hq=8, hk=8, qs=512, ks=512, vs=512, os=512),    # a tile a track
    dict(frames=2 ** 21 - 1, tq=2 ** 27, tk=8, hq=8, hk=8, qs=512, ks=512, vs=512, os=512),
    dict(frames=1, tq=2 ** 31 - 300, tk=8, hq=2, hk=2),
])
def test_attention_rejects_more_workgroups_than_a_launch_holds(kwargs):
    assert attention(**kwargs) == binding.FLOCK_EUNSUPPORTED
    assert "workgroups" in binding.lib().flock_last_error().decode()
    assert attention_back(**dict(kwargs, dqs=512, dks=512, dvs=512)) == binding.FLOCK_EUNSUPPORTED
    assert "workgroups" in binding.lib().flock_last_error().decode()


@pytest.mark.parametrize("kwargs", [
    dict(frames=2 ** 19, tq=2 ** 19, tk=2 ** 19, hq=8, hk=8, qs=512, ks=512, vs=512, os=512),
    dict(frames=1, tq=2 ** 28, tk=8, hq=2, hk=2),
])
def test_attention_takes_batches_within_a_launch(kwargs):
    """What ends such a call here is the missing device, or its other error, not its size."""
    assert attention(**kwargs, lse=FAKE4) == binding.FLOCK_EINVAL
    if not torch.cuda.is_available():
        assert attention(**kwargs) == binding.FLOCK_EDEVICE
        assert attention_back(**dict(kwargs, dqs=512, dks=512, dvs=512)) == binding.FLOCK_EDEVICE


def test_attention_backward_rejects_too_many_keys():
    assert attention_back(tk=2 ** 31 - 1, tq=8, frames=1, hq=2, hk=2, ks=128, vs=128, dks=128, dvs=128) == \
        binding.FLOCK_EUNSUPPORTED


def test_attention_rejects_keys_beyond_its_numbers():
    """A loop over a frame's keys looks up to two tiles of 128 ahead, in 31 bits."""
    most = 2 ** 31 - 256
    assert attention(frames=1, tq=1, tk=most + 1, hq=1, hk=1) == binding.FLOCK_EUNSUPPORTED
    assert "keys" in binding.lib().flock_last_error().decode()
    assert attention(frames=1, tq=1, tk=most, hq=1, hk=1, lse=FAKE4) == binding.FLOCK_EINVAL
    if not torch.cuda.is_available():
        assert attention(frames=1, tq=1, tk=most, hq=1, hk=1) == binding.FLOCK_EDEVICE
