"""What dg_adamw_step, dg_grad_norm and optim.AdamW refuse, and their host side, without a GPU."""
import ctypes
import struct
from array import array

import pytest
import torch

from paper_2104_06700_b200 import binding, optim
from test_host_side import fake, library  # noqa: F401

i64, f32, f64 = ctypes.c_int64, ctypes.c_float, ctypes.c_double
OK, BAD = binding.DG_OK, binding.DG_ERR_INVALID_ARG
FIELDS = dict(numbers="q", param="Q", grad="Q", exp_avg="Q", exp_avg_sq="Q", scales="Q", copy="Q", step="Q", param_type="i",
              grad_type="i", state_bits="i", id="I")       # dg_adamw_list_t, behind `tensors`


def tensor(fake, n=300, **changed):
    a = lambda count: (fake.array(count + 4).value + 15) // 16 * 16  # noqa: E731
    return {**dict(zip(FIELDS, (n, a(n), a(n), a(n), a(n), 0, 0, a(2), 0, 0, 32, 0))), **changed}


def listed(fake, tensors, count=None, absent=()):
    """A dg_adamw_list_t; arrays named in `absent` are NULL."""
    columns = {k: array(code, [t[k] for t in tensors]) for k, code in FIELDS.items()}
    fake.keep.append(columns)
    where = [0 if k in absent else c.buffer_info()[0] for k, c in columns.items()]
    return struct.pack("q12Q", len(tensors) if count is None else count, *where)


def workspace(fake, shift=0):
    return ctypes.c_void_p((fake.array(4096).value + 255) // 256 * 256 + shift)


def step(fake, *tensors, ws=None, lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, decay=0.0, count=None, absent=()):
    return fake.lib.dg_adamw_step(listed(fake, tensors, count, absent), f64(lr), f64(beta1), f64(beta2), f64(eps), f64(decay),
                                  None, ctypes.c_uint64(1), ws or workspace(fake), None)


def norm(fake, *tensors, ws=None, max_norm=1.0, result=True, absent=()):
    return fake.lib.dg_grad_norm(listed(fake, tensors, None, absent), f32(max_norm), ws or workspace(fake),
                                 fake.array(2) if result else None, None)


def test_lists_with_arrays_left_out(fake):
    t = tensor(fake)
    assert step(fake, t, absent=("scales", "copy", "id")) == OK
    assert step(fake, tensor(fake, state_bits=8), absent=("scales",)) == BAD
    for name in set(FIELDS) - {"scales", "copy", "id"}:
        assert step(fake, t, absent=(name,)) == BAD, name
        assert norm(fake, t, absent=(name,)) == (BAD if name in ("numbers", "grad", "grad_type") else OK), name
    assert fake.lib.dg_adamw_step(None, f64(0), f64(0), f64(0), f64(0), f64(0), None, ctypes.c_uint64(1), workspace(fake), None) == BAD
    assert fake.lib.dg_grad_norm(None, f32(1), workspace(fake), fake.array(2), None) == BAD


def test_lists_that_are_refused(fake):
    assert step(fake) == OK and norm(fake) == OK
    scales = fake.array(8).value // 16 * 16 + 16
    assert step(fake, tensor(fake), tensor(fake, state_bits=8, scales=scales), tensor(fake, n=0, param=0, grad=0)) == OK
    for wrong in (dict(param=0), dict(exp_avg=0), dict(exp_avg_sq=0), dict(step=0), dict(state_bits=16),
                  dict(state_bits=8), dict(param_type=2), dict(param_type=1, copy=4096), dict(param=4098), dict(exp_avg=4097),
                  dict(exp_avg_sq=4098), dict(copy=4097), dict(step=4100), dict(state_bits=8, scales=4100)):
        assert step(fake, tensor(fake), tensor(fake, **wrong)) == BAD, wrong
        assert norm(fake, tensor(fake), tensor(fake, **wrong)) == OK, wrong
    for wrong in (dict(grad=0), dict(numbers=-1), dict(numbers=(1 << 40) + 1), dict(grad_type=2), dict(grad=4098),
                  dict(grad_type=1, grad=4097)):
        assert step(fake, tensor(fake, **wrong)) == BAD and norm(fake, tensor(fake, **wrong)) == BAD, wrong
    assert step(fake, count=-1) == BAD and step(fake, tensor(fake), count=(1 << 31) + 1) == BAD
    for shift in (8, 128):
        assert step(fake, tensor(fake), ws=workspace(fake, shift)) == BAD
        assert norm(fake, tensor(fake), ws=workspace(fake, shift)) == BAD
    assert norm(fake, tensor(fake), result=False) == BAD
    odd = ctypes.c_void_p(fake.array(4).value + 2)
    assert fake.lib.dg_grad_norm(listed(fake, [tensor(fake)]), f32(1), workspace(fake), odd, None) == BAD
    assert fake.lib.dg_adamw_step(listed(fake, [tensor(fake)]), f64(0), f64(0), f64(0), f64(0), f64(0), odd, ctypes.c_uint64(1),
                                  workspace(fake), None) == BAD
    assert norm(fake, tensor(fake), max_norm=-1.0) == norm(fake, tensor(fake), max_norm=float("nan")) == BAD


def test_options_that_are_refused(fake):
    nan, inf = float("nan"), float("inf")
    for wrong in [dict(lr=v) for v in (-1.0, nan, inf)] + [dict(eps=v) for v in (-1e-8, nan, inf)] + [
            dict(decay=v) for v in (-1.0, nan, inf)] + [{b: v} for b in ("beta1", "beta2") for v in (-0.1, 1.0, nan)]:
        assert step(fake, tensor(fake), **wrong) == BAD, wrong
    assert step(fake, tensor(fake), lr=0.0, beta1=0.0, beta2=0.0, eps=0.0) == OK


def test_launches_and_their_failures(fake):
    fake.events()
    assert step(fake, *[tensor(fake, n=4)] * 801) == OK
    assert [what.split("kernel")[0][-6:] for what, _, _ in fake.events()] == ["adamw_"] * 3     # no memory of its own
    fake.lib.fake_failing_kernel(b"adamw_kernel")
    assert step(fake, tensor(fake)) == binding.DG_ERR_CUDA
    fake.lib.fake_failing_kernel(b"grad_norm_kernel")
    assert norm(fake, tensor(fake)) == binding.DG_ERR_CUDA


def test_the_optimiser_checks_its_options():
    p = torch.nn.Parameter(torch.zeros(8))
    for wrong in (dict(lr=-1), dict(lr=float("nan")), dict(eps=-1), dict(weight_decay=-1), dict(betas=(0.9, 1.0)),
                  dict(betas=(-0.1, 0.9)), dict(state_bits=4), dict(max_norm=0), dict(max_norm=-1.0)):
        with pytest.raises(ValueError):
            optim.AdamW([p], **wrong)
    with pytest.raises(ValueError, match="twice"):
        optim.AdamW([p, p])
    opt = optim.AdamW([p])
    opt.step()
    p.grad = torch.zeros(8)
    with pytest.raises(ValueError, match="CUDA"):
        opt.step()
    with pytest.raises(ValueError, match="CUDA"):
        binding.AdamwList([p])
