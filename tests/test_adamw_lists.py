"""Lists of tensors for the AdamW calls (binding.AdamwList): what they refuse, and that a refusal leaves them whole, without a GPU."""
import struct

import pytest
import torch

from paper_2104_06700_b200 import binding


@pytest.fixture
def on_cpu(monkeypatch):
    """Lists of CPU tensors: types and sizes are checked, where they lie is not."""
    def check(tensors, dtypes, device, name):
        types = [t.dtype for t in tensors]
        if not dtypes.issuperset(types):
            raise TypeError(name)
        return types
    monkeypatch.setattr(binding, "_check_tensors", check)


def arrays_are_its_own(a, count):
    """What the struct points to are the list's arrays, with as many entries as tensors."""
    got = struct.unpack("q12Q", a.struct)
    assert got[0] == count
    for where, field in zip(got[1:], a._fields):
        assert where == (0 if field is None else field.buffer_info()[0])
        assert field is None or len(field) == count


def test_a_refused_refresh_leaves_the_list_as_it_was(on_cpu):
    n = [5, 300, 7]
    f = lambda dtype=torch.float32: [torch.zeros(k, dtype=dtype) for k in n]  # noqa: E731
    grads, params, copies = f(), f(), f(torch.bfloat16)
    a = binding.AdamwList(grads, params, f(), f(), [torch.zeros((), dtype=torch.int64) for _ in n], copies=copies)
    arrays_are_its_own(a, 3)
    was, fields = a.struct, list(a._fields)
    short = [torch.zeros(k - 1) for k in n]
    for wrong in ((short, params, copies), (f(torch.bfloat16), short, copies), (f(torch.bfloat16), f(torch.bfloat16), short),
                  (grads, params, [c[1:] for c in copies]), (f(torch.float64), params, copies), (grads[:2], params, copies),
                  (grads, params[:2], copies), (grads, params, copies[:2])):
        with pytest.raises((ValueError, TypeError)):
            a.refresh(*wrong)
        assert a.struct == was and all(x is y for x, y in zip(a._fields, fields))
        arrays_are_its_own(a, 3)
    moved = f(torch.bfloat16)
    a.refresh(moved, params, copies)
    arrays_are_its_own(a, 3)
    assert list(a._fields[2]) == [t.data_ptr() for t in moved] and list(a._fields[9]) == [binding.DG_BF16] * 3
    a.refresh(grads, params, None)
    arrays_are_its_own(a, 3)
    assert a._fields[6] is None and list(a._fields[9]) == [binding.DG_F32] * 3


def test_columns_of_another_length_are_refused(on_cpu):
    """The library reads as many entries of every array as there are tensors."""
    n = [5, 300, 7]
    f = lambda dtype=torch.float32, few=3: [torch.zeros(k, dtype=dtype) for k in n[:few]]  # noqa: E731
    steps = [torch.zeros((), dtype=torch.int64) for _ in range(4)]
    given = dict(grads=f(), params=f(), exp_avgs=f(), exp_avg_sqs=f(), steps=steps[:3], scales=[None] * 3,
                 copies=f(torch.bfloat16), ids=[1, 2, 3])
    binding.AdamwList(**given)
    for few in (0, 2):
        for name in given:
            if name != "grads":
                with pytest.raises(ValueError):
                    binding.AdamwList(**{**given, name: given[name][:few]})
    for name, more in (("params", f() + f(few=1)), ("steps", steps), ("scales", [None] * 4), ("copies", [None] * 4), ("ids", [1] * 4)):
        with pytest.raises(ValueError):
            binding.AdamwList(**{**given, name: more})
    e4m3 = [torch.zeros(k, dtype=torch.float8_e4m3fn) for k in n]
    scales = [torch.zeros((k + 255) // 256, 2) for k in n]
    eight = dict(given, exp_avgs=e4m3, exp_avg_sqs=e4m3)
    binding.AdamwList(**{**eight, "scales": scales})
    for wrong in (scales[:2], scales + [None], []):
        with pytest.raises((ValueError, TypeError)):
            binding.AdamwList(**{**eight, "scales": wrong})
