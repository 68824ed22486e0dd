"""Lists of tensors for the AdamW calls (binding.AdamwList): what they refuse, without a GPU."""
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
