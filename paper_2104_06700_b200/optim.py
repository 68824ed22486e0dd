"""AdamW over all parameters, a launch for those of one kind, its states in 32 or 8 bits, with clipping by the norm of all gradients
(dg_adamw_step and dg_grad_norm), behind torch's optimiser interface."""
from __future__ import annotations

import itertools
import operator
from typing import Optional

import torch

from . import binding


_NONE = itertools.repeat(None)


class _Table:
    """The library's list of a group's parameters, with what it was made of."""

    def __init__(self, params, states, entries, grads, ids):
        self.params, self.states, self.entries = list(params), states, entries
        columns = [[s["exp_avg"] for s in states], [s["exp_avg_sq"] for s in states], [s["step"] for s in states],
                   [s.get("scales") for s in states]]
        masters = [s.get("master") for s in states]
        self.targets, self.copies = self.params, None
        if not all(map(operator.is_, masters, _NONE)):
            self.targets = [p if m is None else m for p, m in zip(params, masters)]
            self.copies = [None if m is None else p for p, m in zip(params, masters)]
        self.tensors = [t for column in columns for t in column if t is not None]
        self.places = list(map(binding._data_ptr, self.tensors))
        self.list = binding.AdamwList(grads, self.targets, *columns, self.copies, ids)


def _check_options(options) -> None:
    if options["state_bits"] not in (8, 32):
        raise ValueError(f"state_bits must be 8 or 32, got {options['state_bits']}")
    if not options["lr"] >= 0 or not options["eps"] >= 0 or not options["weight_decay"] >= 0:
        raise ValueError("lr, eps and weight_decay must not be negative")
    if len(options["betas"]) != 2 or not all(0 <= b < 1 for b in options["betas"]):
        raise ValueError(f"betas must be in [0, 1), got {options['betas']}")


class AdamW(torch.optim.Optimizer):
    """torch.optim.AdamW's update (decoupled weight decay) for fp32 and bf16 parameters on one GPU.

    ``state_bits``: 8 keeps the averages of tensors of ``min_8bit_size`` numbers and more in e4m3 with a scale for every
    256 (2.03 bytes a number instead of 8); they are rounded up or down at random, by a hash of ``seed``, the step and the place.
    ``master_weights``: bf16 parameters get fp32 master weights in the state and are their roundings.  Without them a bf16
    parameter itself is rounded at random, so that small steps are not lost.
    ``max_norm``: gradients are scaled as clip_grad_norm_ would (the norm is that of all groups' gradients together); they are
    left as they are.  ``grad_norm`` is the last step's, a tensor of one number that the next step overwrites.

    A parameter's state: ``step`` (int64, on the device: a step can be captured into a CUDA graph once it has run outside one),
    ``exp_avg``, ``exp_avg_sq`` (with 8 bits the square root of it, and ``scales`` (blocks, 2) of both), ``master``.  lr and the
    other options are taken by value: a captured step repeats them.
    """

    def __init__(self, params, lr: float = 1e-3, betas=(0.9, 0.999), eps: float = 1e-8, weight_decay: float = 1e-2,
                 state_bits: int = 32, min_8bit_size: int = 4096, master_weights: bool = False,
                 max_norm: Optional[float] = None, seed: int = 0):
        if max_norm is not None and not max_norm > 0:
            raise ValueError(f"max_norm must be positive, got {max_norm}")
        defaults = dict(lr=lr, betas=betas, eps=eps, weight_decay=weight_decay, state_bits=state_bits,
                        min_8bit_size=min_8bit_size, master_weights=master_weights, seed=seed)
        _check_options(defaults)
        self.max_norm, self.grad_norm = max_norm, None
        self._workspace = self._result = None
        self._tables, self._known_state, self._standing = {}, None, False
        super().__init__(params, defaults)

    def add_param_group(self, group) -> None:
        _check_options({**self.defaults, **group})
        super().add_param_group(group)
        params = self.param_groups[-1]["params"]
        if len(set(params)) != len(params):
            self.param_groups.pop()
            raise ValueError("a parameter stands in its group twice: one launch would update it twice at once")

    def __getstate__(self):     # workspaces are not state
        state = super().__getstate__()
        return {**state, "max_norm": self.max_norm}

    def __setstate__(self, state) -> None:
        super().__setstate__(state)
        self.__dict__.setdefault("max_norm", None)
        self.grad_norm = self._workspace = self._result = None
        self._tables, self._known_state, self._standing = {}, None, False

    def load_state_dict(self, state_dict) -> None:
        """torch's would cast every state to its parameter's type.  The states are new tensors: a step captured before must not be
        replayed afterwards."""
        given = {}      # what the registered hooks made of it: ours comes behind the others, and before theirs when it is loaded
        ours = [self.register_load_state_dict_pre_hook(lambda _, last: given.update(last)),
                self.register_load_state_dict_post_hook(lambda _: self._take_states(given), prepend=True)]
        try:
            super().load_state_dict(state_dict)
        finally:
            for handle in ours:
                handle.remove()

    def _take_states(self, state_dict) -> None:
        saved = state_dict["state"]
        params = [p for group in self.param_groups for p in group["params"]]
        numbers = [i for group in state_dict["param_groups"] for i in group["params"]]
        for i, p in zip(numbers, params):
            if i in saved:
                self.state[p] = {k: v.detach().to(p.device, copy=True).contiguous() if torch.is_tensor(v) else v
                                 for k, v in saved[i].items()}

    def _new_state(self, p: torch.Tensor, group) -> dict:
        if not p.is_cuda or p.dtype not in (torch.float32, torch.bfloat16) or not p.is_contiguous():
            raise ValueError("parameters must be contiguous fp32 or bf16 CUDA tensors")
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("run a step before capturing one: a captured first step would begin anew at every replay")
        eight = group["state_bits"] == 8 and p.numel() >= group["min_8bit_size"]
        dtype = torch.float8_e4m3fn if eight else torch.float32
        state = {"step": torch.zeros((), dtype=torch.int64, device=p.device),
                 "exp_avg": torch.zeros(p.shape, dtype=torch.float32, device=p.device).to(dtype),
                 "exp_avg_sq": torch.zeros(p.shape, dtype=torch.float32, device=p.device).to(dtype)}
        if eight:
            state["scales"] = torch.zeros(((p.numel() + 255) // 256, 2), dtype=torch.float32, device=p.device)
        if group["master_weights"] and p.dtype == torch.bfloat16:
            state["master"] = p.detach().float()
        return state

    def _table(self, at: int, group, first: int):
        """(gradients, the library's list) of the group's parameters that have one; the random bits of the i-th go by first + i.
        The list is made anew when any of its parameters or states is another tensor, or lies elsewhere, than in the last step."""
        ids, params = range(first, first + len(group["params"])), group["params"]
        grads = [p.grad for p in params]
        if any(map(operator.is_, grads, _NONE)):
            some = [(i, p, g) for i, p, g in zip(ids, params, grads) if g is not None]
            if not some:
                return None
            ids, params, grads = zip(*some)
        known = self._tables.get(at)
        same = self._standing and known is not None and len(known.params) == len(params) and all(
            map(operator.is_, known.params, params))
        states = known.states if same else [self.state[p] for p in params]
        entries = list(itertools.chain.from_iterable(map(dict.values, states)))
        same = same and len(entries) == len(known.entries) and all(map(operator.is_, entries, known.entries)) and \
            list(map(binding._data_ptr, known.tensors)) == known.places
        if not same:
            known = None
            if not all(states):
                for p, s in zip(params, states):
                    if not s:
                        s.update(self._new_state(p, group))
                entries = list(itertools.chain.from_iterable(map(dict.values, states)))
        if not all(map(binding._contiguous, grads)):     # sparse ones are not either
            if any(g.layout is not torch.strided for g in grads):
                raise ValueError("sparse gradients are not supported")
            grads = [g.contiguous() for g in grads]      # copies live until the launch, then the allocator's stream order serves
        if known is None:
            known = self._tables[at] = _Table(params, states, entries, grads, ids)
        else:
            known.list.refresh(grads, known.targets, known.copies)
        return grads, known.list

    @torch.no_grad()
    def step(self, closure=None):
        loss = None
        if closure is not None:
            with torch.enable_grad():
                loss = closure()
        device = next((p.device for group in self.param_groups for p in group["params"] if p.grad is not None), None)
        if device is None:
            return loss
        if device.type != "cuda":
            raise ValueError("parameters must be contiguous fp32 or bf16 CUDA tensors")
        if device.index == torch.cuda.current_device():
            self._launch(device)
        else:
            with torch.cuda.device(device):
                self._launch(device)
        return loss

    def _launch(self, device) -> None:
        state = list(self.state), list(self.state.values())
        self._standing = self._known_state is not None and all(
            len(known) == len(now) and all(map(operator.is_, known, now)) for known, now in zip(self._known_state, state))
        self._known_state = state
        parts, first = [], 0
        for at, group in enumerate(self.param_groups):
            table = self._table(at, group, first)
            first += len(group["params"])
            if table is not None:
                parts.append((group, *table))
        if self._workspace is None or self._workspace.device != device:
            if torch.cuda.is_current_stream_capturing():
                raise RuntimeError("run a step before capturing one")
            self._workspace = binding.adamw_workspace(device)
            self._result = torch.zeros(2, dtype=torch.float32, device=device)
            self._norm, self._factor = self._result[0], self._result[1]
        factor = None
        if self.max_norm is not None:
            every = parts[0][2] if len(parts) == 1 else binding.AdamwList([g for _, grads, _ in parts for g in grads])
            binding.dg_grad_norm(every, self.max_norm, self._workspace, self._result)
            self.grad_norm, factor = self._norm, self._factor
        for group, _, table in parts:
            beta1, beta2 = group["betas"]
            binding.dg_adamw_step(table, group["lr"], beta1, beta2, group["eps"], group["weight_decay"], self._workspace,
                                  factor, group["seed"])
            table.forget_gradients()
