"""AdamW over many tensors (dg_adamw_step, dg_grad_norm, optim.AdamW) against the same step in 64 bits: types, sizes around
a task of 256 numbers, alignments, lists longer than a launch takes, states in 8 bits with their roundings."""
import copy

import pytest
import torch

import adamw_util as ref
from paper_2104_06700_b200 import binding, optim

pytestmark = pytest.mark.gpu
DEV = "cuda"
F32, BF16, E4M3 = torch.float32, torch.bfloat16, torch.float8_e4m3fn
U = ref.U
SIZES = [1, 3, 4, 255, 256, 257, 1000, 4097, 40001]
HYPER = dict(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1)


class Tensor:
    """A parameter of n numbers with a gradient and states after `taken` steps, all shifted by `shift` numbers."""

    def __init__(self, n, p_type, g_type, bits, seed, master=False, taken=7, shift=0, spread=1.0):
        gen = torch.Generator(device=DEV).manual_seed(seed)
        r = lambda: torch.randn(n, device=DEV, generator=gen)  # noqa: E731

        def place(t):
            return torch.empty(n + shift, dtype=t.dtype, device=DEV)[shift:].copy_(t)

        self.n, self.bits, self.id = n, bits, seed
        self.grad = place((r() * 1e-2 * torch.exp(spread * r())).to(g_type))
        self.master = place(r() * 0.1) if master else None
        p = self.master if master else r() * 0.1
        self.p = place(p.to(p_type))
        m, u = r() * 3e-3, (r().abs() + 0.1) * 1e-2 * torch.exp(spread * r())
        m[::7], u[::7] = 0, 0            # never reached so far
        self.grad[::14] = 0              # and half of them not now either
        if bits == 8:
            self.scales = torch.stack([ref.scales_of(m), ref.scales_of(u)], 1).float().contiguous()
            each = self.scales.repeat_interleave(256, 0)[:n]
            self.m = place((m / each[:, 0]).to(E4M3))
            self.v = place(torch.where(u > 0, (u / each[:, 1]).clamp(2.0 ** -9, 448), u).to(E4M3))
        else:
            self.scales, self.m, self.v = None, place(m), place(u * u)
        self.step = torch.tensor(taken, device=DEV)

    def snapshot(self):
        if self.bits == 8:
            m, v = ref.decoded(self.m, self.scales, 0), ref.decoded(self.v, self.scales, 1).square()
        else:
            m, v = self.m.double(), self.v.double()
        return (self.p if self.master is None else self.master).double(), m, v, int(self.step)

    def check(self, before, factor=1.0, seed=0, factor_off=0.0, lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1):
        p0, m0, v0, taken = before
        assert int(self.step) == taken + 1
        m, v = ref.moments(self.grad, m0, v0, factor, beta1, beta2)
        p = ref.new_param(p0, m, v, taken + 1, lr, beta1, beta2, eps, weight_decay)
        # decoding, g factor, the difference, the product and the sum; (1 - beta rounded to fp32 among them)
        g = (self.grad.double() * factor).abs()
        d_m = (8 * U + factor_off) * (m0.abs() + g)
        d_v = (10 * U + 2 * factor_off) * v
        # m's error through the quotient, whose own parts are within 12 roundings, then the sum
        update = p - p0 * (1 - lr * weight_decay)
        t = taken + 1
        d_p = (lr / (1 - beta1 ** t) * d_m / (torch.sqrt(v / (1 - beta2 ** t)) + eps)
               + (20 * U + 2 * factor_off) * update.abs() + 4 * U * (p0.abs() + p.abs()))
        d_p = torch.nan_to_num(d_p)
        r = ref.random_bits(seed, taken, self.id, 0, self.n, DEV)
        if self.master is not None:
            ref.close(self.master, p, d_p)
            assert torch.equal(self.p, self.master.to(BF16))
        elif self.p.dtype == BF16:
            ref.check_bf16(self.p.double(), p, d_p, r & 0xFFFF)
        else:
            ref.close(self.p, p, d_p)
        if self.bits == 8:
            u = v.sqrt()
            ref.check_8_bit(ref.decoded(self.m, self.scales, 0), m, d_m, r & 0xFFFF)
            ref.check_8_bit(ref.decoded(self.v, self.scales, 1), u, (8 * U + factor_off) * u, r >> 16, root=True)
            biggest = torch.nn.functional.pad(d_m, (0, -self.n % 256)).view(-1, 256).amax(1)
            ref.close(self.scales[:, 0], ref.scales_of(m), 4 * U * ref.scales_of(m) + biggest / 448)
            ref.close(self.scales[:, 1], ref.scales_of(u), (12 * U + factor_off) * ref.scales_of(u))
        else:
            ref.close(self.m, m, d_m)
            ref.close(self.v, v, d_v + 2.0 ** -149)


def given(tensors):
    masters = [t.p if t.master is None else t.master for t in tensors]
    return binding.AdamwList([t.grad for t in tensors], masters, [t.m for t in tensors], [t.v for t in tensors],
                             [t.step for t in tensors], [t.scales for t in tensors],
                             [None if t.master is None else t.p for t in tensors], [t.id for t in tensors])


def step(tensors, **more):
    binding.dg_adamw_step(given(tensors), workspace=binding.adamw_workspace(DEV), **{**HYPER, **more})


KINDS = [(F32, F32, False), (BF16, BF16, False), (F32, BF16, False), (BF16, F32, False), (BF16, BF16, True), (BF16, F32, True)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_type,g_type,master", KINDS)
@pytest.mark.parametrize("taken", [0, 7, 100000])
def test_one_step(p_type, g_type, master, bits, taken):
    tensors = [Tensor(n, p_type, g_type, bits, n, master, taken) for n in SIZES]
    before = [t.snapshot() for t in tensors]
    step(tensors, seed=2 ** 40 + 5)
    for t, b in zip(tensors, before):
        t.check(b, seed=2 ** 40 + 5)


@pytest.mark.parametrize("shift", [1, 2, 3])
@pytest.mark.parametrize("bits", [32, 8])
def test_any_alignment_and_mixed_lists(bits, shift):
    tensors = [Tensor(n, *kind[:2], b, 10 * n + i, kind[2], shift=s) for n in (300, 5000)
               for i, (kind, b, s) in enumerate((k, b, s) for k in KINDS for b in (bits, 40 - bits) for s in (0, shift))]
    before = [t.snapshot() for t in tensors]
    step(tensors)
    for t, b in zip(tensors, before):
        t.check(b)


@pytest.mark.parametrize("count", [24, 25, 400, 401, 1234])
def test_lists_longer_than_a_launch(count):
    tensors = [Tensor(1 + (37 * i) % 600, F32, F32, (32, 8)[i % 2], i, taken=i % 5) for i in range(count)]
    before = [t.snapshot() for t in tensors]
    norm = torch.zeros(2, device=DEV)
    workspace = binding.adamw_workspace(DEV)
    total = sum(t.grad.double().square().sum() for t in tensors).sqrt()
    listed = given(tensors)
    for _ in range(2):
        binding.dg_grad_norm(listed, 0.5, workspace, norm)
        ref.close(norm[:1], total, 2 * U * total)
        ref.close(norm[1:], 0.5 / (total + 1e-6), 4 * U * norm[1].double())
    binding.dg_adamw_step(listed, workspace=workspace, grad_factor=norm[1:], **HYPER)
    for t, b in zip(tensors, before):
        t.check(b, factor=float(0.5 / (total + 1e-6)), factor_off=8 * U)
    assert not bool(workspace[:8].any())       # the tickets are back at 0


@pytest.mark.parametrize("p_type,bits,sizes", [(F32, 8, [5000011, 257, 1300001, 700000]), (BF16, 8, [1300001, 4096]),
                                               (BF16, 8, [40000 + i for i in range(60)]), (F32, 32, [10000007, 300])])
def test_more_numbers_than_warps_have_in_one_go(p_type, bits, sizes):
    tensors = [Tensor(n, p_type, p_type, bits, i, taken=i) for i, n in enumerate(sizes)]
    before = [t.snapshot() for t in tensors]
    step(tensors, seed=9)
    for t, b in zip(tensors, before):
        t.check(b, seed=9)


@pytest.mark.parametrize("bits", [32, 8])
def test_bf16_parameters_that_are_not_finite_keep_to_themselves(bits):
    t, clean = (Tensor(1000, BF16, BF16, bits, 4) for _ in range(2))
    t.p[[5, 700]], t.p[[300, 999]] = float("nan"), float("-inf")
    before = clean.snapshot()
    step([t])
    step([clean])
    clean.check(before)
    assert t.p[[5, 700]].isnan().all() and t.p[[300, 999]].tolist() == [-float("inf")] * 2
    rest = torch.ones(1000, dtype=torch.bool, device=DEV)
    rest[[5, 700, 300, 999]] = False
    assert torch.equal(t.p[rest], clean.p[rest])
    assert torch.equal(t.m.float(), clean.m.float()) and torch.equal(t.v.float(), clean.v.float())


@pytest.mark.parametrize("sizes,types", [([1], F32), ([5, 0, 256, 70001], F32), ([33, 1000003], BF16)])
def test_norm_of_gradients(sizes, types):
    gen = torch.Generator(device=DEV).manual_seed(1)
    workspace, result = binding.adamw_workspace(DEV), torch.zeros(2, device=DEV)
    for scale in (1.0, 1e-30, 1e25):
        grads = [(torch.randn(n, device=DEV, generator=gen) * scale).to(types) for n in sizes]
        want = torch.cat([g.double() for g in grads]).norm()
        tensors = binding.AdamwList(grads)
        binding.dg_grad_norm(tensors, 1.0, workspace, result)
        first = result.clone()
        ref.close(result[:1], want, 2 * U * want)
        ref.close(result[1:], (1 / (want + 1e-6)).clamp(max=1.0), 4 * U * (1 / (want + 1e-6)).clamp(max=1.0))
        binding.dg_grad_norm(tensors, 1.0, workspace, result)
        assert torch.equal(first, result)
    binding.dg_grad_norm(binding.AdamwList([]), 1.0, workspace, result)
    assert result.tolist() == [0.0, 1.0]
    bad = torch.tensor([1.0, float("nan")], device=DEV)
    binding.dg_grad_norm(binding.AdamwList([bad]), 1.0, workspace, result)
    assert result.isnan().all()


@pytest.mark.parametrize("bits", [32, 8])
def test_numbers_that_are_not_finite_keep_to_themselves(bits):
    t, clean = (Tensor(1000, F32, F32, bits, 3) for _ in range(2))
    for i, bad in ((5, float("nan")), (300, float("inf")), (301, float("-inf"))):
        t.grad[i] = bad
    clean.grad[[5, 300, 301]] = 0
    before = clean.snapshot()
    step([t])
    step([clean])
    hit = torch.zeros(1000, dtype=torch.bool, device=DEV)
    hit[[5, 300, 301]] = True
    clean.check(before)
    assert bool(t.p[hit].isnan().all()) and bool(t.p[~hit].isfinite().all())
    assert not bool(t.m[hit].float().isfinite().any()) and bool(t.m[~hit].float().isfinite().all())
    assert not bool(t.v[hit].float().isfinite().any()) and bool(t.v[~hit].float().isfinite().all())
    assert torch.equal(t.p[~hit], clean.p[~hit])
    if bits == 8:
        assert bool(t.scales.isfinite().all())


def test_gradients_of_zero_and_tiny_blocks():
    """A parameter that no gradient reached only decays; blocks of denormal numbers have scales with a finite inverse."""
    for bits in (32, 8):
        t = Tensor(600, F32, F32, bits, 4)
        t.grad.zero_(), t.m.zero_(), t.v.zero_()
        if bits == 8:
            t.scales.zero_()
        p = t.p.clone()
        step([t])
        ref.close(t.p, p.double() * (1 - 1e-3), 3 * U * p.double().abs())
        assert not bool(t.m.float().any()) and not bool(t.v.float().any())
    t = Tensor(600, F32, F32, 8, 5)
    t.grad.fill_(1e-42), t.m.zero_(), t.v.zero_(), t.scales.zero_()
    step([t])
    assert bool(t.p.isfinite().all()) and bool(t.scales.isfinite().all()) and bool(t.m.float().isfinite().all())


def test_roundings_are_even_handed():
    """Random rounding is right on average: 2^20 numbers halfway and a quarter of the way between neighbours.  The mean of N
    independent roundings is within 5 / (2 sqrt(N)) steps of the number but for one in a million."""
    n = 1 << 20
    for place in (0.5, 0.25, 0.01):
        t = Tensor(n, BF16, F32, 8, 6)
        # lr 0: the parameter stays; m = (1 - beta1) g with beta1 = 0
        t.m.zero_(), t.v.zero_(), t.scales.zero_(), t.p.fill_(1.0)
        t.grad.fill_((8 + place) * 2.0 ** -3)
        t.grad[::256] = 448.0 * 2            # the scale: 2
        step([t], beta1=0.0, lr=0.0)
        y = ref.decoded(t.m, t.scales, 0) / 2
        rest = torch.ones(n, dtype=torch.bool, device=DEV)
        rest[::256] = False
        x = (8 + place) * 2.0 ** -4
        got = y[rest]
        assert set(got.unique().tolist()) == {0.5, 0.5625}
        assert abs(float((got - x).mean()) / 2.0 ** -4) <= 5 / (2 * n ** 0.5) + 2.0 ** -16
    t = Tensor(n, BF16, F32, 32, 7)
    t.p.fill_(1.0)
    step([t], weight_decay=2.0 ** -10, lr=2.0, beta1=0.999999, eps=1e30)    # p becomes 1 - 2^-9: halfway to 1 - 2^-8
    assert set(t.p.unique().tolist()) == {1.0, 1 - 2.0 ** -8}
    assert abs(float(t.p.double().mean()) - (1 - 2.0 ** -9)) <= 2.0 ** -8 * (5 / (2 * n ** 0.5))


@pytest.mark.parametrize("n", [2 ** 32 + 1000])
def test_more_numbers_than_32_bits_count(n):
    p = torch.full((n,), 0.5, dtype=BF16, device=DEV)
    grad = torch.full((n,), 0.25, dtype=BF16, device=DEV)
    m, v = (torch.zeros(n, dtype=torch.uint8, device=DEV).view(E4M3) for _ in range(2))
    scales = torch.zeros((n + 255) // 256, 2, device=DEV)
    count = torch.zeros((), dtype=torch.int64, device=DEV)
    result = torch.zeros(2, device=DEV)
    tensors = binding.AdamwList([grad], [p], [m], [v], [count], [scales], ids=[9])
    workspace = binding.adamw_workspace(DEV)
    binding.dg_grad_norm(tensors, 1e9, workspace, result)
    assert float(result[0]) == pytest.approx(0.25 * n ** 0.5, rel=1e-6)
    binding.dg_adamw_step(tensors, workspace=workspace, grad_factor=result[1:], **HYPER)
    want = ref.new_param(torch.tensor(0.5).double(), torch.tensor(0.025).double(), torch.tensor(0.0625e-3).double(), 1,
                         HYPER["lr"], HYPER["beta1"], HYPER["beta2"], HYPER["eps"], HYPER["weight_decay"])
    for start in (0, 2 ** 31 - 512, 2 ** 32 - 512, 2 ** 32, n - 1000):
        length = min(512, n - start)
        r = ref.random_bits(0, 0, 9, start, length, DEV)
        here = slice(start, start + length)
        ref.check_bf16(p[here].double(), want.to(DEV).expand(length), torch.full((length,), 1e-7, device=DEV).double(), r & 0xFFFF)
        assert bool((m[here].float() == 448).all()) and bool((v[here].float() == 448).all())
    assert bool((scales[:, 0] == scales[0, 0]).all()) and int(count) == 1


# ---- the optimiser ----------------------------------------------------------------------------

def model_params(seed, dtype=F32):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    return [torch.nn.Parameter((torch.randn(*s, device=DEV, generator=gen) * 0.1).to(dtype))
            for s in ((256, 100), (256,), (47, 256), (47,), (1,))]


def set_grads(params, seed, scale=1.0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    for p in params:
        p.grad = (torch.randn(p.shape, device=DEV, generator=gen) * scale).to(p.dtype)


@pytest.mark.parametrize("max_norm", [None, 0.5])
def test_follows_torchs_adamw(max_norm):
    """Twenty steps in two groups against torch's optimiser in fp64."""
    ours = model_params(0)
    theirs = [torch.nn.Parameter(p.detach().double()) for p in ours]
    groups = lambda ps: [dict(params=ps[:2], lr=1e-2), dict(params=ps[2:], weight_decay=0.0)]  # noqa: E731
    a = optim.AdamW(groups(ours), lr=3e-3, betas=(0.8, 0.99), max_norm=max_norm)
    b = torch.optim.AdamW(groups(theirs), lr=3e-3, betas=(0.8, 0.99), weight_decay=1e-2)
    for k in range(20):
        set_grads(ours, k)
        if k < 3:
            ours[1].grad = None               # joins later: its own count of steps
        for p, q in zip(ours, theirs):
            q.grad = None if p.grad is None else p.grad.double()
        if max_norm:
            norm = torch.nn.utils.clip_grad_norm_(theirs, max_norm)
        a.step()
        b.step()
        if max_norm:
            ref.close(a.grad_norm, norm, 2 * U * norm)
    assert int(a.state[ours[1]]["step"]) == 17 and int(a.state[ours[0]]["step"]) == 20
    for p, q in zip(ours, theirs):
        # a step adds 40 roundings of a number no larger than a few lr (m's cancellation among them), and 4 of p
        ref.close(p, q.detach(), 20 * U * (40 * 10 * 1e-2 + 4 * q.detach().abs()))


@pytest.mark.parametrize("bits,dtype,master", [(32, F32, False), (8, F32, False), (8, BF16, False), (8, BF16, True)])
def test_state_dicts_resume_bit_for_bit(bits, dtype, master):
    def steps(params, opt, first, last):
        for k in range(first, last):
            set_grads(params, k)
            opt.step()

    make = lambda ps: optim.AdamW(ps, lr=1e-2, state_bits=bits, min_8bit_size=100, master_weights=master, max_norm=1.0, seed=3)  # noqa: E731
    one = model_params(1, dtype)
    opt = make(one)
    steps(one, opt, 0, 4)
    saved, weights = copy.deepcopy(opt.state_dict()), [p.detach().clone() for p in one]
    steps(one, opt, 4, 8)
    two = [torch.nn.Parameter(w) for w in weights]
    again = make(two)
    again.load_state_dict(saved)
    assert again.state[two[0]]["exp_avg"].dtype == (E4M3 if bits == 8 else F32)
    steps(two, again, 4, 8)
    for p, q in zip(one, two):
        assert torch.equal(p, q)
        for k, s in opt.state[p].items():
            assert torch.equal(s.float(), again.state[q][k].float()), k
    third = copy.deepcopy(again)
    assert third.max_norm == 1.0


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_counts_on(bits):
    a, b = model_params(2), model_params(2)
    oa, ob = (optim.AdamW(ps, lr=1e-2, state_bits=bits, min_8bit_size=100, max_norm=1.0) for ps in (a, b))
    graph = torch.cuda.CUDAGraph()
    set_grads(a, 0)
    with pytest.raises(RuntimeError, match="before capturing"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            oa.step()
    torch.cuda.synchronize()
    oa.step()
    set_grads(b, 0)
    ob.step()
    set_grads(a, 1)
    with torch.cuda.graph(graph):
        oa.step()
    fresh = [p.grad.clone() for p in a]
    for k in range(1, 6):
        set_grads(b, k)
        for p, q in zip(a, b):
            p.grad.copy_(q.grad)
        graph.replay()
        ob.step()
    del fresh, graph
    for p, q in zip(a, b):
        assert torch.equal(p, q) and int(oa.state[p]["step"]) == 6
    assert torch.equal(oa.grad_norm, ob.grad_norm)


def test_states_and_parameters_that_move():
    """Between steps: a state replaced, a state's memory exchanged, a parameter's memory exchanged, a gradient left out."""
    a, b = model_params(4), model_params(4)
    oa, ob = (optim.AdamW(ps, lr=1e-2, state_bits=8, min_8bit_size=100, max_norm=1.0) for ps in (a, b))

    def both_step(k, without=None):
        for ps in (a, b):
            set_grads(ps, k)
            if without is not None:
                ps[without].grad = None
        oa.step(), ob.step()

    both_step(0)
    kept = []
    for change in range(4):
        s = oa.state[a[0]]
        if change == 0:
            s["exp_avg"] = s["exp_avg"].clone()
        elif change == 1:
            kept.append(s["exp_avg_sq"].data)
            s["exp_avg_sq"].data = s["exp_avg_sq"].data.clone()
            kept[-1].view(torch.uint8).zero_()          # what the old memory holds does not matter any more
        elif change == 2:
            a[0].data = a[0].data.clone()
        both_step(1 + change, without=1 if change == 3 else None)
    both_step(9)
    for p, q in zip(a, b):
        assert torch.equal(p, q)
        for k, t in oa.state[p].items():
            assert torch.equal(t.float(), ob.state[q][k].float()), k
    a[0].data = a[0].data[:, :50].contiguous()          # no longer what its states belong to
    a[0].grad = torch.zeros_like(a[0])
    with pytest.raises(ValueError):
        oa.step()


def test_state_dictionaries_that_are_exchanged():
    """Between steps: one parameter's dictionary replaced by a copy, then taken out (it begins anew), a group added."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    start = [torch.randn(n, device=DEV, generator=gen) for n in (700, 700, 33)]
    grads = [[torch.randn(p.numel(), device=DEV, generator=gen) for p in start] for _ in range(5)]
    params = [torch.nn.Parameter(p.clone()) for p in start]
    alone = [torch.nn.Parameter(p.clone()) for p in start]
    together = optim.AdamW(params[:2], lr=1e-2)
    single = [optim.AdamW([p], lr=1e-2) for p in alone]
    for k in range(5):
        if k == 1:
            old = together.state[params[0]]
            together.state[params[0]] = {key: t.clone() for key, t in old.items()}
            for t in old.values():
                t.fill_(7)
        elif k == 2:
            del together.state[params[1]]
            single[1] = optim.AdamW([alone[1]], lr=1e-2)
        elif k == 3:
            together.add_param_group(dict(params=params[2:]))
        for i in range(3 if k >= 3 else 2):
            params[i].grad, alone[i].grad = grads[k][i], grads[k][i].clone()
            single[i].step()
        together.step()
        for p, q in zip(params, alone):
            assert torch.equal(p, q), k


def test_refusals_and_odd_gradients():
    p = torch.nn.Parameter(torch.randn(64, 32, device=DEV))
    q = torch.nn.Parameter(p.detach().clone())
    with pytest.raises(ValueError, match="twice"):
        optim.AdamW([p, p])
    a, b = optim.AdamW([p]), optim.AdamW([q])
    a.step()                                     # no gradient: nothing to do
    assert not a.state
    g = torch.randn(32, 64, device=DEV)
    p.grad, q.grad = g.t(), g.t().contiguous()   # a gradient in another order
    a.step(), b.step()
    assert torch.equal(p, q)
    for bad in (torch.nn.Parameter(torch.randn(8, 8)), torch.nn.Parameter(torch.randn(8, 8, device=DEV).t()),
                torch.nn.Parameter(torch.randn(8, 8, device=DEV).half())):
        bad.grad = torch.zeros_like(bad)
        with pytest.raises((ValueError, TypeError)):
            optim.AdamW([bad]).step()
    r = torch.nn.Parameter(torch.randn(8, 8, device=DEV))
    r.grad = torch.eye(8, device=DEV).to_sparse()
    with pytest.raises(ValueError, match="sparse"):
        optim.AdamW([r]).step()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a.step()
    torch.cuda.current_stream().wait_stream(side)
    b.step()
    assert torch.equal(p, q)
    assert float(a.step(lambda: torch.tensor(3.0))) == 3.0
