"""AdamW on the GPU against its 64-bit form, and the 8-bit states against their definition, bit for bit.

Bounds, with u = 2^-24: m and v are two products and a sum, 4 u (|terms|); the parameter adds the step (a dozen
operations on m, which may have cancelled, so of the step that m's terms' magnitudes would make, a "reach" r: 16 u r and
eps against the root 1e-7 r) to a product: 3 u |p| + 2^-19 r, then its own rounding to 16 bits."""
import numpy as np
import pytest
import torch

import seq_reference as ref
from paper_2606_21101_amd.optim import AdamW

pytestmark = pytest.mark.gpu
DT = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
U = 2.0 ** -24
HYPER = dict(lr=0.01, b1=0.9, b2=0.999, eps=1e-8, wd=0.1)
SIZES = [1, 3, 255, 256, 257, 4096, 4097, 12_345, 0, 70_001]


def near(y, want, bound, what):
    y = y.detach().double().cpu().numpy()
    bad = ~(np.abs(y - want) <= bound)
    assert not bad.any(), f"{what}: {bad.sum()} off, worst {np.abs(y - want)[bad].max()}"


def values(rng, n, dt, sigma=1.0, shift=0):
    t = torch.from_numpy((rng.standard_normal(n + shift) * sigma).astype(np.float32)).to(DT[dt]).cuda()
    return t[shift:]


def arrays(*ts):
    return [t.detach().double().cpu().numpy() for t in ts]


@pytest.mark.parametrize("pdt,gdt,master,shift", [("f32", "f32", False, 0), ("f32", "bf16", False, 1), ("f16", "f16", True, 0),
                                                  ("bf16", "bf16", False, 0), ("bf16", "f32", True, 1), ("f16", "f32", False, 0)])
def test_step_of_many_tensors(pdt, gdt, master, shift):
    rng = np.random.default_rng(7)
    params = [values(rng, n, pdt, shift=shift) for n in SIZES]
    m, v = [values(rng, n, "f32", 0.01) for n in SIZES], [values(rng, n, "f32", 0.1).square() for n in SIZES]
    opt = AdamW(params, masters=True if master else None, m=m, v=v, lr=HYPER["lr"], weight_decay=HYPER["wd"])
    for t in (1, 2, 500):
        grads = [values(rng, n, gdt, shift=shift) for n in SIZES]
        held = opt.masters if master else params
        before = [arrays(p, g, a, b) for p, g, a, b in zip(held, grads, opt.m, opt.v)]
        opt.step(grads, step=t)
        for k, (p, g, a, b) in enumerate(before):
            wp, wm, wv, step = ref.adamw(p, g, a, b, t, **HYPER)
            near(opt.m[k], wm, 4 * U * (np.abs(a) + np.abs(g)), "m")
            near(opt.v[k], wv, 4 * U * (np.abs(b) + g * g), "v")
            bound = 3 * U * (np.abs(p) + step) + 2.0 ** -19 * step
            if master:
                near(opt.masters[k], wp, bound, "master")
                assert torch.equal(params[k], opt.masters[k].to(DT[pdt]))
            else:
                near(params[k], wp, bound + ref.EPS[pdt] * (np.abs(wp) + bound) + ref.TINY[pdt], "param")


def test_more_tensors_than_one_launch_takes_and_missing_gradients():
    rng = np.random.default_rng(1)
    params = [values(rng, 5 + k % 7, "f32") for k in range(600)]
    grads = [None if k % 50 == 0 else values(rng, 5 + k % 7, "f32") for k in range(600)]
    opt = AdamW(params, lr=HYPER["lr"], weight_decay=HYPER["wd"])
    before = arrays(*params)
    opt.step(grads)
    assert opt.step_count == 1
    for k in range(600):
        if grads[k] is None:
            assert np.array_equal(before[k], arrays(params[k])[0]) and not opt.m[k].any()
        else:
            z = np.zeros_like(before[k])
            wp, _, _, step = ref.adamw(before[k], arrays(grads[k])[0], z, z, 1, **HYPER)
            near(params[k], wp, 3 * U * (np.abs(before[k]) + step) + 2.0 ** -19 * step, k)


def as_codes(t):
    return t.view(torch.uint8).reshape(-1).cpu().numpy()


@pytest.mark.parametrize("pdt,gdt,master", [("f32", "f32", False), ("f16", "f16", True), ("bf16", "f32", False)])
def test_states_of_8_bits_are_what_they_are_defined_to_be(pdt, gdt, master):
    """Each step's codes and scales equal the definition's on the states before it, in binary32 and integers."""
    rng = np.random.default_rng(3)
    f = np.float32
    params = [values(rng, n, pdt) for n in SIZES]
    opt = AdamW(params, masters=True if master else None, state_bits=8, lr=HYPER["lr"], weight_decay=HYPER["wd"], seed=99)
    for t in (1, 2, 3, 1000):
        grads = [values(rng, n, gdt, 10.0 ** rng.integers(-3, 2)) for n in SIZES]
        for g in (g for g in grads if g.numel()):
            g[g.abs() < 0.3 * g.abs().max()] *= 1e-3      # small beside large in one block
        held = opt.masters if master else params
        before = [(as_codes(a), as_codes(b), s.cpu().numpy(), r.cpu().numpy(), *arrays(p, g))
                  for a, b, s, r, p, g in zip(opt.m, opt.v, opt.m_scale, opt.v_scale, held, grads)]
        opt.step(grads, step=t)
        for k, (mc, vc, ms, vs, p, g) in enumerate(before):
            n = len(mc)
            m = ref.decode(mc).astype(f) * np.repeat(ms, 256)[:n]
            v = ref.decode(vc).astype(f) * np.repeat(vs, 256)[:n]
            g = g.astype(f)
            m2 = m * f(0.9) + g * f(1 - 0.9)
            v2 = v * f(0.999) + (g * g) * f(1 - 0.999)
            rm, rv = ref.random_bits(n, 99, t, k)
            for name, z, r, small in (("m", m2, rm, False), ("v", v2, rv, True)):
                codes, scale = ref.store8(z, r, small)
                assert np.array_equal(as_codes(getattr(opt, name)[k]), codes), (name, k, t)
                assert np.array_equal(getattr(opt, name + "_scale")[k].cpu().numpy(), scale), (name, k, t)
            wp, _, _, step = ref.adamw(p, g, m, v, t, **HYPER)
            bound = 3 * U * (np.abs(p) + step) + 2.0 ** -19 * step
            if master:
                near(opt.masters[k], wp, bound, "master")
            else:
                near(params[k], wp, bound + ref.EPS[pdt] * (np.abs(wp) + bound) + ref.TINY[pdt], "param")


def test_rounding_keeps_the_mean_and_a_nonzero_second_moment_is_not_lost():
    """2^20 equal small moments beside one large one a block: the codes' mean is the moment (a code is off by at most
    one step, 1/8 of its value, with an independent sign: 5 sigma of the mean are 5/16 / 2^10 of it)."""
    n = 1 << 20
    p = torch.zeros(n, device="cuda")
    opt = AdamW([p], state_bits=8, betas=(0.0, 0.0))
    g = torch.full((n,), 0.0133, device="cuda")
    g[::256] = 1.0
    opt.step([g])
    small = torch.ones(n, dtype=torch.bool, device="cuda")
    small[::256] = False
    for codes, scale, want in ((opt.m[0], opt.m_scale[0], 0.0133), (opt.v[0], opt.v_scale[0], 0.0133 ** 2)):
        got = (codes.to(torch.float32).view(-1, 256) * scale[:, None]).view(-1)[small].double()
        assert abs(float(got.mean()) / want - 1) < 5 / 16 / 2 ** 10 + 1e-5
        assert len(torch.unique(got)) == 2
    g[small] = 1e-6                      # far below the smallest code of its block
    opt.step([g])
    held = opt.v[0].view(torch.uint8)[small]
    assert bool((held == 1).all())


def test_training_with_8_bits_follows_32():
    """A quadratic with gradients of very different sizes: both forms bring the loss down alike."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    scale = torch.logspace(-2, 1, 4096, device="cuda")
    target = torch.randn(4096, generator=gen, device="cuda")
    losses = {}
    for bits in (32, 8):
        p = torch.zeros(4096, device="cuda")
        opt = AdamW([p], state_bits=bits, lr=0.02, betas=(0.9, 0.99), weight_decay=0.0)
        for _ in range(300):
            opt.step([scale * (p - target)])
        losses[bits] = float((0.5 * scale * (p - target) ** 2).sum())
    start = float((0.5 * scale * target ** 2).sum())
    assert losses[32] < 1e-3 * start and losses[8] < 1e-2 * start, (start, losses)


def test_gradients_that_are_not_finite_are_seen():
    for bits in (32, 8):
        p = torch.ones(1024, device="cuda")
        opt = AdamW([p], state_bits=bits)
        g = torch.ones(1024, device="cuda")
        g[300] = float("nan")
        opt.step([g])
        assert torch.isnan(p[300]) and int(torch.isnan(p).sum()) == 1
        opt.step([torch.ones(1024, device="cuda")])
        lost = torch.isnan(p)
        assert bool(lost[300]) and not bool(lost[:256].any()) and not bool(lost[512:].any())


def test_step_replays_in_a_graph_and_runs_on_another_stream():
    p, q = torch.ones(5000, device="cuda"), torch.ones(5000, device="cuda")
    a, b = AdamW([p]), AdamW([q])
    g = torch.randn(5000, device="cuda")
    a.step([g], step=1)
    b.step([g], step=1)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    with torch.cuda.graph(graph, stream=side):
        a.step([g], step=2)
    for _ in range(3):
        g.normal_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        b.step([g], step=2, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(p, q)
