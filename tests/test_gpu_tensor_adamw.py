"""AdamW over a list of tensors against the formulas.

Tolerances with fp32 moments: some ten roundings of 2^-24 in a row, of the magnitudes
that a result is made of.  8-bit codes are checked exactly: the same single fp32
operations in torch give the same moments, and a plain table of the 128 (256) values
that codes stand for says which one is nearest.  The quotient m / (sqrt(v) r + eps) goes
through the hardware's square root and reciprocal, 2^-23 each, and three roundings of
2^-24: less than 2^-21 of it, and a parameter takes two more roundings of its own."""
from __future__ import annotations

import pytest
import torch

from paper_2509_21271_b200 import binding as B
from paper_2509_21271_b200 import build as so_build
from paper_2509_21271_b200.tensor_adamw import TensorAdamW
from test_gpu_operators import BF16, FP16, FP32, gen, randn, same_bits

pytestmark = pytest.mark.gpu
BLOCK = B.SO_TENSOR_BLOCK


class HP:
    lr, beta1, beta2, eps, weight_decay, max_grad_norm = 1e-2, 0.9, 0.99, 1e-8, 0.1, 0.0

    def __init__(self, **kw):
        for k, v in kw.items():
            setattr(self, k, v)


@pytest.fixture(scope="module", autouse=True)
def _built():
    so_build.build_library()
    torch.cuda.set_device(0)


RAGGED = [1, 7, 255, 256, 257, 1000, 4097, 100_003, 8, 2048]


def make(seed, sizes, grad=BF16, copy=BF16, bits=32, offset=0):
    """Tensors `offset` elements into buffers of their own."""
    g = gen(seed)
    cut = lambda n, t, s: (randn(g, n + offset + 8) * s).to(t)[offset:offset + n]  # noqa: E731
    params = [cut(n, FP32, 0.1) for n in sizes]
    grads = [cut(n, grad, 0.01) for n in sizes]
    copies = [cut(n, copy, 1.0) for n in sizes] if copy else None
    return g, TensorAdamW(params, grads, copies=copies, state_bits=bits)


def f32(x):
    return torch.tensor(x, dtype=FP32, device="cuda")


def plain_update(p, grad, m, v, t, hp, factor=1.0):
    """The same single operations, each rounded to fp32."""
    g = grad.float() * f32(factor)
    m = m * f32(hp.beta1) + g * f32(1.0 - hp.beta1)
    v = v * f32(hp.beta2) + g * f32(1.0 - hp.beta2) * g
    u = m / (v.sqrt() * f32((1.0 - hp.beta2 ** t) ** -0.5) + f32(hp.eps))
    return p - (p * f32(hp.lr * hp.weight_decay) + u * f32(hp.lr / (1.0 - hp.beta1 ** t))), m, v


def same_parameters(got, want, before, hp):
    """See above; what is left of a parameter's change without the decay is the quotient's part."""
    quotient = (want - before).abs() + hp.lr * hp.weight_decay * before.abs()
    return ((got - want).abs() <= 2.0 ** -21 * quotient + 2.0 ** -22 * want.abs()).all()


def exact_update(p, grad, m, v, t, hp, factor=1.0):
    g = grad.double() * factor
    m, v = hp.beta1 * m.double() + (1 - hp.beta1) * g, hp.beta2 * v.double() + (1 - hp.beta2) * g * g
    u = m / (1 - hp.beta1 ** t) / ((v / (1 - hp.beta2 ** t)).sqrt() + hp.eps)
    return p.double() * (1 - hp.lr * hp.weight_decay) - hp.lr * u, m, v


def pieces(opt, arena):
    out = []
    for i, p in enumerate(opt.params):
        at = opt.block_of(i) * BLOCK
        out.append(arena[at:at + p.numel()])
    return out


@pytest.mark.parametrize("grad", [BF16, FP16, FP32])
@pytest.mark.parametrize("copy", [BF16, FP16, None])
@pytest.mark.parametrize("offset", [0, 8, 1, 3])
def test_fp32_moments(grad, copy, offset):
    g, opt = make(3, RAGGED, grad, copy, offset=offset)
    hp = HP()
    state = [(p.clone(), torch.zeros_like(p), torch.zeros_like(p)) for p in opt.params]
    for t in (1, 2, 3):
        for x in opt.grads:
            x.copy_(randn(g, x.numel()) * 0.01)
        opt.step(hp, clip=False)
        state = [exact_update(p, x, m, v, t, hp) for (p, m, v), x in zip(state, opt.grads)]
        for (p, m, v), q, qm, qv in zip(state, opt.params, pieces(opt, opt.m), pieces(opt, opt.v)):
            e = 16 * t * 2.0 ** -24
            assert (q - p).abs().max() <= (e * (p.abs() + hp.lr * 10)).max()
            assert ((qm - m).abs() <= e * 0.05).all() and ((qv - v).abs() <= e * v.abs() + 1e-30).all()
    if copy:
        assert all(same_bits(c, p.to(copy)) for c, p in zip(opt.copies, opt.params))
    assert opt.step_count == 3
    for i, p in enumerate(opt.params):                    # behind a tensor's end the arenas stay zero
        lo, hi = opt.block_of(i) * BLOCK + p.numel(), opt.block_of(i + 1) * BLOCK
        assert (opt.m[lo:hi] == 0).all() and (opt.v[lo:hi] == 0).all()


def values(bits, top):
    """What the codes stand for, in units."""
    k = torch.arange(1 << bits, device="cuda")
    return torch.where(k < 16, k, (16 + k % 16) << (k // 16 - 1).clamp(min=0)).double()


def nearest(x, scale, table):
    """Codes of magnitudes: the nearest value, halves up.  A value is first held in steps of
    2^-19 of a unit where it is below 16 units (fp32's spacing there, see the kernel), so
    that one less than 2^-20 below a half counts as the half: 4.4999995 becomes 5."""
    units = x.double() / torch.exp2(scale.double() - 127)[:, None]
    units = torch.where(units < 16, (units * 2.0 ** 19).round() * 2.0 ** -19, units)
    middle = (table[1:] + table[:-1]) / 2
    return torch.bucketize(units, middle, right=True)


def scale_of(x, largest):
    """The smallest power of two in which the largest magnitude of a block fits, biased."""
    most = x.abs().amax(1).double()
    e = torch.ceil(torch.log2(most / largest))
    e = torch.where(most > torch.exp2(e) * largest, e + 1, e)
    return torch.where(most == 0, torch.zeros_like(e), (e + 127).clamp(min=1))


def padded(opt, tensors):
    out = torch.zeros(opt.blocks * BLOCK, device="cuda")
    for i, x in enumerate(tensors):
        at = opt.block_of(i) * BLOCK
        out[at:at + x.numel()] = x
    return out


def decoded(opt):
    m, v = opt.moments()
    return m.float(), v.float()


@pytest.mark.parametrize("grad", [BF16, FP32])
@pytest.mark.parametrize("offset", [0, 1])
def test_8_bit_codes_are_the_nearest(grad, offset):
    g, opt = make(4, RAGGED, grad, FP16, bits=8, offset=offset)
    hp = HP(beta2=0.9)
    tm, tv = values(7, 1984), values(8, 507904)
    assert tm[-1] == 1984 and tv[-1] == 507904
    p = padded(opt, opt.params)
    m = v = torch.zeros_like(p)
    for t in (1, 2, 3, 4):
        for x in opt.grads:
            x.copy_(randn(g, x.numel()) * 10.0 ** (3 * randn(g, x.numel())) * 1e-3)   # over many binades
        before = p
        p, m, v = plain_update(p, padded(opt, opt.grads), m, v, t, hp)
        opt.step(hp, clip=False)
        assert same_parameters(padded(opt, opt.params), p, before, hp)
        p = padded(opt, opt.params)
        for name, x, table, scale in (("m", m, tm, opt.m_scale), ("v", v, tv, opt.v_scale)):
            x = x.view(-1, BLOCK)
            assert torch.equal(scale.double(), scale_of(x, table[-1])), name
            want = nearest(x.abs(), scale, table)
            want = torch.where((want == 0) & (x > 0), 1, want) if name == "v" else want
            code = getattr(opt, name).view(-1, BLOCK).long()
            assert torch.equal(code & 127 if name == "m" else code, want), name
        m, v = decoded(opt)
        # bf16 held them exactly
        units = tm[(opt.m.view(-1, BLOCK).long() & 127)] * torch.exp2(opt.m_scale.double() - 127)[:, None]
        sign = torch.where(opt.m.view(-1, BLOCK) >= 128, -1.0, 1.0)
        assert torch.equal(m.view(-1, BLOCK).double(), units * sign * (opt.m_scale > 0)[:, None])


def test_stochastic_rounding_keeps_the_mean():
    """n values of one code's distance d, each up with probability f: the mean is off by less than
    six standard deviations, 6 d / (2 sqrt n), and by 2^-17 d; only the two neighbours occur."""
    n = 1 << 16
    param, grad = torch.zeros(n, device="cuda"), torch.full((n,), 0.37, device="cuda")
    hp = HP(lr=0.0, weight_decay=0.0, beta1=0.5, beta2=0.5)
    for seed in (0, 1, 2 ** 40 + 5):
        opt = TensorAdamW([param], [grad], state_bits=8)
        grad[::BLOCK] = 1.0                                 # what the block's scale goes by
        opt.step(hp, clip=False, seed=seed)
        m, v = decoded(opt)
        for got, exact in ((m, 0.5 * 0.37), (v, 0.5 * 0.37 ** 2)):
            got = got.view(-1, BLOCK)[:, 1:].reshape(-1).double()
            low, high = got.min(), got.max()
            assert low < exact < high and got.unique().numel() == 2
            share = (exact - low) / (high - low)
            assert abs((got == high).double().mean() - share) <= 6 * 0.5 / got.numel() ** 0.5 + 2.0 ** -17
        again = TensorAdamW([param], [grad], state_bits=8)
        again.step(hp, clip=False, seed=seed)
        assert torch.equal(opt.m, again.m) and torch.equal(opt.v, again.v)
        before = opt.v.clone()
        opt.set_step(0)
        other = TensorAdamW([param], [grad], state_bits=8)
        other.step(hp, clip=False, seed=seed + 1)
        assert 0.2 < (other.v != before).float().mean() < 0.6


def test_an_average_that_moves_slowly_still_moves():
    """beta2 = 0.999 from a large v: rounded to nearest it never falls, stochastically it follows
    the average, whose noise after 400 steps over 4096 elements is far below a tenth."""
    hp = HP(lr=0.0, beta2=0.999)
    n = 4096
    ends = {}
    for seed in (None, 7):
        param, grad = torch.zeros(n, device="cuda"), torch.ones(n, device="cuda")
        opt = TensorAdamW([param], [grad], state_bits=8)
        opt.step(HP(lr=0.0, beta2=0.0), clip=False)                  # v = 1
        grad.fill_(0.1)
        for _ in range(400):
            opt.step(hp, clip=False, seed=seed)
        ends[seed] = decoded(opt)[1].mean().item()
    want = 0.01 + 0.99 * 0.999 ** 400
    assert ends[None] == 1.0 and abs(ends[7] - want) < 0.1 * want


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("grad", [BF16, FP16, FP32])
def test_norm_and_clipping(bits, grad):
    g, opt = make(5, RAGGED + [300_000], grad, BF16, bits=bits)
    hp = HP(max_grad_norm=0.5)
    flat = torch.cat([x.double() for x in opt.grads])
    norm = flat.norm().item() * 0.25
    p = padded(opt, opt.params)
    stats = opt.step(hp, grad_scale=0.25)
    assert abs(stats[0].item() - norm) <= 2.0 ** -22 * norm and stats[2].item() == 0
    coef = min(1.0, 0.5 / (norm + 1e-6))
    assert coef < 1 and abs(stats[1].item() - coef) <= 2.0 ** -22
    want, m, v = plain_update(p, padded(opt, opt.grads), torch.zeros_like(p), torch.zeros_like(p), 1, hp,
                              (stats[1] * 0.25).item())
    assert same_parameters(padded(opt, opt.params), want, p, hp)
    if bits == 32:
        assert torch.equal(opt.m, m) and torch.equal(opt.v, v)
    stats = opt.step(HP(max_grad_norm=0.0))
    assert stats[1].item() == 1.0 and opt.step_count == 2


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), 1e30])
def test_a_step_that_is_not_finite_is_skipped(bits, bad):
    g, opt = make(6, [1000, 3000], FP32, FP16, bits=bits)
    opt.step(HP())
    tensors = [*opt.params, *opt.copies, opt.m, opt.v] + ([opt.m_scale, opt.v_scale] if bits == 8 else [])
    before = [t.clone() for t in tensors]
    opt.grads[1][1234] = bad
    stats = opt.step(HP(max_grad_norm=1.0), seed=3 if bits == 8 else None)
    assert stats[2].item() == 1.0 and opt.step_count == 1
    assert all(same_bits(a, b) for a, b in zip(tensors, before))
    opt.grads[1][1234] = 0.0
    stats = opt.step(HP(max_grad_norm=1.0))
    assert stats[2].item() == 0.0 and opt.step_count == 2
    # without a look the block is marked, and the others are as ever
    if bits == 8:
        opt.grads[1][1234] = float("nan")
        opt.step(HP(), clip=False)
        block = opt.block_of(1) + 1234 // BLOCK
        m, v = opt.moments()
        gone = torch.isnan(m.view(-1, BLOCK)).all(1) & torch.isnan(v.view(-1, BLOCK)).all(1)
        assert gone.nonzero()[:, 0].tolist() == [block] and opt.m_scale[block] == 255
        assert torch.isnan(opt.params[1]).nonzero()[:, 0].tolist() == [1234]


def test_blocks_of_zeros_tiny_and_huge_values():
    n = 4 * BLOCK
    param, grad = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    grad[BLOCK:2 * BLOCK] = 1e-18                            # v near 1e-36
    grad[2 * BLOCK:3 * BLOCK] = 1e18
    grad[3 * BLOCK:] = torch.logspace(-30, 0, BLOCK)         # beyond what a block spans
    opt = TensorAdamW([param], [grad], state_bits=8)
    opt.step(HP(beta1=0.0, beta2=0.0), clip=False)
    m, v = (t.view(4, BLOCK) for t in decoded(opt))
    assert (m[0] == 0).all() and (v[0] == 0).all() and opt.m_scale[0] == 0 and opt.v_scale[0] == 0
    for i, x in ((1, 1e-18), (2, 1e18)):
        assert ((m[i] - x).abs() <= 2.0 ** -5 * x).all() and ((v[i] - x * x).abs() <= 2.0 ** -5 * x * x + 1e-38).all()
    there = grad[3 * BLOCK:] ** 2 > 0                        # 1e-30 has no square in fp32
    assert torch.equal(v[3] > 0, there) and 0 < there.sum() < BLOCK
    assert v[3][there].min() >= 2.0 ** -20 and (m[3][:64] == 0).all()
    assert torch.isfinite(param).all()


def test_more_tensors_than_a_launch_takes():
    sizes = [(i * 37) % 700 + (i % 5 == 0) * 300 for i in range(1500)]
    sizes[3] = sizes[4] = sizes[900] = sizes[-1] = 0
    g, opt = make(7, sizes, BF16, BF16, bits=8)
    assert opt.blocks == sum(-(-n // BLOCK) for n in sizes)
    hp = HP(max_grad_norm=0.1)
    p, grads = padded(opt, opt.params), padded(opt, opt.grads)
    stats = opt.step(hp)
    norm = grads.double().norm().item()
    assert abs(stats[0].item() - norm) <= 2.0 ** -22 * norm
    want, _, _ = plain_update(p, grads, torch.zeros_like(p), torch.zeros_like(p), 1, hp, stats[1].item())
    assert same_parameters(padded(opt, opt.params), want, p, hp)


def test_neighbours_are_left_alone():
    for bits in (8, 32):
        buf = torch.full((5000,), 3.0, device="cuda")
        low = torch.full((5000,), 3.0, dtype=BF16, device="cuda")
        opt = TensorAdamW([buf[11:1011], buf[1500:1777]], [torch.ones(1000, device="cuda"), torch.ones(277, device="cuda")],
                          copies=[low[9:1009], low[2000:2277]], state_bits=bits)
        opt.step(HP())
        for t, runs in ((buf, ((11, 1011), (1500, 1777))), (low, ((9, 1009), (2000, 2277)))):
            hole = torch.ones(5000, dtype=torch.bool, device="cuda")
            for lo, hi in runs:
                hole[lo:hi] = False
            assert (t[hole] == 3.0).all() and (t[~hole] != 3.0).all()


def test_captured_steps_go_on_from_the_device():
    """A replayed graph takes the next step, with its own bias corrections and random numbers."""
    g, opt = make(8, RAGGED, BF16, BF16, bits=8)
    g2, twin = make(8, RAGGED, BF16, BF16, bits=8)
    hp = HP(max_grad_norm=0.3)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            opt.step(hp, seed=11)
    torch.cuda.current_stream().wait_stream(side)
    assert opt.step_count == 0
    for t in (1, 2, 3):
        for a, b in zip(opt.grads, twin.grads):
            a.copy_(randn(g, a.numel()) * 0.01)
            b.copy_(a)
        graph.replay()
        twin.step(hp, seed=11, stream=torch.cuda.current_stream())
        assert opt.step_count == t
        for a, b in zip((*opt.params, *opt.copies, opt.m, opt.v, opt.m_scale, opt.v_scale, opt.stats),
                        (*twin.params, *twin.copies, twin.m, twin.v, twin.m_scale, twin.v_scale, twin.stats)):
            assert same_bits(a, b)


def test_gradients_may_change_and_parameters_require_grad():
    p = torch.nn.Parameter(torch.ones(600, device="cuda"))
    opt = TensorAdamW([p], [torch.zeros(600, device="cuda")])
    y = p.exp()
    (y * y).sum().backward()
    opt.set_grads([p.grad])
    version = p._version
    opt.step(HP())
    assert p._version == version + 1 and (p != 1).all()


def test_refusals():
    p, g = torch.zeros(8, device="cuda"), torch.zeros(8, device="cuda")
    bad = [lambda: TensorAdamW([], []), lambda: TensorAdamW([p], [g], state_bits=16), lambda: TensorAdamW([p], []),
           lambda: TensorAdamW([p.half()], [g]), lambda: TensorAdamW([p], [g[:7]]), lambda: TensorAdamW([p[::2]], [g[:4]]),
           lambda: TensorAdamW([p], [g.long()]), lambda: TensorAdamW([p, p], [g, g.half()]),
           lambda: TensorAdamW([p], [g], copies=[p]), lambda: TensorAdamW([p], [g], copies=[]),
           lambda: TensorAdamW([p], [g.cpu()]), lambda: TensorAdamW([p, p], [g, g]), lambda: TensorAdamW([p.cpu()], [g]),
           lambda: TensorAdamW([p], [g]).step(HP(), seed=1), lambda: TensorAdamW([p], [g]).set_step(-1)]
    for name, value in (("lr", -1.0), ("lr", float("nan")), ("beta1", 1.0), ("beta2", -0.1), ("eps", 0.0), ("eps", 1e-60),
                        ("weight_decay", -1.0), ("max_grad_norm", float("nan"))):
        bad.append(lambda name=name, value=value: TensorAdamW([p], [g]).step(HP(**{name: value})))
    bad.append(lambda: TensorAdamW([p], [g]).step(HP(), grad_scale=float("inf")))
    for call in bad:
        with pytest.raises(B.SuperOffloadError) as err:
            call()
        assert err.value.status == B.SO_ERR_INVALID_ARG


@pytest.mark.parametrize("bits", [8, 32])
def test_no_elements(bits):
    """Tensors without elements are passed over; a list of nothing else still counts its steps."""
    none = torch.zeros(0, device="cuda")
    opt = TensorAdamW([none, none], [none, none], state_bits=bits)
    assert opt.blocks == 0
    for clip in (True, False):
        stats = opt.step(HP(max_grad_norm=1.0), clip=clip)
        assert stats.tolist() == [0.0, 1.0, 0.0]
    assert opt.step_count == 2


def test_what_is_written_must_not_overlap():
    arena = torch.zeros(1000, device="cuda")
    a, b, c = arena[:300], arena[299:600], arena[600:1000]
    grads = [torch.zeros_like(t) for t in (a, b)]
    with pytest.raises(B.SuperOffloadError, match="overlap"):
        TensorAdamW([a, b], grads)
    with pytest.raises(B.SuperOffloadError, match="overlap"):      # one copy for two parameters
        copy = torch.zeros(300, device="cuda", dtype=BF16)
        TensorAdamW([arena[:300], arena[300:600]], [grads[0]] * 2, copies=[copy, copy])
    with pytest.raises(B.SuperOffloadError, match="overlap"):      # a copy inside a parameter
        TensorAdamW([c], [torch.zeros_like(c)], copies=[c.view(BF16)[:400]])
    # neighbours are apart, an empty tensor anywhere is, and a gradient may serve two parameters
    TensorAdamW([arena[300:600], arena[:300], arena[100:100]], [grads[0], grads[0], arena[:0]])
