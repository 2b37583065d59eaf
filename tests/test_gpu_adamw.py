"""The optimizer's step on the GPU: AdamW with moments in 32 and 8 bits over many tensors, the norm of the gradients, against the
plain forms (tests/adapters_util.py)."""
import numpy as np
import pytest
import torch

import adapters_util as au

pytestmark = pytest.mark.gpu

B1, B2, EPS = 0.9, 0.999, 1e-8
SIZES = [1, 3, 255, 256, 257, 511, 4096, 4097, 8191, 0, 5000]


@pytest.fixture(scope="module")
def qb():
    from paper_2407_17029_amd import binding
    return binding


class Tensors:
    """Weights, gradients and moments of several tensors, on the host in float64 (exact fp32 or bf16 values) and on the device."""

    def __init__(self, seed, sizes, bits, form, shift=0):
        r = np.random.Generator(np.random.Philox(key=[seed, 21]))
        f32 = lambda x: np.asarray(x, np.float32).astype(np.float64)  # noqa: E731
        self.sizes, self.bits, self.form = sizes, bits, form
        self.g = [f32(r.standard_normal(n) * 10.0 ** r.uniform(-6, 2)) for n in sizes]
        self.w = [f32(r.standard_normal(n)) for n in sizes]
        if form == "param":
            self.w = [au.bf16(w) for w in self.w]
        self.m = [f32(0.1 * r.standard_normal(n)) for n in sizes]
        self.v = [f32(r.standard_normal(n) ** 2) for n in sizes]
        for x in (*self.g, *self.m, *self.v):
            x[r.random(len(x)) < 0.05] = 0.0
        self.rate = [1.0 + 0.5 * (i % 3) for i in range(len(sizes))]
        self.decay = [0.1 * (i % 2) for i in range(len(sizes))]

        def place(x, dtype):                                 # `shift` elements into its memory
            out = torch.zeros(len(x) + shift, dtype=dtype, device=au.DEV)[shift:]
            out.copy_(torch.from_numpy(np.asarray(x, np.float32)))
            return out

        self.d_g = [place(x, torch.float32) for x in self.g]
        self.d_w = [place(x, torch.float32) for x in self.w] if form != "param" else None
        self.d_p = [place(x, torch.bfloat16) for x in self.w] if form != "master" else None
        self.d_ms = self.d_vs = None
        if bits == 8:
            # moments that 8 bits hold
            one = np.uint64(0x8000) * np.ones(1, np.uint64)
            stored = [au.Moments8(m, v, np.repeat(one * np.uint64(65537), len(m))) for m, v in zip(self.m, self.v)]
            self.d_m = [place(s.m, torch.float32).to(torch.float8_e4m3fn) for s in stored]
            self.d_v = [place(s.v, torch.float32).to(torch.float8_e5m2) for s in stored]
            self.d_ms, self.d_vs = ([place(x, torch.float32) for x in y] for y in ([s.m_scale for s in stored], [s.v_scale for s in stored]))
            self.m = [s.m * np.repeat(s.m_scale, 256)[:len(s.m)] for s in stored]
            self.v = [s.v * np.repeat(s.v_scale, 256)[:len(s.v)] for s in stored]
        else:
            self.d_m, self.d_v = ([place(x, torch.float32) for x in y] for y in (self.m, self.v))

    def list(self, qb):
        none = [None] * len(self.sizes)
        return qb.qblora_adamw_list(self.d_p or none, self.d_g, self.d_m, self.d_v, master=self.d_w, m_scale=self.d_ms, v_scale=self.d_vs,
                                    rate=self.rate, decay=self.decay)

    def check(self, step, lr, seed, factor=1.0):
        """The device's state against a step from the host's.  The weight: g * f, m and v are off by a few 2^-24 of what they add up,
        the root, the quotient and the product by as much; eight roundings of the step and two of the weight."""
        for i, n in enumerate(self.sizes):
            f32 = np.float64(np.float32(factor))
            w, m, v = au.adamw(self.w[i], self.m[i], self.v[i], self.g[i], step, lr, B1, B2, EPS, self.rate[i], self.decay[i], f32)
            m1, v1 = au.moments32(self.m[i], self.v[i], self.g[i], B1, B2, factor)
            bits = au.random_bits(n, i, step, seed)
            # what the moment adds up may cancel: its error counts by the sizes, in units of the denominator
            size = (B1 * np.abs(self.m[i]) + (1 - B1) * np.abs(np.where(np.isfinite(self.g[i]), self.g[i], 0.0)) * f32)
            c1, c2 = 1 - B1 ** step, 1 - B2 ** step
            move = lr * self.rate[i] / c1 * size / (np.sqrt(v / c2) + EPS)
            allowed = 12 * 2.0 ** -24 * move + 3 * 2.0 ** -24 * np.abs(self.w[i]) + 1e-37
            if self.form != "param":
                got = self.d_w[i].cpu().numpy().astype(np.float64)
                assert (np.abs(got - w) <= allowed).all(), f"weight of {i}: {np.abs(got - w).max()}"
                if self.d_p:
                    assert torch.equal(self.d_p[i], self.d_w[i].to(torch.bfloat16)), f"param of {i}"
            else:                                            # one of the two neighbours, the upper if the random bits carry
                got = au.host(self.d_p[i])
                step_ = 2 * au.half_step(np.where(w == 0, 1e-30, w))
                assert (np.abs(got - w) <= step_ + allowed).all(), f"param of {i}"
                low = (np.floor(np.abs(w) / step_) * step_)
                part = (np.abs(w) - low) / step_
                r16 = ((bits * np.uint64(0x9E3779B1)) & np.uint64(0xffffffff)) >> np.uint64(16)
                sure = np.abs(part + r16.astype(np.float64) / 65536.0 - 1.0) > allowed / step_ + 2.0 ** -16
                up = part + r16.astype(np.float64) / 65536.0 >= 1.0
                want = np.copysign(np.where(up, low + step_, low), w)
                assert np.array_equal(got[sure], want[sure]), f"param of {i}"
            if self.bits == 32:
                assert np.array_equal(self.d_m[i].cpu().numpy(), m1), f"m of {i}"
                assert np.array_equal(self.d_v[i].cpu().numpy(), v1), f"v of {i}"
            else:
                want = au.Moments8(m1.astype(np.float64), v1.astype(np.float64), bits)
                assert np.array_equal(self.d_ms[i].cpu().numpy(), want.m_scale), f"scale of m of {i}"
                assert np.array_equal(self.d_vs[i].cpu().numpy(), want.v_scale), f"scale of v of {i}"
                assert np.array_equal(au.host(self.d_m[i]), want.m), f"m of {i}"
                assert np.array_equal(au.host(self.d_v[i]), want.v), f"v of {i}"


@pytest.mark.parametrize("shift", [0, 1, 3])
@pytest.mark.parametrize("form", ["both", "master", "param"])
@pytest.mark.parametrize("bits", [8, 32])
def test_step(qb, bits, form, shift):
    t = Tensors(bits + shift, SIZES, bits, form, shift)
    lst = t.list(qb)
    qb.qblora_adamw_step(lst, 3, 1e-2, B1, B2, EPS, seed=77)
    t.check(3, 1e-2, 77)


@pytest.mark.parametrize("bits", [8, 32])
def test_first_steps_from_nothing(qb, bits):
    """Moments of zero, then three steps; the second and third start from what the device holds."""
    t = Tensors(5, [700, 4200], bits, "both")
    for x in (*t.d_m, *t.d_v, *(t.d_ms or []), *(t.d_vs or [])):
        x.zero_()
    lst = t.list(qb)
    for step in (1, 2, 3):
        scales = [[np.repeat(s.cpu().numpy().astype(np.float64), 256)[:n] for s, n in zip(x, t.sizes)] if x else [1.0] * 2 for x in (t.d_ms, t.d_vs)]
        t.m, t.v = ([au.host(x) * s for x, s in zip(y, sc)] for y, sc in zip((t.d_m, t.d_v), scales))
        t.w = [x.cpu().numpy().astype(np.float64) for x in t.d_w]
        qb.qblora_adamw_step(lst, step, 1e-3, B1, B2, EPS, seed=step)
        t.check(step, 1e-3, step)


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("max_norm", [1e-3, 1e9])
def test_clipped_step(qb, bits, max_norm):
    t = Tensors(9, SIZES, bits, "both")
    lst = t.list(qb)
    clip = qb.qblora_grad_norm(lst, max_norm)
    norm = np.sqrt(sum((g * g).sum() for g in t.g))
    got = clip.cpu().numpy()
    assert abs(got[0] - norm) <= 2.0 ** -24 * norm * 1.01
    want = min(1.0, max_norm / (norm + 1e-6))
    assert abs(got[1] - want) <= 2.0 ** -24 * want * 1.01
    qb.qblora_adamw_step(lst, 2, 1e-2, B1, B2, EPS, clip=clip, seed=1)
    t.check(2, 1e-2, 1, factor=got[1])


def test_norm_of_many_units(qb):
    """More units than partial sums; the same bits every time."""
    n = [4096 * 1500 + 5, 4096 * 1200, 3]
    g = [torch.randn(k, device=au.DEV, generator=torch.Generator(au.DEV).manual_seed(i)) for i, k in enumerate(n)]
    zeros = [torch.zeros(k, device=au.DEV) for k in n]
    lst = qb.qblora_adamw_list([None] * 3, g, zeros, zeros, master=zeros)
    a, b = qb.qblora_grad_norm(lst, 1.0), qb.qblora_grad_norm(lst, 1.0)
    norm = float(sum((x.double() ** 2).sum() for x in g)) ** 0.5
    assert torch.equal(a, b) and abs(float(a[0]) - norm) <= 2.0 ** -23 * norm


@pytest.mark.parametrize("units", [1, 3, 4, 5, 31, 32, 33])
def test_norm_around_its_rule(qb, units):
    """Lists of few units, which one workgroup adds up, and of more; the last unit is not a whole one."""
    g = [torch.randn(4096 * (units - 1) + 100, device=au.DEV, generator=torch.Generator(au.DEV).manual_seed(units))]
    zeros = [torch.zeros_like(x) for x in g]
    got = qb.qblora_grad_norm(qb.qblora_adamw_list([None], g, zeros, zeros, master=zeros), 1.0)
    norm = float((g[0].double() ** 2).sum()) ** 0.5
    assert abs(float(got[0]) - norm) <= 2.0 ** -23 * norm


def test_norm_of_large_and_small_gradients(qb):
    """Squares that pass fp32 both ways."""
    for scale in (1e30, 1e-30):
        t = Tensors(3, [1000, 77], 32, "both")
        for x in t.d_g:
            x.fill_(scale)
        got = qb.qblora_grad_norm(t.list(qb), scale).cpu().numpy().astype(np.float64)
        norm = float(np.float32(scale)) * 1077 ** 0.5
        assert abs(got[0] - norm) <= 2.0 ** -23 * norm
        want = min(1.0, float(np.float32(scale)) / (norm + 1e-6))
        assert abs(got[1] - want) <= 2.0 ** -23 * want


@pytest.mark.parametrize("bits", [8, 32])
def test_broken_gradients(qb, bits):
    """With the norm in front, a step with a NaN changes nothing; without it, only elements with a finite gradient move."""
    t = Tensors(4, [600, 300], bits, "both")
    t.g[0][5], t.g[0][300], t.g[1][299] = np.nan, np.inf, -np.inf
    for d, g in zip(t.d_g, t.g):
        d.copy_(torch.from_numpy(g.astype(np.float32)))
    lst = t.list(qb)
    state = [x for y in (t.d_w, t.d_p, t.d_m, t.d_v, t.d_ms or [], t.d_vs or []) for x in y]
    before = [x.clone().view(torch.uint8) for x in state]
    clip = qb.qblora_grad_norm(lst, 1.0)
    assert not torch.isfinite(clip[0]) and torch.isnan(clip[1])
    qb.qblora_adamw_step(lst, 3, 1e-2, B1, B2, EPS, clip=clip)
    assert all(torch.equal(x.view(torch.uint8), y) for x, y in zip(state, before))
    qb.qblora_adamw_step(lst, 3, 1e-2, B1, B2, EPS, seed=5)
    t.check(3, 1e-2, 5)
    assert t.d_w[0][5] == float(np.float32(t.w[0][5]))


@pytest.mark.parametrize("bits", [8, 32])
def test_huge_gradients(qb, bits):
    """A square that passes fp32 leaves v at 2^127, in 8 bits too; so does a gradient near fp32's end with m, step after step."""
    t = Tensors(6, [300], bits, "both")
    t.g[0][10] = np.float64(np.float32(3e38))
    t.d_g[0][10] = 3e38
    for step in range(3, 60):
        qb.qblora_adamw_step(t.list(qb), step, 1e-2, B1, B2, EPS, seed=5)
    assert torch.isfinite(t.d_w[0]).all()
    m = t.d_m[0].float() * (t.d_ms[0].repeat_interleave(256)[:300] if bits == 8 else 1.0)
    assert torch.isfinite(m).all() and m[10] > 1e38
    v = t.d_v[0].float() * (t.d_vs[0].repeat_interleave(256)[:300] if bits == 8 else 1.0)
    assert torch.isfinite(v).all() and v[10] > 1e38


def test_small_moments_next_to_large_ones(qb):
    """v of a block with one huge value: it is never rounded to zero where a gradient has been, so that a weight's step stays small."""
    n = 512
    g = torch.full((n,), 1e-6, device=au.DEV)
    g[0] = 1e4
    w = torch.zeros(n, device=au.DEV)
    m, v = torch.zeros(n, dtype=torch.float8_e4m3fn, device=au.DEV), torch.zeros(n, dtype=torch.float8_e5m2, device=au.DEV)
    ms, vs = torch.zeros(2, device=au.DEV), torch.zeros(2, device=au.DEV)
    lst = qb.qblora_adamw_list([None], [g], [m], [v], master=[w], m_scale=[ms], v_scale=[vs])
    for step in (1, 2, 3):
        qb.qblora_adamw_step(lst, step, 1e-2, seed=step)
    assert (v.float() > 0).all() and (w.abs() <= 3.5e-2).all()


def test_chance_keeps_small_steps(qb):
    """A bf16 weight of 1 that steps by a 2^-12 each time, a sixteenth of its spacing: after 64 steps the mean has moved by 64 of
    them, to within five standard deviations (spacing 2^-8 below one; 64 roundings of at most half of it, 65536 elements)."""
    n, steps, lr = 65536, 64, 2.0 ** -12
    p = torch.ones(n, dtype=torch.bfloat16, device=au.DEV)
    g = torch.ones(n, device=au.DEV)
    m, v = torch.zeros(n, device=au.DEV), torch.zeros(n, device=au.DEV)
    lst = qb.qblora_adamw_list([p], [g], [m], [v])
    for step in range(1, steps + 1):
        qb.qblora_adamw_step(lst, step, lr, seed=9)          # with a constant gradient every step is lr
    moved = 1.0 - p.double().mean().item()
    assert abs(moved - steps * lr) <= 5 * (steps ** 0.5 * 0.5 * 2.0 ** -8) / n ** 0.5 + steps * lr * 1e-5


def test_plan_of_many_tensors(qb):
    """More tensors than one launch describes, empty ones among them, and their neighbours' memory."""
    sizes = [(i * 37) % 600 for i in range(101)] + [0, 9000, 0]
    t = Tensors(8, sizes, 8, "both")
    qb.qblora_adamw_step(t.list(qb), 4, 1e-2, B1, B2, EPS, seed=3)
    t.check(4, 1e-2, 3)


def test_neighbours_stay(qb):
    """Tensors cut out of the middle of arrays: what lies around them keeps its bits."""
    n, around = 4099, 64
    arrays = {k: torch.full((n + 2 * around,), 3.0, device=au.DEV).to(d) for k, d in
              dict(g=torch.float32, w=torch.float32, p=torch.bfloat16, m=torch.float8_e4m3fn, v=torch.float8_e5m2).items()}
    scales = [torch.full((17 + 2 * around,), 0.5, device=au.DEV) for _ in range(2)]
    cut = {k: x[around:around + n] for k, x in arrays.items()}
    sc = [s[around:around + 17] for s in scales]
    lst = qb.qblora_adamw_list([cut["p"]], [cut["g"]], [cut["m"]], [cut["v"]], master=[cut["w"]], m_scale=[sc[0]], v_scale=[sc[1]])
    qb.qblora_adamw_step(lst, 1, 1e-2)
    for x in arrays.values():
        assert (x[:around].float() == 3.0).all() and (x[around + n:].float() == 3.0).all()
    for s in scales:
        assert (s[:around] == 0.5).all() and (s[around + 17:] == 0.5).all()
    assert (cut["w"] != 3.0).all()


@pytest.mark.parametrize("bits", [8, 32])
def test_captured_step(qb, bits):
    """Step number and rate on the device: replays of one graph are the eager steps."""
    a, b = Tensors(12, [3000, 77], bits, "both"), Tensors(12, [3000, 77], bits, "both")
    la, lb = a.list(qb), b.list(qb)
    step, lr = torch.zeros(1, dtype=torch.int64, device=au.DEV), torch.zeros(1, device=au.DEV)

    def run():
        step.add_(1)
        qb.qblora_adamw_step(lb, step, lr, B1, B2, EPS, clip=qb.qblora_grad_norm(lb, 0.5), seed=4)

    keep = [x.clone() for y in (b.d_w, b.d_p, b.d_m, b.d_v, b.d_ms or [], b.d_vs or []) for x in y]
    run()
    for x, k in zip([x for y in (b.d_w, b.d_p, b.d_m, b.d_v, b.d_ms or [], b.d_vs or []) for x in y], keep):
        x.copy_(k)
    step.zero_()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for i in range(1, 5):
        rate = float(np.float32(1e-2 / i))
        lr.fill_(rate)
        torch.cuda.synchronize()
        graph.replay()
        qb.qblora_adamw_step(la, i, rate, B1, B2, EPS, clip=qb.qblora_grad_norm(la, 0.5), seed=4)
        torch.cuda.synchronize()
        for x, y in zip((a.d_m, a.d_v, a.d_ms or [], a.d_vs or []), (b.d_m, b.d_v, b.d_ms or [], b.d_vs or [])):
            assert all(torch.equal(u.view(torch.uint8), w.view(torch.uint8)) for u, w in zip(x, y)), i
        for u, w in zip(a.d_w, b.d_w):                       # factors by the host's power function and the device's: a rounding apart
            assert (u - w).abs().max() <= 1e-6
        assert int(step) == i


def test_more_elements_than_32_bits_count(qb):
    """A tensor of 2^32 elements and some: its ends and the places around 2^31 and 2^32, by a step of cut-out pieces."""
    n, step, lr = (1 << 32) + 777, 3, 1e-2
    g = torch.zeros(n, device=au.DEV)
    p = torch.zeros(n, dtype=torch.bfloat16, device=au.DEV)
    m, v = torch.zeros(n, dtype=torch.float8_e4m3fn, device=au.DEV), torch.zeros(n, dtype=torch.float8_e5m2, device=au.DEV)
    ms, vs = torch.zeros(-(-n // 256), device=au.DEV), torch.zeros(-(-n // 256), device=au.DEV)
    r = np.random.Generator(np.random.Philox(key=[3, 3]))
    places = [0, (1 << 31) - 256, (1 << 32) - 256, 1 << 32, n - 9 - 256]
    values = {}
    for at in places:
        at -= at % 256
        k = min(512, n - at)
        values[at] = np.asarray(r.standard_normal(k), np.float32).astype(np.float64)
        g[at:at + k] = torch.from_numpy(values[at]).float()
    lst = qb.qblora_adamw_list([p], [g], [m], [v], m_scale=[ms], v_scale=[vs])
    norm = qb.qblora_grad_norm(lst, 1e9)
    # overlapping pieces hold the last values written
    kept = {at: g[at:at + len(x)].cpu().numpy().astype(np.float64) for at, x in values.items()}
    qb.qblora_adamw_step(lst, step, lr, B1, B2, EPS, seed=2)
    assert norm[0] > 10 and torch.isfinite(norm).all()
    bits = {at: au.random_bits_at(np.arange(at, at + len(x)), 0, step, 2) for at, x in kept.items()}
    for at, x in kept.items():
        zero = np.zeros(len(x))
        w, _, _ = au.adamw(zero, zero, zero, x, step, lr, B1, B2, EPS)
        m1, v1 = au.moments32(zero, zero, x, B1, B2)
        want = au.Moments8(m1.astype(np.float64), v1.astype(np.float64), bits[at])
        assert np.array_equal(au.host(m[at:at + len(x)]), want.m) and np.array_equal(au.host(v[at:at + len(x)]), want.v), at
        got = au.host(p[at:at + len(x)])
        assert (np.abs(got - w) <= 2 * au.half_step(np.where(w == 0, 1e-30, w)) + 1e-7).all(), at


def test_empty_list(qb):
    lst = qb.qblora_adamw_list([], [], [], [], master=[])
    out = qb.qblora_grad_norm(lst, 2.0)
    assert out.tolist() == [0.0, 1.0]
    qb.qblora_adamw_step(lst, 1, 1e-3)


def test_refusals_of_the_binding(qb):
    t = Tensors(2, [100], 8, "both")
    good = dict(params=t.d_p, grads=t.d_g, m=t.d_m, v=t.d_v, master=t.d_w, m_scale=t.d_ms, v_scale=t.d_vs)
    for bad in (dict(params=t.d_w), dict(grads=[t.d_g[0][:50]]), dict(grads=[t.d_g[0][::2]]), dict(v=t.d_m), dict(m_scale=[t.d_ms[0].double()]),
                dict(m_scale=[torch.zeros(2, device=au.DEV)]), dict(master=[t.d_w[0].cpu()]), dict(m=t.d_m * 2)):
        with pytest.raises(AssertionError):
            qb.qblora_adamw_list(**{**good, **bad})
    lst = qb.qblora_adamw_list(**good)
    with pytest.raises(qb.QBLoRAError):
        qb.qblora_adamw_step(lst, 0, 1e-3)
    with pytest.raises(qb.QBLoRAError):
        qb.qblora_grad_norm(lst, 0.0)
    with pytest.raises(AssertionError):
        qb.qblora_adamw_step(lst, 1, 1e-3, clip=torch.zeros(1, device=au.DEV))
