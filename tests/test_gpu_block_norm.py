"""What stands between two blocks, h = x + s norm(y) w_post act(u), n = norm(h) w_pre, and its backward pass, through the C ABI against
the fp64 oracle.

Tolerances: everything is fp32 between loads and stores.  A row's value passes about ten roundings of 2^-24 and two inverse square roots
good to 2^-22, on sums of squares whose relative error is below 2^-20 for 16384 terms added up in a tree: 1e-5 of a row's RMS covers
them.  dx and dy are differences of two terms, r p and r y^ mean(p y^), of one size, which cancel where a row has few features (with one,
all but eps / y^2 of them): the roundings are those of the terms, so 1e-5 of their RMS counts too.  du has act'(u) as a factor, itself a sum
of two terms of size 1 that cancel at u = -1.28: what it multiplies counts likewise.  Sums over tokens: 1e-5 of the root of the sum of squares of what is summed (rows^1/2 times a term's RMS) and of the result's
own RMS.  A result in bf16 is off by half a step besides."""
import numpy as np
import pytest
import torch

from oracle import delta_oracle as orc
from paper_2307_14995_b200 import binding as la

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
GATES = [None, la.LA_GATE_PLAIN, la.LA_GATE_SIGMOID, la.LA_GATE_SILU]


def near(got, ref, what, sums=None):
    g = got.double().cpu().numpy()
    assert g.shape == ref.shape and np.all(np.isfinite(g)), what
    rms = np.sqrt(np.mean(ref * ref, -1, keepdims=True)) + (0.0 if sums is None else sums)
    bound = 1e-5 * rms + (2.0 ** -8 if got.dtype is BF16 else 2.0 ** -23) * np.abs(ref)
    assert np.all(np.abs(g - ref) <= bound), "%s: %.3g of the bound" % (what, np.max(np.abs(g - ref) / np.maximum(bound, 1e-300)))


class Case:
    def __init__(self, rows, D, dtype, res, gate, weights=True, eps=1e-6, post_norm=True, seed=0):
        gen = torch.Generator()
        gen.manual_seed(seed)
        new = lambda *s: torch.randn(*s, generator=gen)
        self.x, self.dh = (2 * new(rows, D)).to(res), new(rows, D).to(res)
        self.y, self.dn = (3 * new(rows, D)).to(dtype), new(rows, D).to(dtype)
        self.u = None if gate is None else new(rows, D).to(dtype)
        self.w = [0.5 + torch.rand(D, generator=gen) for _ in range(3)] if weights else [None] * 3
        self.more = dict(eps=eps, gate=gate or 0, post_norm=post_norm)
        self.shape = la.make_block_norm_shape(rows, D, dtype, res, **self.more)
        self.rows, self.D, self.dtype, self.res = rows, D, dtype, res
        self.margins = []

    def out(self, dtype, *size):
        n = int(np.prod(size))
        whole = torch.full((n + 64,), float("nan"), dtype=dtype, device=DEV)
        self.margins.append(whole[n:])
        return whole[:n].view(size)

    def dev(self, x):
        return None if x is None else x.to(DEV)

    def inputs(self):
        return [self.dev(t) for t in (self.x, self.y, self.u, *self.w)]

    def fwd(self):
        h, n = self.out(self.res, self.rows, self.D), self.out(self.dtype, self.rows, self.D)
        la.la_block_norm_fwd(self.shape, *self.inputs(), h, n)
        return h, n

    def bwd(self, dh=True, dn=True):
        self.grads = [self.out(self.res, self.rows, self.D), self.out(self.dtype, self.rows, self.D),
                      None if self.u is None else self.out(self.dtype, self.rows, self.D)] + [self.out(F32, self.D) for _ in range(3)]
        ws = torch.full((la.block_norm_workspace_bytes(self.shape),), 255, dtype=torch.uint8, device=DEV)
        la.la_block_norm_bwd(self.shape, *self.inputs(), self.dev(self.dh) if dh else None, self.dev(self.dn) if dn else None, *self.grads, ws)
        return self.grads

    def done(self):
        torch.cuda.synchronize()
        assert all(torch.isnan(m).all() for m in self.margins)

    def terms(self, dh, dn, dx):
        """RMS by row of what dx, dy and du are the differences of; dx's terms are scaled by dy's factors on their way to dy and du."""
        f64 = lambda v: v.double().numpy()
        rms = lambda v: np.sqrt(np.mean(v * v, -1, keepdims=True))
        eps = self.more["eps"]
        inv = lambda v: 1 / np.sqrt(np.mean(v * v, -1, keepdims=True) + max(eps, 1e-30))
        h = orc.block_norm_fwd(self.x, self.y, self.u, *self.w, **self.more)[0]
        w_post, s, w_pre = (1.0 if w is None else f64(w) for w in self.w)
        act = 1.0 if self.u is None else orc.ACT[self.more["gate"]][0](f64(self.u))
        of_x = rms(f64(self.dn) * w_pre) * inv(h) if dn else 0.0
        ry = inv(f64(self.y)) if self.more["post_norm"] else 1.0
        on_u = s * f64(self.y) * ry * w_post
        return (of_x, ry * (rms(dx * s * act * w_post) + of_x * rms(np.ones_like(dx) * s * act * w_post)),
                rms(dx * on_u) + of_x * rms(np.ones_like(dx) * on_u))

    def check(self, dh=True, dn=True):
        for name, got, ref in zip(("h", "n"), self.fwd(), orc.block_norm_fwd(self.x, self.y, self.u, *self.w, **self.more)):
            near(got, ref, name)
        ref = orc.block_norm_bwd(self.x, self.y, self.u, *self.w, self.dh if dh else None, self.dn if dn else None, **self.more)
        terms = dict(zip(("dx", "dy", "du"), self.terms(dh, dn, ref[0])))
        for name, got, want in zip(("dx", "dy", "du", "dw_post", "ds", "dw_pre"), self.bwd(dh, dn), ref):
            if want is not None:
                near(got, want, name, terms.get(name, None) if want.ndim == 2 else np.sqrt(self.rows))
        self.done()


@pytest.mark.parametrize("dtype,res", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("D", [1, 7, 64, 100, 256, 257, 512, 768, 1003, 1024, 2048, 4096, 5000, 8192, 16384])
def test_widths(D, dtype, res):
    Case(5, D, dtype, res, la.LA_GATE_SILU, seed=D).check()


@pytest.mark.parametrize("rows", [1, 2, 8, 9, 441, 1000, 3001])
@pytest.mark.parametrize("D", [128, 1024, 999])
def test_numbers_of_rows(rows, D):
    Case(rows, D, BF16, F32, la.LA_GATE_SIGMOID, seed=rows).check()


@pytest.mark.parametrize("dtype,res", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("D", [2049, 4099, 8191, 8201, 16383])
def test_wide_rows_of_no_round_width(D, dtype, res):
    Case(5, D, dtype, res, la.LA_GATE_SILU, seed=D).check()


@pytest.mark.parametrize("dtype,res", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("D", [200, 301, 512, 1000, 1537, 2048, 2999, 4096, 5600, 8192])
def test_many_rows_of_each_width(D, dtype, res):
    """Enough of them (5 MB of residual stream) that every thread block takes several, an odd number."""
    rows = 5 * 2 ** 20 // (D * (2 if res is BF16 else 4)) | 1
    Case(rows, D, dtype, res, la.LA_GATE_SILU, seed=D).check()


@pytest.mark.parametrize("dtype,res", [(BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("D", [96, 2048])
def test_many_rows_in_other_forms(D, dtype, res):
    rows = 6 * 2 ** 20 // (D * (2 if res is BF16 else 4))
    for gate, weights, post_norm, dh, dn in ((None, True, True, True, False), (la.LA_GATE_PLAIN, False, True, False, True), (la.LA_GATE_SIGMOID, True, False, True, True)):
        Case(rows, D, dtype, res, gate, weights, post_norm=post_norm, seed=4).check(dh, dn)


@pytest.mark.parametrize("gate", GATES)
@pytest.mark.parametrize("weights", [True, False])
@pytest.mark.parametrize("post_norm", [True, False])
def test_forms(gate, weights, post_norm):
    for dh, dn in ((True, True), (True, False), (False, True)):
        Case(33, 320, BF16, BF16, gate, weights, post_norm=post_norm, seed=3).check(dh, dn)


def test_either_output_alone():
    c = Case(10, 512, BF16, BF16, None)
    h, n = c.fwd()
    for want_h in (True, False):
        out = c.out(BF16, 10, 512)
        la.la_block_norm_fwd(c.shape, *c.inputs(), out if want_h else None, None if want_h else out)
        assert torch.equal(out, h if want_h else n)
    c.done()


@pytest.mark.parametrize("D", [96, 101, 2048])
def test_rows_of_zeros(D):
    """Without eps a row of zeros has no direction: zeros, and no NaN among the gradients."""
    c = Case(6, D, F32, F32, la.LA_GATE_SILU, eps=0.0)
    c.y[1:3] = 0
    c.x[2] = 0
    c.check()
    assert not c.grads[1][1:3].any()


def test_large_and_small_gates():
    """The gate's exponential at both ends: exp(-u) overflows to infinity and vanishes."""
    c = Case(4, 64, F32, F32, la.LA_GATE_SILU)
    c.u[:, :4] = torch.tensor([100.0, -100.0, 88.0, -60.0])
    with np.errstate(over="ignore"):
        c.check()


def test_bad_rows_stay_alone():
    c = Case(40, 640, BF16, BF16, la.LA_GATE_SILU)
    h, n = (t.clone() for t in c.fwd())
    dx = c.bwd()[0].clone()
    c.y[7], c.y[20, 3] = float("nan"), float("inf")
    others = [i for i in range(40) if i not in (7, 20)]
    h2, n2 = c.fwd()
    dx2 = c.bwd()[0]
    for a, b in ((h, h2), (n, n2), (dx, dx2)):
        assert torch.equal(a[others], b[others]) and torch.isnan(b[7]).all()


def test_same_bits_from_graphs_and_streams():
    c = Case(700, 1024, BF16, F32, la.LA_GATE_SILU)
    inputs, dh, dn = c.inputs(), c.dev(c.dh), c.dev(c.dn)
    ws = la.alloc_block_norm_workspace(c.shape, DEV)
    h, n = c.out(F32, 700, 1024), c.out(BF16, 700, 1024)
    grads = [g.clone() for g in c.bwd()]
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=stream):
        la.la_block_norm_fwd(c.shape, *inputs, h, n)
        la.la_block_norm_bwd(c.shape, *inputs, dh, dn, *c.grads, ws)
    for g in c.grads:
        g.fill_(float("nan"))
    graph.replay()
    c.done()
    assert all(torch.equal(a, b) for a, b in zip(grads, c.grads))


def test_offsets_past_32_bits():
    past_32_bits()
    torch.cuda.empty_cache()


def past_32_bits():
    """More than 2^31 values to a tensor: the last rows have what they have alone."""
    D, last = 4096, 6
    rows = 2 ** 31 // D + 7
    c = Case(last, D, BF16, BF16, la.LA_GATE_SILU)
    shape = la.make_block_norm_shape(rows, D, BF16, BF16, **c.more)

    def whole(x):
        big = torch.zeros(rows, D, dtype=BF16, device=DEV)
        big[-last:] = x.to(DEV)
        return big

    x, y, u, dh, dn = (whole(t) for t in (c.x, c.y, c.u, c.dh, c.dn))
    w = [t.to(DEV) for t in c.w]
    h, n, dx, dy, du = (torch.empty_like(x) for _ in range(5))
    dw = [torch.empty(D, device=DEV) for _ in range(3)]
    la.la_block_norm_fwd(shape, x, y, u, *w, h, n)
    la.la_block_norm_bwd(shape, x, y, u, *w, dh, dn, dx, dy, du, *dw, la.alloc_block_norm_workspace(shape, DEV))
    ref = orc.block_norm_fwd(c.x, c.y, c.u, *c.w, **c.more) + orc.block_norm_bwd(c.x, c.y, c.u, *c.w, c.dh, c.dn, **c.more)
    terms = (None, None) + c.terms(True, True, ref[2])
    for name, got, want, more in zip(("h", "n", "dx", "dy", "du"), (h, n, dx, dy, du), ref, terms):
        near(got[-last:], want, name, more)
    for name, got, want in zip(("dw_post", "ds", "dw_pre"), dw, ref[5:]):  # (the rows before are zeros)
        near(got, want, name, np.sqrt(last))


def test_gradient_against_differences():
    """Central differences of the forward pass along a random direction: the rest of third order is 1e-6 of the loss's scale at this
    step, the forward pass's roundings (1e-6 of a value, random signs) are divided by it."""
    c = Case(6, 200, F32, F32, la.LA_GATE_SILU)
    grads = [g.double().cpu() for g in c.bwd()]
    gen = torch.Generator()
    gen.manual_seed(3)
    step = 2.0 ** -8
    at = [(lambda v: setattr(c, "x", v), c.x, 0), (lambda v: setattr(c, "y", v), c.y, 1), (lambda v: setattr(c, "u", v), c.u, 2)]
    at += [(lambda v, i=i: c.w.__setitem__(i, v), c.w[i], 3 + i) for i in range(3)]
    for put, x, i in at:
        way = torch.randn(x.shape, generator=gen)
        loss = []
        for sign in (1, -1):
            put(x + sign * step * way)
            h, n = c.fwd()
            loss.append(((h.double().cpu() * c.dh.double()).sum() + (n.double().cpu() * c.dn.double()).sum()).item())
        put(x)
        want = (grads[i] * way.double()).sum().item()
        assert abs((loss[0] - loss[1]) / (2 * step) - want) <= 2e-3 * np.sqrt(6 * 200) + 2e-3 * abs(want)


def test_wrong_tensors_are_refused():
    c = Case(4, 64, BF16, F32, la.LA_GATE_SILU)
    x, y, u, *w = c.inputs()
    h, n = c.out(F32, 4, 64), c.out(BF16, 4, 64)
    launched = la.launch_count()
    for bad in ((x.bfloat16(), y, u, *w), (x, y.float(), u, *w), (x, y[:2].contiguous(), u, *w), (x, y, u, w[0].double(), w[1], w[2]),
                (x, y, u, w[0][:32].contiguous(), w[1], w[2]), (x, y, u.cpu(), *w)):
        with pytest.raises(ValueError):
            la.la_block_norm_fwd(c.shape, *bad, h, n)
    with pytest.raises(la.LaError):
        la.la_block_norm_fwd(c.shape, x, y, u, *w, None, None)
    with pytest.raises(la.LaError):  # a gate without its gradient
        la.la_block_norm_bwd(c.shape, x, y, u, *w, c.dev(c.dh), None, h, n, None, None, None, None, la.alloc_block_norm_workspace(c.shape, DEV))
    with pytest.raises(TypeError):
        la.la_block_norm_fwd(la.make_shape(1, 2, 64, 64, 64, BF16, F32), x, y, u, *w, h, n)
    assert la.launch_count() == launched


@pytest.mark.parametrize("dtype,res", [(BF16, BF16), (BF16, F32), (F32, F32)])
@pytest.mark.parametrize("D", [8190, 8201, 12288])
def test_wide_rows_in_turn(D, dtype, res):
    """More rows than thread blocks (9472) where the ring does not go, so that one takes several: the bits of calls in which each has one
    row, with one sum to a row (no post norm, or h alone) and with two."""
    rows, part = 2 * 9472 + 5, 9472
    gen = torch.Generator(DEV)
    gen.manual_seed(D)
    new = lambda dt: torch.empty(rows, D, dtype=dt, device=DEV).normal_(generator=gen)
    x, y, w = new(res), new(dtype), [0.5 + torch.rand(D, generator=gen, device=DEV) for _ in range(3)]
    y *= torch.rand(rows, 1, generator=gen, device=DEV).to(dtype)  # (rows of different sizes)
    for post_norm, want_h, want_n in ((False, True, True), (False, False, True), (True, True, False), (True, True, True)):
        def run(a, b):
            shape = la.make_block_norm_shape(b - a, D, dtype, res, eps=1e-6, post_norm=post_norm)
            h = torch.empty(b - a, D, dtype=res, device=DEV) if want_h else None
            n = torch.empty(b - a, D, dtype=dtype, device=DEV) if want_n else None
            la.la_block_norm_fwd(shape, x[a:b], y[a:b], None, *w, h, n)
            return h, n

        whole = run(0, rows)
        for a in range(0, rows, part):
            b = min(rows, a + part)
            for got, want in zip(whole, run(a, b)):
                assert got is None or torch.equal(got[a:b], want), (post_norm, want_h, want_n)
        del whole


@pytest.mark.parametrize("post_norm", [True, False])
@pytest.mark.parametrize("D,dtype,res,rows", [
    (8190, BF16, BF16, 901), (8190, BF16, F32, 601), (8190, F32, F32, 601), (8201, BF16, BF16, 301), (8201, F32, F32, 449), (12288, BF16, F32, 301),
    (16384, BF16, BF16, 301), (16384, F32, F32, 301), (5700, F32, F32, 601), (6144, F32, F32, 901), (8192, F32, F32, 601)])
def test_gradients_of_wide_rows_in_turn(D, dtype, res, rows, post_norm):
    """Gradients where the ring does not go, with several rows to a thread block: 148 of more than 8192 features, else 296."""
    Case(rows, D, dtype, res, la.LA_GATE_SILU, post_norm=post_norm, seed=D).check()


@pytest.mark.parametrize("dh,dn", [(True, False), (False, True)])
def test_either_gradient_of_wide_rows_in_turn(dh, dn):
    Case(301, 8201, BF16, BF16, la.LA_GATE_SIGMOID, seed=5).check(dh, dn)


@pytest.mark.parametrize("gate", [la.LA_GATE_SIGMOID, la.LA_GATE_SILU])
@pytest.mark.parametrize("D,rows,dtype", [(1024, 9, F32), (1024, 1200, F32), (1003, 9, F32), (8200, 3, F32), (1024, 9, BF16), (1024, 1200, BF16), (8200, 3, BF16)])
def test_gates_relative_to_their_own_size(D, rows, dtype, gate):
    """The gate and its derivative alone (x = 0, y = 1, no norm), in the direct forms and the ring's.  The exponential is good to 2^-22, the
    reciprocal to 2^-23, three roundings to 2^-24 each: 5.4e-7 of a sigmoid, however small; two factors round once more.  The derivatives
    are sums of two terms where u is small: where they are not (|u| >= 3, negative), those of a sigmoid have two such errors, and those
    of SiLU, s + u s (1 - s), 2.9 + 1 of them over 1.9.  Below exp(-87) values are subnormal.  With u in bf16 the ring's exponent is a
    product rounded once, 2^-24 of it, of a constant that is off by 1.34e-8 of itself: |u| 7.3e-8 more, twice that for the derivatives,
    and those are rounded to bf16."""
    c = Case(rows, D, dtype, F32, gate, weights=False, post_norm=False)
    c.x[:], c.y[:], c.dh[:] = 0.0, 1.0, 1.0
    c.u[:] = torch.linspace(-120.0, 120.0, rows * D).view(rows, D)[:, torch.randperm(D, generator=torch.Generator().manual_seed(2))]
    c.u[0, :4] = torch.tensor([-np.inf, np.inf, -2.0 ** 127, 2.0 ** 127])
    u = c.u.double().numpy()
    bf16 = dtype is BF16
    more = np.minimum(np.abs(u), 130) * (7.3e-8 if bf16 else 0.0)
    with np.errstate(over="ignore", invalid="ignore"):
        want, slope = (f(u) for f in orc.ACT[gate])
    odd = np.zeros_like(u, dtype=bool)
    odd[0, :4] = True
    h = torch.empty(rows, D, device=DEV)
    la.la_block_norm_fwd(c.shape, *c.inputs(), h, None)
    got = h.double().cpu().numpy()
    off = np.abs(got[~odd] - want[~odd]) - ((6.5e-7 + more) * np.abs(want))[~odd] - 2.0 ** -126 * np.maximum(1, np.abs(u[~odd]))
    assert off.max() <= 0
    if gate == la.LA_GATE_SIGMOID:
        assert np.array_equal(got[odd], [0, 1, 0, 1])
    else:
        assert np.isnan(got[0, 0]) and got[0, 1] == np.inf and got[0, 2] == 0 and got[0, 3] == 2.0 ** 127
    c.u[0, :4] = -50.0
    u[0, :4], more[0, :4] = -50.0, 50 * 7.3e-8 if bf16 else 0.0
    slope = orc.ACT[gate][1](np.clip(u, -700, 700))
    du = c.bwd(dn=False)[2].double().cpu().numpy()
    some = u <= -3
    off = np.abs(du - slope)[some] - ((2e-6 + 2 * more + (2.0 ** -8 if bf16 else 0.0)) * np.abs(slope))[some] - 2.0 ** -126 * np.maximum(1, np.abs(u[some]))
    assert off.max() <= 0
    c.done()
