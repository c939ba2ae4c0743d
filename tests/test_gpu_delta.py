"""The gated delta rule through the C ABI against the fp64 oracle: la_delta_fwd, la_delta_bwd, la_delta_steps.

Tolerances, in units of the RMS of each (batch, head) slice of the result.  CUDA cores: fp32 throughout, the library's 1e-4 for its fp32
workload.  Tensor cores: operands that are formed on chip are rounded to two bf16 terms, at most 2^-16 of each value (each term leaves
2^-8 / sqrt(3) of the rest on the root of the mean square, times 0.72 for values spread over a binade: 2.7e-6 for both); a result passes
six such operands forward and twelve backward, 9e-6, its largest error is five times that, and the inverse of a unit triangle with
entries below 1 enlarges it by 4 at most on these inputs: 2e-4, and half as much again for the products of lo terms that are left out.  A result in bf16 is off by half a step of its own besides, 2^-8 of its value."""
import numpy as np
import pytest
import torch

from oracle import delta_oracle as orc
from paper_2307_14995_b200 import binding as la

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
HEADS, TOKENS = la.LA_LAYOUT_BHND, la.LA_LAYOUT_BNHD


def draw(B, H, Hk, N, d, seed, dtype=BF16, rates=None):
    """Heads first, on the CPU: q, k of unit length, v, do normal, beta in (0, 1), one rate of forgetting per head."""
    gen = torch.Generator()
    gen.manual_seed(seed)
    new = lambda *s: torch.randn(*s, generator=gen)
    q, k = (torch.nn.functional.normalize(torch.nn.functional.silu(new(B, Hk, N, d)), dim=-1).to(dtype) for _ in range(2))
    v, do = new(B, H, N, d).to(dtype), new(B, H, N, d).to(dtype)
    rates = torch.logspace(-3, 0.5, H) if rates is None else torch.tensor(rates)
    g = -rates.view(1, H, 1) * (0.5 + torch.rand(B, H, N, generator=gen))
    return q, k, v, g, torch.sigmoid(new(B, H, N)), do


def tol(shape_path, dtype):
    return 1e-4 if dtype is F32 or shape_path == la.LA_PATH_SIMT else 3e-4


def near(got, ref, tol, what):
    assert tuple(got.shape) == ref.shape, what
    g, r = got.double().cpu().numpy(), np.asarray(ref)
    assert np.all(np.isfinite(g)), what
    rms = np.sqrt(np.mean((r * r).reshape(*r.shape[:2], -1), -1)).reshape(r.shape[:2] + (1,) * (r.ndim - 2))
    off = np.abs(g - r) - (2.0 ** -8 * np.abs(r) if got.dtype is BF16 else 0.0)
    worst = np.max(off / np.maximum(rms, 1e-30))
    assert worst <= tol, "%s: %.2e of the RMS, %.1e allowed" % (what, worst, tol)


class Call:
    """One layer's tensors on the GPU, with a margin behind each output that has to stay as it is."""

    def __init__(self, data, out=F32, layout=HEADS, scale=0.25, path=la.LA_PATH_AUTO, kv_in=None, grad_kv_out=None):
        self.tokens = layout == TOKENS
        q, k, v, g, beta, do = data
        self.B, self.Hk, self.N, self.d = q.shape
        self.H = v.shape[1]
        self.inputs = [self.move(x).to(DEV) for x in (q, k, v, g, beta)]
        self.do = self.move(do).to(DEV)
        self.shape = la.make_delta_shape(self.B, self.H, self.N, self.d, self.d, q.dtype, out, Hk=self.Hk, scale=scale, path=path, layout=layout)
        self.states = {n: None if x is None else x.to(DEV) for n, x in (("kv_in", kv_in), ("grad_kv_out", grad_kv_out))}
        self.margins = []
        self.o, self.dv = (self.output(out, self.H, self.d) for _ in range(2))
        self.dq, self.dk = (self.output(out, self.Hk, self.d) for _ in range(2))
        self.dg, self.dbeta = (self.output(F32, self.H) for _ in range(2))
        self.kv_out, self.grad_kv_in = (self.buffer(F32, (self.B, self.H, self.d, self.d)) for _ in range(2))
        self.ws_f, self.ws_b = (torch.full((la.delta_workspace_bytes(op, self.shape),), 255, dtype=torch.uint8, device=DEV)
                                for op in (la.LA_OP_FWD, la.LA_OP_BWD))  # NaN in every type

    def move(self, x):
        return x.transpose(1, 2).contiguous() if self.tokens else x.contiguous()

    def buffer(self, dtype, size):
        n = int(np.prod(size))
        whole = torch.full((n + 256,), float("nan"), dtype=dtype, device=DEV)
        self.margins.append(whole[n:])
        return whole[:n].view(size)

    def output(self, dtype, heads, *more):
        return self.buffer(dtype, (self.B, self.N, heads, *more) if self.tokens else (self.B, heads, self.N, *more))

    def fwd(self, **more):
        la.la_delta_fwd(self.shape, *self.inputs, self.o, self.states["kv_in"], self.kv_out, self.ws_f, **more)

    def bwd(self, reuse=True, **more):
        la.la_delta_bwd(self.shape, *self.inputs, self.do, self.dq, self.dk, self.dv, self.dg, self.dbeta, **self.states,
                        grad_kv_in=self.grad_kv_in, workspace=self.ws_b, fwd_workspace=self.ws_f if reuse else None, **more)

    def done(self):
        torch.cuda.synchronize()
        la.device_status()
        assert all(torch.isnan(m).all() for m in self.margins)

    def results(self):
        back = lambda x: x.transpose(1, 2) if self.tokens else x
        return dict(o=back(self.o), kv_out=self.kv_out, dq=back(self.dq), dk=back(self.dk), dv=back(self.dv), dg=back(self.dg),
                    dbeta=back(self.dbeta), grad_kv_in=self.grad_kv_in)


def reference(data, scale=0.25, kv_in=None, grad_kv_out=None):
    *args, do = data
    o, kv = orc.delta_fwd(*args, scale=scale, kv_in=kv_in)
    return dict(zip(("o", "kv_out", "dq", "dk", "dv", "dg", "dbeta", "grad_kv_in"),
                    (o, kv) + orc.delta_bwd(*args, do, scale=scale, kv_in=kv_in, grad_kv_out=grad_kv_out)))


def check(call, ref, tolerance, only=None):
    for name, got in call.results().items():
        if only is None or name in only:
            near(got, ref[name], tolerance, name)


def states(B, H, d, seed):
    gen = torch.Generator()
    gen.manual_seed(seed)
    return [torch.randn(B, H, d, d, generator=gen) for _ in range(2)]


KINDS = [(BF16, la.LA_PATH_AUTO), (BF16, la.LA_PATH_SIMT), (F32, la.LA_PATH_AUTO)]


@pytest.mark.parametrize("dtype,path", KINDS)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N", [1, 2, 63, 64, 65, 127, 128, 129, 300, 515])
def test_lengths(N, d, dtype, path):
    """Forward and backward with states in and out, on the forward pass's workspace and without."""
    data = draw(2, 3, 3, N, d, 10 + N, dtype)
    kv_in, grad = states(2, 3, d, N)
    call = Call(data, kv_in=kv_in, grad_kv_out=grad, path=path)
    ref = reference(data, kv_in=kv_in, grad_kv_out=grad)
    call.fwd()
    call.bwd()
    call.done()
    check(call, ref, tol(path, dtype))
    first = {n: x.clone() for n, x in call.results().items()}
    call.ws_b.fill_(255)
    call.bwd(reuse=False)
    call.done()
    assert all(torch.equal(first[n], x) for n, x in call.results().items())


@pytest.mark.parametrize("dtype,path", KINDS)
@pytest.mark.parametrize("layout", [HEADS, TOKENS])
@pytest.mark.parametrize("H,Hk", [(1, 1), (4, 2), (6, 2), (8, 1)])
def test_shared_heads_and_layouts(H, Hk, layout, dtype, path):
    out = F32 if dtype is F32 else BF16
    data = draw(2, H, Hk, 200, 128, H, dtype)
    call = Call(data, out=out, layout=layout, path=path)
    call.fwd()
    call.bwd()
    call.done()
    check(call, reference(data), tol(path, dtype))


@pytest.mark.parametrize("dtype,path", KINDS)
def test_long_sequence(dtype, path):
    """Many chunks, rates from hardly any forgetting to a few tokens' memory."""
    data = draw(1, 4, 4, 2500, 128, 5, dtype, rates=[0.0, 1e-3, 0.1, 3.0])
    call = Call(data, path=path)
    call.fwd()
    call.bwd()
    call.done()
    check(call, reference(data), tol(path, dtype))


@pytest.mark.parametrize("dtype,path", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_gates_at_their_ends(d, dtype, path):
    """Forgetting everything (g = -inf, and so strongly that it is the same in fp32), idle tokens (beta = 0), whole idle chunks,
    beta of 1 and 2, keys that repeat, keys and queries of zero."""
    q, k, v, g, beta, do = draw(1, 3, 3, 400, d, 77, dtype)
    g[:, 0, [0, 5, 64, 127, 128, 300]] = -np.inf
    g[:, 1, 10:20] = -500.0
    beta[:, :, ::7] = 0.0
    beta[:, 1, 128:256] = 0.0
    beta[:, 2, 1::3] = 1.0
    beta[:, 0, 2::50] = 2.0
    k[:, :, 30:36] = k[:, :, 30:31]
    k[:, :, 60:62] = 0
    q[:, :, 61] = 0
    data = (q, k, v, g, beta, do)
    kv_in, grad = states(1, 3, d, 3)
    call = Call(data, kv_in=kv_in, grad_kv_out=grad, path=path)
    call.fwd()
    call.bwd()
    call.done()
    check(call, reference(data, kv_in=kv_in, grad_kv_out=grad), tol(path, dtype))


@pytest.mark.parametrize("dtype,path", KINDS)
def test_packed_sequences(dtype, path):
    """Sequences one after the other, g = -inf at the first token of each: every one as on its own, forward and backward."""
    lengths = [1, 130, 64, 5, 200]
    data = list(draw(1, 4, 2, sum(lengths), 128, 61, dtype))
    first = np.cumsum([0] + lengths)
    data[3][:, :, first[:-1]] = -np.inf
    call = Call(data, path=path)
    call.fwd()
    call.bwd()
    call.done()
    got = call.results()
    for a, b in zip(first[:-1], first[1:]):
        ref = reference([x[:, :, a:b].contiguous() for x in data])
        for name in ("o", "dq", "dk", "dv", "dbeta"):
            near(got[name][:, :, a:b], ref[name], tol(path, dtype) * (1 if b - a > 5 else 4), name)  # (an RMS of few values)


@pytest.mark.parametrize("dtype,path", KINDS)
def test_gradient_against_differences(dtype, path):
    """The backward pass against differences of the forward pass of the same kernels: along a random direction of g, beta and kv_in,
    which are fp32 and can be moved by little.  Of a central difference with step 2^-7 the rest is of third order, 2^-14 / 6 of the
    function's third derivative, and the forward pass's own error is divided by the step: 2^7 times its 3e-4 of an output's RMS, on
    independent outputs summed up with random signs: n^-1/2 of the sum of their sizes."""
    B, H, N, d = 1, 2, 150, 64
    data = draw(B, H, H, N, d, 21, dtype, rates=[0.01, 0.2])
    kv_in, _ = states(B, H, d, 4)
    base = Call(data, kv_in=kv_in, path=path)
    base.fwd()
    base.bwd()
    base.done()
    gen = torch.Generator()
    gen.manual_seed(1)
    step = 2.0 ** -7
    for i, grad in ((3, "dg"), (4, "dbeta"), (None, "grad_kv_in")):
        way = torch.randn(data[i].shape if i else kv_in.shape, generator=gen) * 0.1
        loss = []
        for sign in (1, -1):
            moved = list(data)
            start = kv_in
            if i:
                moved[i] = data[i] + sign * step * way
            else:
                start = kv_in + sign * step * way
            call = Call(moved, kv_in=start, path=path)
            call.fwd()
            call.done()
            loss.append((call.o.double() * call.do.double()).sum().item())
        want = (base.results()[grad].double().cpu() * way.double()).sum().item()
        size = (base.o.double().square().mean().sqrt() * np.sqrt(base.o.numel())).item()
        assert abs((loss[0] - loss[1]) / (2 * step) - want) <= 1e-3 * abs(want) + 4 * size * 3e-4 / (2 * step) / np.sqrt(8)


def steps_tol(N):
    """A token rounds every element of the state twice, half a step of 2^-24 of at most 5 RMS: 6e-7; and adds beta k_i times a sum of
    128 products made in 24 additions, 24 x 2^-24 of an RMS times at most a half: 7e-7.  An output is such a sum once more."""
    return 1.3e-6 * N + 1.5e-6


@pytest.mark.parametrize("dtype,out", [(BF16, F32), (BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("N", [1, 2, 8, 9, 20])
@pytest.mark.parametrize("layout", [HEADS, TOKENS])
def test_steps(N, d, dtype, out, layout):
    """Decoding: against the oracle, and N calls with one token give the bits of one call with N."""
    B, H, Hk = 3, 4, 2
    data = draw(B, H, Hk, N, d, N, dtype)
    kv0 = states(B, H, d, 9)[0]
    call = Call(data, out=out, layout=layout, kv_in=kv0)
    kv = kv0.to(DEV)
    la.la_delta_steps(call.shape, *call.inputs, kv, call.o)
    call.done()
    ref, ref_kv = orc.delta_fwd(*data[:5], scale=0.25, kv_in=kv0)
    near(call.results()["o"], ref, steps_tol(N), "o")
    near(kv, ref_kv, steps_tol(N), "kv")
    one = la.make_delta_shape(B, H, 1, d, d, dtype, out, Hk=Hk, scale=0.25, layout=layout)
    axis = 1 if layout == TOKENS else 2
    kv1 = kv0.to(DEV)
    for t in range(N):
        o = torch.empty_like(call.o.select(axis, t).contiguous())
        la.la_delta_steps(one, *(x.select(axis, t).contiguous() for x in call.inputs), kv1, o)
        assert torch.equal(o, call.o.select(axis, t))
    assert torch.equal(kv1, kv)


def test_steps_with_gates_at_their_ends():
    data = list(draw(1, 2, 2, 6, 128, 3))
    data[3][:, 0, 2], data[4][:, 1, :] = -np.inf, 0.0
    kv0 = states(1, 2, 128, 2)[0]
    call = Call(data)
    kv = kv0.to(DEV)
    la.la_delta_steps(call.shape, *call.inputs, kv, call.o)
    ref, ref_kv = orc.delta_fwd(*data[:5], scale=0.25, kv_in=kv0)
    near(call.o, ref, steps_tol(6), "o")
    near(kv, ref_kv, steps_tol(6), "kv")


def test_prompt_then_decoding_then_prompt():
    """A run as a server makes it: a prompt, drafted tokens, a further prompt from the state, against one pass over all of it."""
    B, H, d = 1, 4, 128
    data = draw(B, H, 2, 400, d, 31)
    whole = reference(data)
    parts, kv = [(0, 250), (250, 254), (254, 255), (255, 400)], torch.zeros(B, H, d, d)
    outs = []
    for a, b in parts:
        call = Call([x[:, :, a:b].contiguous() for x in data], kv_in=kv, layout=TOKENS)
        if b - a < 10:
            state = kv.to(DEV)
            la.la_delta_steps(call.shape, *call.inputs, state, call.o)
            call.kv_out = state
        else:
            call.fwd()
        call.done()
        outs.append(call.results()["o"].cpu())
        kv = call.kv_out.cpu()
    near(torch.cat(outs, 2), whole["o"], 3e-4, "o")
    near(kv, whole["kv_out"], 3e-4, "kv_out")


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_layer_between_two_norms(dtype):
    """A layer of a model as it is used: block norm, delta rule, gate, block norm, each reading what the one before it wrote."""
    B, H, N, d = 1, 4, 300, 64
    D = H * d
    gen = torch.Generator()
    gen.manual_seed(8)
    x, y = (torch.randn(B * N, D, generator=gen).to(dtype) for _ in range(2))
    q, k, _, g, beta, _ = draw(B, H, H, N, d, 12, dtype)
    norm = la.make_block_norm_shape(B * N, D, dtype, dtype, eps=1e-6)
    xg, yg = x.to(DEV), y.to(DEV)
    h, n, h2, n2, o, gated = (torch.empty_like(xg) for _ in range(6))
    shape = la.make_delta_shape(B, H, N, d, d, dtype, dtype, layout=TOKENS)
    heads = lambda t: t.view(B, N, H, d)
    gate = la.make_shape(B, H, N, d, d, dtype, dtype, layout=TOKENS)
    args = [t.transpose(1, 2).contiguous().to(DEV) for t in (q, k, g, beta)]
    la.la_block_norm_fwd(norm, xg, yg, h=h, n=n)
    la.la_delta_fwd(shape, args[0], args[1], heads(n), args[2], args[3], heads(o), workspace=la.alloc_delta_workspace(la.LA_OP_FWD, shape, DEV))
    la.la_gate_fwd(gate, heads(o), heads(n), heads(gated))
    la.la_block_norm_fwd(norm, h, gated, h=h2, n=n2)
    torch.cuda.synchronize()
    la.device_status()
    # each stage against the oracle on what the stage before it wrote
    first = orc.block_norm_fwd(x, y, eps=1e-6)
    near(h.view(B, N, D), first[0].reshape(B, N, D), 1e-5, "h")
    near(n.view(B, N, D), first[1].reshape(B, N, D), 1e-5, "n")
    v = heads(n.cpu()).transpose(1, 2)
    near(heads(o).transpose(1, 2), orc.delta_fwd(q, k, v, g, beta)[0], 3e-4, "o")
    second = orc.block_norm_fwd(h.cpu(), gated.cpu(), eps=1e-6)
    near(h2.view(B, N, D), second[0].reshape(B, N, D), 1e-5, "h2")
    near(n2.view(B, N, D), second[1].reshape(B, N, D), 1e-5, "n2")


@pytest.mark.parametrize("path", [la.LA_PATH_AUTO, la.LA_PATH_SIMT])
def test_offsets_past_32_bits(path):
    past_32_bits(path)
    torch.cuda.empty_cache()


def past_32_bits(path):
    """More than 2^31 values and 2^32 bytes to a tensor, ten times that to a workspace.  The last head's last tokens stand alone behind a token that
    forgets everything, so that they have a reference of their own."""
    H, N, d, last = 64, 262800 + 200, 128, 200
    gen = torch.Generator(DEV)
    gen.manual_seed(8)
    q, k = (torch.nn.functional.normalize(torch.randn(1, 1, N, d, generator=gen, device=DEV), dim=-1).to(BF16) for _ in range(2))
    v, do = (torch.empty(1, H, N, d, dtype=BF16, device=DEV).normal_(generator=gen) for _ in range(2))
    g, beta = (torch.rand(1, H, N, generator=gen, device=DEV) for _ in range(2))
    g *= -0.1
    g[:, :, N - last] = -np.inf
    shape = la.make_delta_shape(1, H, N, d, d, BF16, BF16, Hk=1, scale=0.25, path=path)
    o, dv = torch.empty_like(v), torch.empty_like(v)
    dq, dk, dg, dbeta = torch.empty_like(q), torch.empty_like(k), torch.empty_like(g), torch.empty_like(g)
    ws_f = la.alloc_delta_workspace(la.LA_OP_FWD, shape, DEV)
    la.la_delta_fwd(shape, q, k, v, g, beta, o, workspace=ws_f)
    ws_b = torch.empty(la.delta_workspace_bytes(la.LA_OP_BWD, shape) - ws_f.numel(), dtype=torch.uint8, device=DEV)
    la.la_delta_bwd(shape, q, k, v, g, beta, do, dq, dk, dv, dg, dbeta, workspace=ws_b, fwd_workspace=ws_f)
    torch.cuda.synchronize()
    la.device_status()
    tail = lambda x: x[:, -1:, N - last:].cpu()
    data = [tail(x) for x in (q, k, v, g, beta, do)]
    data[3][:, :, 0] = 0.0  # (on a state of zeros it makes no difference)
    ref = reference(data)
    for name, got in (("o", o), ("dv", dv), ("dg", dg), ("dbeta", dbeta)):
        near(tail(got), ref[name], tol(path, BF16), name)


@pytest.mark.parametrize("dtype,path", KINDS)
def test_streams_and_graphs(dtype, path):
    """The same bits on a stream of the caller's and from a captured graph that is replayed on new inputs, two graphs on one workspace
    replayed one after the other included; the calls allocate nothing."""
    data = draw(1, 4, 2, 700, 128, 41, dtype)
    call = Call(data, path=path)
    call.fwd()
    call.bwd()
    call.done()
    want = {n: x.clone() for n, x in call.results().items()}
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    call.fwd(stream=stream)
    call.bwd(stream=stream)
    call.done()
    assert all(torch.equal(want[n], x) for n, x in call.results().items())
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph, stream=stream):
            call.fwd()
            call.bwd()
    before = torch.cuda.memory_allocated()
    for x in call.inputs[:3]:
        x.copy_(torch.flip(x, [0, 1]))
    graphs[0].replay()
    graphs[1].replay()
    call.done()
    assert torch.cuda.memory_allocated() <= before + (1 << 20)
    other = {n: x.clone() for n, x in call.results().items()}
    call.fwd()
    call.bwd()
    call.done()
    assert all(torch.equal(other[n], x) for n, x in call.results().items())


@pytest.mark.parametrize("dtype,path", KINDS)
def test_two_calls_at_once(dtype, path):
    """On two streams, each with its workspaces and beside an ordinary attention call on a third: the bits that each has alone."""
    calls = [Call(draw(2, 8, 4, 900, 128, 60 + i, dtype), path=path) for i in range(2)]
    wants = []
    for call in calls:
        call.fwd()
        call.bwd()
        call.done()
        wants.append({n: x.clone() for n, x in call.results().items()})
    q, k, v = (torch.randn(2, 8, 900, 128, device=DEV).to(BF16) for _ in range(3))
    lam = np.full(8, 0.97, np.float32)
    o = la.fwd(q, k, v, lam)
    o = (o[0] if isinstance(o, tuple) else o).clone()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(5):
        for call, stream in zip(calls, streams):
            call.fwd(stream=stream)
            call.bwd(stream=stream)
        with torch.cuda.stream(streams[2]):
            again = la.fwd(q, k, v, lam)
    for call, want in zip(calls, wants):
        call.done()
        assert all(torch.equal(want[n], x) for n, x in call.results().items())
    assert torch.equal(again[0] if isinstance(again, tuple) else again, o)


@pytest.mark.parametrize("dtype,path", KINDS)
def test_a_bad_row_stays_where_it_belongs(dtype, path):
    """NaN and infinity in one sequence's and one head's tokens reach no other, and tokens before them stay as they are."""
    data = list(draw(2, 4, 2, 300, 128, 51, dtype))
    call = Call(data, path=path)
    call.fwd()
    call.done()
    want = call.o.clone()
    data[2][0, 1, 200] = float("nan")
    data[2][1, 2, 290, 5] = float("inf")
    bad = Call(data, path=path)
    bad.fwd()
    bad.done()
    o = bad.o
    assert torch.equal(o[0, [0, 2, 3]], want[0, [0, 2, 3]]) and torch.equal(o[1, [0, 1, 3]], want[1, [0, 1, 3]])
    chunk = 64 if path == la.LA_PATH_SIMT or dtype is F32 else 128
    assert torch.equal(o[0, 1, :200 // chunk * chunk], want[0, 1, :200 // chunk * chunk])
    assert torch.isnan(o[0, 1, 200:]).all()


def test_wrong_tensors_are_refused():
    """Types, sizes and devices that are not the shape's, before anything is launched."""
    data = draw(1, 2, 2, 64, 64, 1)
    call = Call(data)
    launched = la.launch_count()
    q, k, v, g, beta = call.inputs
    for bad in ([q.float(), k, v, g, beta], [q, k[:, :1].contiguous(), v, g, beta], [q, k, v, g.bfloat16(), beta],
                [q, k, v, g, beta[:, :, :10].contiguous()], [q, k, v.cpu(), g, beta], [q, k, v.transpose(2, 3), g, beta]):
        with pytest.raises(ValueError):
            la.la_delta_fwd(call.shape, *bad, call.o, workspace=call.ws_f)
    with pytest.raises(TypeError):
        la.la_delta_fwd(la.make_shape(1, 2, 64, 64, 64, BF16, F32), *call.inputs, call.o, workspace=call.ws_f)
    with pytest.raises(la.LaError):
        la.la_delta_fwd(call.shape, *call.inputs, call.o, workspace=call.ws_f[:-256])
    with pytest.raises(la.LaError):
        la.la_delta_bwd(call.shape, *call.inputs, call.do, call.dq, call.dk, call.dv, call.dg, call.dbeta, workspace=call.ws_b,
                        fwd_workspace=call.ws_f[:-256])
    assert la.launch_count() == launched


@pytest.mark.parametrize("d,B,H,Hk", [(64, 5, 16, 16), (64, 5, 16, 4), (128, 2, 20, 20), (128, 4, 12, 6)])
@pytest.mark.parametrize("layout", [HEADS, TOKENS])
def test_more_heads_than_run_at_once(d, B, H, Hk, layout):
    """From 75 heads of 64 features and 38 of 128 on, a thread block of the chain has 64 columns of a state: every output, states in and out."""
    data = draw(B, H, Hk, 300, d, H, rates=np.logspace(-3, 0.5, H).tolist())
    kv_in, grad = states(B, H, d, 6)
    call = Call(data, layout=layout, kv_in=kv_in, grad_kv_out=grad)
    call.fwd()
    call.bwd()
    call.done()
    check(call, reference(data, kv_in=kv_in, grad_kv_out=grad), tol(la.LA_PATH_AUTO, BF16))


@pytest.mark.parametrize("dtype,path", KINDS)
@pytest.mark.parametrize("H,Hk", [(4, 2), (6, 2), (8, 1)])
def test_shared_heads_of_64_features(H, Hk, dtype, path):
    data = draw(2, H, Hk, 200, 64, H, dtype)
    kv_in, grad = states(2, H, 64, 7)
    call = Call(data, layout=TOKENS, path=path, kv_in=kv_in, grad_kv_out=grad)
    call.fwd()
    call.bwd()
    call.done()
    check(call, reference(data, kv_in=kv_in, grad_kv_out=grad), tol(path, dtype))


@pytest.mark.parametrize("dtype,path", KINDS)
def test_packed_sequences_gradients_of_gates(dtype, path):
    """dg of packed sequences: every one as on its own, and nothing at all where everything is forgotten."""
    lengths = [40, 130, 64, 1, 200]
    data = list(draw(1, 4, 2, sum(lengths), 128, 62, dtype))
    first = np.cumsum([0] + lengths)
    data[3][:, :, first[:-1]] = -np.inf
    call = Call(data, path=path)
    call.fwd()
    call.bwd()
    call.done()
    assert not call.dg[:, :, first[:-1]].any()
    for a, b in zip(first[:-1], first[1:]):
        if b - a > 1:
            near(call.dg[:, :, a:b], reference([x[:, :, a:b].contiguous() for x in data])["dg"], tol(path, dtype), "dg")


@pytest.mark.parametrize("dtype,path", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_precision_that_is_stated(d, dtype, path):
    """The relative 2-norm of the error of fp32 results.  Tensor cores: operands formed on chip are off by 2.7e-6 on the root of the mean
    square, of which a result passes six forward and twelve backward, 6.6e-6 and 9.4e-6 with random signs, and half as much again for the
    products of lo terms that are left out.  CUDA cores: a product's sum of 128 terms rounds 128 times, each by 2^-24 / 3^1/2 of a partial sum
    at most, whose size grows as the root of its terms: 2^-24 (128 / 6)^1/2 = 2.8e-7; six of them 6.7e-7, twelve 9.5e-7."""
    data = draw(2, 4, 2, 515, d, 14, dtype, rates=[1e-3, 0.03, 0.3, 2.0])
    kv_in, grad = states(2, 4, d, 8)
    call = Call(data, kv_in=kv_in, grad_kv_out=grad, path=path)
    call.fwd()
    call.bwd()
    call.done()
    ref = reference(data, kv_in=kv_in, grad_kv_out=grad)
    tensor = dtype is BF16 and path == la.LA_PATH_AUTO
    for name, got in call.results().items():
        error = np.linalg.norm(got.double().cpu().numpy() - ref[name]) / np.linalg.norm(ref[name])
        forward = name in ("o", "kv_out")
        print(name, error)
        assert error <= ((1e-5 if forward else 1.4e-5) if tensor else (7e-7 if forward else 1e-6)), (name, error)


@pytest.mark.parametrize("dtype,path", KINDS)
@pytest.mark.parametrize("d", [64, 128])
def test_gradient_along_itself_against_differences(d, dtype, path):
    """As above, but along the gradient, where the loss changes by as much as it can.  The fp64 oracle's own central differences at these
    steps are off by 7e-4 of the derivative at most (third order; dg), and the forward pass's error, 1e-5 of the outputs' size, divided by
    twice the step is 2e-4 of it: 2e-3 leaves twice that."""
    B, H, N = 1, 2, 150
    data = draw(B, H, H, N, d, 21, dtype, rates=[0.01, 0.2])
    kv_in, _ = states(B, H, d, 4)
    base = Call(data, kv_in=kv_in, path=path)
    base.fwd()
    base.bwd()
    base.done()
    for i, grad, step in ((3, "dg", 2.0 ** -7), (4, "dbeta", 0.25), (None, "grad_kv_in", 0.25)):
        along = base.results()[grad].double().cpu()
        way, loss = along / along.norm(), []
        for sign in (1, -1):
            moved = [(x.double() + sign * step * way).float() if j == i else x for j, x in enumerate(data)]
            call = Call(moved, kv_in=kv_in if i else (kv_in.double() + sign * step * way).float(), path=path)
            call.fwd()
            call.done()
            loss.append((call.o.double() * call.do.double()).sum().item())
        want = along.norm().item()
        assert abs((loss[0] - loss[1]) / (2 * step) - want) <= 2e-3 * want, grad
