"""The operators of a gated delta rule layer and of the block around it, as they are timed: calls of the library's entry points
(paper_2307_14995_b200.binding) beside plain forms in elementary torch operations.

  delta_train    la_delta_fwd then la_delta_bwd on the workspace the forward pass left: one layer's token mixer in a training step
  delta_prefill  la_delta_fwd with the state handed in and out: a prompt, or a chunk of one, before decoding
  delta_decode   la_delta_steps on a state that is updated in place: one token, or a few drafted ones
  norm           la_block_norm_fwd: what stands between two blocks, norm and gate of the one's output, residual scale and sum,
                 norm of the next one's input; where it trains la_block_norm_bwd too

The gated delta rule, per value head, with q and k of key head h // (H / Hk):

  S_t = exp(g_t) (S_{t-1} - beta_t k_t (k_t^T S_{t-1})) + beta_t k_t v_t^T,    o_t = scale S_t^T q_t

Between two blocks, per token:

  z = y / rms(y) (.) w_post (.) silu(u),    h = x + s (.) z,    n = h / rms(h) (.) w_pre,    rms(a)^2 = mean(a^2) + eps

Values are drawn as such a layer sees them: q, k = SiLU(N(0,1)) of unit length, v, do ~ N(0,1), beta = sigmoid(N(0,1)),
g = -a softplus(N(0,1) + dt) with one rate a and one step dt per head.  Everything is made on the GPU from the seed.
"""
import torch

own = False

_DTYPE = {"bf16": torch.bfloat16, "fp32": torch.float32}
_BYTES = {"bf16": 2, "fp32": 4}


def _delta(kind, B, H, N, d, **more):
    c = {"kind": kind, "B": B, "H": H, "Hk": H, "N": N, "d": d, "inp": "bf16", "out": "bf16", "layout": "tokens"}
    c.update(more)
    return c


def _norm(rows, D, **more):
    c = {"kind": "norm", "rows": rows, "D": D, "inp": "bf16", "res": "bf16", "gate": True, "backward": True}
    c.update(more)
    return c


def listed():
    cases = [
        # the fp32 reference configuration: the smallest training call
        ("delta_train_fp32_ref", _delta("delta_train", 1, 2, 256, 64, inp="fp32", out="fp32", layout="heads")),
        # one training step of a layer of the 385M-like and of the 1B-like configuration
        ("delta_train_385m", _delta("delta_train", 4, 16, 2048, 64, out="fp32", layout="heads")),
        ("delta_train_1b", _delta("delta_train", 2, 16, 8192, 128)),
        # two value heads to a key head, a length of no round size
        ("delta_train_ragged", _delta("delta_train", 3, 8, 3001, 128, Hk=4)),
        # serving: a short prompt continuing an earlier state, and one of the long-context 7B-like configuration
        ("delta_prefill_short", _delta("delta_prefill", 1, 32, 777, 128)),
        ("delta_prefill_long", _delta("delta_prefill", 1, 32, 65536, 128)),
        # serving: a single conversation, a full batch
        ("delta_decode_single", _delta("delta_decode", 1, 32, 1, 128)),
        ("delta_decode_batch64", _delta("delta_decode", 64, 32, 1, 128, Hk=16)),
        # one token of the 7B-like configuration while decoding
        ("norm_token", _norm(1, 4096, backward=False)),
        # a training step of the 1B-like configuration with the residual stream in fp32, and one of no round size without a gate
        ("norm_train_1b", _norm(16384, 2048, res="fp32")),
        ("norm_train_odd", _norm(3001, 1003, gate=False)),
        # the 7B-like configuration over its long context
        ("norm_train_7b_long", _norm(65536, 4096)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log_int(rng, low, high):
    return int(round(low * (high / low) ** rng.random()))


def draw(rng):
    kind = rng.choice(("delta_train", "delta_train", "delta_prefill", "delta_decode", "norm", "norm"))
    if kind == "norm":
        D = _log_int(rng, 64, 8192)
        if rng.random() < 0.6:  # models have such widths
            D = max(64, D // 64 * 64)
        inp = rng.choice(("bf16", "bf16", "fp32"))
        return _norm(_log_int(rng, 1, max(1, min(65536, (1 << 27) // D))), D, inp=inp, res="fp32" if inp == "fp32" else rng.choice(("bf16", "fp32")),
                     gate=rng.random() < 0.7, backward=rng.random() < 0.7)
    d = rng.choice((64, 128, 128))
    H = rng.choice((4, 8, 16, 32))
    form = {"Hk": H // rng.choice((1, 1, 2, 4)), "out": rng.choice(("fp32", "bf16", "bf16")), "layout": rng.choice(("heads", "tokens"))}
    if kind == "delta_decode":
        return _delta(kind, _log_int(rng, 1, 64), H, rng.choice((1, 1, 1, 2, 3, 4, 8)), d, **form)
    if kind == "delta_prefill":
        return _delta(kind, rng.choice((1, 1, 2)), H, _log_int(rng, 16, 16384), d, **form)
    if rng.random() < 0.25:  # full precision: checks and small models
        form.update(inp="fp32", out="fp32")
        return _delta(kind, rng.choice((1, 2)), H, _log_int(rng, 16, 1024), d, **form)
    B = rng.choice((1, 1, 2, 3))
    return _delta(kind, B, H, _log_int(rng, 100, min(8192, 262144 // (B * H))), d, **form)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(dev)
    gen.manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=gen, device=dev)

    def empty(dtype, *shape):
        return torch.empty(shape, dtype=dtype, device=dev)

    s = {"case": case}
    inp = _DTYPE[case["inp"]]
    if case["kind"] == "norm":
        rows, D, res = case["rows"], case["D"], _DTYPE[case["res"]]
        s["x"], s["y"] = (4 * normal(rows, D)).to(res), normal(rows, D).to(inp)
        s["u"] = normal(rows, D).to(inp) if case["gate"] else None
        s["w_post"], s["w_pre"] = 1 + 0.1 * normal(D), 1 + 0.1 * normal(D)
        s["s"] = 0.5 + 0.1 * normal(D)
        if case["backward"]:
            s["dh"], s["dn"] = normal(rows, D).to(res), normal(rows, D).to(inp)
        if own:  # the outputs' buffers and the workspace, which a program keeps from step to step
            from paper_2307_14995_b200 import binding as la
            s["shape"] = la.make_block_norm_shape(rows, D, inp, res, eps=1e-6, gate=la.LA_GATE_SILU)
            s["h"], s["n"] = empty(res, rows, D), empty(inp, rows, D)
            if case["backward"]:
                s["dx"], s["dy"], s["du"] = empty(res, rows, D), empty(inp, rows, D), empty(inp, rows, D) if case["gate"] else None
                s["dw_post"], s["ds"], s["dw_pre"] = (empty(torch.float32, D) for _ in range(3))
                s["ws"] = la.alloc_block_norm_workspace(s["shape"], dev)
        return s
    B, H, Hk, N, d = (case[x] for x in ("B", "H", "Hk", "N", "d"))
    out, tokens = _DTYPE[case["out"]], case["layout"] == "tokens"

    def size(heads, *more):
        return (B, N, heads, *more) if tokens else (B, heads, N, *more)

    def unit(*shape):
        x = torch.nn.functional.silu(normal(*shape))
        return (x / x.square().sum(-1, keepdim=True).sqrt()).to(inp)

    def per_head(x):
        return x.view(H) if tokens else x.view(H, 1)

    s["q"], s["k"], s["v"] = unit(*size(Hk, d)), unit(*size(Hk, d)), normal(*size(H, d)).to(inp)
    s["beta"] = torch.sigmoid(normal(*size(H)))
    # rates of 1 to 16 and steps of 0.001 to 0.1, as such layers are initialised
    rate = 1 + 15 * torch.rand(H, generator=gen, device=dev)
    step = 0.001 * 100 ** torch.rand(H, generator=gen, device=dev)
    s["g"] = -per_head(rate) * torch.nn.functional.softplus(0.5 * normal(*size(H)) + per_head(step.expm1().log()))
    if case["kind"] != "delta_train":
        s["kv"] = normal(B, H, d, d)  # what an earlier prompt left
    else:
        s["do"] = normal(*size(H, d)).to(inp)
    if own:  # the outputs' buffers and the workspaces, which a program keeps from step to step
        from paper_2307_14995_b200 import binding as la
        shape = s["shape"] = la.make_delta_shape(B, H, N, d, d, inp, out, Hk=Hk, scale=d ** -0.5,
                                                 layout=la.LA_LAYOUT_BNHD if tokens else la.LA_LAYOUT_BHND)
        s["o"] = empty(out, *size(H, d))
        if case["kind"] != "delta_decode":
            s["ws_f"] = la.alloc_delta_workspace(la.LA_OP_FWD, shape, dev)
            s["kv_out"] = empty(torch.float32, B, H, d, d)
        if case["kind"] == "delta_train":
            s["ws_b"] = la.alloc_delta_workspace(la.LA_OP_BWD, shape, dev)
            s["dq"], s["dk"], s["dv"] = empty(out, *size(Hk, d)), empty(out, *size(Hk, d)), empty(out, *size(H, d))
            s["dg"], s["dbeta"] = empty(torch.float32, *size(H)), empty(torch.float32, *size(H))
    return s


def run(s):
    c = s["case"]
    if not own:
        return _plain_norm(s) if c["kind"] == "norm" else _plain_delta(s)
    from paper_2307_14995_b200 import binding as la
    shape = s["shape"]
    if c["kind"] == "norm":
        la.la_block_norm_fwd(shape, s["x"], s["y"], s["u"], s["w_post"], s["s"], s["w_pre"], s["h"], s["n"])
        if not c["backward"]:
            return s["h"], s["n"]
        la.la_block_norm_bwd(shape, s["x"], s["y"], s["u"], s["w_post"], s["s"], s["w_pre"], s["dh"], s["dn"], s["dx"], s["dy"], s["du"],
                             s["dw_post"], s["ds"], s["dw_pre"], s["ws"])
        return s["h"], s["n"], s["dx"], s["dy"], s["du"], s["dw_post"], s["ds"], s["dw_pre"]
    data = (s["q"], s["k"], s["v"], s["g"], s["beta"])
    if c["kind"] == "delta_decode":
        la.la_delta_steps(shape, *data, s["kv"], s["o"])
        return s["o"], s["kv"]
    if c["kind"] == "delta_prefill":
        la.la_delta_fwd(shape, *data, s["o"], s["kv"], s["kv_out"], s["ws_f"])
        return s["o"], s["kv_out"]
    la.la_delta_fwd(shape, *data, s["o"], workspace=s["ws_f"])
    la.la_delta_bwd(shape, *data, s["do"], s["dq"], s["dk"], s["dv"], s["dg"], s["dbeta"], workspace=s["ws_b"], fwd_workspace=s["ws_f"])
    return s["o"], s["dq"], s["dk"], s["dv"], s["dg"], s["dbeta"]


def work(case):
    """Every input read once and every output written once; flops of the token recurrence where that is what a call runs, else of
    chunks of 64 tokens (half of each score tile): k k^T, q k^T, the inverse times k and v, three products with the state
    forward; backward twice that, as for any product."""
    i = _BYTES[case["inp"]]
    if case["kind"] == "norm":
        n, r = case["rows"] * case["D"], _BYTES[case["res"]]
        t = n * (2 * r + i * (3 if case["gate"] else 2)) + 12 * case["D"]
        if case["backward"]:
            t += n * (3 * r + i * (5 if case["gate"] else 3)) + 24 * case["D"]
        return {"bytes": t, "flops": n * (45 if case["backward"] else 15)}
    B, H, Hk, N, d = (case[x] for x in ("B", "H", "Hk", "N", "d"))
    o, rows, state = _BYTES[case["out"]], B * N * H, B * H * d * d * 4
    qk = 2 * B * N * Hk * d
    fwd = {"bytes": qk * i + rows * d * (i + o) + 8 * rows, "flops": rows * (5 * 64 * d + 6 * d * d)}
    if case["kind"] == "delta_decode":
        return {"bytes": fwd["bytes"] + 2 * state, "flops": rows * 7 * d * d}
    if case["kind"] == "delta_prefill":
        return {"bytes": fwd["bytes"] + 2 * state, "flops": fwd["flops"]}
    return {"bytes": fwd["bytes"] + qk * o + rows * d * (i + o) + 8 * rows, "flops": 3 * fwd["flops"]}


# ---- plain forms, in 32 bits -------------------------------------------------------------------------------------------------

def _plain_norm(s):
    c = s["case"]
    inp, res = _DTYPE[c["inp"]], _DTYPE[c["res"]]

    def rms_norm(a, w):
        return a * (a.square().mean(-1, keepdim=True) + 1e-6).rsqrt() * w

    names = ["x", "y"] + (["u"] if c["gate"] else []) + ["w_post", "s", "w_pre"]
    a = {n: s[n].float().detach().requires_grad_(c["backward"]) for n in names}
    z = rms_norm(a["y"], a["w_post"])
    if c["gate"]:
        z = z * a["u"] / (1 + (-a["u"]).exp())
    h = a["x"] + a["s"] * z
    n = rms_norm(h, a["w_pre"])
    if not c["backward"]:
        return h.to(res), n.to(inp)
    grads = dict(zip(names, torch.autograd.grad((h, n), [a[k] for k in names], (s["dh"].float(), s["dn"].float()))))
    return (h.detach().to(res), n.detach().to(inp), grads["x"].to(res), grads["y"].to(inp), grads["u"].to(inp) if c["gate"] else None,
            grads["w_post"], grads["s"], grads["w_pre"])


_C = 64  # tokens of a chunk of the plain form


def _inverse(a):
    """(I + a)^-1 for strictly lower triangular a [..., 64, 64]: blocks of 1, 2, .. 32 merged in pairs, which keeps to the size of
    the result where powers of a would not."""
    x, n = torch.ones_like(a[..., :1, :1]).expand(*a.shape[:-1], 1).unsqueeze(-1), 1
    while n < _C:
        pairs = torch.stack(a.unflatten(-2, (-1, 2 * n)).unflatten(-1, (-1, 2 * n)).unbind(-2), -3).diagonal(dim1=-4, dim2=-3).movedim(-1, -3)
        first, second = x[..., 0::2, :, :], x[..., 1::2, :, :]
        low = -second @ pairs[..., n:, :n] @ first
        x = torch.cat((torch.cat((first, torch.zeros_like(first)), -1), torch.cat((low, second), -1)), -2)
        n *= 2
    return x.squeeze(-3)


def _chunks(q, k, v, g, beta, kv, scale):
    """Heads first, q and k already one per value head: o and the state after the last token."""
    N, d = q.shape[2:]
    pad = -N % _C
    if pad:  # tokens that write nothing and forget nothing
        q, k, v = (torch.nn.functional.pad(x, (0, 0, 0, pad)) for x in (q, k, v))
        g, beta = (torch.nn.functional.pad(x, (0, pad)) for x in (g, beta))
    q, k, v = (x.unflatten(2, (-1, _C)) for x in (q * scale, k, v))
    g, beta = g.unflatten(2, (-1, _C)), beta.unflatten(2, (-1, _C))
    total = g.double().cumsum(-1)  # differences of long sums
    rows = torch.arange(_C, device=q.device)
    lower = rows.view(-1, 1) >= rows
    decay = torch.where(lower, total.unsqueeze(-1) - total.unsqueeze(-2), -torch.inf).float().exp()
    since, until = total.float().exp().unsqueeze(-1), (total[..., -1:] - total).float().exp().unsqueeze(-1)
    t = _inverse((beta.unsqueeze(-1) * (k @ k.mT) * decay).tril(-1))
    w, u = t @ (beta.unsqueeze(-1) * since * k), t @ (beta.unsqueeze(-1) * v)
    scores, late, last = (q @ k.mT) * decay, (k * until).mT, total[..., -1].float().exp()
    q, o = q * since, []
    for i in range(q.shape[2]):  # a recurrence: each chunk starts from the state that the one before it left
        new = u[:, :, i] - w[:, :, i] @ kv
        o.append(q[:, :, i] @ kv + scores[:, :, i] @ new)
        kv = last[:, :, i, None, None] * kv + late[:, :, i] @ new
    return torch.cat(o, 2)[:, :, :N], kv


def _plain_delta(s):
    c = s["case"]
    H, Hk, d, tokens, train = c["H"], c["Hk"], c["d"], c["layout"] == "tokens", c["kind"] == "delta_train"
    out = _DTYPE[c["out"]]
    leaves = [s[n].float().detach().requires_grad_(train) for n in ("q", "k", "v", "g", "beta")]
    q, k, v, g, beta = (x.transpose(1, 2) if tokens else x for x in leaves)
    q, k = (x.repeat_interleave(H // Hk, 1) for x in (q, k))
    kv = s["kv"] if not train else torch.zeros(c["B"], H, d, d, device=q.device)
    if c["kind"] == "delta_decode":
        o = []
        for t in range(c["N"]):  # token by token, as the definition has it
            kv = g[:, :, t, None, None].exp() * kv
            kv = kv + k[:, :, t, :, None] * (beta[:, :, t, None] * (v[:, :, t] - (k[:, :, t, :, None] * kv).sum(-2)))[:, :, None, :]
            o.append((q[:, :, t, :, None] * kv).sum(-2) * d ** -0.5)
        s["kv"].copy_(kv)
        o = torch.stack(o, 2)
        return (o.transpose(1, 2) if tokens else o).to(out), s["kv"]
    o, kv = _chunks(q, k, v, g, beta, kv, d ** -0.5)
    o = o.transpose(1, 2) if tokens else o
    if not train:
        return o.to(out).contiguous(), kv
    grads = torch.autograd.grad(o, leaves, s["do"].float())
    return (o.detach().to(out).contiguous(),) + tuple(x.to(out) for x in grads[:3]) + tuple(grads[3:])


# ---- definitions, in 64 bits ---------------------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return _exact_norm(s) if case["kind"] == "norm" else _exact_delta(s)


def _exact_norm(s):
    c = s["case"]
    parts = []
    for at in range(0, c["rows"], 8192):  # (64-bit copies of a few thousand rows at a time)
        x, y = (s[n][at:at + 8192].double() for n in ("x", "y"))
        w_post, res, w_pre = (s[n].double() for n in ("w_post", "s", "w_pre"))
        ry = 1 / torch.sqrt((y * y).mean(-1, keepdim=True) + 1e-6)
        if c["gate"]:
            u = s["u"][at:at + 8192].double()
            sig = torch.sigmoid(u)
            a, da = u * sig, sig + u * sig * (1 - sig)
        else:
            a = torch.ones_like(y)
        yn = y * ry
        z = yn * w_post * a
        h = x + res * z
        rh = 1 / torch.sqrt((h * h).mean(-1, keepdim=True) + 1e-6)
        hn = h * rh
        if not c["backward"]:
            parts.append((h, hn * w_pre))
            continue
        dh, dn = (s[n][at:at + 8192].double() for n in ("dh", "dn"))
        dhn = dn * w_pre
        dx = dh + rh * (dhn - hn * (dhn * hn).mean(-1, keepdim=True))
        dyn = dx * res * a * w_post
        dy = ry * (dyn - yn * (dyn * yn).mean(-1, keepdim=True))
        du = dx * res * yn * w_post * da if c["gate"] else None
        parts.append((h, hn * w_pre, dx, dy, du, (dx * res * a * yn).sum(0), (dx * z).sum(0), (dn * hn).sum(0)))
    rows, sums = (5, 8) if c["backward"] else (2, 2)
    cat = [None if parts[0][i] is None else torch.cat([p[i] for p in parts]) for i in range(rows)]
    return tuple(cat + [sum(p[i] for p in parts) for i in range(rows, sums)])


def _exact_delta(s):
    """The recurrence token by token, and its adjoint: with E the gradient of the state after token t, r = v_t - S^T k_t on the decayed
    state S, n = beta_t r,  E += scale q do^T;  dk = E n;  dn = E^T k;  dv = beta dn;  dbeta = dn . r;  dk -= S dv;  E -= k dv^T;
    dg = <S, E>;  E *= exp(g)."""
    c = s["case"]
    B, H, Hk, N, d, tokens = c["B"], c["H"], c["Hk"], c["N"], c["d"], c["layout"] == "tokens"
    train, G, scale = c["kind"] == "delta_train", H // Hk, d ** -0.5

    def steps(x, heads):  # one [B * H, ...] slice for each token
        x = (x if tokens else x.transpose(1, 2)).double()
        x = x.repeat_interleave(G, 2) if heads == Hk and G > 1 else x
        return x.transpose(0, 1).reshape(N, B * H, *x.shape[3:])

    q, k, v = steps(s["q"], Hk) * scale, steps(s["k"], Hk), steps(s["v"], H)
    g, beta = steps(s["g"], -1).exp().unsqueeze(-1), steps(s["beta"], -1).unsqueeze(-1)
    S = s["kv"].double().reshape(B * H, d, d) if not train else torch.zeros(B * H, d, d, dtype=torch.float64, device=q.device)

    def forth(S, t):  # the decayed state, v - S^T k, the state after the token
        S = S * g[t].unsqueeze(-1)
        r = v[t] - torch.bmm(k[t].unsqueeze(1), S).squeeze(1)
        return S, r, torch.baddbmm(S, k[t].unsqueeze(2), (beta[t] * r).unsqueeze(1))

    o, kept = torch.empty_like(v), []
    for t in range(N):
        if train and t % 64 == 0:
            kept.append(S)
        S = forth(S, t)[2]
        torch.bmm(q[t].unsqueeze(1), S, out=o[t].unsqueeze(1))

    def back(x, heads=H):
        x = x.view(N, B, heads, *x.shape[2:]).transpose(0, 1)
        return x if tokens else x.transpose(1, 2)

    if not train:
        return back(o), S.view(B, H, d, d)
    do = steps(s["do"], H)
    dq, dk, dv, dg, dbeta = (torch.empty_like(x) for x in (q, k, v, g.squeeze(-1), beta.squeeze(-1)))
    E = torch.zeros_like(S)
    for t0 in range((N - 1) // 64 * 64, -1, -64):
        S, past = kept.pop(), []
        for t in range(t0, min(N, t0 + 64)):
            before, r, S = forth(S, t)
            past.append((before, r, S))
        for t in range(min(N, t0 + 64) - 1, t0 - 1, -1):
            before, r, S = past[t - t0]
            dq[t] = torch.bmm(S, do[t].unsqueeze(2)).squeeze(2) * scale
            E = torch.baddbmm(E, q[t].unsqueeze(2), do[t].unsqueeze(1))
            dn = torch.bmm(k[t].unsqueeze(1), E).squeeze(1)
            dv[t] = beta[t] * dn
            dbeta[t] = (dn * r).sum(-1)
            dk[t] = torch.bmm(E, (beta[t] * r).unsqueeze(2)).squeeze(2) - torch.bmm(before, dv[t].unsqueeze(2)).squeeze(2)
            E = torch.baddbmm(E, k[t].unsqueeze(2), dv[t].unsqueeze(1), alpha=-1)
            dg[t] = (before * E).sum((1, 2))
            E = E * g[t].unsqueeze(-1)
    dq, dk = (x.view(N, B * Hk, G, d).sum(2) for x in (dq, dk))
    return back(o), back(dq, Hk), back(dk, Hk), back(dv), back(dg), back(dbeta)
