"""The operators of a causal model over item histories that this library is timed on, apart from `perf/cases.py`:
the gated delta rule (training, whole histories, single tokens) and the embedding of item ids with its gradient.

A case is a dict of
    op               "delta" or "embed"
    direction        "forward", "train" (forward and backward) or, for "delta", "step" (one token per sequence against
                     the states that a server keeps, which the step replaces)
    via              how the program calls the library: "call" the binding's functions, "autograd" the differentiable
                     functions and `torch.autograd.grad`
    dtype            "f32", "bf16" or "f16": histories and tables; decays, betas and states are always f32
  delta:
    B, H, N, d       sizes
    layout           "bhnd" or "bnhd"
    lengths          "full" (no mask) or "uniform" (5 ... N valid tokens per sequence, from a quarter of N on for long
                     histories; padding on the left)
    states           an initial state comes in and the final one goes out (backward: their gradients the other way)
  embed:
    B, N, D, V       sequences, tokens of each, width, rows of the table (row 0 is the padding's)
    ids              "i64" or "i32"
    positions        a table of positions is added, and gets its gradient
Ids follow a power law, as the popularity of items does.
"""
import math

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELEM_BYTES = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-6
MOST_DELTA = 16 * 4 * 4096 * 64      # elements of a tensor of the largest listed training case
MOST_EMBED = 1024 * 200 * 256        # values gathered by the largest listed embedding


def _delta(name, B, H, N, d, dtype, direction, via="call", layout="bhnd", lengths="uniform", states=False):
    c = dict(op="delta", direction=direction, via=via, dtype=dtype, B=B, H=H, N=N, d=d, layout=layout,
             lengths=lengths, states=states)
    return c if name is None else dict(c, name=name)


def _embed(name, B, N, D, V, dtype, direction, via="call", ids="i64", positions=True):
    c = dict(op="embed", direction=direction, via=via, dtype=dtype, B=B, N=N, D=D, V=V, ids=ids, positions=positions)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # next-item serving, a handful of users: latency of one call
        _delta("step_b4_f32", 4, 2, 1, 32, "f32", "step", lengths="full", states=True),
        # the same for many users at a time: the states stream through
        _delta("step_b512_bf16", 512, 4, 1, 64, "bf16", "step", lengths="full", states=True),
        # short histories taken in whole, fp32
        _delta("forward_n50_f32", 256, 2, 50, 32, "f32", "forward"),
        # long histories taken in before serving starts: the state is what is wanted
        _delta("forward_long_bf16", 16, 4, 4096, 64, "bf16", "forward", states=True),
        # training, embedding 256 with four heads under mixed precision
        _delta("train_n200_bf16", 128, 4, 200, 64, "bf16", "train"),
        # training, embedding 64, fp32, inside a model
        _delta("train_n200_f32", 256, 2, 200, 32, "f32", "train", via="autograd", layout="bnhd"),
        # embedding 256 with two heads, fp16, odd length, histories continued from earlier states
        _delta("train_n197_f16", 64, 2, 197, 128, "f16", "train", layout="bnhd", states=True),
        # training on long histories
        _delta("train_long_bf16", 16, 4, 4096, 64, "bf16", "train"),
        # the newest item of a few users
        _embed("embed_b4_f32", 4, 1, 64, 3700, "f32", "forward"),
        # training with a large catalogue, fp32
        _embed("embed_v120k_f32", 128, 200, 256, 120000, "f32", "train"),
        # a large batch under mixed precision, inside a model
        _embed("embed_b1024_bf16", 1024, 200, 256, 16600, "bf16", "train", via="autograd"),
        # odd width, short histories, no positions
        _embed("embed_odd_f16", 77, 50, 99, 3700, "f16", "train", ids="i32", positions=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    dtype = rng.choice(["f32", "bf16", "bf16", "f16"])
    if rng.random() < 0.4:
        while True:
            B, N, V = _log_int(rng, 1, 1024), _log_int(rng, 1, 400), _log_int(rng, 50, 120000)
            D = rng.choice([32, 64, 128, 256, rng.randint(17, 300)])
            if B * N * D <= MOST_EMBED:
                break
        return _embed(None, B, N, D, V, dtype, rng.choice(["forward", "train", "train"]),
                      rng.choice(["call", "call", "autograd"]), rng.choice(["i64", "i64", "i32"]), rng.random() < 0.7)
    direction = rng.choice(["step", "forward", "forward", "train", "train", "train"])
    while True:
        d, H = rng.choice([16, 32, 64, 64, 128]), rng.choice([1, 2, 2, 3, 4, 8])
        B = _log_int(rng, 1, 1024)
        N = 1 if direction == "step" else _log_int(rng, 1, 4096)
        # (the states of all chunks of a plain backward have to fit as well)
        if B * H * N * d <= MOST_DELTA and B * H * N * d * d <= MOST_DELTA * 64:
            break
    if direction == "step":
        return _delta(None, B, H, 1, d, dtype, "step", "call", rng.choice(["bhnd", "bnhd"]), "full", True)
    via = rng.choice(["call", "call", "autograd"]) if direction == "train" else "call"
    return _delta(None, B, H, N, d, dtype, direction, via, rng.choice(["bhnd", "bnhd"]),
                  rng.choice(["uniform", "uniform", "full"]), rng.random() < 0.4)


def _length_range(N):
    return min(N, 5 if N <= 512 else N // 4), N


def work(case):
    """Each input read once and each output written once, over a forward and its backward together; the operations of the
    recurrences as they are defined."""
    e = ELEM_BYTES[case["dtype"]]
    if case["op"] == "embed":
        tokens, D, V = case["B"] * case["N"], case["D"], case["V"]
        rows = min(tokens, V)
        n_bytes = tokens * ((8 if case["ids"] == "i64" else 4) + D * e) + rows * D * e
        flops = 2 * tokens * D
        if case["positions"]:
            n_bytes += case["N"] * D * e
        if case["direction"] == "train":
            n_bytes += tokens * D * e + V * D * e + (case["N"] * D * e if case["positions"] else 0)
            flops += 2 * tokens * D
        return {"bytes": n_bytes, "flops": flops}
    B, H, N, d = case["B"], case["H"], case["N"], case["d"]
    lo, hi = _length_range(N)
    f = 1.0 if case["lengths"] == "full" else (lo + hi) / 2 / N
    rows, state = B * H * N, B * H * d * d * 4
    n_bytes = rows * ((2 + 2 * f) * d * e + 8 * f) + (2 * state if case["states"] else 0)
    if case["lengths"] != "full":
        n_bytes += B * N
    flops = rows * (2 + 4 * f) * d * d
    if case["direction"] == "train":
        n_bytes += rows * (4 * d * e + 8) + (2 * state if case["states"] else 0)
        flops += rows * (4 + 10 * f) * d * d
    return {"bytes": n_bytes, "flops": flops}


class _State:
    """What the program holds."""


def prepare(case, seed):
    device = torch.device("cuda", torch.cuda.current_device())
    gen = torch.Generator(device=device)
    gen.manual_seed(int(seed))
    dtype = DTYPES[case["dtype"]]
    s = _State()
    s.case = dict(case)
    train = case["direction"] == "train"

    def normal(*shape, scale=1.0, to=dtype):
        return (torch.randn(shape, generator=gen, device=device) * scale).to(to)

    def uniform(*shape):
        return torch.rand(shape, generator=gen, device=device, dtype=torch.float64)

    if case["op"] == "embed":
        B, N, D, V = case["B"], case["N"], case["D"], case["V"]
        ids = torch.exp(uniform(B, N) * math.log(V)).long().clamp(1, V - 1)
        lo, hi = _length_range(N)
        lengths = (lo + torch.floor(uniform(B) * (hi - lo + 1))).clamp(lo, hi).long()
        s.ids = torch.where(torch.arange(N, device=device)[None, :] >= (N - lengths)[:, None], ids, 0)
        s.ids = s.ids.to(torch.int64 if case["ids"] == "i64" else torch.int32)
        s.scale = math.sqrt(D)
        s.W = normal(V, D, scale=0.02)
        s.P = normal(N + 7, D, scale=0.02) if case["positions"] else None   # room for histories that grow
        s.dE = normal(B, N, D) if train else None
        if case["via"] == "autograd":
            s.W.requires_grad_(True)
            if s.P is not None:
                s.P.requires_grad_(True)
        return s
    B, H, N, d = case["B"], case["H"], case["N"], case["d"]
    lead = (B, H, N) if case["layout"] == "bhnd" else (B, N, H)
    s.q, s.k, s.v = (normal(*lead, d) for _ in range(3))
    # decays between a thousandth and one e-fold a token; betas as a sigmoid leaves them
    s.g = -torch.exp((uniform(*lead) - 1.0) * math.log(1000.0)).float()
    s.beta = torch.sigmoid(normal(*lead, scale=1.5, to=torch.float32))
    s.mask = None
    if case["lengths"] != "full":
        lo, hi = _length_range(N)
        lengths = (lo + torch.floor(uniform(B) * (hi - lo + 1))).clamp(lo, hi).long()
        s.mask = (torch.arange(N, device=device)[None, :] >= (N - lengths)[:, None]).to(torch.uint8)
    s.scale = 1.0 / math.sqrt(d) if case["direction"] != "step" else 1.0
    s.S0 = normal(B, H, d, d, scale=0.2, to=torch.float32) if case["states"] else None
    s.S1 = torch.empty(B, H, d, d, device=device) if case["states"] and case["direction"] != "step" else None
    s.dO = normal(*lead, d) if train else None
    s.dS1 = normal(B, H, d, d, scale=0.2, to=torch.float32) if train and case["states"] else None
    if case["via"] == "autograd":
        for t in (s.q, s.k, s.v, s.g, s.beta) + ((s.S0,) if s.S0 is not None else ()):
            t.requires_grad_(True)
    return s


# ---- the plain forms: elementary operations in 32 bits ----------------------------------------------------

def _embed_plain(s):
    c = s.case
    with torch.no_grad():
        W, ids = s.W.float(), s.ids.long()
        live = (ids != 0).unsqueeze(-1)
        E = torch.where(live, W[ids] * s.scale, 0.0)
        if s.P is not None:
            E = E + s.P[:c["N"]].float()
        out = {"E": E.to(s.W.dtype)}
        if c["direction"] == "train":
            dE = s.dE.float()
            dW = torch.zeros_like(W)
            dW.index_add_(0, ids.reshape(-1), torch.where(live, dE * s.scale, 0.0).reshape(-1, c["D"]))
            out["dW"] = dW.to(s.W.dtype)
            if s.P is not None:
                dP = torch.zeros(s.P.shape, device=dE.device)
                dP[:c["N"]] = dE.sum(0)
                out["dP"] = dP.to(s.P.dtype)
    return out


def _heads_first(t, layout):
    return t if layout == "bhnd" else t.transpose(1, 2)


def _delta_plain(s):
    """The recurrence token by token, and its adjoint token by token in reverse order."""
    c = s.case
    lay, B, H, N, d = c["layout"], c["B"], c["H"], c["N"], c["d"]
    with torch.no_grad():
        q, k, v = (_heads_first(t, lay).float() for t in (s.q, s.k, s.v))
        g, beta = (_heads_first(t, lay) for t in (s.g, s.beta))
        if s.mask is not None:
            live = (s.mask != 0)[:, None, :]
            k, v = (torch.where(live.unsqueeze(-1), t, 0.0) for t in (k, v))
            g, beta = (torch.where(live, t, 0.0) for t in (g, beta))
        rq = torch.rsqrt((q * q).sum(-1, keepdim=True) + EPS)
        rk = torch.rsqrt((k * k).sum(-1, keepdim=True) + EPS)
        q, k, a = q * rq, k * rk, torch.exp(g)
        S = torch.zeros(B, H, d, d, device=q.device) if s.S0 is None else s.S0
        if c["direction"] == "step":
            S.mul_(a[:, :, 0, None, None])
            u = beta[:, :, 0, None] * (v[:, :, 0] - (k[:, :, 0, :, None] * S).sum(-2))
            S.add_(k[:, :, 0, :, None] * u.unsqueeze(-2))
            O = (s.scale * (q[:, :, 0, :, None] * S).sum(-2)).unsqueeze(2)
            return {"O": _heads_first(O, lay).to(s.q.dtype), "S": S}
        train = c["direction"] == "train"
        O = torch.empty_like(q)
        before, delta = [], []
        for t in range(N):
            S = S * a[:, :, t, None, None]
            kt = k[:, :, t, :, None]
            e = v[:, :, t] - (kt * S).sum(-2)
            if train:
                before.append(S)
                delta.append(e)
            S = S + kt * (beta[:, :, t, None] * e).unsqueeze(-2)
            O[:, :, t] = (q[:, :, t, :, None] * S).sum(-2)
        out = {"O": _heads_first(O * s.scale, lay).to(s.q.dtype).contiguous()}
        if s.S0 is not None:
            out["S1"] = S
        if not train:
            return out
        dO = _heads_first(s.dO, lay).float() * s.scale
        dS = torch.zeros_like(S) if s.dS1 is None else s.dS1
        dq, dk, dv = torch.empty_like(q), torch.empty_like(q), torch.empty_like(q)
        dg, db = torch.empty_like(a), torch.empty_like(a)
        for t in range(N - 1, -1, -1):
            kt, do, e, bt = k[:, :, t, :, None], dO[:, :, t].unsqueeze(-2), delta[t], beta[:, :, t, None]
            u = (bt * e).unsqueeze(-2)
            dq[:, :, t] = ((before[t] + kt * u) * do).sum(-1)
            dS = dS + q[:, :, t, :, None] * do
            du = (kt * dS).sum(-2)
            db[:, :, t] = (du * e).sum(-1)
            de = (bt * du).unsqueeze(-2)
            dv[:, :, t] = de.squeeze(-2)
            dk[:, :, t] = (dS * u - before[t] * de).sum(-1)
            dS = dS - kt * de
            dg[:, :, t] = (dS * before[t]).sum((-1, -2))
            dS = dS * a[:, :, t, None, None]
        dq = (dq - q * (q * dq).sum(-1, keepdim=True)) * rq
        dk = (dk - k * (k * dk).sum(-1, keepdim=True)) * rk
        if s.mask is not None:
            dk, dv = (torch.where(live.unsqueeze(-1), t, 0.0) for t in (dk, dv))
            dg, db = (torch.where(live, t, 0.0) for t in (dg, db))
        out.update({n: _heads_first(t, lay).to(s.q.dtype).contiguous() for n, t in (("dQ", dq), ("dK", dk), ("dV", dv))})
        out.update({n: _heads_first(t, lay).contiguous() for n, t in (("dg", dg), ("dbeta", db))})
        if s.S0 is not None:
            out["dS0"] = dS
    return out


# ---- the library's calls ----------------------------------------------------------------------------------

def _embed_own(s):
    from paper_2602_06935_amd import autograd, binding
    c = s.case
    if c["via"] == "autograd":
        E = autograd.item_embedding(s.ids, s.W, s.P, scale=s.scale, padding_idx=0)
        out = {"E": E}
        if c["direction"] == "train":
            leaves = (s.W,) if s.P is None else (s.W, s.P)
            grads = torch.autograd.grad(E, leaves, s.dE)
            out.update(zip(("dW", "dP"), grads))
        return out
    out = {"E": binding.cotten_embed_fwd(s.ids, s.W, s.P, scale=s.scale, padding_idx=0)}
    if c["direction"] == "train":
        dP = None if s.P is None else torch.empty_like(s.P)
        out["dW"] = binding.cotten_embed_bwd(s.ids, s.dE, c["V"], dP=dP, scale=s.scale, padding_idx=0)
        if dP is not None:
            out["dP"] = dP
    return out


def _delta_own(s):
    from paper_2602_06935_amd import autograd, binding
    c = s.case
    if c["direction"] == "step":
        O = binding.cotten_delta_fwd(s.q, s.k, s.v, s.g, s.beta, None, scale=s.scale, eps=EPS, layout=c["layout"],
                                     initial_state=s.S0, final_state=s.S0)
        return {"O": O, "S": s.S0}
    if c["via"] == "autograd":
        leaves = [s.q, s.k, s.v, s.g, s.beta]
        got = autograd.gated_delta_attention(*leaves, s.mask, scale=s.scale, eps=EPS, layout=c["layout"],
                                             initial_state=s.S0, return_state=s.S0 is not None)
        if s.S0 is None:
            out, grads = {"O": got}, torch.autograd.grad(got, leaves, s.dO)
        else:
            out = {"O": got[0], "S1": got[1]}
            grads = torch.autograd.grad(got, leaves + [s.S0], (s.dO, s.dS1))
        out.update(zip(("dQ", "dK", "dV", "dg", "dbeta", "dS0"), grads))
        return out
    opts = dict(scale=s.scale, eps=EPS, layout=c["layout"], initial_state=s.S0)
    train = c["direction"] == "train"
    kept = binding.cotten_delta_kept(s.q, layout=c["layout"]) if train else None
    out = {"O": binding.cotten_delta_fwd(s.q, s.k, s.v, s.g, s.beta, s.mask, final_state=s.S1, kept=kept, **opts)}
    if s.S1 is not None:
        out["S1"] = s.S1
    if train:
        dS0 = None if s.S0 is None else torch.empty_like(s.S0)
        grads = binding.cotten_delta_bwd(s.q, s.k, s.v, s.g, s.beta, s.mask, s.dO, dfinal_state=s.dS1,
                                         dinitial_state=dS0, kept=kept, **opts)
        out.update(zip(("dQ", "dK", "dV", "dg", "dbeta"), grads))
        if dS0 is not None:
            out["dS0"] = dS0
    return out


def run(state):
    if state.case["op"] == "embed":
        return _embed_own(state) if own else _embed_plain(state)
    return _delta_own(state) if own else _delta_plain(state)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------

def _embed_exact(s):
    c = s.case
    B, N, D, V = c["B"], c["N"], c["D"], c["V"]
    W = s.W.detach().double()
    W[0] = 0.0
    at = s.ids.reshape(-1).long()
    E = (s.scale * torch.index_select(W, 0, at)).reshape(B, N, D)
    if s.P is not None:
        E = E + s.P.detach().double()[:N].expand(B, N, D)
    out = {"E": E}
    if c["direction"] == "train":
        # one 1 per token in a sparse V x tokens matrix, times the upstream rows
        one = torch.sparse_coo_tensor(torch.stack([at, torch.arange(B * N, device=at.device)]),
                                      torch.ones(B * N, dtype=torch.float64, device=at.device), (V, B * N))
        dW = torch.sparse.mm(one, s.dE.double().reshape(B * N, D)) * s.scale
        dW[0] = 0.0
        out["dW"] = dW
        if s.P is not None:
            out["dP"] = torch.cat([s.dE.double().sum(0), torch.zeros(s.P.shape[0] - N, D, device=at.device,
                                                                     dtype=torch.float64)])
    return out


def _delta_exact(s):
    """S_t = a_t (I - beta_t k_t k_t^T) S_{t-1} + beta_t k_t v_t^T by matrix products in 64 bits, gradients by
    differentiating that."""
    c = s.case
    B, H, N, d = c["B"], c["H"], c["N"], c["d"]

    def rows(t):
        t = t.detach().double()
        return t if c["layout"] == "bhnd" else t.movedim(1, 2)

    leaves = [rows(t).clone().requires_grad_(True) for t in (s.q, s.k, s.v)]
    gates = [rows(t).clone().requires_grad_(True) for t in (s.g, s.beta)]
    S0 = (torch.zeros(B, H, d, d, dtype=torch.float64, device=s.q.device) if s.S0 is None
          else s.S0.detach().double().clone())
    S0.requires_grad_(True)
    train = c["direction"] == "train"
    with torch.set_grad_enabled(train):
        q, k, v = leaves
        g, beta = gates
        qn = q / torch.sqrt(q.square().sum(-1, keepdim=True) + EPS)
        kn = k / torch.sqrt(k.square().sum(-1, keepdim=True) + EPS)
        if s.mask is not None:
            m = s.mask.double()[:, None, :]
            g, beta = g * m, beta * m
        alpha = g.exp()
        S, o = S0.reshape(B * H, d, d), []
        flat = [t.reshape(B * H, N, d).unbind(1) for t in (qn, kn, v)]
        al, be = (t.reshape(B * H, N, 1, 1).unbind(1) for t in (alpha, beta))
        for t in range(N):
            qt, kt, vt = (x[t].unsqueeze(1) for x in flat)
            S = al[t] * S
            S = torch.baddbmm(S, kt.transpose(1, 2) * be[t], vt - torch.bmm(kt, S))
            o.append(torch.bmm(qt, S))
        O = s.scale * torch.cat(o, 1).reshape(B, H, N, d)
    S = S.reshape(B, H, d, d)

    def back(t):
        return t if c["layout"] == "bhnd" else t.movedim(1, 2)

    if c["direction"] == "step":
        return {"O": back(O).detach(), "S": S.detach()}
    out = {"O": back(O).detach()}
    if c["states"]:
        out["S1"] = S.detach()
    if train:
        upstream = (rows(s.dO),) if s.dS1 is None else (rows(s.dO), s.dS1.double())
        outputs = (O,) if s.dS1 is None else (O, S)
        grads = torch.autograd.grad(outputs, leaves + gates + [S0], upstream)
        out.update({n: back(x) for n, x in zip(("dQ", "dK", "dV", "dg", "dbeta"), grads)})
        if c["states"]:
            out["dS0"] = grads[5]
    return out


def exact(case, seed):
    state = prepare(case, seed)
    return _embed_exact(state) if case["op"] == "embed" else _delta_exact(state)
