"""The learner's operators next to the actor step, as timed cases.

What a learner does with the episodes that ``Actor.ring_sample`` hands it, before it publishes a new model:

  logprob  ``marl_policy_logprob`` / ``_backward``: rows of action values -> log probability of the action taken, entropy,
           the best alternatives; ``train`` adds the gradient of the rows
  scan     ``marl_linear_scan`` / ``_backward``: the gated linear recurrence over a batch of episodes, forwards (a recurrent
           layer without the products of a GRU) or backwards in time (discounted returns); ``train`` adds the gradients
  ortho    ``marl_orthogonalise``: the update of a network's weight matrices, orthogonalised by Newton-Schulz products
"""
import math

import torch

own = False  # False: the operators in elementary torch operations; True: the framework's entry points

DTYPE = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
NS_COEFFS = (3.4445, -4.7750, 2.0315)
NS_EPS = 1e-7
DISCOUNT, LAMBDA = 0.99, 0.95


def listed():
    return [
        # one decision of a small worker (eight games of three agents), with its alternatives: latency
        dict(name="logprob_3m_step", op="logprob", B=8, L=1, n=3, A=9, dtype="fp32", mask=True, top=3, temperature=1.0, pad=0, train=False),
        # a learner's batch: sampled episodes of ragged length, unavailable actions, with the gradient
        dict(name="logprob_8m_train", op="logprob", B=1024, L=96, n=8, A=14, dtype="fp32", mask=True, top=4, temperature=0.7, pad=0, train=True),
        # a wide discrete action space of odd size: rows that start anywhere, many equal values
        dict(name="logprob_wide", op="logprob", B=2048, L=1, n=1, A=65537, dtype="bf16", mask=False, top=8, temperature=1.0, pad=0, train=False),
        # the same with unavailable actions, rows of a wider buffer and the gradient
        dict(name="logprob_wide_train", op="logprob", B=1000, L=1, n=1, A=32001, dtype="fp16", mask=True, top=1, temperature=1.3, pad=7, train=True),
        # one step of a recurrent layer for a small batch: the serving form
        dict(name="scan_step", op="scan", B=24, L=1, C=64, dtype="fp32", form="blend", reverse=False, done=True, ragged=False, train=False),
        # discounted returns of a batch of episodes: one channel, backwards in time, a constant gate
        dict(name="scan_returns", op="scan", B=1024, L=96, C=1, dtype="fp32", form="raw", reverse=True, done=True, ragged=True, train=False),
        # a recurrent layer over sampled episodes (8 agents of 64 units a game), with gradients
        dict(name="scan_8m_train", op="scan", B=64, L=256, C=512, dtype="bf16", form="blend", reverse=False, done=True, ragged=True, train=True),
        # one very long episode: few channels, all of the parallelism is along time
        dict(name="scan_long", op="scan", B=1, L=65521, C=128, dtype="fp32", form="raw", reverse=False, done=False, ragged=False, train=False),
        # the weight matrices of one network of hidden size 64
        dict(name="ortho_8m", op="ortho", K=1, H=64, D=80, n=8, A=14, dtype="fp32"),
        # a network per unit type, hidden size 128
        dict(name="ortho_typed_h128", op="ortho", K=4, H=128, D=80, n=5, A=11, dtype="fp32"),
        # a population of learners, updates kept in bf16
        dict(name="ortho_population", op="ortho", K=64, H=64, D=55, n=5, A=12, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["logprob", "logprob", "scan", "scan", "ortho"])
    if op == "logprob":
        c = dict(op=op, dtype=rng.choice(["fp32", "bf16", "fp16"]), mask=rng.random() < 0.7, top=rng.choice([0, 1, 2, 4, 8, 16]),
                 temperature=rng.choice([0.5, 1.0, 1.7]), pad=rng.choice([0, 0, 1, 8]), train=rng.random() < 0.5)
        if rng.random() < 0.5:   # sampled episodes
            B, L, n, A = _log(rng, 1, 1024), _log(rng, 1, 128), rng.randint(1, 10), rng.randint(1, 32)
        else:                    # wide rows
            A = _log(rng, 33, 131072)
            B, L, n = _log(rng, 1, max(1, min(8192, 2048 * 32768 // A))), 1, 1
        return dict(c, B=B, L=L, n=n, A=A)
    if op == "scan":
        C = _log(rng, 1, 1024)
        L = _log(rng, 1, 16384)
        return dict(op=op, B=_log(rng, 1, max(1, min(2048, 8000000 // (L * C)))), L=L, C=C, dtype=rng.choice(["fp32", "bf16", "fp16"]),
                    form=rng.choice(["raw", "blend"]), reverse=rng.random() < 0.4, done=rng.random() < 0.6, ragged=rng.random() < 0.6,
                    train=rng.random() < 0.5)
    return dict(op=op, K=_log(rng, 1, 24), H=rng.choice([64, 128]), D=_log(rng, 8, 256), n=rng.randint(2, 12), A=rng.randint(2, 32),
                dtype=rng.choice(["fp32", "bf16"]))


def _lengths(B, L, ragged, g):
    if not ragged:
        return None
    return torch.randint(1, L + 1, (B,), generator=g, device="cuda", dtype=torch.int32)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPE[case["dtype"]]
    rand = lambda *s: torch.rand(s, generator=g, device="cuda")  # noqa: E731
    randn = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    st = dict(case=dict(case))
    if case["op"] == "logprob":
        B, L, n, A = case["B"], case["L"], case["n"], case["A"]
        R = B * L * n
        # action values of a policy that has learned something: a spread of two, and a row of a wider buffer where `pad` says so
        buf = (2.0 * randn(R, A + case["pad"])).to(dt)
        st["logits"] = buf[:, :A]
        avail = None
        if case["mask"]:
            avail = (rand(R, A) < 0.7).to(torch.uint8)
            avail[:, 0] = 1                                    # action 0 is always there in a live step ...
            if L > 1:                                          # ... and nothing is behind an episode's end
                live = torch.arange(L, device="cuda")[None, :] < _lengths(B, L, True, g)[:, None]
                avail *= live[:, :, None].expand(B, L, n).reshape(R, 1).to(torch.uint8)
        st["avail"] = avail
        act = torch.randint(0, A, (R,), generator=g, device="cuda")
        if avail is not None:
            act = torch.where(avail.gather(1, act[:, None])[:, 0] > 0, act, torch.zeros_like(act))
        st["action"] = act.to(torch.int32)
        if case["train"]:
            st["g_logp"], st["g_entropy"] = randn(R), 0.01 * (1.0 + rand(R))
        return st
    if case["op"] == "scan":
        B, L, C = case["B"], case["L"], case["C"]
        returns = case["form"] == "raw" and C == 1
        if returns:        # discounted returns: the same decay everywhere, rewards and bootstrap values as input
            st["gate"] = torch.full((1, 1, 1), DISCOUNT * LAMBDA, device="cuda").to(dt).expand(B, L, 1)
            st["x"] = (randn(B, L, 1) + DISCOUNT * (1 - LAMBDA) * 5.0 * randn(B, L, 1)).to(dt)
        elif case["form"] == "raw":
            st["gate"] = (1.0 - 0.2 * rand(B, L, C)).to(dt)
            st["x"] = (0.3 * randn(B, L, C)).to(dt)
        else:              # gate and candidate come out of one projection and lie side by side
            both = randn(B, L, 2 * C)
            both[..., :C] = 1.5 * both[..., :C] + 1.0
            both = both.to(dt)
            st["gate"], st["x"] = both[..., :C], both[..., C:]
        st["h0"] = randn(B, C)
        st["done"] = (rand(B, L) < 0.05).to(torch.uint8) if case["done"] else None
        st["length"] = _lengths(B, L, case["ragged"], g)
        if case["train"]:
            st["dy"], st["dlast"] = randn(B, L, C).to(dt), randn(B, C)
        return st
    K, H, D, n, A = case["K"], case["H"], case["D"], case["n"], case["A"]
    st["mats"] = []
    for r, c in ((H, D + n + A), (3 * H, H), (3 * H, H), (A, H)):
        k = max(1, min(r, c) // 4)   # a momentum: a few strong directions over noise
        m = randn(K, r, k) @ randn(K, k, c) / math.sqrt(k) + 0.3 * randn(K, r, c)
        st["mats"].append((1e-3 * m).to(dt))
    return st


# ---- plain forms -----------------------------------------------------------------------------------------------------
def _plain_logprob(st):
    c = st["case"]
    x = st["logits"].float()
    R, A = x.shape
    live = x != -math.inf
    if st["avail"] is not None:
        live = live & (st["avail"] != 0)
    some = live.any(1)
    z = torch.where(live, x, torch.full_like(x, -math.inf))
    m = torch.where(some, z.max(1).values, torch.zeros_like(z[:, 0]))
    u = (z - m[:, None]) / c["temperature"]
    e = torch.exp(u)
    logs = torch.log(torch.where(some, e.sum(1), torch.ones_like(m)))
    lp = u - logs[:, None]
    p = torch.exp(lp)
    plp = torch.where(p > 0, p * lp, torch.zeros_like(p))
    entropy = -plp.sum(1)
    act = st["action"].long()
    logp = torch.where(some, lp.gather(1, act[:, None])[:, 0], torch.zeros_like(m))
    out = dict(logp=logp, entropy=entropy)
    k = c["top"]
    if k:
        kk = min(k, A)
        bits = (z + 0.0).view(torch.int32)                    # ordered like the values, lowest index first among equals
        bits = (bits ^ ((bits >> 31) & 0x7FFFFFFF)).long()
        key = (bits << 32) | (0xFFFFFFFF - torch.arange(A, device=x.device))
        idx = torch.topk(key, kk, dim=1).indices
        ok = live.gather(1, idx)
        out["top_index"] = torch.full((R, k), -1, dtype=torch.int32, device=x.device)
        out["top_logp"] = torch.full((R, k), -math.inf, device=x.device)
        out["top_index"][:, :kk] = torch.where(ok, idx, torch.full_like(idx, -1)).to(torch.int32)
        out["top_logp"][:, :kk] = torch.where(ok, lp.gather(1, idx), torch.full_like(m[:, None], -math.inf))
    if c["train"]:
        chosen = torch.arange(A, device=x.device)[None, :] == act[:, None]
        gl = st["g_logp"][:, None]
        lpz = torch.where(p > 0, lp, torch.zeros_like(p))
        d = (gl * (chosen.float() - p) - st["g_entropy"][:, None] * p * (lpz + entropy[:, None])) / c["temperature"]
        out["dlogits"] = torch.where(live & some[:, None], d, torch.zeros_like(d)).to(st["logits"].dtype)
    return out


def _doubling(a, b):
    """h[t] = a[t] h[t-1] + b[t] along dim 1 with h[-1] = 0, in log2(L) sweeps."""
    d, L = 1, a.shape[1]
    while d < L:
        b = torch.cat([b[:, :d], b[:, d:] + a[:, d:] * b[:, :-d]], 1)
        a = torch.cat([a[:, :d], a[:, d:] * a[:, :-d]], 1)
        d *= 2
    return b


def _masks(st):
    """live[b][t]: the step is inside the sequence; cut[b][t]: no state comes in from the step before (in scan order)."""
    c = st["case"]
    B, L = c["B"], c["L"]
    t = torch.arange(L, device="cuda")
    live = torch.ones(B, L, dtype=torch.bool, device="cuda") if st["length"] is None else t[None, :] < st["length"][:, None]
    done = torch.zeros(B, L, dtype=torch.bool, device="cuda") if st["done"] is None else st["done"] != 0
    if c["reverse"]:
        cut = done
    else:
        cut = torch.cat([torch.zeros_like(done[:, :1]), done[:, :-1]], 1)
    last = L - 1 if st["length"] is None else st["length"].long() - 1
    rows = torch.arange(B, device="cuda")
    gone = torch.zeros(B, dtype=torch.bool, device="cuda") if c["reverse"] else done[rows, last]   # nothing passes on behind the end
    return live, cut, gone, last, rows


def _plain_scan(st):
    c = st["case"]
    dt = st["x"].dtype
    live, cut, gone, last, rows = _masks(st)
    live, cut = live[:, :, None], cut[:, :, None]
    g, x = st["gate"].float(), st["x"].float()
    blend = c["form"] == "blend"
    z = torch.sigmoid(g) if blend else g
    a = torch.where(live & ~cut, z, torch.zeros_like(z))
    b = torch.where(live, torch.sigmoid(-g) * x if blend else x, torch.zeros_like(x))
    first = live.clone()                                # the step that h0 enters
    L = c["L"]
    if c["reverse"]:
        first[:, :-1] = live[:, :-1] & ~live[:, 1:]
    else:
        first[:, 1:] = False
    h0 = st["h0"][:, None, :]
    b0 = b + torch.where(first, a * h0, torch.zeros_like(b))
    aa = torch.where(first, torch.zeros_like(a), a)     # beyond the end (reverse) everything is zero
    if c["reverse"]:
        y = _doubling(aa.flip(1), b0.flip(1)).flip(1)
        out_last = y[:, 0]
    else:
        y = _doubling(aa, b0)
        out_last = torch.where(gone[:, None], torch.zeros_like(st["h0"]), y[rows, last])
        y = torch.where(live, y, torch.zeros_like(y))
    out = dict(y=y.to(dt), last=out_last)
    if c["train"]:
        G = torch.where(live, st["dy"].float(), torch.zeros_like(y))
        dl = torch.where(gone[:, None], torch.zeros_like(h0[:, 0]), st["dlast"])
        if c["reverse"]:
            G[:, 0] += dl
            nxt = torch.cat([torch.zeros_like(aa[:, :1]), aa[:, :-1]], 1)      # dh[t] += a[t-1] dh[t-1]
            G = _doubling(nxt, G)
            prev = torch.cat([y[:, 1:], torch.zeros_like(y[:, :1])], 1)
        else:
            G[rows, last] += dl
            nxt = torch.cat([aa[:, 1:], torch.zeros_like(aa[:, :1])], 1)       # dh[t] += a[t+1] dh[t+1]
            G = _doubling(nxt.flip(1), G.flip(1)).flip(1)
            prev = torch.cat([torch.zeros_like(y[:, :1]), y[:, :-1]], 1)
        G = torch.where(live, G, torch.zeros_like(G))
        prev = torch.where(first, h0.expand_as(prev), prev)
        prev = torch.where(cut, torch.zeros_like(prev), prev)
        dz = G * (prev - x) if blend else torch.where(cut, torch.zeros_like(G), G * prev)
        dg = dz * z * torch.sigmoid(-g) if blend else dz
        dx = G * torch.sigmoid(-g) if blend else G
        zero = torch.zeros_like(G)
        out["dgate"], out["dx"] = torch.where(live, dg, zero).to(dt), torch.where(live, dx, zero).to(dt)
        out["dh0"] = torch.where(first, a * G, zero).sum(1)
    return out


def _newton_schulz(X, steps=5):
    a, b, c = NS_COEFFS
    tall = X.shape[-2] > X.shape[-1]
    if tall:
        X = X.transpose(-1, -2)
    X = X / (X.square().sum((-1, -2), keepdim=True).sqrt() + NS_EPS)
    for _ in range(steps):
        S = X @ X.transpose(-1, -2)
        X = a * X + (b * S + c * (S @ S)) @ X
    return X.transpose(-1, -2) if tall else X


def run(state):
    c = state["case"]
    if not own:
        if c["op"] == "logprob":
            return _plain_logprob(state)
        if c["op"] == "scan":
            return _plain_scan(state)
        return [_newton_schulz(m.float()).to(m.dtype) for m in state["mats"]]
    from paper_2205_05248_b200 import binding
    if c["op"] == "logprob":
        r = binding.marl_policy_logprob(state["logits"], state["action"], avail=state["avail"], temperature=c["temperature"], top=c["top"])
        out = dict(logp=r["logp"], entropy=r["entropy"])
        if c["top"]:
            out["top_index"], out["top_logp"] = r["top_index"], r["top_logp"]
        if c["train"]:
            out["dlogits"] = binding.marl_policy_logprob_backward(
                state["logits"], state["action"], r["stats"], r["entropy"], g_logp=state["g_logp"], g_entropy=state["g_entropy"],
                avail=state["avail"], temperature=c["temperature"])
        return out
    if c["op"] == "scan":
        kw = dict(h0=state["h0"], done=state["done"], length=state["length"], form=c["form"], reverse=c["reverse"])
        r = binding.marl_linear_scan(state["gate"], state["x"], keep=c["train"], **kw)
        out = dict(y=r["y"], last=r["last"])
        if c["train"]:
            d = binding.marl_linear_scan_backward(state["gate"], state["x"], r["states"], state["dy"], dlast=state["dlast"], **kw)
            out["dgate"], out["dx"], out["dh0"] = d["dgate"], d["dx"], d["dh0"]
        return out
    return binding.marl_orthogonalise(state["mats"], steps=5, coeffs=NS_COEFFS, eps=NS_EPS)


def work(case):
    es = 4 if case["dtype"] == "fp32" else 2
    if case["op"] == "logprob":
        R, A = case["B"] * case["L"] * case["n"], case["A"]
        by = R * (A * (es + case["mask"]) + 4 + 8 + 8 * case["top"])
        fl = 6 * R * A
        if case["train"]:
            by += R * (A * es + 8)
            fl += 8 * R * A
        return {"bytes": by, "flops": fl}
    if case["op"] == "scan":
        B, L, C = case["B"], case["L"], case["C"]
        N = B * L * C
        returns = case["form"] == "raw" and C == 1            # the gate is one number
        flags = (B * L if case["done"] else 0) + (4 * B if case["ragged"] else 0)
        by = N * es * (2 if returns else 3) + 8 * B * C + flags
        fl = 2 * N if case["form"] == "raw" else 10 * N
        if case["train"]:
            by += 3 * N * es + 8 * B * C
            fl += 8 * N
        return {"bytes": by, "flops": fl}
    by = fl = 0
    for r, c in ((case["H"], case["D"] + case["n"] + case["A"]), (3 * case["H"], case["H"]), (3 * case["H"], case["H"]), (case["A"], case["H"])):
        m, n = min(r, c), max(r, c)
        by += 2 * es * r * c
        fl += 5 * (2 * m * m * n + 2 * m ** 3 + 2 * m * m * n)
    return {"bytes": case["K"] * by, "flops": case["K"] * fl}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------
def _exact_logprob(st):
    c = st["case"]
    R, A = st["logits"].shape
    per = max(1, (1 << 25) // A)
    parts = []
    for r0 in range(0, R, per):
        s = slice(r0, min(R, r0 + per))
        x = st["logits"][s].double() / c["temperature"]
        off = torch.isneginf(x)
        if st["avail"] is not None:
            off = off | (st["avail"][s] == 0)
        x = x.masked_fill(off, -math.inf)
        empty = off.all(1)
        lp = (x - torch.logsumexp(x, 1, keepdim=True)).masked_fill(off, -math.inf)
        p = lp.exp()
        H = -(p * lp.masked_fill(off, 0.0)).sum(1)
        a = st["action"][s].long()
        logp = lp.gather(1, a[:, None]).squeeze(1).masked_fill(empty, 0.0)
        row = [logp, H]
        if c["top"]:
            top = torch.full((x.shape[0], c["top"]), -math.inf, dtype=torch.float64, device=x.device)
            kk = min(A, c["top"])
            top[:, :kk] = torch.topk(lp, kk, 1).values
            row.append(top)
        if c["train"]:
            hot = torch.zeros_like(p).scatter_(1, a[:, None], 1.0)
            d = st["g_logp"][s].double()[:, None] * (hot - p) - st["g_entropy"][s].double()[:, None] * p * (lp.masked_fill(off, 0.0) + H[:, None])
            row.append((d / c["temperature"]).masked_fill(off, 0.0))
        parts.append(row)
    cols = [torch.cat(v) for v in zip(*parts)]
    out = dict(logp=cols[0], entropy=cols[1])
    if c["top"]:
        out["top_index"], out["top_logp"] = None, cols[2]
    if c["train"]:
        out["dlogits"] = cols[-1]
    return out


def _exact_scan(st):
    c = st["case"]
    B, L, C = c["B"], c["L"], c["C"]
    dev = st["x"].device
    n = torch.full((B,), L, device=dev) if st["length"] is None else st["length"].long()
    done = torch.zeros(B, L, dtype=torch.bool, device=dev) if st["done"] is None else st["done"].bool()
    blend = c["form"] == "blend"
    gate, x = st["gate"].double(), st["x"].double()
    order = range(L - 1, -1, -1) if c["reverse"] else range(L)
    h = st["h0"].double()
    y = torch.zeros(B, L, C, dtype=torch.float64, device=dev)
    came = torch.zeros_like(y) if c["train"] else None
    for t in order:
        inside = (t < n)[:, None]
        if c["reverse"]:
            h = h.masked_fill(done[:, t, None] & inside, 0.0)
        elif t:
            h = h.masked_fill(done[:, t - 1, None] & inside, 0.0)
        if came is not None:
            came[:, t] = h
        a = gate[:, t].sigmoid() if blend else gate[:, t]
        new = (1 - a) * x[:, t] + a * h if blend else a * h + x[:, t]
        h = torch.where(inside, new, h)
        y[:, t] = torch.where(inside, new, torch.zeros_like(new))
    end = torch.zeros(B, dtype=torch.bool, device=dev) if c["reverse"] else done[torch.arange(B, device=dev), n - 1]
    out = dict(y=y, last=h.masked_fill(end[:, None], 0.0))
    if c["train"]:
        dg, dx = torch.zeros_like(y), torch.zeros_like(y)
        G = st["dlast"].double().masked_fill(end[:, None], 0.0)       # gradient of the state that a step passes on
        for t in reversed(order):
            inside = (t < n)[:, None]
            a = gate[:, t].sigmoid() if blend else gate[:, t]
            G2 = G + st["dy"][:, t].double()
            if blend:
                dgt, dxt = G2 * (came[:, t] - x[:, t]) * a * (1 - a), G2 * (1 - a)
            else:
                dgt, dxt = G2 * came[:, t], G2
            back = a * G2
            cut = done[:, t] if c["reverse"] else (done[:, t - 1] if t else torch.zeros_like(done[:, 0]))
            back = back.masked_fill(cut[:, None], 0.0)
            dg[:, t], dx[:, t] = dgt * inside, dxt * inside
            G = torch.where(inside, back, G)
        out["dgate"], out["dx"], out["dh0"] = dg, dx, G
    return out


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "logprob":
        return _exact_logprob(st)
    if case["op"] == "scan":
        return _exact_scan(st)
    res = []
    for m in st["mats"]:
        X = m.double()
        if m.shape[1] > m.shape[2]:
            X = X.mT
        X = X / (torch.linalg.matrix_norm(X, keepdim=True) + NS_EPS)
        for _ in range(5):
            S = X @ X.mT
            X = NS_COEFFS[0] * X + NS_COEFFS[1] * (S @ X) + NS_COEFFS[2] * (S @ (S @ X))
        res.append(X.mT if m.shape[1] > m.shape[2] else X)
    return res
