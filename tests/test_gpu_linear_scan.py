"""marl_linear_scan and its gradient against the recurrence in 64 bits, step by step.

Tolerances.  u = 2^-24.  A step's gate enters at most four products of maps (steps of a thread, lanes, warps, chunks) and its input at
most four sums; a blend's gate pair comes from ex2.approx (2^-22) and an approximate quotient (2 ulp), below 6 u.  So a step adds at
most 16 u (|a h| + |b|) to an error that it otherwise multiplies by |a|: the bound below runs that recurrence beside the
states.  The gradient's state R has the same bound from its own recurrence; a gradient is a product of G, h and z terms, each with
its relative error (G and h from the bounds), then the rounding to its type: half a step."""
import pytest
import torch

from paper_2205_05248_b200 import binding

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
U = 2.0 ** -24


def _make(B, L, C, dt, form, seed, done=True, ragged=True, fused=False):
    g = torch.Generator().manual_seed(seed)
    gate = torch.randn(B, L, C, generator=g) * 2 if form == "blend" else 1 - 0.3 * torch.rand(B, L, C, generator=g)
    x = torch.randn(B, L, C, generator=g)
    if fused:
        both = torch.cat([gate, x], 2).to(DT[dt]).cuda()
        gate, x = both[..., :C], both[..., C:]
    else:
        gate, x = gate.to(DT[dt]).cuda(), x.to(DT[dt]).cuda()
    kw = dict(h0=torch.randn(B, C, generator=g).cuda(), done=None, length=None)
    if done:
        kw["done"] = (torch.rand(B, L, generator=g) < 0.08).to(torch.uint8).cuda()
        if L:
            kw["done"][0, L - 1] = 255
    if ragged:
        n = torch.randint(0, L + 1, (B,), generator=g)
        n[0] = L
        if B > 1:
            n[1] = 0
        if B > 2:
            n[2] = min(1, L)
        kw["length"] = n.to(torch.int32).cuda()
    dy, dlast = torch.randn(B, L, C, generator=g).to(DT[dt]).cuda(), torch.randn(B, C, generator=g).cuda()
    return gate, x, kw, dy, dlast


def _want(gate, x, kw, form, reverse, dy=None, dlast=None):
    B, L, C = x.shape
    dev = x.device
    n = torch.full((B,), L, device=dev) if kw["length"] is None else kw["length"].long()
    done = torch.zeros(B, L, dtype=torch.bool, device=dev) if kw["done"] is None else kw["done"] != 0
    g, xd = gate.double(), x.double()
    z = torch.sigmoid(g) if form == "blend" else g
    rest = torch.sigmoid(-g) if form == "blend" else torch.ones_like(g)
    h = torch.zeros(B, C, dtype=torch.float64, device=dev) if kw["h0"] is None else kw["h0"].double()
    E = torch.zeros_like(h)
    y, Ey, came, Ecame = (torch.zeros(B, L, C, dtype=torch.float64, device=dev) for _ in range(4))
    cuts = done if reverse else torch.nn.functional.pad(done, (1, 0))[:, :L]
    order = list(range(L - 1, -1, -1)) if reverse else list(range(L))
    for t in order:
        live = (t < n)[:, None]
        cut = cuts[:, t, None] & live
        hin, Ein = h.masked_fill(cut, 0.0), E.masked_fill(cut, 0.0)
        came[:, t], Ecame[:, t] = hin, Ein
        a, b = z[:, t], rest[:, t] * xd[:, t]
        hn = a * hin + b
        En = a.abs() * Ein + 16 * U * ((a * hin).abs() + b.abs()) + 1e-40
        h, E = torch.where(live, hn, h), torch.where(live, En, E)
        y[:, t], Ey[:, t] = torch.where(live, hn, torch.zeros_like(hn)), torch.where(live, En, torch.zeros_like(En))
    gone = torch.zeros(B, dtype=torch.bool, device=dev)
    if not reverse and L:
        gone = (n > 0) & done[torch.arange(B, device=dev), (n - 1).clamp(min=0)]
    out = dict(y=(y, Ey), last=(h.masked_fill(gone[:, None], 0.0), E.masked_fill(gone[:, None], 0.0)))
    if dy is None:
        return out
    R = dlast.double().masked_fill(gone[:, None], 0.0)
    ER = torch.zeros_like(R)
    dg, Eg, dx, Ex = (torch.zeros_like(y) for _ in range(4))
    for t in reversed(order):
        live = (t < n)[:, None]
        cut = cuts[:, t, None] & live
        G, a = R + dy[:, t].double(), z[:, t]
        EG = ER + 2 * U * (R.abs() + dy[:, t].double().abs())
        if form == "blend":
            diff, zr = came[:, t] - xd[:, t], z[:, t] * rest[:, t]
            v = G * diff * zr
            e = (EG * diff.abs() + G.abs() * (Ecame[:, t] + U * (came[:, t].abs() + xd[:, t].abs()))) * zr + 24 * U * v.abs()
            w, ew = G * rest[:, t], EG * rest[:, t] + 16 * U * (G * rest[:, t]).abs()
        else:
            v = G * came[:, t]
            e = EG * came[:, t].abs() + G.abs() * Ecame[:, t] + 4 * U * v.abs()
            w, ew = G, EG
        zero = torch.zeros_like(v)
        dg[:, t], Eg[:, t] = torch.where(live, v, zero), torch.where(live, e, zero)
        dx[:, t], Ex[:, t] = torch.where(live, w, zero), torch.where(live, ew, zero)
        Rn = (a * G).masked_fill(cut, 0.0)
        En = (a.abs() * EG + 16 * U * (a.abs() * (R.abs() + dy[:, t].double().abs()))).masked_fill(cut, 0.0)
        R, ER = torch.where(live, Rn, R), torch.where(live, En, ER)
    out.update(dgate=(dg, Eg), dx=(dx, Ex), dh0=(R, ER))
    return out


def _close(got, want, what):
    v, e = want
    tol = e * 1.01 + torch.finfo(got.dtype).eps / 2 * (v.abs() + e) + (2.0 ** -25 if got.dtype == torch.float16 else 1e-44)
    err = (got.double() - v).abs()
    assert bool((err <= tol).all()), (what, float((err - tol).max()), float(err.max()))


def _check(gate, x, kw, dy, dlast, form, reverse, grads=True):
    r = binding.marl_linear_scan(gate, x, form=form, reverse=reverse, keep=grads, **kw)
    w = _want(gate, x, kw, form, reverse, dy if grads else None, dlast)
    if grads:
        r.update(binding.marl_linear_scan_backward(gate, x, r["states"], dy, dlast=dlast, form=form, reverse=reverse, **kw))
    for k in w:
        _close(r[k], w[k], k)
    return r


SHAPES = [(1, 1, 1), (3, 1, 64), (2, 2, 3), (5, 7, 1), (4, 8, 32), (3, 9, 33), (4, 63, 2), (3, 64, 66), (2, 65, 31), (4, 96, 1), (2, 129, 128),
          (3, 200, 5), (2, 300, 17), (4, 513, 1), (2, 700, 10)]


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,L,C", SHAPES)
def test_scan_and_gradient(B, L, C, dt):
    for form in ("raw", "blend"):
        for reverse in (False, True):
            for done, ragged, fused in ((True, True, False), (False, False, True)):
                gate, x, kw, dy, dlast = _make(B, L, C, dt, form, B + L + C, done, ragged, fused)
                _check(gate, x, kw, dy, dlast, form, reverse)


@pytest.mark.parametrize("B,L,C,dt,form", [(1, 4100, 32, "fp32", "raw"), (2, 5003, 6, "bf16", "blend"), (1, 9001, 1, "fp32", "blend"),
                                           (3, 2500, 70, "fp16", "raw"), (1, 3333, 64, "bf16", "raw"),
                                           (1, 5001, 200, "fp32", "blend"), (2, 3100, 72, "fp16", "blend")])
def test_time_divided_over_blocks(B, L, C, dt, form):
    for reverse in (False, True):
        gate, x, kw, dy, dlast = _make(B, L, C, dt, form, L, done=reverse, ragged=B > 1)
        s = binding._scan_args(gate, x, None, None, None, form, reverse)
        assert binding._scan_work(s, x.device)[1] > 0
        _check(gate, x, kw, dy, dlast, form, reverse)
    gate, x, kw, dy, dlast = _make(B, L, C, dt, form, L + 1, done=True, ragged=False)
    kw["done"][:, 100:L - 100] = 0     # cuts at the ends only: maps without one over many blocks
    _check(gate, x, kw, dy, dlast, form, False)


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,L,C", [(3, 32, 48), (4, 64, 64), (3, 65, 72), (5, 127, 128), (4, 300, 200), (2, 1000, 64), (300, 40, 64)])
def test_rows_on_16_byte_boundaries(B, L, C, dt):
    """Tiles by asynchronous copies: whole and partial tiles and groups of channels, either direction, cuts and ends."""
    for form in ("raw", "blend"):
        for reverse in (False, True):
            for done, ragged, fused in ((True, True, False), (False, True, True), (True, False, True)):
                gate, x, kw, dy, dlast = _make(B, L, C, dt, form, B + L + C, done, ragged, fused)
                _check(gate, x, kw, dy, dlast, form, reverse)


@pytest.mark.parametrize("form", ["raw", "blend"])
@pytest.mark.parametrize("C", [1, 6, 64])
def test_two_windows_are_one_run(form, C):
    """[0, s) and then [s, L) with the state that was passed on; a cut on the border included."""
    gate, x, kw, _, _ = _make(3, 150, C, "fp32", form, 9, True, False)
    kw["done"][1, 69] = 1
    one = binding.marl_linear_scan(gate, x, form=form, **kw)
    for s in (1, 64, 70, 149):
        a = binding.marl_linear_scan(gate[:, :s].contiguous(), x[:, :s], h0=kw["h0"], done=kw["done"][:, :s].contiguous(), form=form)
        b = binding.marl_linear_scan(gate[:, s:], x[:, s:], h0=a["last"], done=kw["done"][:, s:].contiguous(), form=form)
        y = torch.cat([a["y"], b["y"]], 1)
        assert float((y - one["y"]).abs().max()) < 1e-5 and float((b["last"] - one["last"]).abs().max()) < 1e-5


def test_step_by_step_is_the_scan():
    """The serving form: one step a call, the state carried by the caller."""
    gate, x, kw, _, _ = _make(24, 20, 64, "fp32", "blend", 1, True, False)
    whole = binding.marl_linear_scan(gate, x, **kw)
    h = kw["h0"]
    for t in range(20):
        r = binding.marl_linear_scan(gate[:, t:t + 1], x[:, t:t + 1], h0=h, done=kw["done"][:, t:t + 1].contiguous())
        assert float((r["y"][:, 0] - whole["y"][:, t]).abs().max()) < 1e-5
        h = r["last"]


@pytest.mark.parametrize("reverse", [False, True])
@pytest.mark.parametrize("B,L,C", [(2, 90, 64), (2, 90, 1), (1, 5000, 2)])
def test_nothing_crosses_a_cut_an_end_or_a_channel(reverse, B, L, C):
    """NaN and infinities behind the end of a sequence are not read; those in front of a cut (in scan order) stay there."""
    gate, x, kw, dy, dlast = _make(B, L, C, "fp32", "raw", 4, False, False)
    n = L - 10
    kw["length"] = torch.full((B,), n, dtype=torch.int32, device="cuda")
    kw["done"] = torch.zeros(B, L, dtype=torch.uint8, device="cuda")
    kw["done"][:, 40] = 1
    clean = _check(gate, x, kw, dy, dlast, "raw", reverse)
    x2, g2, d2 = x.clone(), gate.clone(), dy.clone()
    for t in (x2, g2, d2):
        t[:, n:] = float("nan")
    bad = 60 if reverse else 30
    x2[:, bad, 0] = float("inf")
    g2[0, bad, 0] = float("nan")
    r = binding.marl_linear_scan(g2, x2, form="raw", reverse=reverse, keep=True, **kw)
    r.update(binding.marl_linear_scan_backward(g2, x2, r["states"], d2, dlast=dlast, form="raw", reverse=reverse, **kw))
    side = slice(0, 41) if reverse else slice(41, n)      # behind the cut, in scan order
    for k in ("y", "dgate", "dx"):
        assert torch.equal(r[k][:, side], clean[k][:, side]), k
        assert torch.equal(r[k][:, :, 1:], clean[k][:, :, 1:]), k
        assert bool((r[k][:, n:] == 0).all()), k
    assert not bool(torch.isfinite(r["y"][:, bad, 0]).any())


def test_large_gates_before_anything_arrives():
    """Gates above 1 over a stretch of zero state: the state stays 0 (a thread's few steps are the longest product that meets it)."""
    x = torch.zeros(2, 64, 32, device="cuda")
    x[:, 60] = 1.0
    gate = torch.full((2, 64, 32), 30.0, device="cuda")
    r = binding.marl_linear_scan(gate, x, form="raw")
    assert bool((r["y"][:, :60] == 0).all()) and bool((r["y"][:, 63] == 27000.0).all())


def test_expanded_gates_and_odd_starts():
    """One decay for everything, one for each row, one for all channels; 16-bit rows that start off 4-byte boundaries."""
    B, L, C = 3, 140, 6
    for dt in ("fp32", "bf16"):
        _, x, kw, dy, dlast = _make(B, L, C, dt, "raw", 2)
        for gate in (torch.full((1, 1, 1), 0.9), 0.5 + 0.5 * torch.rand(B, 1, 1), 0.5 + 0.5 * torch.rand(B, L, 1), torch.rand(1, L, C)):
            _check(gate.to(DT[dt]).cuda().expand(B, L, C), x, kw, dy, dlast, "raw", True)
        for off in (1, 2, 3):
            buf = torch.empty(B * L * (C + 3) + 8, dtype=DT[dt], device="cuda")
            v = buf[off:off + B * L * (C + 3)].view(B, L, C + 3)[..., :C]
            v.copy_(x)
            _check(torch.full((1, 1, 1), 0.9, dtype=DT[dt], device="cuda").expand(B, L, C), v, kw, dy, dlast, "raw", False)
        t = x.transpose(0, 1).contiguous().transpose(0, 1)       # time-major storage
        _check(t.abs().clamp(max=1), t, kw, dy.transpose(0, 1).contiguous().transpose(0, 1), dlast, "raw", False)


def test_gradient_against_differences():
    gate, x, kw, dy, dlast = _make(2, 70, 3, "fp32", "blend", 5)
    for reverse in (False, True):
        r = binding.marl_linear_scan(gate, x, reverse=reverse, keep=True, **kw)
        d = binding.marl_linear_scan_backward(gate, x, r["states"], dy, dlast=dlast, reverse=reverse, **kw)

        def f(g, xx, h0):
            w = _want(g, xx, dict(kw, h0=h0), "blend", reverse)
            return float((w["y"][0] * dy.double()).sum() + (w["last"][0] * dlast.double()).sum())

        g0, x0, h0, e = gate.double(), x.double(), kw["h0"].double(), 1e-5
        for k in range(12):
            b, t, c = k % 2, (k * 13) % 70, k % 3
            for name, base in (("dgate", 0), ("dx", 1)):
                v = [g0.clone(), x0.clone()]
                v[base][b, t, c] += e
                up = f(v[0], v[1], h0)
                v[base][b, t, c] -= 2 * e
                assert abs((up - f(v[0], v[1], h0)) / (2 * e) - float(d[name][b, t, c])) < 1e-4, (name, b, t, c)
        for b in range(2):
            h1 = h0.clone()
            h1[b, 1] += e
            up = f(g0, x0, h1)
            h1[b, 1] -= 2 * e
            assert abs((up - f(g0, x0, h1)) / (2 * e) - float(d["dh0"][b, 1])) < 1e-4


def test_lengths_outside_the_batch_and_missing_arrays():
    gate, x, kw, dy, dlast = _make(3, 33, 8, "fp32", "blend", 6, False, False)
    wild = dict(kw, length=torch.tensor([-5, 40, 33], dtype=torch.int32, device="cuda"))
    tame = dict(kw, length=torch.tensor([0, 33, 33], dtype=torch.int32, device="cuda"))
    a, b = (binding.marl_linear_scan(gate, x, **k) for k in (wild, tame))
    assert torch.equal(a["y"], b["y"]) and torch.equal(a["last"], b["last"])
    _check(gate, x, dict(h0=None, done=None, length=None), dy, dlast, "blend", False)
    r = binding.marl_linear_scan(gate, x, keep=True)
    d0 = binding.marl_linear_scan_backward(gate, x, r["states"], dy)
    d1 = binding.marl_linear_scan_backward(gate, x, r["states"], dy, dlast=torch.zeros_like(dlast))
    assert all(torch.equal(d0[k], d1[k]) for k in d0)
    e = binding.marl_linear_scan(gate[:, :0], x[:, :0], h0=kw["h0"], keep=True)
    assert torch.equal(e["last"], kw["h0"])
    d = binding.marl_linear_scan_backward(gate[:, :0], x[:, :0], e["states"], dy[:, :0], dlast=dlast)
    assert torch.equal(d["dh0"], dlast)
    assert binding.marl_linear_scan(gate[:0], x[:0])["y"].shape == (0, 33, 8)


def test_captured_and_replayed_beside_another_graph():
    """Two captured calls with scratch of their own, replayed on two streams at once."""
    runs = []
    for k in range(2):
        gate, x, kw, dy, dlast = _make(1, 6000, 8, "fp32", "raw", 20 + k, False, False)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            r = binding.marl_linear_scan(gate, x, form="raw", keep=True, **kw)
            r.update(binding.marl_linear_scan_backward(gate, x, r["states"], dy, dlast=dlast, form="raw", **kw))
        runs.append((g, torch.cuda.Stream(), r, (gate, x, kw, dy, dlast)))
    torch.cuda.synchronize()
    for _ in range(5):
        for g, s, _, _ in runs:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for _, _, r, (gate, x, kw, dy, dlast) in runs:
        w = binding.marl_linear_scan(gate, x, form="raw", keep=True, **kw)
        w.update(binding.marl_linear_scan_backward(gate, x, w["states"], dy, dlast=dlast, form="raw", **kw))
        for k in ("y", "last", "dgate", "dx", "dh0"):
            assert torch.equal(r[k], w[k]), k


def test_offsets_beyond_32_bits():
    B, L, C = 3, 11000, 70000                   # 2.3e9 elements
    x = torch.zeros(B, L, C, dtype=torch.bfloat16, device="cuda")
    x[B - 1, L - 2, C - 1] = 2.0
    gate = torch.full((1, 1, 1), 0.5, dtype=torch.bfloat16, device="cuda").expand(B, L, C)
    r = binding.marl_linear_scan(gate, x, form="raw")
    assert float(r["y"][B - 1, L - 1, C - 1]) == 1.0 and float(r["y"][B - 1, L - 2, C - 1]) == 2.0
    assert float(r["last"].abs().sum()) == 1.0 and float(r["last"][B - 1, C - 1]) == 1.0


def test_refusals():
    gate, x, kw, dy, dlast = _make(2, 5, 4, "fp32", "blend", 0)
    f, e = binding.marl_linear_scan, binding.MarlError
    for bad in (dict(h0=kw["h0"].double()), dict(h0=kw["h0"][:1]), dict(done=kw["done"].float()), dict(done=kw["done"][:, :4]),
                dict(length=kw["length"].long()), dict(length=kw["length"].cpu()), dict(form="gru")):
        with pytest.raises(e):
            f(gate, x, **{**kw, **bad})
    for a in ((gate.half(), x), (gate[:, :4], x), (gate.double(), x.double()), (gate[0], x[0]), (gate, x.transpose(1, 2).contiguous().transpose(1, 2))):
        with pytest.raises(e):
            f(*a, **kw)
    r = f(gate, x, keep=True, **kw)
    g = binding.marl_linear_scan_backward
    for a in ((r["states"][:, :0], dy), (r["states"], dy.half()), (r["states"], dy[:, :4])):
        with pytest.raises(e):
            g(gate, x, *a, **kw)


def test_gradient_arrays_on_other_boundaries_than_the_inputs():
    """The states that the forward pass kept serve every form of the gradient: dy that starts off a 16-byte boundary, and strided dy."""
    for dt, B, L, C in (("fp32", 3, 150, 64), ("bf16", 2, 200, 72)):
        gate, x, kw, dy, dlast = _make(B, L, C, dt, "blend", 3)
        r = binding.marl_linear_scan(gate, x, keep=True, **kw)
        want = binding.marl_linear_scan_backward(gate, x, r["states"], dy, dlast=dlast, **kw)
        for off, pad in ((1, 0), (8, 3), (0, 8)):
            buf = torch.empty(B * L * (C + pad) + 16, dtype=DT[dt], device="cuda")
            v = buf[off:off + B * L * (C + pad)].view(B, L, C + pad)[..., :C]
            v.copy_(dy)
            got = binding.marl_linear_scan_backward(gate, x, r["states"], v, dlast=dlast, **kw)
            w = _want(gate, x, kw, "blend", False, dy, dlast)
            for k in ("dgate", "dx", "dh0"):
                _close(got[k], w[k], k)
                assert float((got[k].float() - want[k].float()).abs().max()) < 0.1


@pytest.mark.parametrize("B,L,C", [(3, 1, 200), (2, 40, 3), (2, 64, 64), (1, 1000, 64)])
def test_gates_far_from_zero(B, L, C):
    """z = 1 / (1 + e^-g) and 1 - z where one of them is small, up to where e^-g leaves the normal numbers.

    u = 2^-24.  g log2 e is rounded once and its constant is off by 0.23 u, so e^-g is off by 1.23 |g| u relative, and ex2.approx by 4 u.
    With e = e^-g: d ln z = -e / (1 + e) d ln e and d ln (1 - z) = 1 / (1 + e) d ln e, to which the sum adds u and the quotient 2 u
    (1 ulp), and 1 - z one product more.  So both are within (1.23 |g| + 8) u relative, and a result that multiplies them once more by
    an input, or each other, within that sum and 2 u a product.  2^v below 2^-126 is flushed, and 1 - z is e z: both are off by up to 2^-126 there."""
    n = B * L * C
    g = torch.linspace(-100.0, 100.0, n).view(B, L, C)[:, torch.randperm(L, generator=torch.Generator().manual_seed(1))].contiguous().cuda()
    x = (1.0 + torch.rand(B, L, C, generator=torch.Generator().manual_seed(2))).cuda()
    cut = torch.ones(B, L, dtype=torch.uint8, device="cuda")                 # every step by itself: y = (1 - z) x
    z, rest = torch.sigmoid(g.double()), torch.sigmoid(-g.double())
    e = (1.23 * g.double().abs() + 8) * U

    def close(got, want, rel, what):
        err = (got.double() - want).abs()
        tol = rel * want.abs() + 2.0 ** -125
        assert bool((err <= tol).all()), (what, float((err / tol).max()))

    for reverse in (False, True):
        r = binding.marl_linear_scan(g, x, done=cut, form="blend", reverse=reverse, keep=True)
        close(r["y"], rest * x.double(), e + 2 * U, "y")
        dy = torch.ones_like(x)
        d = binding.marl_linear_scan_backward(g, x, r["states"], dy, done=cut, form="blend", reverse=reverse)
        close(d["dx"], rest, e + 2 * U, "dx")
        close(d["dgate"], -x.double() * z * rest, 2 * e + 6 * U, "dgate")
    if L == 1:
        h0 = torch.ones(B, C, device="cuda")
        close(binding.marl_linear_scan(g, torch.zeros_like(x), h0=h0, form="blend")["last"], z[:, 0], e[:, 0] + 2 * U, "z")
