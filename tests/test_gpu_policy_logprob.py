"""marl_policy_logprob and its gradient against their definition in 64 bits.

Tolerances.  With U = (largest - smallest live value) / temperature, an exponent's error is below 3 U 2^-24 (difference, product,
constant), ex2.approx is within 2^-22, and a lane adds up to A/32 terms one after the other, the rest in a tree: the relative
error of S is below 2^-23 (A/64 + 2 U + 16), which is the absolute error of log S; (x_a - m) / T adds 2 U 2^-24 and each stored number half a step.
Entropy is log S - V / S: V's terms carry another factor u <= U, so (1 + U) times that.  A gradient p (g + h (log p + H)) has p's
relative error and h p times the errors of log p and H, then the rounding to its type, half a step relative (and half the
smallest subnormal of fp16, 2^-25).  Probabilities below 2^-126 are flushed to 0."""
import math

import pytest
import torch

from paper_2205_05248_b200 import binding

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def _make(R, A, dt, seed, mask=True, pad=0, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    buf = (spread * torch.randn(R, A + pad, generator=g)).to(DT[dt]).cuda()
    x = buf[:, :A]
    av = None
    if mask:
        av = (torch.rand(R, A, generator=g) < 0.6).to(torch.uint8)
        av[R // 2] = 0                                     # an empty row
        if A > 2:
            av[0] = 0
            av[0, A - 1] = 7                               # one entry, any non-zero byte
        av = av.cuda()
    act = torch.randint(-1, A + 1, (R,), generator=g).to(torch.int32).cuda()   # none in front, none behind
    return x, av, act


def _want(x, av, act, T, top):
    z = x.double() / T
    on = ~torch.isneginf(z)
    if av is not None:
        on &= av != 0
    z = z.masked_fill(~on, -math.inf)
    empty = ~on.any(1)
    m = z.max(1, keepdim=True).values.masked_fill(empty[:, None], 0.0)
    S = (z - m).exp().sum(1, keepdim=True)
    lp = (z - m - S.log()).masked_fill(~on, -math.inf)
    p = lp.exp()
    H = -(p * lp.masked_fill(~on, 0.0)).sum(1)
    has = (act >= 0) & (act < x.shape[1])
    a = act.long().clamp(0, x.shape[1] - 1)
    logp = lp.gather(1, a[:, None])[:, 0].masked_fill(empty | ~has, 0.0)
    order = torch.argsort(z, dim=1, descending=True, stable=True)[:, :top]
    ti = torch.where(on.gather(1, order), order, torch.full_like(order, -1))
    tl = lp.gather(1, order)
    if top > x.shape[1]:
        fill = top - x.shape[1]
        ti = torch.nn.functional.pad(ti, (0, fill), value=-1)
        tl = torch.nn.functional.pad(tl, (0, fill), value=-math.inf)
    U = (m[:, 0] - torch.where(on, z, m.expand_as(z)).min(1).values)
    return dict(logp=logp, H=H, ti=ti, tl=tl, p=p, lp=lp, on=on, has=has, a=a, empty=empty, U=U)


def _close(got, want, tol, what):
    inf = torch.isinf(want)
    assert torch.equal(got.double()[inf], want[inf]), what
    err = (got.double() - want)[~inf].abs()
    lim = tol.expand_as(want)[~inf]
    assert bool((err <= lim).all()), (what, float((err - lim).max()))


def _check(x, av, act, T=1.0, top=0, grads=True, gl=None, ge=None, out=None):
    r = binding.marl_policy_logprob(x, act, avail=av, temperature=T, top=top)
    w = _want(x, av, act, T, top)
    A = x.shape[1]
    e = 2.0 ** -23 * (A / 64 + 2 * w["U"] + 16)
    half = 2.0 ** -24
    _close(r["logp"], w["logp"], e + 2 * w["U"] * half + half * w["logp"].abs().nan_to_num(posinf=0), "logp")
    _close(r["entropy"], w["H"], (1 + w["U"]) * e + half * w["H"], "entropy")
    if top:
        assert torch.equal(r["top_index"].long(), w["ti"]), "top_index"
        _close(r["top_logp"], w["tl"], (e + 3 * w["U"] * half)[:, None], "top_logp")
    assert torch.equal(torch.isneginf(r["stats"][:, 1]), w["empty"])
    if not grads:
        return r, w
    g = torch.Generator().manual_seed(A)
    R = x.shape[0]
    gl = torch.randn(R, generator=g).cuda() if gl is None else gl
    ge = torch.randn(R, generator=g).cuda() if ge is None else ge
    d = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=gl, g_entropy=ge, avail=av, temperature=T, out=out)
    gd, hd = gl.double()[:, None], ge.double()[:, None]
    hot = torch.zeros_like(w["p"]).scatter_(1, w["a"][:, None], 1.0) * w["has"][:, None]
    lp0 = w["lp"].masked_fill(~w["on"], 0.0)
    want = (gd * w["has"][:, None] * (hot - w["p"]) - hd * w["p"] * (lp0 + w["H"][:, None])) / T
    want = want.masked_fill(~w["on"], 0.0)
    rel = (2 * e + 4 * w["U"] * half + 2.0 ** -21)[:, None]
    mag = (gd.abs() * (hot + w["p"]) + hd.abs() * w["p"] * (lp0.abs() + w["H"][:, None] + 2 + w["U"][:, None])) / T
    tol = rel * mag + torch.finfo(x.dtype).eps / 2 * want.abs() + (2.0 ** -25 if x.dtype == torch.float16 else 1e-44)
    # ex2 flushes: a probability below 2^-126 counts as 0, which takes up to 2^-126 (|g| + |h| |log p + H|) / T from its gradient
    tol = tol + 2.0 ** -126 * (gd.abs() + hd.abs() * (lp0.abs() + w["H"][:, None])) / T
    _close(d, want, tol, "dlogits")
    assert bool((d[~w["on"]] == 0).all())
    return r, w


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("R,A", [(1, 1), (3, 2), (24, 9), (129, 14), (128, 16), (300, 17), (127, 31), (257, 32)])
@pytest.mark.parametrize("mask", [True, False])
def test_small_rows(R, A, dt, mask):
    x, av, act = _make(R, A, dt, R + A, mask, pad=A % 3)
    _check(x, av, act, T=0.7, top=min(A + 2, 32))


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("R,A,top", [(1, 33, 1), (9, 40, 32), (8, 255, 5), (17, 256, 0), (5, 1000, 31), (3, 2048, 8), (4, 2049, 8),
                                     (3, 4099, 32), (7, 20001, 1), (2, 65537, 16)])
@pytest.mark.parametrize("mask,pad", [(True, 0), (False, 3), (True, 8)])
def test_wide_rows(R, A, top, dt, mask, pad):
    x, av, act = _make(R, A, dt, R + A + pad, mask, pad)
    _check(x, av, act, T=1.3, top=top)


@pytest.mark.parametrize("A", [9, 33, 700, 9001])
def test_every_start_of_a_row(A):
    """Rows and availability rows that start at every offset from a 16-byte boundary."""
    for dt in ("fp32", "bf16"):
        for off in range(0, 9):
            x, av, act = _make(3, A, dt, off, True, pad=0)
            bx = torch.empty(3 * A + 32, dtype=x.dtype, device="cuda")
            ba = torch.empty(3 * A + 32, dtype=torch.uint8, device="cuda")
            xo, ao = bx[off:off + 3 * A].view(3, A), ba[off:off + 3 * A].view(3, A)
            xo.copy_(x)
            ao.copy_(av)
            _check(xo, ao, act, top=4)


@pytest.mark.parametrize("order", ["ascending", "descending", "equal", "few"])
@pytest.mark.parametrize("A", [20, 500, 10007])
@pytest.mark.parametrize("dt", ["fp32", "bf16"])
def test_alternatives_of_ordered_and_equal_values(order, A, dt):
    v = torch.arange(A, dtype=torch.float32)
    v = {"ascending": v / A, "descending": -v / A, "equal": torch.full((A,), -0.0), "few": (v * 7 % 5).floor()}[order]
    x = torch.stack([v, v.roll(3), v.flip(0)]).to(DT[dt]).cuda()
    if order == "equal":
        x[:, ::2] = 0.0                                     # +0 and -0 are equal
    _check(x, None, torch.tensor([0, A - 1, A // 2], dtype=torch.int32, device="cuda"), top=min(32, A))


@pytest.mark.parametrize("A", [6, 32, 100, 3001])
def test_lowest_values_and_infinities(A):
    """Masks written into the values: the type's lowest number everywhere is a uniform row; -infinity is unavailable; an infinite or
    NaN value of an unavailable entry has no effect."""
    low = torch.finfo(torch.float32).min
    g = torch.Generator().manual_seed(A)
    x = torch.randn(6, A, generator=g)
    av = torch.ones(6, A, dtype=torch.uint8)
    x[0] = low
    x[1, 1:] = low
    x[2] = -math.inf
    x[3, ::2] = -math.inf
    av[4, 1::2] = 0
    x[4, 1::2] = math.nan
    av[5, 1:3] = 0
    x[5, 1], x[5, 2] = math.inf, -math.inf
    act = torch.tensor([0, 0, 0, 1, 2, 3], dtype=torch.int32)
    x, av, act = x.cuda(), av.cuda(), act.cuda()
    for T in (1.0, 0.25, 3.0):
        r = binding.marl_policy_logprob(x, act, avail=av, temperature=T, top=3)
        assert abs(float(r["logp"][0]) + math.log(A)) < 1e-4 and abs(float(r["entropy"][0]) - math.log(A)) < 1e-4
        assert float(r["logp"][1]) == 0.0 and float(r["entropy"][1]) == 0.0
        assert float(r["logp"][2]) == 0.0 and float(r["entropy"][2]) == 0.0 and bool((r["top_index"][2] == -1).all())
        assert r["top_index"][0].tolist() == [0, 1, 2]
        _check(x[3:].clone(), av[3:].clone(), act[3:].clone(), T=T, top=3)
        d = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=torch.ones(6, device="cuda"),
                                                 g_entropy=torch.ones(6, device="cuda"), avail=av, temperature=T)
        assert bool(torch.isfinite(d).all()) and bool((d[2] == 0).all())
        assert abs(float(d[0, 0]) - (1 - 1 / A) / T) < 1e-5 and abs(float(d[0, 1]) + 1 / A / T) < 1e-5


@pytest.mark.parametrize("A", [7, 64, 5000])
def test_not_a_number_and_infinity_stay_in_their_row(A):
    x, av, act = _make(5, A, "fp32", 3, mask=False)
    act[:] = 1
    x[1, A // 2] = math.nan
    x[3, A - 1] = math.inf
    r = binding.marl_policy_logprob(x, act, top=2)
    d = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=torch.ones(5, device="cuda"))
    for k in (1, 3):
        assert math.isnan(r["logp"][k]) and math.isnan(r["entropy"][k]) and bool(torch.isnan(d[k]).all())
    assert int(r["top_index"][1, 0]) == A // 2 and int(r["top_index"][3, 0]) == A - 1
    keep = torch.tensor([0, 2, 4], device="cuda")
    s, _ = _check(x[keep], None, act[keep], top=2)
    for k in ("logp", "entropy", "stats", "top_index", "top_logp"):
        assert torch.equal(s[k], r[k][keep])


def test_gradient_against_differences():
    """d/dx of a weighted sum of logp and entropy, by central differences of the definition in 64 bits."""
    x, av, act = _make(4, 11, "fp32", 1, True)
    act[:] = torch.tensor([10, 1, 2, 3])
    av[torch.arange(4), act.long()] = 1
    gl, ge = torch.tensor([1.0, -2.0, 0.5, 3.0]).cuda(), torch.tensor([0.3, 1.0, -1.0, 0.0]).cuda()
    r = binding.marl_policy_logprob(x, act, avail=av, temperature=0.9)
    d = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=gl, g_entropy=ge, avail=av, temperature=0.9)
    h = 1e-5

    def f(y):
        w = _want(y, av, act, 0.9, 0)
        return w["logp"] * gl.double() + w["H"] * ge.double()

    for j in range(11):
        step = torch.zeros(4, 11, dtype=torch.float64, device="cuda")
        step[:, j] = h
        diff = (f(x.double() + step) - f(x.double() - step)) / (2 * h)
        assert bool(((diff - d[:, j].double()).abs() < 1e-5).all())


def test_batch_shapes_broadcast_rows_and_wider_gradient_rows():
    x = torch.randn(3, 4, 5, 14, device="cuda")
    av = (torch.rand(14, device="cuda") < 0.5).expand(3, 4, 5, 14)      # one availability for all rows
    act = torch.randint(0, 14, (3, 4, 5), dtype=torch.int32, device="cuda")
    r = binding.marl_policy_logprob(x, act, avail=av, top=2)
    flat, _ = _check(x.view(60, 14), av.reshape(60, 14).to(torch.uint8).contiguous(), act.view(60), top=2)
    for k in ("logp", "entropy", "top_index", "top_logp"):
        assert torch.equal(r[k].reshape(flat[k].shape), flat[k])
    for A in (14, 100):
        x, avm, a = _make(9, A, "bf16", 0, True)
        wide = torch.full((9, A + 5), 3.0, dtype=torch.bfloat16, device="cuda")
        _check(x, avm, a, out=wide[:, :A])
        assert bool((wide[:, A:] == 3.0).all())
    e = binding.marl_policy_logprob(torch.empty(0, 6, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"), top=2)
    assert e["logp"].shape == (0,) and e["top_index"].shape == (0, 2)


def test_captured_and_replayed_on_another_stream():
    x, av, act = _make(50, 300, "bf16", 5, True)
    gl = torch.randn(50, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            r = binding.marl_policy_logprob(x, act, avail=av, top=4)
            d = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=gl, avail=av)
    for seed in (6, 7):
        y, av2, act2 = _make(50, 300, "bf16", seed, True)
        x.copy_(y)
        av.copy_(av2)
        act.copy_(act2)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            g.replay()
        torch.cuda.synchronize()
        want = binding.marl_policy_logprob(x, act, avail=av, top=4)
        dw = binding.marl_policy_logprob_backward(x, act, want["stats"], want["entropy"], g_logp=gl, avail=av)
        for k in want:
            assert torch.equal(r[k], want[k]), k
        assert torch.equal(d, dw)


def test_offsets_beyond_32_bits():
    """More than 2^32 bytes and 2^31 elements of rows: the last ones are read where they lie."""
    A, R = 65537, 33000
    x = torch.zeros(R, A, dtype=torch.bfloat16, device="cuda")
    x[R - 1, 5] = 4.0
    x[R - 1, A - 1] = 3.0
    act = torch.full((R,), A - 1, dtype=torch.int32, device="cuda")
    r = binding.marl_policy_logprob(x, act, top=3)
    assert r["top_index"][R - 1].tolist() == [5, A - 1, 0] and r["top_index"][R - 2].tolist() == [0, 1, 2]
    s = math.log(math.exp(4) + math.exp(3) + A - 2)
    assert abs(float(r["logp"][R - 1]) - (3 - s)) < 1e-4
    d = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=torch.ones(R, device="cuda"), out=x)
    want = 1 - math.exp(3 - s)
    assert abs(float(d[R - 1, A - 1]) - want) < want * 2 ** -8
    assert abs(float(d[R - 1, 5]) + math.exp(4 - s)) < math.exp(4 - s) * 2 ** -7


def test_refusals():
    x, av, act = _make(4, 9, "fp32", 0, True)
    f, e = binding.marl_policy_logprob, binding.MarlError
    for bad in (dict(top=33), dict(top=-1), dict(temperature=0.0), dict(avail=av[:, :8]), dict(avail=av.float()), dict(avail=av.cpu())):
        with pytest.raises(e):
            f(x, act, **{**dict(avail=av), **bad})
    for args in ((x.double(), act), (x, act.long()), (x, act[:3]), (x.t().contiguous().t(), act), (x, act.cpu())):
        with pytest.raises(e):
            f(*args)
    r = f(x, act)
    with pytest.raises(e):
        binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=torch.ones(3, device="cuda"))
    with pytest.raises(e):
        binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], out=x.half())


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("R,A,top", [(300, 4097, 8), (400, 9001, 1), (1200, 5000, 20), (297, 20011, 3)])
@pytest.mark.parametrize("mask", [True, False])
def test_many_long_rows(R, A, top, dt, mask):
    x, av, act = _make(R, A, dt, R, mask, pad=R % 2)
    _check(x, av, act, T=0.8, top=top)


@pytest.mark.parametrize("R,A", [(3, 1500), (2, 40000), (310, 16385)])
def test_large_values_in_few_lanes(R, A):
    """Periods at which one lane of a warp, or of a block, meets nearly all large values: more candidates than there is room for."""
    j = torch.arange(A)
    rows = []
    for period in (32 * 8, 256 * 8, 32 * 4, 512 * 8, 1024 * 8):
        rows.append(torch.where(j % period < 8, 100.0 + (j * 37 % 101) / 64, -(j % 13) / 4.0))
    v = torch.stack(rows)
    for dt in ("fp32", "bf16"):
        x = v.to(DT[dt]).cuda().repeat(-(-R // 5), 1)[:R].contiguous()
        act = torch.zeros(R, dtype=torch.int32, device="cuda")
        for top in (1, 5, 32):
            _check(x, None, act, top=top, grads=False)


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("A", [13, 600, 9000])
def test_temperatures_from_greedy_to_uniform(A, dt):
    """Temperatures at which one value takes all, and at which the largest and the lowest number of the type are alike."""
    x, av, act = _make(6, A, dt, A, True)
    for T in (1e-4, 0.05, 40.0, 3e3, 1e6, 1e30):
        _check(x, av, act, T=T, top=4)
    x[1] = torch.finfo(x.dtype).min
    x[2, ::3] = torch.finfo(x.dtype).min
    av[1:3] = 1
    for T in (0.5, 1e6, 1e30):
        r = binding.marl_policy_logprob(x, act, avail=av, temperature=T, top=min(A, 32))
        w = _want(x, av, act, T, min(A, 32))
        assert torch.equal(r["top_index"].long(), w["ti"])
        for k, v in (("logp", w["logp"]), ("entropy", w["H"])):
            # (a log probability below fp32's lowest number is -infinity there; otherwise it has that many of its own steps, and
            # log S and the entropy their errors as above, U being below 150 where a term counts)
            f = torch.isfinite(v.float())
            lim = 1e-3 * (1 + math.log(A)) + 2.0 ** -20 * v.abs()
            assert torch.equal(torch.isfinite(r[k]), f) and bool(((r[k].double() - v).abs() < lim)[f].all()), (T, k)


def test_a_gradient_that_is_not_finite_stays_in_its_row():
    for A in (14, 500):
        x, av, act = _make(6, A, "fp32", 0, True)
        act[:] = 0
        r = binding.marl_policy_logprob(x, act, avail=av)
        g = torch.ones(6, device="cuda")
        clean = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=g, avail=av)
        g[2], g[3] = math.nan, math.inf                      # row 3 is empty
        d = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=g, avail=av)
        keep = torch.tensor([0, 1, 3, 4, 5], device="cuda")
        assert torch.equal(d[keep], clean[keep]) and bool((d[3] == 0).all()) and bool(torch.isnan(d[2]).any())


@pytest.mark.parametrize("A", [5, 14, 32, 40])
def test_neighbouring_numbers_are_ranked_exactly(A):
    """Values one step of fp32 apart, in ascending and in mixed order, around powers of two, zero and below it."""
    for base in (1.0, -1.0, 2.0 ** -20, 1024.0):
        b = torch.tensor([base], dtype=torch.float32).view(torch.int32)
        j = torch.arange(A, dtype=torch.int32)
        rows = torch.stack([b + j, b - j, b + (j * 7) % A, b + j // 2, b + (A - j) // 3])
        x = rows.view(torch.float32).cuda()
        _check(x, None, torch.zeros(5, dtype=torch.int32, device="cuda"), top=min(A, 32), grads=False)
    tiny = (torch.arange(A, dtype=torch.int32) * 3 % A).view(torch.float32)          # subnormal numbers and zero
    _check(torch.stack([tiny, -tiny]).cuda(), None, torch.zeros(2, dtype=torch.int32, device="cuda"), top=min(A, 32), grads=False)


def _crowded_rows(A, seed):
    """fp32 rows of numbers a few steps apart: whatever a ranking leaves out of their last bits, it has to look at them."""
    g = torch.Generator().manual_seed(seed)
    rows = []
    for base in (1.0, -1.0, 2.0 ** -20, 1024.0):
        b = torch.tensor([base], dtype=torch.float32).view(torch.int32)
        for span in (2, 4, 12, 33, 41):                               # steps between the least and the largest, equal ones among them
            j = torch.randint(0, span, (20, A), generator=g, dtype=torch.int32)
            rows.append((b + j).view(torch.float32))
        up = torch.tensor([0, 0, 1, 2, 1, 3, 40, 1], dtype=torch.int32)   # the largest last, behind a prefix that does not ascend
        for k in range(4):
            rows.append((b + up.roll(k).repeat(5)[:A][None]).view(torch.float32))
    rows.append(20.0 + 1e-4 * torch.randn(100, A, generator=g))       # heads that are nearly equal
    rows.append(10000.0 + 0.01 * torch.randn(100, A, generator=g))
    half = 2.0 * torch.randn(100, A, generator=g)                     # half of a row close together, the rest apart
    near = half.max() + 1.0 + 2.0 ** -20 * torch.randint(0, 16, (100, A), generator=g)
    rows.append(torch.where(torch.rand(100, A, generator=g) < 0.5, near, half))
    return torch.cat(rows)


@pytest.mark.parametrize("A", [2, 3, 5, 8, 9, 14, 16, 17, 31, 32, 33])
def test_fewer_alternatives_than_close_values_are_ranked_exactly(A):
    """The best few of rows in which more values than those lie close together, with and without a mask."""
    x = _crowded_rows(A, A)
    R = x.shape[0]
    av = (torch.rand(R, A, generator=torch.Generator().manual_seed(1)) < 0.8).to(torch.uint8)
    act = torch.zeros(R, dtype=torch.int32).cuda()
    buf = torch.zeros(R, A + 3)
    buf[:, :A] = x
    for top in sorted({1, 2, 3, 4, A // 2, A - 2, A - 1} - {0, -1}):
        for rows in (x.cuda(), buf.cuda()[:, :A]):                    # without gaps, and rows of a wider buffer
            for mask in (None, av.cuda()):
                _check(rows, mask, act, top=top, grads=False)


@pytest.mark.parametrize("dt", ["bf16", "fp16"])
def test_close_values_of_16_bit_types_are_ranked_exactly(dt):
    for A in (3, 14, 32):
        g = torch.Generator().manual_seed(A)
        one = torch.ones(1, dtype=DT[dt]).view(torch.int16)
        x = (one + torch.randint(-3, 4, (200, A), generator=g, dtype=torch.int16)).view(DT[dt]).cuda()
        for top in (1, 2, A - 1):
            _check(x, None, torch.zeros(200, dtype=torch.int32, device="cuda"), top=top, grads=False)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("A", [14, 500, 9000])
def test_the_gradient_of_a_row_that_is_not_a_number(A, dt):
    """A NaN or +infinity among the available entries makes its own row NaN, all of it; an unavailable one has no effect."""
    x, av, act = _make(8, A, dt, 3, True)
    av[:, :3] = 1
    av[4] = 0                                                     # an empty row
    act[:] = 1
    g = torch.ones(8, device="cuda")
    kw = dict(g_logp=g, g_entropy=g, avail=av)
    av[6, 2] = 0
    r = binding.marl_policy_logprob(x, act, avail=av)
    clean = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], **kw)
    x[1, 0], x[2, 2], x[6, 2], x[4, 5] = math.nan, math.inf, math.nan, math.nan
    r = binding.marl_policy_logprob(x, act, avail=av)
    d = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], **kw)
    bad = torch.zeros(8, dtype=torch.bool, device="cuda")
    bad[1:3] = True
    assert torch.equal(torch.isnan(r["logp"]), bad) and torch.equal(torch.isnan(r["entropy"]), bad)
    assert bool(torch.isnan(d[1:3]).all()) and torch.equal(d[~bad], clean[~bad])
