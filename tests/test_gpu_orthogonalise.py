"""marl_orthogonalise against its definition in 64 bits.

Tolerance.  The kernel makes the same fp32 products as the definition does when torch evaluates it in fp32, with sums in another
order; both errors are sums of many independent roundings, amplified alike by the polynomial's slope at small singular
values.  So the kernel may be off by at most three times the error of that fp32 evaluation (2-norm over the matrix; twice for the
spread of the two sums, once more for a slice's sum that is added up in parts), plus half a step of the output's type (relative), and
fp32's own rounding of the scaled result."""
import pytest
import torch

from paper_2205_05248_b200 import binding, workloads

pytestmark = pytest.mark.gpu
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
CO = (3.4445, -4.7750, 2.0315)


def _formula(m, steps=5, coeffs=CO, eps=1e-7):
    X = m.mT if m.shape[-2] > m.shape[-1] else m
    X = X / (X.square().sum((-1, -2), keepdim=True).sqrt() + eps)
    for _ in range(steps):
        S = X @ X.mT
        X = coeffs[0] * X + (coeffs[1] * S + coeffs[2] * (S @ S)) @ X
    return X.mT if m.shape[-2] > m.shape[-1] else X


def _check(got, m, scale=1.0, **kw):
    want = _formula(m.double(), **kw) * scale
    off32 = (_formula(m.float(), **kw).double() * scale - want).flatten(-2).norm(dim=-1)
    err = (got.double() - want).flatten(-2).norm(dim=-1)
    n = want.flatten(-2).norm(dim=-1)
    tol = 3 * off32 + (torch.finfo(got.dtype).eps / 2 + 2.0 ** -22) * n
    if got.dtype == torch.float16:
        tol = tol + 2.0 ** -25 * (m.shape[-1] * m.shape[-2]) ** 0.5
    assert bool((err <= tol).all()), (tuple(m.shape), float((err / tol).max()))


def _rand(*shape, seed=0, rank=None):
    g = torch.Generator().manual_seed(seed)
    m = torch.randn(*shape, generator=g)
    if rank:
        m = 0.1 * m + torch.randn(*shape[:-1], rank, generator=g) @ torch.randn(*shape[:-2], rank, shape[-1], generator=g)
    return m.cuda()


SHAPES = [(1, 1), (1, 7), (5, 1), (3, 2), (16, 16), (17, 16), (15, 33), (31, 64), (64, 14), (64, 102), (192, 64), (65, 64), (65, 66), (128, 128),
          (128, 96), (384, 128), (11, 128), (100, 577), (1024, 128), (127, 1023), (1024, 3)]


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("r,c", SHAPES)
def test_one_matrix(r, c, dt):
    m = (1e-2 * _rand(r, c, seed=r + c, rank=3)).to(DT[dt])
    _check(binding.marl_orthogonalise([m])[0], m)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("K", [1, 3, 12, 40, 150])
def test_lists_of_mixed_shapes(K, dt):
    """All weight matrices of K networks of either hidden size in one call, whatever the blocks a matrix gets."""
    for H in (64, 128):
        mats = [(1e-3 * _rand(K, r, c, seed=K + r, rank=5)).to(DT[dt]) for r, c in ((H, 102), (3 * H, H), (3 * H, H), (14, H))]
        mats.append(_rand(9, H, seed=1).to(DT[dt]))
        out = binding.marl_orthogonalise(mats, scale=[1.0, 0.5, -2.0, 1.0, 3.0])
        for m, o, s in zip(mats, out, (1.0, 0.5, -2.0, 1.0, 3.0)):
            _check(o, m, scale=s)
        again = binding.marl_orthogonalise(mats, scale=[1.0, 0.5, -2.0, 1.0, 3.0])
        assert all(torch.equal(a, b) for a, b in zip(out, again))


def test_more_entries_than_a_launch_holds():
    mats = [_rand(4 + k % 9, 3 + k % 17, seed=k) for k in range(70)]
    for m, o in zip(mats, binding.marl_orthogonalise(mats)):
        _check(o, m)


def test_singular_values_are_drawn_to_one():
    for r, c in ((64, 102), (384, 128), (14, 64)):
        o = binding.marl_orthogonalise([_rand(r, c, seed=r)])[0]
        s = torch.linalg.svdvals(o.double())
        assert float(s.min()) > 0.6 and float(s.max()) < 1.25
        o = binding.marl_orthogonalise([_rand(r, c, seed=r)], steps=25, coeffs=(1.875, -1.25, 0.375))[0]
        s = torch.linalg.svdvals(o.double())
        assert float((s - 1).abs().max()) < 1e-4      # the quintic that has 1 as a fixed point of order three


@pytest.mark.parametrize("steps", [0, 1, 2, 9])
def test_steps_and_coefficients(steps):
    m = [_rand(40, 70, seed=1), _rand(130, 90, seed=2)]
    kw = dict(steps=steps, coeffs=(1.5, -0.5, 0.0), eps=0.0)
    for a, o in zip(m, binding.marl_orthogonalise(m, **kw)):
        _check(o, a, **kw)


def test_zeros_extremes_and_not_a_number():
    """Zeros give zeros; the scale of a matrix does not matter, near overflow and below the normal numbers; a NaN or infinity stays in its matrix."""
    base = _rand(20, 33, seed=3)
    mats = torch.stack([torch.zeros(20, 33, device="cuda"), base, base * 1e37, base * 1e-39, base.clone(), base.clone()])
    mats[4, 7, 8] = float("nan")
    mats[5, 0, 32] = float("-inf")
    for eps in (0.0, 1e-30):
        o = binding.marl_orthogonalise([mats], eps=eps)[0]
        assert bool((o[0] == 0).all())
        _check(o[1], mats[1], eps=eps)
        assert float((o[2] - o[1]).abs().max()) < 1e-5
        if eps == 0.0:
            _check_small = _formula(mats[3].double(), eps=0.0)
            assert float((o[3].double() - _check_small).norm() / _check_small.norm()) < 1e-4
        assert bool(torch.isnan(o[4:]).all())


def test_strides_in_place_and_untouched_neighbours():
    for dt in ("fp32", "bf16"):
        buf = _rand(5, 70, 90, seed=4).to(DT[dt])
        v = buf[1:4, 3:67, 5:40]                                  # rows that start off any boundary
        want = v.clone()
        keep = buf.clone()
        out = binding.marl_orthogonalise([v], out=[v])[0]
        _check(out, want)
        keep[1:4, 3:67, 5:40] = out
        assert torch.equal(keep, buf)
        one = want[:1].expand(3, 64, 35)                          # one matrix three times
        _check(binding.marl_orthogonalise([one])[0], one)


def test_captured_on_two_streams():
    m = [_rand(192, 64, seed=k) for k in range(2)]
    graphs = []
    for k in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            o = binding.marl_orthogonalise([m[k]])[0]
        graphs.append((g, torch.cuda.Stream(), o))
    for a in m:
        a.mul_(-3.0).add_(0.01)
    torch.cuda.synchronize()
    for _ in range(4):
        for g, s, _ in graphs:
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for a, (_, _, o) in zip(m, graphs):
        assert torch.equal(o, binding.marl_orthogonalise([a])[0])


def test_refusals():
    e, f = binding.MarlError, binding.marl_orthogonalise
    a = _rand(8, 9)
    for bad in ([a.double()], [a, a.half()], [a, a.cpu()], [a.t()], [a[0]], [a[:0]], [_rand(129, 129)], [_rand(2, 1025)]):
        with pytest.raises(e):
            f(bad)
    for kw in (dict(steps=65), dict(steps=-1), dict(eps=-1.0), dict(coeffs=(1.0, 2.0)), dict(scale=[1.0, 2.0]), dict(out=[]),
               dict(out=[a.half()]), dict(out=[a[:, :1].expand(8, 9)])):
        with pytest.raises(e):
            f([a], **kw)


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("r,c", [(1, 2), (20, 33), (64, 102), (128, 1024)])
@pytest.mark.parametrize("top", [3e38, 1e38, 2e36])
def test_norms_beyond_fp32(r, c, top, dt):
    """Finite matrices whose norm is not a number of fp32, beside one whose norm is.  Their scale is taken out in 64 bits for the fp32 evaluation that
    the tolerance counts from; eps is as large as the entries once."""
    base = _rand(r, c, seed=r)
    m = (base / base.abs().max() * top).to(DT[dt])
    assert bool(torch.isfinite(m).all())
    for eps in (0.0, 1e-7, 1e38):
        got = binding.marl_orthogonalise([m, base.to(DT[dt])], eps=eps)[0]
        small = (m.double() * 2.0 ** -120).float()                       # exact
        want = _formula(m.double(), eps=eps)
        off32 = (_formula(small, eps=eps * 2.0 ** -120).double() - want).norm()
        err, n = (got.double() - want).norm(), want.norm()
        assert float(n) > 0.1
        # (the quotients of the scaled norm and eps round twice more: 2^-23, and the polynomial passes a relative change of scale on by at most
        # its largest slope a step where singular values are small: 3.4445^5 = 485 of those)
        assert float(err) <= float(3 * off32 + (torch.finfo(got.dtype).eps / 2 + 2.0 ** -22 + 485 * 2.0 ** -23) * n), (eps, float(err / n))


def test_norms_below_the_normal_numbers():
    """Without eps the scale does not matter, however few bits the norm would have as a number of fp32."""
    for r, c in ((1, 2), (20, 33), (100, 64)):
        m = _rand(r, c, seed=c) * 1e-43
        assert float(m.abs().max()) > 0
        got = binding.marl_orthogonalise([m], eps=0.0)[0]
        want = _formula(m.double(), eps=0.0)
        off32 = (_formula((m.double() * 2.0 ** 120).float(), eps=0.0).double() - want).norm()
        err, n = (got.double() - want).norm(), want.norm()
        assert float(err) <= float(3 * off32 + (2.0 ** -22 + 485 * 2.0 ** -23) * n), (r, c, float(err / n))
