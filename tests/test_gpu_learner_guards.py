"""The learner's operators write their outputs, all of them and nothing else: every output lies between guard bytes and starts as NaN (the
stand-in for a memory checker)."""
import math

import pytest
import torch

from paper_2205_05248_b200 import binding

pytestmark = pytest.mark.gpu
PAD = 64                      # elements: keeps 16-byte boundaries
DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


class Guarded:
    def __init__(self):
        self.all = []

    def new(self, shape, dtype, dev):
        n = math.prod(shape)
        full = torch.empty(n + 2 * PAD, dtype=dtype, device=dev)
        full.view(torch.uint8).fill_(0xA5)
        t = full[PAD:PAD + n].view(tuple(shape))
        t.fill_(float("nan") if dtype.is_floating_point else -77)
        self.all.append((full, n))
        return t

    def check(self, unwritten=()):
        torch.cuda.synchronize()
        for full, n in self.all:
            b = full.view(torch.uint8)
            e = full.element_size()
            assert bool((b[:PAD * e] == 0xA5).all()) and bool((b[(PAD + n) * e:] == 0xA5).all())
        self.all = []


@pytest.fixture
def guarded(monkeypatch):
    g = Guarded()
    monkeypatch.setattr(binding, "_new", g.new)
    return g


def _written(t, what):
    assert not bool(torch.isnan(t).any() if t.is_floating_point() else (t == -77).any()), what


@pytest.mark.parametrize("dt", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("R,A,pad", [(1, 1, 0), (127, 9, 0), (129, 14, 0), (130, 32, 1), (9, 33, 0), (17, 1000, 3), (5, 4096, 0), (3, 4097, 0),
                                     (1, 70001, 0), (2, 131072, 8), (310, 5003, 0)])
def test_log_probabilities(guarded, R, A, pad, dt):
    g = torch.Generator().manual_seed(A)
    x = torch.randn(R, A + pad, generator=g).to(DT[dt]).cuda()[:, :A]
    av = (torch.rand(R, A, generator=g) < 0.7).to(torch.uint8).cuda()
    av[:, 0] = 1
    act = torch.zeros(R, dtype=torch.int32, device="cuda")
    for mask in (av, None):
        for top in (0, 1, 4, 7, 32):
            r = binding.marl_policy_logprob(x, act, avail=mask, top=top)
            guarded.check()
            for k, v in r.items():
                if v is not None:
                    _written(v, k)
        d = binding.marl_policy_logprob_backward(x, act, r["stats"], r["entropy"], g_logp=torch.ones(R, device="cuda"), avail=mask)
        guarded.check()
        _written(d, "dlogits")


@pytest.mark.parametrize("dt", ["fp32", "bf16"])
@pytest.mark.parametrize("B,L,C", [(3, 1, 5), (2, 1, 64), (5, 7, 1), (3, 65, 3), (2, 100, 33), (3, 64, 64), (3, 129, 72), (1, 3000, 2), (1, 3001, 64),
                                   (2, 70, 200), (9, 33, 48)])
def test_recurrence(guarded, B, L, C, dt):
    g = torch.Generator().manual_seed(L)
    gate, x = (torch.randn(B, L, C, generator=g).to(DT[dt]).cuda() for _ in range(2))
    n = torch.randint(0, L + 1, (B,), generator=g).to(torch.int32).cuda()
    done = (torch.rand(B, L, generator=g) < 0.1).to(torch.uint8).cuda()
    for reverse in (False, True):
        for length in (None, n):
            kw = dict(h0=torch.zeros(B, C, device="cuda"), done=done, length=length, reverse=reverse)
            r = binding.marl_linear_scan(gate, x, keep=True, **kw)
            guarded.check()
            _written(r["y"], "y")
            _written(r["last"], "last")
            if length is None:
                _written(r["states"], "states")
            d = binding.marl_linear_scan_backward(gate, x, r["states"], x, **kw)
            guarded.check()
            for k, v in d.items():
                _written(v, k)


@pytest.mark.parametrize("dt", ["fp32", "fp16"])
def test_updates(guarded, dt):
    for shapes in ([(1, 1)], [(3, 64, 102), (3, 192, 64), (3, 14, 64)], [(128, 1024)], [(40, 17, 5)], [(1024, 9), (2, 100, 130), (16, 33)]):
        mats = [torch.randn(*s).to(DT[dt]).cuda() for s in shapes]
        out = binding.marl_orthogonalise(mats)
        guarded.check()
        for o in out:
            _written(o, "out")
