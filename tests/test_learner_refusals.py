"""Argument checks of the learner's operators that need no GPU: every refusal is an error code with a text, made before any device
work; empty calls succeed."""
import ctypes as C

import pytest
import torch

from paper_2205_05248_b200 import binding, build

EINVAL, EALIGN = -1, -2
GOOD = 1 << 20  # a well-aligned address that is never used: the calls below are refused first


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def _rows(**over):
    p = dict(logits=GOOD, avail=GOOD, action=GOOD, rows=4, row_stride=9, avail_stride=9, n_actions=9, dtype=0, temperature=1.0,
             reserved=0)
    p.update(over)
    return binding.PolicyRows(*[p[k] for k, _ in binding.PolicyRows._fields_])


def _p(v):
    return None if v is None else C.c_void_p(v)


BAD_ROWS = [(dict(rows=-1), EINVAL), (dict(n_actions=0), EINVAL), (dict(n_actions=(1 << 30) + 1), EINVAL), (dict(dtype=3), EINVAL),
            (dict(dtype=-1), EINVAL), (dict(temperature=0.0), EINVAL), (dict(temperature=-1.0), EINVAL),
            (dict(temperature=float("nan")), EINVAL), (dict(temperature=float("inf")), EINVAL), (dict(temperature=1e-39), EINVAL),
            (dict(logits=None), EINVAL), (dict(action=None), EINVAL), (dict(row_stride=-9), EINVAL), (dict(avail_stride=-1), EINVAL),
            (dict(logits=GOOD + 2), EALIGN), (dict(logits=GOOD + 1, dtype=1), EALIGN), (dict(action=GOOD + 2), EALIGN)]


@pytest.mark.parametrize("over,code", BAD_ROWS)
def test_policy_rows_are_refused(lib, over, code):
    r = _rows(**over)
    assert lib.marl_policy_logprob(None, C.byref(r), 2, *[_p(GOOD)] * 5) == code and lib.marl_last_error()
    assert lib.marl_policy_logprob_backward(None, C.byref(r), *[_p(GOOD)] * 5, 9) == code


def test_policy_outputs_are_refused(lib):
    r = _rows()
    f = lib.marl_policy_logprob
    for top in (-1, 33):
        assert f(None, C.byref(r), top, *[_p(GOOD)] * 5) == EINVAL
    for k in range(5):
        ptr = [_p(GOOD)] * 5
        ptr[k] = None
        assert f(None, C.byref(r), 2, *ptr) == EINVAL
        ptr[k] = _p(GOOD + (4 if k == 2 else 2))
        assert f(None, C.byref(r), 2, *ptr) == EALIGN
    g = lib.marl_policy_logprob_backward
    for k in (0, 1, 4):
        ptr = [_p(GOOD)] * 5
        ptr[k] = None
        assert g(None, C.byref(r), *ptr, 9) == EINVAL
    for k in range(5):
        ptr = [_p(GOOD)] * 5
        ptr[k] = _p(GOOD + (4 if k == 0 else 2))
        assert g(None, C.byref(r), *ptr, 9) == EALIGN
    assert g(None, C.byref(r), *[_p(GOOD)] * 5, 8) == EINVAL
    assert f(None, None, 0, *[_p(GOOD)] * 5) == EINVAL and g(None, None, *[_p(GOOD)] * 5, 9) == EINVAL


def test_policy_rows_of_an_empty_batch(lib):
    r = _rows(rows=0, logits=None, action=None, avail=None)
    assert lib.marl_policy_logprob(None, C.byref(r), 0, None, None, None, None, None) == 0
    assert lib.marl_policy_logprob_backward(None, C.byref(r), None, None, None, None, None, 9) == 0


def test_rows_of_a_tensor():
    t = torch.zeros(4, 6, 8, 16)
    assert binding._rows_of(t, "t") == (192, 16)
    assert binding._rows_of(t[..., :9], "t") == (192, 16)
    assert binding._rows_of(t[1, 2, 3], "t") == (1, 16)
    assert binding._rows_of(t[:, 2:3, 1], "t") == (4, 6 * 8 * 16)
    assert binding._rows_of(torch.zeros(1, 5).expand(7, 5), "t") == (7, 0)
    assert binding._rows_of(torch.zeros(3, 0, 5), "t") == (0, 5)
    for bad in (t.transpose(-1, -2), t[:, 1:], t.transpose(0, 1)):
        with pytest.raises(binding.MarlError):
            binding._rows_of(bad, "t")


def test_tensors_without_a_gpu_are_refused():
    x = torch.zeros(3, 5)
    a = torch.zeros(3, dtype=torch.int32)
    with pytest.raises(binding.MarlError):
        binding.marl_policy_logprob(x, a)


def _scan(**over):
    p = dict(gate=GOOD, x=GOOD, gate_b=40, gate_t=8, x_b=40, x_t=8, gate_c=1, x_c=1, h0=GOOD, done=GOOD, length=GOOD, B=2, L=5, C=8,
             dtype=0, form=1, reverse=0)
    p.update(over)
    return binding.Scan(*[p[k] for k, _ in binding.Scan._fields_])


@pytest.mark.parametrize("over,code", [
    (dict(B=-1), EINVAL), (dict(L=-1), EINVAL), (dict(C=-1), EINVAL), (dict(L=(1 << 30) + 1), EINVAL), (dict(dtype=3), EINVAL),
    (dict(form=2), EINVAL), (dict(gate_b=-1), EINVAL), (dict(x_t=-1), EINVAL), (dict(gate_c=2), EINVAL), (dict(x_c=-1), EINVAL),
    (dict(gate=None), EINVAL), (dict(x=None), EINVAL), (dict(gate=GOOD + 2), EALIGN), (dict(x=GOOD + 1, dtype=2), EALIGN),
    (dict(h0=GOOD + 2), EALIGN), (dict(length=GOOD + 2), EALIGN)])
def test_scans_are_refused(lib, over, code):
    s = _scan(**over)
    assert lib.marl_linear_scan(None, C.byref(s), _p(GOOD), _p(GOOD), _p(GOOD), None, 0) == code and lib.marl_last_error()
    assert lib.marl_linear_scan_backward(None, C.byref(s), _p(GOOD), _p(GOOD), 40, 8, _p(GOOD), _p(GOOD), _p(GOOD), _p(GOOD), None, 0) == code


def test_scan_outputs_and_work_are_refused(lib):
    s = _scan()
    f, g = lib.marl_linear_scan, lib.marl_linear_scan_backward
    for y, last, code in ((None, GOOD, EINVAL), (GOOD, None, EINVAL), (GOOD + 2, GOOD, EALIGN), (GOOD, GOOD + 2, EALIGN)):
        assert f(None, C.byref(s), _p(y), _p(last), None, None, 0) == code
    for k in (0, 1, 3, 4):
        a = [GOOD] * 6
        a[k] = None
        assert g(None, C.byref(s), _p(a[0]), _p(a[1]), 40, 8, _p(a[2]), _p(a[3]), _p(a[4]), _p(a[5]), None, 0) == EINVAL
    for k in range(6):
        a = [GOOD] * 6
        a[k] = GOOD + 2
        assert g(None, C.byref(s), _p(a[0]), _p(a[1]), 40, 8, _p(a[2]), _p(a[3]), _p(a[4]), _p(a[5]), None, 0) == EALIGN
    assert g(None, C.byref(s), *[_p(GOOD)] * 2, -40, 8, *[_p(GOOD)] * 4, None, 0) == EINVAL
    assert f(None, None, None, None, None, None, 0) == EINVAL
    long = _scan(B=1, L=100000)                             # few channels, many steps: needs scratch
    need, kept = C.c_size_t(), C.c_size_t()
    assert lib.marl_linear_scan_query(C.byref(long), C.byref(kept), C.byref(need)) == 0
    assert need.value > 0 and kept.value == 4 * 8 * -(-100000 // 64)
    assert f(None, C.byref(long), _p(GOOD), _p(GOOD), None, None, 0) == -4
    assert f(None, C.byref(long), _p(GOOD), _p(GOOD), None, _p(GOOD), need.value - 1) == -4
    assert f(None, C.byref(long), _p(GOOD), _p(GOOD), None, _p(GOOD + 4), need.value) == EALIGN


def test_scans_of_nothing(lib):
    for over in (dict(B=0), dict(C=0)):
        s = _scan(gate=None, x=None, h0=None, done=None, length=None, **over)
        assert lib.marl_linear_scan(None, C.byref(s), None, None, None, None, 0) == 0
        assert lib.marl_linear_scan_backward(None, C.byref(s), None, None, 0, 0, None, None, None, None, None, 0) == 0


def test_sizes_of_scans_of_nothing(lib):
    """No sequences or channels, however long: no scratch (and no division by the number of blocks)."""
    for over in (dict(B=0, L=100000), dict(C=0, L=100000), dict(B=0, C=0, L=1 << 20), dict(L=0)):
        need, kept = C.c_size_t(7), C.c_size_t(7)
        assert lib.marl_linear_scan_query(C.byref(_scan(**over)), C.byref(kept), C.byref(need)) == 0
        assert need.value == 0 and kept.value == 0


def test_scan_tensors_without_a_gpu_are_refused():
    x = torch.zeros(2, 3, 4)
    with pytest.raises(binding.MarlError):
        binding.marl_linear_scan(x, x)


def _matrix(**over):
    p = dict(in_=GOOD, out=GOOD, in_batch=64, in_row=8, out_batch=64, out_row=8, batch=2, rows=8, cols=8, scale=1.0)
    p.update(over)
    return binding.Matrix(*[p[k] for k, _ in binding.Matrix._fields_])


def _ortho(lib, entries, count=None, dtype=0, steps=5, coeffs=(3.4, -4.7, 2.0), eps=1e-7):
    arr = (binding.Matrix * max(1, len(entries)))(*entries)
    co = (C.c_float * 3)(*coeffs) if coeffs is not None else None
    return lib.marl_orthogonalise(None, arr, len(entries) if count is None else count, dtype, steps, co, eps)


@pytest.mark.parametrize("over,code", [
    (dict(batch=-1), EINVAL), (dict(rows=0), EINVAL), (dict(cols=0), EINVAL), (dict(rows=129, cols=129), EINVAL),
    (dict(rows=1025, cols=4), EINVAL), (dict(rows=4, cols=1025), EINVAL), (dict(in_=None), EINVAL), (dict(out=None), EINVAL),
    (dict(in_row=-1), EINVAL), (dict(in_batch=-1), EINVAL), (dict(out_row=7), EINVAL), (dict(out_batch=63), EINVAL),
    (dict(in_=GOOD + 2), EALIGN), (dict(out=GOOD + 2), EALIGN)])
def test_matrices_are_refused(lib, over, code):
    assert _ortho(lib, [_matrix(**over)]) == code and lib.marl_last_error()
    assert _ortho(lib, [_matrix(batch=0), _matrix(**over)]) == code


def test_orthogonalise_arguments_are_refused(lib):
    m = [_matrix()]
    assert _ortho(lib, m, dtype=3) == EINVAL and _ortho(lib, m, steps=-1) == EINVAL and _ortho(lib, m, steps=65) == EINVAL
    assert _ortho(lib, m, eps=-1.0) == EINVAL and _ortho(lib, m, eps=float("nan")) == EINVAL and _ortho(lib, m, eps=float("inf")) == EINVAL
    assert _ortho(lib, m, coeffs=None) == EINVAL and _ortho(lib, m, count=-1) == EINVAL
    assert lib.marl_orthogonalise(None, None, 1, 0, 5, (C.c_float * 3)(1, 1, 1), 0.0) == EINVAL
    assert _ortho(lib, []) == 0 and _ortho(lib, [_matrix(batch=0, in_=None, out=None)]) == 0


def test_two_results_in_one_place_are_refused(lib):
    a, b = _matrix(), _matrix(in_=GOOD + 4096)
    assert _ortho(lib, [a, b]) == EINVAL and b"same output" in lib.marl_last_error()
    assert _ortho(lib, [a, _matrix(out=GOOD + 8192), a]) == EINVAL


def test_matrices_without_a_gpu_are_refused():
    with pytest.raises(binding.MarlError):
        binding.marl_orthogonalise([torch.zeros(4, 4)])
    assert binding.marl_orthogonalise([]) == []


def test_a_list_with_an_entry_too_many_is_refused_whole(lib):
    """The refusal of a later entry comes before any work on the ones in front of it, however the list is cut into launches."""
    big = dict(out=GOOD + 65536, batch=(1 << 24) + 1)
    assert _ortho(lib, [_matrix(**big)]) == EINVAL
    assert _ortho(lib, [_matrix(), _matrix(**big)]) == EINVAL and b"2^24" in lib.marl_last_error()
    assert _ortho(lib, [_matrix(out=GOOD + (1 << 16) * k) for k in range(40)] + [_matrix(**dict(big, out=GOOD + (1 << 30)))]) == EINVAL
