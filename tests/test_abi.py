"""The C ABI library builds, loads without a GPU, and exports every symbol
that include/gmc.h declares; the binding declares the same names."""
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def _declared():
    src = open(os.path.join(ROOT, "include", "gmc.h")).read()
    src = re.sub(r"/\*.*?\*/", "", src, flags=re.S)
    return sorted(set(re.findall(r"\b(gmc_[a-z0-9_]+)\s*\(", src)))


@pytest.fixture(scope="module")
def lib():
    from paper_1905_12948_gb300 import build, gmc
    build.build()
    return gmc.load()


def test_header_declares_the_api():
    names = _declared()
    for must in ("gmc_create", "gmc_step", "gmc_get_params", "gmc_destroy", "gmc_check"):
        assert must in names


def test_library_exports_every_declared_symbol(lib):
    for name in _declared():
        assert hasattr(lib, name), name


def test_binding_covers_the_header(lib):
    from paper_1905_12948_gb300 import gmc
    assert sorted(gmc.exported_symbols()) == _declared()


def test_strerror_without_gpu(lib):
    assert lib.gmc_strerror(0) == b"success"
    assert lib.gmc_strerror(1) == b"invalid argument"
    assert lib.gmc_kernel_name(0) == b"accumulate"


def test_invalid_arguments_rejected_without_gpu(lib):
    import ctypes
    h = ctypes.c_void_p()
    # d = 0 (empty), K = 0, beta = 1, eta = 0, ratio = 0 / > 1, bad compressor, RBGS block 0
    bad = [(0, 4, 0.9, 0.1, 0, 0.01, 1), (10, 0, 0.9, 0.1, 0, 0.01, 1),
           (10, 2, 1.0, 0.1, 0, 0.01, 1), (10, 2, 0.9, 0.0, 0, 0.01, 1),
           (10, 2, 0.9, 0.1, 0, 0.0, 1), (10, 2, 0.9, 0.1, 0, 1.5, 1),
           (10, 2, 0.9, 0.1, 7, 0.01, 1), (10, 2, 0.9, 0.1, 1, 0.01, 0),
           (1 << 31, 2, 0.9, 0.1, 0, 0.01, 1), (10, 2, float("nan"), 0.1, 0, 0.01, 1)]
    for args in bad:
        assert lib.gmc_create(ctypes.byref(h), *args) == 1, args
        assert h.value is None
    assert lib.gmc_step(None, None, None) == 1
    assert lib.gmc_set_params(None, None, None) == 1


def test_failure_hooks_without_gpu(lib):
    """The allocation hook round-trips without a device (no handle holds
    memory), the timeout has its own status and message, and the copy hook
    refuses a NULL handle."""
    assert lib.gmc_test_fail_alloc(3) == 0
    assert lib.gmc_test_fail_alloc(-1) == 0
    assert lib.gmc_strerror(8).startswith(b"a bounded wait")
    assert lib.gmc_strerror(9) == b"unknown status"
    assert lib.gmc_test_withhold_copy(None, 0, 0, 1000) == 1
    assert lib.gmc_test_pass(None) == -1
    assert lib.gmc_test_leave_barrier(None, 2_000_000_001) == 1
    assert lib.gmc_test_refuse_cooperative(-1) == 1
    assert lib.gmc_test_refuse_cooperative(0) == 0
    assert lib.gmc_check(None) == 1


def test_operators_module_loads_and_refuses_without_gpu(lib):
    """The compiled Python module of the operators: loads, wants init() once, and refuses
    what is not a CUDA tensor with an exception of Python's."""
    torch = pytest.importorskip("torch")
    from paper_1905_12948_gb300 import dropout, token_logp, tokens
    with pytest.raises(TypeError, match="logits must be a CUDA tensor"):
        token_logp(torch.zeros(2, 3), torch.zeros(2, dtype=torch.int64))
    with pytest.raises(TypeError, match="x must be a CUDA tensor"):
        dropout(3.0, 0.1, seed=1)
    module = tokens._load()
    with pytest.raises(TypeError, match="expected"):
        module.policy(1, 2)
    with pytest.raises(ValueError):
        module.init(RuntimeError, 0, 0, 0, 0, 0)


def test_operators_refuse_bad_arguments_without_gpu(lib):
    import ctypes
    buf = ctypes.create_string_buffer(4096)
    p = ctypes.addressof(buf) + 16 - ctypes.addressof(buf) % 16
    # type, stride, alignment, vocabulary, scale: refused before anything is launched
    for args in [(p, 3, 4, 10, 10, 1.0), (p, 0, 4, 10, 9, 1.0), (p + 2, 0, 4, 10, 10, 1.0), (p, 0, 4, 0, 10, 1.0),
                 (p, 0, 4, 10, 10, 0.0), (p, 0, 4, 10, 10, float("inf")), (None, 0, 4, 10, 10, 1.0),
                 (p, 0, -1, 10, 10, 1.0), (p, 0, 4, 1 << 31, 1 << 31, 1.0)]:
        assert lib.gmc_token_logp(*args, p, p, None, None) == 1, args
    assert lib.gmc_token_logp(None, 0, 0, 10, 10, 1.0, None, None, None, None) == 0     # no rows: nothing to do
    assert lib.gmc_dropout(p, 8, None, 0, p, 8, 0, 0, 2, 8, 1.5, 0, 0, 0, None) == 1
    assert lib.gmc_dropout(None, 0, None, 0, None, 0, 0, 0, 0, 8, 0.5, 0, 0, 0, None) == 0
    assert lib.gmc_policy_loss(None, p, 0, 4, 10, 10, 1.0, p, p, None, p, None, 0.2, 0.2, 0.0, p, None, None, None, 10,
                               None) == 1
    lib.gmc_loss_destroy(None)
