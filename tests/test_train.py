"""Host-side checks of the trainer-side operators (include/dte_train.h) that
need no GPU: argument errors come before any device work, empty calls are
legal, workspace sizes, the range check of Newton-Schulz coefficients, and
what the built kernels may not contain."""
import ctypes
import os
import subprocess

import pytest

from paper_2608_00455_amd import binding as B
from paper_2608_00455_amd import build as dte_build
from paper_2608_00455_amd import train

F32, BF16 = B.DTE_TYPE_F32, B.DTE_TYPE_BF16
P = 4096   # an address that no call may follow


def st(fn, *a):
    return B.raw_status(fn, *a)


def test_embedding_arguments():
    fwd = lambda *a: st("dte_embedding_forward", *a)  # noqa: E731
    good = [P, BF16, 10, 8, 8, P, 4, 1.0, P, 8, None]
    for k, v in ((0, None), (1, 2), (1, -1), (2, -1), (2, 1 << 31), (3, -1), (4, 7), (4, 1 << 22),
                 (5, None), (6, -1), (6, 1 << 31), (7, float("nan")), (8, None), (9, 7)):
        bad = list(good)
        bad[k] = v
        assert fwd(*bad) == B.DTE_ERR_ARG, (k, v)
    assert fwd(None, BF16, 10, 8, 8, None, 0, 1.0, None, 8, None) == B.DTE_OK
    assert fwd(None, F32, 10, 0, 0, None, 4, 1.0, None, 0, None) == B.DTE_OK

    bwd = lambda *a: st("dte_embedding_backward", *a)  # noqa: E731
    need = B.dte_embedding_workspace_bytes(4, 10, 8)
    assert need > 0
    good = [P, BF16, 8, P, 4, 10, 8, 1.0, P, F32, 8, 1, P, need, None]
    for k, v in ((0, None), (1, 3), (2, 7), (3, None), (4, -1), (5, -1), (6, 9), (7, float("inf")),
                 (8, None), (9, 9), (9, BF16), (10, 7), (12, None), (12, P + 8), (13, need - 1)):
        bad = list(good)
        bad[k] = v
        assert bwd(*bad) == B.DTE_ERR_ARG, (k, v)
    assert bwd(None, F32, 8, None, 0, 10, 8, 1.0, None, F32, 8, 1, None, 0, None) == B.DTE_OK
    assert bwd(None, F32, 8, None, 4, 0, 8, 1.0, None, F32, 8, 0, None, 0, None) == B.DTE_OK
    assert B.dte_embedding_workspace_bytes(-1, 10, 8) == -1
    assert B.dte_embedding_workspace_bytes(0, 10, 8) == 0
    # partial rows, sorted pairs twice, flags: a bounded share of the gradient
    n, vocab, d = 16384, 151936, 4096
    assert B.dte_embedding_workspace_bytes(n, vocab, d) < n * d + 2 * 8 * n + vocab + (1 << 20)


def ce(**kw):
    c = B.dte_linear_ce(P, P, P, 8, 8, 4, 10, 8, 1.0, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


BAD_CE = [dict(tokens=-1), dict(tokens=1 << 31), dict(vocab=0), dict(vocab=1 << 31), dict(dim=0),
          dict(dim=1 << 20, hidden_ld=1 << 20, weight_ld=1 << 20), dict(hidden_ld=7),
          dict(weight_ld=7), dict(weight_ld=1 << 22), dict(scale=float("nan")), dict(reserved=1)]


@pytest.mark.parametrize("bad", BAD_CE)
def test_linear_ce_bad_sizes(bad):
    c = ce(**bad)
    assert B.dte_linear_ce_workspace_bytes(c, 0) == -1
    assert B.dte_linear_ce_workspace_bytes(c, 1, F32) == -1
    assert st("dte_linear_ce_forward", ctypes.byref(c), P, P, P, 1 << 40, None) == B.DTE_ERR_ARG
    assert st("dte_linear_ce_backward", ctypes.byref(c), P, P, P, 8, P, F32, 8, 0, P, 1 << 40,
              None) == B.DTE_ERR_ARG


def test_linear_ce_arguments():
    c = ce()
    need = B.dte_linear_ce_workspace_bytes(c, 0)
    assert need > 0
    fwd = lambda c, *a: st("dte_linear_ce_forward", ctypes.byref(c), *a)  # noqa: E731
    for name in ("hidden", "weight", "targets"):
        assert fwd(ce(**{name: None}), P, P, P, 1 << 30, None) == B.DTE_ERR_ARG
    assert fwd(c, None, P, P, need, None) == B.DTE_ERR_ARG
    assert fwd(c, P, None, P, need, None) == B.DTE_ERR_ARG
    assert fwd(c, P, P, None, need, None) == B.DTE_ERR_ARG
    assert fwd(c, P, P, P + 128, need, None) == B.DTE_ERR_ARG
    assert fwd(c, P, P, P, need - 1, None) == B.DTE_ERR_ARG
    assert fwd(ce(tokens=0, hidden=None, targets=None), None, None, None, 0, None) == B.DTE_OK
    assert st("dte_linear_ce_forward", None, P, P, P, need, None) == B.DTE_ERR_ARG

    need = B.dte_linear_ce_workspace_bytes(c, 1, F32)
    assert need > B.dte_linear_ce_workspace_bytes(c, 1, BF16) > 0
    assert B.dte_linear_ce_workspace_bytes(c, 1, 2) == -1
    good = [P, P, P, 8, P, F32, 8, 1, P, need, None]
    bwd = lambda *a: st("dte_linear_ce_backward", ctypes.byref(c), *a)  # noqa: E731
    for k, v in ((0, None), (1, None), (3, 7), (5, 5), (5, BF16), (6, 7), (8, None), (8, P + 16),
                 (9, need - 1)):
        bad = list(good)
        bad[k] = v
        assert bwd(*bad) == B.DTE_ERR_ARG, (k, v)
    # nothing wanted
    assert bwd(P, P, None, 0, None, F32, 0, 0, None, 0, None) == B.DTE_OK


def test_linear_ce_workspace_is_bounded_by_pieces_not_logits():
    T, V, d = 8192, 151936, 4096
    c = ce(hidden_ld=d, weight_ld=d, tokens=T, vocab=V, dim=d)
    logits = T * V * 2
    for args in ((0, F32), (1, BF16), (1, F32)):
        assert B.dte_linear_ce_workspace_bytes(c, *args) < logits // 2
    # rows that cannot be read in place cost a packed copy of a piece (and the
    # statistics of the pieces' last, partial tiles)
    odd = ce(hidden_ld=d, weight_ld=d + 1, tokens=T, vocab=V, dim=d)
    more = B.dte_linear_ce_workspace_bytes(odd, 0) - B.dte_linear_ce_workspace_bytes(c, 0)
    assert 0 < more <= (1 << 28) + 64 * 8 * T


def test_orthogonalise_arguments():
    ns = train.newton_schulz()
    need = B.dte_orthogonalise_workspace_bytes(2, 8, 16)
    good = [P, F32, 2, 8, 16, 16, 128, ctypes.byref(ns), P, 16, 128, P, need, None]
    call = lambda *a: st("dte_orthogonalise", *a)  # noqa: E731
    for k, v in ((0, None), (1, 7), (2, -1), (2, 1 << 16), (3, -1), (3, 1 << 16), (4, -1),
                 (5, 15), (6, 127), (7, None), (8, None), (9, 15), (10, 127), (11, None),
                 (11, P + 4), (12, need - 1)):
        bad = list(good)
        bad[k] = v
        assert call(*bad) == B.DTE_ERR_ARG, (k, v)
    for zero in (2, 3, 4):
        a = list(good)
        a[zero] = 0
        a[0] = a[8] = a[11] = None
        assert call(*a) == B.DTE_OK
    assert B.dte_orthogonalise_workspace_bytes(-1, 8, 8) == -1
    assert B.dte_orthogonalise_workspace_bytes(1, 0, 8) == 0


@pytest.mark.parametrize("coefficients,ok", [
    (train.QUINTIC, True), ((1.875, -1.25, 0.375), True), ((16.0, 0.0, 0.0), False),
    ((1.0, 0.0, 0.0), True), ((1.5, -0.5, 0.0), True), ((0.0, 0.0, 0.0), True),
    ((17.0, 0.0, 0.0), False), ((float("nan"), 0.0, 0.0), False), ((1.0, 0.0, 5.0), False),
    # large coefficients that cancel at both ends but not between
    ((200.0, -400.0, 200.0), False),
])
def test_range_of_coefficients(coefficients, ok):
    """The iterates' singular values must stay at or below 16 (16 x: only the
    first of five iterations does)."""
    ns = train.newton_schulz(5, coefficients)
    got = st("dte_orthogonalise", None, F32, 0, 8, 16, 16, 128, ctypes.byref(ns), None, 16, 128,
             None, 0, None)
    assert got == (B.DTE_OK if ok else B.DTE_ERR_ARG)


@pytest.mark.parametrize("field,value", [
    ("lr", -1.0), ("lr", float("nan")), ("momentum", 1.0), ("momentum", -0.1),
    ("weight_decay", float("inf")), ("weight_decay", 1e9), ("update_scale", float("nan")),
    ("reserved", 1)])
def test_muon_arguments(field, value):
    hp = train.MuonStep(lr=1e-3).c()
    call = lambda: st("dte_muon_forward", None, None, None, 0, 4, 4, ctypes.byref(hp), None,  # noqa: E731
                      None, 0, None)
    assert call() == B.DTE_OK
    setattr(hp, field, value)
    assert call() == B.DTE_ERR_ARG


def test_muon_step_structs():
    hp = train.MuonStep(lr=1e-2, weight_decay=0.1, update_scale=3.0, steps=3,
                        coefficients=[(1, 0, 0), (2, 0, 0), (3, -1, 0)])
    c = hp.c()
    assert c.ns.steps == 3 and list(c.ns.coefficients[2]) == [3.0, -1.0, 0.0]
    inv = hp.inverse()
    sc = B.dte_derive_scalars(inv)
    assert sc.rbc2 == 1.0 and sc.eps == 0.0
    assert abs(sc.lrb1 - 0.03) < 1e-8 and abs(sc.decay - 0.999) < 1e-7
    with pytest.raises(ValueError):
        train.MuonStep(lr=1.0, update_scale=-1.0).inverse()
    with pytest.raises(ValueError):
        train.newton_schulz(4, [(1, 0, 0)] * 3)


def test_device_code(tmp_path):
    """No packed binary32 arithmetic, no scalar-cache writes, no scratch, and
    no LDS of the compiler's own beside the products' tiles."""
    import re
    if not os.path.exists(dte_build.hipcc()):
        pytest.skip("hipcc not available")
    flags = [f for f in dte_build.HIPCC_FLAGS if f not in ("-shared", "-fPIC")]
    names = ["embedding", "linear_ce", "orthogonalise"]
    procs = []
    for n in names:
        cmd = [dte_build.hipcc()] + flags + ["--cuda-device-only", "-S", "-o",
                                             str(tmp_path / (n + ".s")),
                                             os.path.join(dte_build.SRC, n + ".hip")]
        procs.append(subprocess.Popen(cmd, stdout=subprocess.DEVNULL, stderr=subprocess.PIPE))
    for p in procs:
        err = p.communicate(timeout=900)[1]
        assert p.returncode == 0, err.decode()[-2000:]
    products = 0
    for n in names:
        text = (tmp_path / (n + ".s")).read_text()
        assert not re.search(r"^\s+v_pk_(add|mul|fma)_f32\b", text, re.M), n
        assert not re.search(r"^\s+s_(store|atomic|buffer_store|scratch_store|dcache_wb|"
                             r"dcache_discard)", text, re.M), n
        meta = text[text.index("amdhsa.kernels:"):]
        for entry in meta.split("\n  - ")[1:]:
            f = dict(re.findall(r"\.(\w+):\s+(\S+)", entry))
            if "name" not in f or "private_segment_fixed_size" not in f:
                continue
            assert int(f["private_segment_fixed_size"]) == 0, f["name"]
            if "product_kernel" in f["name"]:
                products += 1
                assert int(f["group_segment_fixed_size"]) == 0, f["name"]
                assert int(f["vgpr_count"]) <= 256, f["name"]
    assert products >= 20
