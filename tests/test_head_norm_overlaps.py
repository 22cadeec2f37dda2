"""Norms of query and key heads: outputs and the workspace on weights, positions or frequencies are refused (before any
CUDA call), and memory beside them is not.  No GPU: a call that passes the checks ends at the device query, and where
there is a GPU such calls, with made-up addresses, are not made."""
import ctypes

import pytest
import torch

from paper_2605_28283_gb300 import binding as pp
from paper_2605_28283_gb300 import build as ppbuild

A = 0x100000  # an aligned address that nothing dereferences
T, H, HKV, D = 4, 4, 2, 128
Q, K = 2 * H * D, 2 * HKV * D  # bytes of a row, in bf16


@pytest.fixture(scope="module")
def lib():
    ppbuild.build()
    return pp.load()


def call(lib, grad, **kw):
    """Every tensor at an address of its own, unless given."""
    names = ["qg", "kg", "freq", "pos", "q", "k", "gq", "gk", "qo", "ko", "dgq", "dgk", "ws"]
    d = {n: (i + 1) * 16 * A for i, n in enumerate(names)}
    d.update(qs=H * D, dtype=pp.PP_BF16)
    d.update(kw)
    norm, rot = pp.pp_head_norm(1e-6, d["qg"], d["kg"]), pp.pp_rotation(D, 0, 1.0, d["freq"])
    head = (d["dtype"], ctypes.byref(norm), ctypes.byref(rot), d["pos"], T, H, HKV, D, d["q"], H * D, d["k"], HKV * D)
    if grad:
        return lib.pp_head_norm_rope_grad(*head, d["gq"], H * D, d["gk"], HKV * D, d["qo"], d["qs"], d["ko"], HKV * D, d["dgq"],
                                          d["dgk"], d["ws"], 1 << 30, None)
    return lib.pp_head_norm_rope(*head, d["qo"], d["qs"], d["ko"], HKV * D, None)


def passes(lib, grad, **kw):
    """The call gets past the checks."""
    if torch.cuda.is_available():
        pytest.skip("made-up addresses would be launched")
    return call(lib, grad, **kw) == pp.PP_ERR_CUDA


# what an output may not lie on: (name, bytes)
SMALL = [("qg", 2 * D), ("kg", 2 * D), ("freq", 2 * D), ("pos", 4 * T)]


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("name,size", SMALL)
@pytest.mark.parametrize("out,row", [("qo", Q), ("ko", K)])
def test_outputs_on_parameters(lib, grad, name, size, out, row):
    at = 5 * A
    for off in (0, 16 - size, row, T * row - 16):  # at the start, over it, on the second row, at the end
        assert call(lib, grad, **{out: at, name: at + off}) == pp.PP_ERR_INVALID_ARG, off


@pytest.mark.parametrize("name,size", SMALL)
@pytest.mark.parametrize("out", ["dgq", "dgk"])
def test_weight_gradients_on_parameters(lib, name, size, out):
    at = 5 * A
    for off in (0, 16 - size, 4 * D - 16):
        assert call(lib, True, **{out: at, name: at + off}) == pp.PP_ERR_INVALID_ARG, off


@pytest.mark.parametrize("name,size", SMALL + [("q", T * Q), ("k", T * K), ("gq", T * Q), ("gk", T * K), ("qo", T * Q), ("ko", T * K),
                                               ("dgq", 4 * D), ("dgk", 4 * D)])
def test_workspace_on_tensors(lib, name, size):
    ws = 5 * A
    need = pp.pp_head_norm_workspace_size(D)
    for off in (0, 16 - size, need - 16):
        assert call(lib, True, ws=ws, **{name: ws + off}) == pp.PP_ERR_INVALID_ARG, off
    # without gradients of weights it is not looked at
    if name not in ("dgq", "dgk"):
        assert passes(lib, True, ws=ws, dgq=None, dgk=None, **{name: ws})


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("name,size", SMALL)
def test_memory_beside_outputs_and_between_their_rows(lib, grad, name, size):
    at = 5 * A
    for off in (-size, T * Q):
        assert passes(lib, grad, qo=at, **{name: at + off})
    for row in range(T):  # rows twice as far apart
        off = 2 * Q * row + Q
        assert passes(lib, grad, qo=at, qs=2 * H * D, **{name: at + off})
        assert call(lib, grad, qo=at, qs=2 * H * D, **{name: at + off - 16}) == pp.PP_ERR_INVALID_ARG
