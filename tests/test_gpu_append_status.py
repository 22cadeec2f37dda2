"""GPU tests of what the append records on the device."""
import numpy as np
import pytest

from test_gpu_attention import to_dev
from test_gpu_cache import AppendCase

pytestmark = pytest.mark.gpu


def test_append_reports_sequences_that_no_token_belongs_to(pp):
    """Lengths that cannot be right are recorded also for a sequence without new tokens, and where the starts descend
    behind the last token; the other sequences are appended."""
    import torch
    for how in ("ctx_negative", "ctx_long", "descending"):
        c = AppendCase([(2, 30), (0, 4), (3, 9)], 4, 2, 64, 16, "f32", 64, "half")
        _, wk, wv, _, tc = c.want(c.default_pos)
        if how == "ctx_negative":
            c.ctx[1] = -1
        elif how == "ctx_long":
            c.ctx[1] = 16 * c.pages.shape[1] + 1
        else:
            # a fourth sequence that ends before it begins
            c.starts = np.append(c.starts, 4).astype(np.int32)
            c.ctx = np.append(c.ctx, 0).astype(np.int32)
            c.pages = np.concatenate([c.pages, c.pages[:1]])
        cache, batch, rot = c.device(pp)
        ws = pp.alloc_attn_workspace(cache)
        q = to_dev(c.q)
        pp.pp_kv_append(cache, batch, rot, None, q, to_dev(c.k), to_dev(c.v), torch.empty_like(q), ws)
        assert pp.pp_get_device_status(ws) == pp.PP_ERR_INVALID_ARG, how
        if how != "descending":
            assert (np.abs(cache.k.cpu().numpy() - wk) <= tc).all(), how
            assert np.array_equal(cache.v.cpu().numpy(), wv), how


def test_append_reports_nothing_for_padding_and_empty_sequences(pp):
    for pad in (0, 5):
        AppendCase([(0, 0), (2, 30), (0, 4), (0, 0), (3, 9), (0, 0)], 4, 2, 64, 16, "bf16", 64, "half", pad=pad).check(pp)
        AppendCase([(0, 1)] * 70 + [(1, 3)] + [(0, 2)] * 70, 2, 1, 64, 16, "bf16", 64, "half", pad=pad).check(pp)
