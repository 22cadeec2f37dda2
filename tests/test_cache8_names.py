"""Names of the 8-bit cache's calls in the binding: both sets, and every name that the case files call (no GPU)."""
import os
import re

import pytest

from paper_2605_28283_gb300 import binding as pp

PERF = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "perf")


@pytest.mark.parametrize("first,now", [("alloc_attn8_workspace", "alloc_kvq_workspace"), ("pp_kv8_append", "pp_kvq_append"),
                                       ("pp_kv8_read", "pp_kvq_read"), ("pp_tree_attention8", "pp_kvq_tree_attention"),
                                       ("pp_kv8_commit", "pp_kvq_commit")])
def test_both_names_are_one_call(first, now):
    assert getattr(pp, first) is getattr(pp, now)


@pytest.mark.parametrize("name", ["operators.py", "more_operators.py"])
def test_case_files_call_what_exists(name):
    text = open(os.path.join(PERF, name)).read()
    called = set(re.findall(r"\bpp\.(\w+)", text))
    assert called and not [n for n in sorted(called) if not hasattr(pp, n)]
