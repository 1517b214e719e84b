"""The operators together, as examples/answer_from_memory.py calls them."""
import os
import sys

import pytest

pytestmark = pytest.mark.gpu

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("kw", [dict(n_layers=3, frames=12, question=5, answer=3, group_tokens=50, q_heads=14, kv_heads=2, hidden=256, top_k=4),
                                dict(n_layers=2, frames=7, question=40, answer=2, group_tokens=9, q_heads=4, kv_heads=4, head_dim=64, hidden=128, top_k=16)])
def test_stored_shortened_forked_and_asked(kw):
    sys.path.insert(0, os.path.join(ROOT, "examples"))
    try:
        import answer_from_memory as example
    finally:
        sys.path.pop(0)
    r = example.main(**kw)
    assert r["kept"] == kw["frames"] - kw["frames"] // 4 and r["forked"] == min(8, r["kept"]) and r["finite"]
    # the buffer's rows are rounded to bfloat16, scores of a few units so move by 2^-7 and outputs by as much and 2^-8
    assert max(r["apart"]) <= 0.03
