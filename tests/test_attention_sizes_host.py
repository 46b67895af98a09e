"""Sizes past 32 bits are refused by the attention calls before anything is planned with them (no GPU).

Each case runs in a process of its own: a wrapped tile count once ended the caller's in a division by zero."""
import os
import subprocess
import sys

import pytest

pytest.importorskip("paper_2208_01944_gb300.binding", reason="libpalquant.so not built")
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
from paper_2208_01944_gb300 import binding as B
v = dict(type=1, B=2, Hq=4, max_q=1, max_len=32, causal=1, window=0, table_pitch=2, scale=0.1, q_token_stride=256,
         q_head_stride=64, o_token_stride=256, o_head_stride=64, cu_q_dev=64, len_dev=64, page_table_dev=64)
v.update({changes})
a = B.KV8Attn(*[v[n] for n, _ in B.KV8Attn._fields_])
c = B.KV8Cache(4, 16, 2, 64, 64, 64, 64, 64)
assert B.palquant_kv8_attention_scratch_bytes(c, a) == 0
try:
    B.palquant_kv8_attention(c, 64, 64, a, 64, 1 << 62, stream=0)
except B.PalquantError as e:
    assert e.status == B.PQ_EUNSUPPORTED, e
else:
    raise AssertionError("not refused")
"""


def _refused(**changes):
    subprocess.run([sys.executable, "-c", PROGRAM.format(changes=changes)], cwd=ROOT, check=True)


ROWS = [dict(type=0, Hq=128, max_q=1 << 30), dict(Hq=128, max_q=1 << 30), dict(max_q=0x7FFFFFFF), dict(B=0x7FFFFFFF, max_q=0x7FFFFFFF),
        dict(type=2, B=1 << 20, Hq=128, max_q=1 << 10), dict(type=0, B=1, Hq=128, max_q=1 << 25, max_len=1 << 20)]


@pytest.mark.parametrize("changes", ROWS, ids=str)
def test_too_many_query_rows(changes):
    _refused(**changes)


@pytest.mark.parametrize("changes", [dict(max_len=(1 << 30) + 1), dict(max_len=0x7FFFFFFF), dict(type=0, max_len=0x7FFFFFFF, window=5),
                                     dict(B=1, Hq=2, max_q=(1 << 30) - 1, max_len=0x7FFFFF80)], ids=str)
def test_positions_past_the_parts_ends(changes):
    _refused(**changes)
