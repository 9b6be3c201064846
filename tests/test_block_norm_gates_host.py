"""How many workgroups the gradients of norms with gates of their own have: one gate more does not leave half of a card of 256 compute units idle.
No GPU is needed."""
import re

import pytest

from paper_2409_11902_amd import binding as B


def workgroups(D, rows, gates):
    d = B.make_block_norm_desc(rows * gates, D, post=B.NORM_RMS, pre=B.NORM_LAYER, gate_rows=rows)
    return int(re.match(r"(\d+) workgroups", B.cac_block_norm_describe_plan(d, B.BLOCK_NORM_BWD)).group(1))


@pytest.mark.parametrize("D,rows,gates", [(2048, 49, 256), (1024, 16, 512), (4608, 196, 128), (512, 49, 1024), (16384, 49, 128)])
def test_one_gate_more(D, rows, gates):
    assert workgroups(D, rows, gates - 1) >= 250 and workgroups(D, rows, gates) >= workgroups(D, rows, gates - 1)


@pytest.mark.parametrize("D,rows,gates,slots", [(128, 49, 4095, 32), (2048, 1, 5000, 2), (512, 7, 2048, 8), (2048, 49, 512, 2)])
def test_many_gates_are_shared_out_among_slots(D, rows, gates, slots):
    assert workgroups(D, rows, gates) == min(256, -(-gates // slots))
