"""The table of the buffers that updates are scattered into: the kernels know the plan's sizes alone, so tensors that do not have
them are refused when the table is made."""
import pytest
import torch

import paper_2608_00455_b200 as dte


def layout(*numels):
    lay = dte.Layout.__new__(dte.Layout)              # sizes and device only: no handle, no GPU
    lay.device, lay.shard_numels = torch.device("cpu"), list(numels)
    return lay


def shards(*numels):
    return [None if n is None else torch.empty(n, dtype=torch.bfloat16) for n in numels]


def test_tensors_of_the_plan_are_taken():
    t = shards(64, None, 0, 9)
    table = layout(64, 128, 0, 5).shard_table(t)
    assert [p or 0 for p in table] == [t[0].data_ptr(), 0, t[2].data_ptr(), t[3].data_ptr()]
    assert len(layout().shard_table([])) == 1         # never an empty array
    assert layout(64).shard_table([torch.empty(64, dtype=torch.int16)])[0]


@pytest.mark.parametrize("plan,given,word", [((64,), (63,), "shard 0"), ((64, 8), (64, 0), "shard 1"), ((64, 8), (64,), "2 shards"),
                                             ((64, 8), (), "2 shards")])
def test_tensors_smaller_than_the_plan_and_short_tables_are_refused(plan, given, word):
    with pytest.raises(ValueError, match=word):
        layout(*plan).shard_table(shards(*given))
