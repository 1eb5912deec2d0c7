"""driver.paged4_step over whole prompts: lengths that are not the numbers of rows are refused with the index checks on, before anything
is stored (the attention of whole prompts sees the call's own rows alone)."""
import pytest
import torch

from paper_2609_29812_amd import driver
from paper_2609_29812_amd import flashloop as fl


@pytest.fixture
def calls(monkeypatch):
    made = []
    monkeypatch.setattr(fl, "paged4_append", lambda *a, **kw: made.append("append"))
    monkeypatch.setattr(fl, "packed_attn", lambda *a, **kw: made.append("packed"))
    monkeypatch.setattr(fl, "paged4_attn", lambda *a, **kw: made.append("cache"))
    on = fl.index_checks()
    yield made
    fl.set_index_checks(on)


def step(lens, whole):
    x = torch.zeros(5, 2, 64, dtype=torch.bfloat16)
    driver.paged4_step((None,) * 4, x, x, x, torch.tensor([0, 2, 5], dtype=torch.int32), torch.tensor(lens, dtype=torch.int32), None, whole=whole)


def test_whole_prompts_have_as_many_rows_as_positions(calls):
    fl.set_index_checks(True)
    assert fl.index_checks()
    step([2, 3], True)
    assert calls == ["append", "packed"]
    for lens in ([2, 4], [9, 3], [1, 3]):
        with pytest.raises(fl.FlashLoopError, match="FL_E_RANGE"):
            step(lens, True)
    assert calls == ["append", "packed"]
    step([2, 4], False)
    assert calls[2:] == ["append", "cache"]


def test_nothing_is_looked_at_with_the_checks_off(calls):
    fl.set_index_checks(False)
    assert not fl.index_checks()
    step([2, 4], True)
    assert calls == ["append", "packed"]
