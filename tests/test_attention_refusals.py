"""Host-only checks of arguments that the attention calls must not take at their word: the binding's and the entry
points' refusals beyond those of tests/test_attention_args.py. Fake device pointers are never read."""
import pytest

import paper_2607_02525_amd as P

torch = pytest.importorskip("torch")


def test_tables_whose_rows_overlap_are_refused():
    """A row expanded to all sequences, or rows closer than they are wide, have no stride that the calls take."""
    i32 = torch.int32
    row = torch.arange(6, dtype=i32)
    for t in (row[None].expand(3, -1), row.as_strided((3, 4), (1, 1)), row[None, :1].expand(4, -1)):
        with pytest.raises(ValueError, match="overlap"):
            P._table(t, t.shape[0])
    # rows of any stride from their width on get as far as the check for a device tensor, as do single and empty ones
    wide = torch.zeros(3, 9, dtype=i32)
    for t in (wide, wide[:, :4], wide[::2], wide[:1, :4], row[None].expand(1, -1), torch.zeros(3, 0, dtype=i32)):
        with pytest.raises(ValueError, match="device tensor"):
            P._table(t, t.shape[0])
