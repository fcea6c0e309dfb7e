"""What the Python binding refuses of shared prefixes and norms with rotation: tensors that hold fewer entries, or others, than
the call reads or writes (no GPU: every refusal comes before the device is asked)."""
import pytest
import torch

import paper_2607_28069_amd as pic

def test_token_rows_refuse_one_row_for_all():
    """A step of 0 from token to token stands for dense rows in the call, which would read past the one row there is."""
    one = torch.zeros(1, 4, 64)
    for t in (one.expand(5, 4, 64), one.expand(2, 5, 4, 64)):
        with pytest.raises(ValueError, match="one place"):
            pic._token_rows(t, 4, 64, "q", -1)
    assert pic._token_rows(one, 4, 64, "q", -1)[1] == 0
    assert pic._token_rows(torch.zeros(0, 4, 64), 4, 64, "q", -1)[0] is not None
