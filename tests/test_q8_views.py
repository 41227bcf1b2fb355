"""Which views of keys, values, queries and outputs the binding takes."""
import pytest
import torch

from paper_2601_20357_amd import binding

view = binding._heads_view


def test_strides_of_a_single_row_or_token_do_not_count():
    """A part of a wider row and a tensor of its own are the same to a call of one row and one token, of one token each, or of one row."""
    for rows, T in ((1, 1), (1, 5), (4, 1)):
        wide = torch.zeros(rows, T, 3 * 256)
        part, own = wide[:, :, 256:512], torch.zeros(rows, T, 256)
        if rows == 1 and T == 1:
            assert view(part, rows, T, 4, 64, "k")[1:] == view(own, rows, T, 4, 64, "v")[1:] == (256, 256)
        elif T == 1:
            assert view(part, rows, T, 4, 64, "k")[1:] == (768, 256) and view(own, rows, T, 4, 64, "k")[1:] == (256, 256)
        else:
            assert view(part, rows, T, 4, 64, "k")[2] == 768 and view(own, rows, T, 4, 64, "k")[2] == 256
    step = torch.zeros(4, 7, 256)[:, 3:4]                              # a token of longer rows, and the same rows side by side
    assert view(step, 4, 1, 4, 64, "k")[1:] == (7 * 256, 256)
    for t, rows, T in ((torch.zeros(1, 1, 255), 1, 1), (torch.zeros(1, 3, 256).expand(1, 3, 256)[:, :1].expand(1, 3, 256), 1, 3)):
        with pytest.raises(binding.TabedError):
            view(t, rows, T, 4, 64, "k")
