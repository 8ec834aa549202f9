"""A cache and a call's sequences hold the addresses of their tensors: the tensors cannot be replaced in them, where the old ones' memory would be read on after it
was freed.  No GPU: stand-ins for tensors, and nothing reaches the library.
"""
import pytest

from test_more_operator_arguments import I32, SEQUENCES, WIDE, Stub, cache, sequences

NAMES = [(cache, name) for name in ("k", "v", "k_scales", "v_scales", "pages", "heads", "page_tokens", "head_dim", "device", "_struct")] + \
        [(sequences, name) for name in ("starts", "lengths", "table", "device", "_struct")]


@pytest.mark.parametrize("make, name", NAMES)
def test_what_they_hold_stays(make, name):
    held = make()
    before = getattr(held, name)
    with pytest.raises(AttributeError):
        setattr(held, name, before)
    with pytest.raises(AttributeError):
        delattr(held, name)
    assert getattr(held, name) is before


def test_addresses_are_the_tensors():
    class At(Stub):
        def __init__(self, *args, at):
            super().__init__(*args)
            self.at = at

        def data_ptr(self):
            return self.at

    held = sequences(At((SEQUENCES + 1,), I32, at=0x10), At((SEQUENCES,), I32, at=0x20), At((SEQUENCES, WIDE), I32, at=0x30))
    told = held._struct
    assert (told.d_starts, told.d_lengths, told.d_table) == tuple(t.data_ptr() for t in (held.starts, held.lengths, held.table)) == (0x10, 0x20, 0x30)
