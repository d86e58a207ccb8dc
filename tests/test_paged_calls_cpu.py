"""Calls of the paged-cache operators that do nothing, which need no device either."""
from test_paged_cpu import attend, lib, ragged, write  # noqa: F401 (lib is a fixture)


def test_a_batch_of_none_needs_no_arrays(lib):  # noqa: F811
    """No sequences: the arrays have no elements, and a framework's tensors of none have no address."""
    none = ragged(B=0, seq_lens=None, block_table=None)
    assert write(lib, r=none) == 0 and write(lib, r=none, read=True) == 0 and attend(lib, r=none) == 0
    assert write(lib, r=ragged(B=1, seq_lens=None)) == -2
