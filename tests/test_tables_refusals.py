"""What the tables' calls refuse on the host beside the arguments of test_8bit_refusals (no GPU)."""
import pytest

from test_8bit_refusals import PTR, _tables


@pytest.fixture(scope="module")
def B():
    from paper_2509_16495_amd import binding
    if not binding.is_built():
        import __graft_entry__
        __graft_entry__.build()
    binding.lib()
    return binding


def test_rows_of_chunks_stay_below_the_end_of_32_bits(B):
    """Sums of lengths saturate at 2^31 - 1: with as many rows a sum beyond them would pass for one that fits."""
    call = lambda total, rows, pre: B.lib().shiftattn_tables_append(_tables(B), PTR, pre, total, rows, PTR, PTR, PTR, PTR, B.tables_workspace_bytes(3), None)
    assert call(2 ** 31 - 1, 2 ** 31 - 1, 3) == B.EINVAL and "2^31 - 2" in B.last_error()
    assert call(2 ** 31 - 2, 2 ** 31 - 1, 1) == B.EINVAL and "do not fit" in B.last_error()   # (as before: the decode rows)
