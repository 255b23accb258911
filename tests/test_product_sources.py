"""The products' reads of a tensor that is not the library's: none behind its last row, none left out."""
from test_host_indexing import needs_hipcc, run_host_program

pytestmark = needs_hipcc


def test_rows_of_any_length_are_read_whole_and_nothing_behind_them(tmp_path):
    word, reads = run_host_program(tmp_path, "product_sources")
    assert word == "ok" and int(reads) > 10 ** 6
