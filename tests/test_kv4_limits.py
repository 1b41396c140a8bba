"""Lengths at which the 4-bit cache attention's 32-bit positions end, on the CPU: refused before anything is enqueued."""
import pytest

from paper_2604_26412_gb300 import build as kbuild
from paper_2604_26412_gb300 import kvshot
from tests.test_kv4_boundary import SHAPE, UNSUPPORTED, _attn

NULL = kvshot.KVSHOT_ERR_NULL
LONG = dict(num_caches=1, num_seqs=1, hkv=1, hq=4, page_size=1 << 20, max_pages_per_seq=2047, num_pages=1)
ROOM = 2047 << 20  # tokens of a full table


@pytest.fixture(scope="module", autouse=True)
def lib():
    kbuild.build()


@pytest.mark.parametrize("kw,code", [
    # (what the limits let pass ends at the missing q)
    (dict(max_seq_len=ROOM), NULL), (dict(max_seq_len=2 ** 31 - 1), NULL),
    (dict(max_seq_len=2 ** 31 - 1, page_size=16, max_pages_per_seq=2 ** 27 - 1), UNSUPPORTED),
    (dict(max_seq_len=2 ** 31 - 16, page_size=16, max_pages_per_seq=2 ** 27 - 1), UNSUPPORTED),
    (dict(max_seq_len=2 ** 31 - 129 - 16, page_size=16, max_pages_per_seq=2 ** 27 - 1), NULL),
    (dict(max_seq_len=2 ** 31 - 129 - 15, page_size=16, max_pages_per_seq=2 ** 27 - 1), UNSUPPORTED),
    (dict(max_seq_len=ROOM, n_nodes=10 ** 6, n_max=10 ** 6, tree=False), UNSUPPORTED),
    (dict(max_seq_len=ROOM, n_nodes=500_000, n_max=500_000, tree=False), NULL),
    (dict(max_seq_len=2 ** 31 - 16, ptrs=dict(pt=None), l_cap=2 ** 31 - 16), UNSUPPORTED),
    (dict(max_seq_len=-1), SHAPE),
])
def test_lengths_at_the_end_of_32_bits(kw, code):
    kw = {**LONG, **kw}
    kw["ptrs"] = {"q": None, **kw.get("ptrs", {})}
    assert _attn(**kw) == code
