"""The longest block tables that the block-scaled calls take: the end of a context's last tile of 128 keys, and of the two pages
that an append may look past its last one, still are int32 positions."""

import pytest

from test_block_refusals import append, attend


@pytest.fixture(scope="module")
def wc():
    import paper_2607_28699_gb300 as w
    return w


LONGEST = 2 ** 27 - 64      # pages: 2^31 - 1024 positions


@pytest.mark.parametrize("call", [append, attend, lambda wc, **kw: attend(wc, extend=True, **kw)])
@pytest.mark.parametrize("pages", [LONGEST + 1, 2 ** 27 - 8, 2 ** 27 - 1])
def test_refused(wc, call, pages):
    # the bound is checked before anything that these calls lack
    st, message = call(wc, mp=pages, bt=None)
    assert st == 2 and b"max_pages" in message


@pytest.mark.parametrize("call", [append, attend, lambda wc, **kw: attend(wc, extend=True, **kw)])
def test_taken(wc, call):
    st, message = call(wc, mp=LONGEST, bt=None)
    assert st == 1 and b"block_table" in message


def test_ends_fit():
    keys = 16 * LONGEST
    assert (keys + 127) // 128 * 128 + 128 < 2 ** 31 and keys + 3 * 16 < 2 ** 31
