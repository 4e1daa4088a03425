"""tt_cache_append on the host: as many requests as a CTA's threads can share out."""
from test_lib_append import append, lib  # noqa: F401

UNSUPPORTED = 2


def test_too_many_requests_are_refused(lib):  # noqa: F811
    """The list of requests is cut into runs by numbers of 32 bits."""
    far = 1 << 40  # (outputs away from the inputs)
    for B in ((1 << 30) + 1, (1 << 31) - 256, (1 << 31) - 1):
        assert append(lib, B=B, new_len=far, status=2 * far) == UNSUPPORTED
        assert append(lib, B=B, new_len=far, status=2 * far, max_len=0, page_table=None) == UNSUPPORTED
