"""What the binding's classes for the expert sublayer do on the host: no GPU is needed (addresses are never followed)."""
import pytest

from paper_2601_21198_b200 import build


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def test_capture_id_wants_somewhere_to_put_it(zb):
    assert zb._lib.zipmoe_stream_capture_id(None, None) == zb.ERR_INVALID_ARG
