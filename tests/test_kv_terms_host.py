"""The tolerances of tests/test_gpu_kv_terms.py see what they are meant to see: a low term left out of the float64 form."""
import pytest

from tests import kv_terms as K


@pytest.mark.parametrize("what, fmt, G, shared", K.ALL)
def test_a_missing_term_would_show(what, fmt, G, shared):
    t = K.Terms(what, fmt, G, shared, seed=G)
    cos, sin = (x.double() for x in K.tables(K.ROWS))
    if what == "window":
        assert t.differs("key", cos, sin) and t.differs("query", cos, sin)
    else:
        assert t.differs("digit" if fmt == "i8" else "query", cos, sin)
