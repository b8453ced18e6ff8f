"""None where a call of shared prefixes, accumulated weights or eviction needs a tensor is a ValueError."""
import pytest

from tests.test_cache_binding import evict, prompt, shared, weights
from tests.test_window_binding import kv  # noqa: F401  (fixture)


@pytest.mark.parametrize("call,name", [(shared, n) for n in ("q", "bt", "lens", "out", "ws")]
                         + [(weights, n) for n in ("q", "bt", "lens", "out", "w", "ws")]
                         + [(prompt, n) for n in ("q", "cu", "ctx", "bt", "w", "pos", "ws")]
                         + [(evict, n) for n in ("lens", "bt", "nextp", "w", "pos", "nextl")])
def test_refused(kv, call, name):  # noqa: F811
    with pytest.raises(ValueError):
        call(kv, **{name: None})
