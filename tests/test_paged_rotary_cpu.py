"""PagedCache.rotary's own arguments, on a cache whose library only counts its calls."""
import pytest

from paper_2403_00835_amd import binding
from tests.test_paged_binding_cpu import cache  # noqa: F401
from tests.test_paged_forms_cpu import counted

torch = pytest.importorskip("torch")


@pytest.mark.parametrize("form", [dict(), dict(layout="interleaved", dim=8), dict(scaling="linear", factor=8.0)])
def test_the_base_is_the_caches_unless_one_is_given(cache, form):  # noqa: F811
    c = counted(cache)
    c.rope_base = 500000.0
    c.rotary(**form)
    c.rotary(**form, base=10000.0)
    assert [x[1][1]._obj.base for x in c.calls] == [500000.0, 10000.0]


def test_a_cache_without_rotation_has_no_base(cache):  # noqa: F811
    assert binding.PagedCache.rope_base == 0.0
    c = counted(cache)
    c.rotary()  # (the library refuses it: there are no factors to make again)
    assert c.calls[0][1][1]._obj.base == 0.0
