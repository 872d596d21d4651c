"""GPU tests of the form of the rotation as a cache keeps it, against the float64 references of tests/test_gpu_paged_forms.py."""
import pytest

from tests.test_gpu_paged import host, ints, make
from tests.test_gpu_paged_forms import angles, check

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


@pytest.fixture(scope="module")
def binding():
    from paper_2403_00835_amd import binding as b
    return b


@pytest.mark.parametrize("form", [dict(), dict(layout="interleaved", dim=20), dict(scaling="linear", factor=4.0), dict(base=10000.0)])
def test_the_base_is_the_caches_unless_one_is_given(binding, form):
    c = make(binding, page=16, n_pages=20, max_seqs=1, max_ctx=300, max_rows=40, heads=4, kv=2, hd=64, dtype="f32", rope_base=500000.0)
    c.rotary(**form)
    c.plan(ints([0]), ints([200]), ints([40]), rows=40)
    q, k = torch.randn(40, 4, 64, device="cuda"), torch.randn(40, 2, 64, device="cuda")
    out, pools = torch.empty_like(q), [torch.zeros(c.pool_shape, device="cuda") for _ in range(2)]
    c.append(q, k, k, out, *pools)
    kw = {"base": 500000.0, **{x: form[x] for x in form if x in ("base", "scaling", "factor")}}
    check(host(out), host(q), None, 0, list(range(200, 240)), angles(form.get("dim", 64), **kw), form.get("layout", "half"), c.dtype)
