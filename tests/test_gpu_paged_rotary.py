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


@pytest.mark.parametrize("own", [dict(), dict(dim=32), dict(layout="interleaved", dim=20)], ids=["whole", "part", "neighbours"])
@pytest.mark.parametrize("norms", [False, True])
def test_a_captured_append_behind_another_form(binding, own, norms):
    """The factors of another layout or width are not those that the graph reads by its own: it does nothing and the status
    says so, until the form is its own again. Appends that are called, and plans, go on in between."""
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        c = make(binding, page=16, n_pages=20, max_seqs=2, max_ctx=300, max_rows=40, heads=4, kv=2, hd=64, dtype="f32", rope_base=10000.0)
        q, k = torch.randn(40, 4, 64, device="cuda"), torch.randn(40, 2, 64, device="cuda")
        gain, out = torch.randn(64, device="cuda") if norms else None, torch.empty_like(q)
        pools = [torch.zeros(c.pool_shape, device="cuda") for _ in range(2)]

        def step():
            c.plan(ints([0]), ints([200]), ints([40]), rows=40)
            c.append(q, k, k, out, *pools, q_gain=gain, k_gain=gain)

        def right(form):
            keys = pools[0].transpose(1, 2).reshape(-1, 2, 64)[c.row_slot[:40].long()]
            for got, raw in ((out, q), (keys, k)):
                check(host(got), host(raw), host(gain) if norms else None, 1e-6, list(range(200, 240)), angles(form.get("dim", 64)),
                      form.get("layout", "half"), c.dtype)

        seq, ctx, new = ints([0]), ints([200]), ints([40])
        c.rotary(**own)
        step()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            c.plan(seq, ctx, new, rows=40)
            c.append(q, k, k, out, *pools, q_gain=gain, k_gain=gain)
        for other in (dict(dim=16), dict(layout="interleaved"), dict(layout="interleaved", dim=32), dict(dim=20)):
            c.rotary(**other)
            for x in (out, *pools):
                x.fill_(9)
            graph.replay()
            with pytest.raises(binding.CllmError, match="ERR_STATE.*form of the rotation"):
                c.status()
            assert all((x == 9).all() for x in (out, *pools))
            step()
            assert c.status()[0] == 40
            right(other)
            c.rotary(**own)
            graph.replay()
            assert c.status()[0] == 40
            right(own)
        side.synchronize()
        del graph
