"""GPU tests of the form of the rotation as a cache keeps it, and of the norms' largest eps, against the float64 references of
tests/test_gpu_paged_forms.py."""
import numpy as np
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


@pytest.mark.parametrize("dtype,hd", [("bf16", 64), ("f32", 64), ("f32", 16)])
@pytest.mark.parametrize("eps", [1e-6, 1e30, 1e38, 3e38, float(np.finfo(np.float32).max)])
def test_means_and_eps_whose_sum_passes_fp32(binding, dtype, hd, eps):
    """Heads of 1, 1e15, and mean squares at, near and far above eps."""
    sizes = [1.0, 1e15, 1e18, 1.5e19, 1.8e19, 3e19, 1e20, 1e30]
    c = make(binding, page=16, n_pages=2, max_seqs=1, max_ctx=32, max_rows=4, heads=8, kv=8, hd=hd, dtype=dtype, rope_base=10000.0)
    c.plan(ints([0]), ints([3]), ints([2]), rows=2)
    g = torch.Generator(device="cuda").manual_seed(hd)
    x = (torch.randn(2, 8, hd, generator=g, device="cuda") * torch.tensor(sizes, device="cuda")[:, None]).to(c.dtype)
    gain, out = torch.randn(hd, generator=g, device="cuda"), torch.empty_like(x)
    pools = [torch.zeros(c.pool_shape, device="cuda", dtype=c.dtype) for _ in range(2)]
    c.append(x, x, x, out, *pools, q_gain=gain, k_gain=gain, eps=eps)
    keys = pools[0].transpose(1, 2).reshape(-1, 8, hd)[c.row_slot[:2].long()]
    for got in (out, keys):
        check(host(got), host(x), host(gain), float(np.float32(eps)), [3, 4], angles(hd), "half", c.dtype)
