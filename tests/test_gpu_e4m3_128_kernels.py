"""Every kernel of the products with a scale per 128, each with its tiles and cuts along K, against 64 bits: shapes and
choice in gemm128_shapes.py, problems and tolerances as in test_gpu_e4m3_128.py."""
import pytest
import torch

from .gemm128_shapes import CODES, GATED, PLAIN, choice, flat
from .gpu_helpers import lib_ready
from .test_gpu_e4m3_128 import Problem, check, check_codes, count, gated_exact, run_gated, run_gemm

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    return lib_ready()


def sms():
    return torch.cuda.get_device_properties(0).multi_processor_count


def name(s):
    return "%s%d-cut%d-%dx%dx%d" % s


@pytest.mark.parametrize("shape", flat(PLAIN), ids=name)
def test_gemm_of_every_kernel(H, shape):
    kernel, rows, k, n = shape[:3], *shape[3:]
    assert choice(rows, k, n, num_sms=sms()) == kernel
    p = Problem(rows, k, n)
    want, off = p.exact()
    for out in ("f32", "bf16", "f16"):
        check(run_gemm(H, p, out), want, off, out, out)


@pytest.mark.parametrize("shape", flat(GATED), ids=name)
def test_gated_of_every_kernel(H, shape):
    kernel, rows, k, n = shape[:3], *shape[3:]
    assert choice(rows, k, n, gated=True, num_sms=sms()) == kernel
    p = Problem(rows, k, n, two=True)
    for act, outs in (("silu", ("f32", "bf16")), ("gelu", ("f16",))):
        h, off = gated_exact(p, act)
        for out in outs:
            check(run_gated(H, p, act, out)[0], h, off, out, out)


@pytest.mark.parametrize("shape", flat(CODES), ids=name)
def test_gated_to_codes_of_every_kernel(H, shape):
    kernel, rows, k, n = shape[:3], *shape[3:]
    assert choice(rows, k, n, gated=True, codes=True, num_sms=sms()) == kernel
    p = Problem(rows, k, n, two=True)
    for act in ("silu", "gelu"):
        h, off = gated_exact(p, act)
        y, sc = run_gated(H, p, act, "e4m3")
        check_codes(y, sc, h, off)
        assert (sc[:, rows:] == -7).all()


def counted(shape, **kw):
    """A problem of the shape's capacity of which the device counts fewer rows, with strides of its own and NaN codes and
    scales behind the rows and in the padding: the last tile of rows is short, or not there."""
    rows, k, n = shape[3:]
    spare = rows // 3 if rows > 2 else 0
    return Problem(rows - spare, k, n, spare=spare, pad=48, **kw)


@pytest.mark.parametrize("shape", [s[-1] for s in ([(*k, *v) for v in shapes] for k, shapes in PLAIN.items())], ids=name)
def test_gemm_counts_rows_in_every_kernel(H, shape):
    p = counted(shape)
    assert choice(p.cap, p.k, p.n, num_sms=sms()) == shape[:3]
    want, off = p.exact()
    for out, opad in (("bf16", 16), ("f32", 32)):
        y = run_gemm(H, p, out, n_rows=count(p.rows), opad=opad)
        check(y[:p.rows, :p.n], want, off, out)
        assert (y[p.rows:] == 3).all() and (y[:, p.n:] == 3).all()
    y = run_gemm(H, p, "f32", n_rows=count(0))
    assert (y == 3).all()


@pytest.mark.parametrize("codes,shape", [(t is CODES, (*k, *shapes[-1])) for t in (GATED, CODES) for k, shapes in t.items()],
                         ids=lambda v: name(v) if isinstance(v, tuple) else "codes" if v else "bits")
def test_gated_counts_rows_in_every_kernel(H, codes, shape):
    p = counted(shape, two=True)
    assert choice(p.cap, p.k, p.n, gated=True, codes=codes, num_sms=sms()) == shape[:3]
    h, off = gated_exact(p, "gelu")
    for out, opad in (("e4m3", 16), ("e4m3", 32)) if codes else (("bf16", 16), ("f32", 32)):
        y, sc = run_gated(H, p, "gelu", out, n_rows=count(p.rows), opad=opad)
        if codes:
            check_codes(y[:, :p.n], sc, h, off)
            assert (sc[:, p.rows:] == -7).all()
        else:
            check(y[:p.rows, :p.n], h, off, out)
        assert (y[p.rows:] == 3).all() and (y[:, p.n:] == 3).all()


@pytest.mark.parametrize("shape", [(*k, *shapes[0]) for k, shapes in PLAIN.items()], ids=name)
def test_every_kernel_repeats_itself_and_replays(H, shape):
    """Bit for bit: eagerly with another problem in between, and from a graph whose inputs change under it."""
    rows, k, n = shape[3:]
    p, q = Problem(rows, k, n), Problem(rows, k, n, seed=1)
    want, other = run_gemm(H, p, "f32"), run_gemm(H, q, "f32")
    y = torch.zeros_like(want)
    for _ in range(5):
        run_gemm(H, q, "f32", into=y)
        assert torch.equal(y, other)
        run_gemm(H, p, "f32", into=y)
        assert torch.equal(y, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for _ in range(3):
            run_gemm(H, p, "f32", into=y)
    graph.replay()
    assert torch.equal(y, want)
    p.a.copy_(q.a)
    p.a_scale.copy_(q.a_scale)
    p.w[0].copy_(q.w[0])
    p.w_scale[0].copy_(q.w_scale[0])
    p.bias[0].copy_(q.bias[0])
    graph.replay()
    assert torch.equal(y, other)


@pytest.mark.parametrize("shape", [(*k, *shapes[-1]) for k, shapes in CODES.items()], ids=name)
def test_every_gated_kernel_repeats_itself(H, shape):
    rows, k, n = shape[3:]
    p, q = Problem(rows, k, n, two=True), Problem(rows, k, n, two=True, seed=1)
    (y, sc), (z, sz) = run_gated(H, p, "silu", "e4m3"), run_gated(H, q, "silu", "e4m3")
    into = torch.zeros_like(y), torch.zeros_like(sc)
    for _ in range(5):
        for problem, codes, scales in ((q, z, sz), (p, y, sc)):
            run_gated(H, problem, "silu", "e4m3", into=into)
            assert torch.equal(into[0], codes) and torch.equal(into[1][:, :rows], scales[:, :rows])
