"""The layer operators at the ends of what they take."""
import ctypes
import types

import pytest
import torch

import paper_2609_14706_amd as ffe

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


# few tokens, k split over 16 and 4 parts and joined, tiles alone
@pytest.mark.parametrize("T,m", [(3, 5), (40, 5), (70, 5), (1000, 1000), (2048, 2048)])
def test_q8_sums_of_two_to_the_31(gpu, T, m):
    """131072 products of (-128)^2 are 2^31 exactly, one more than 32 bits hold."""
    n = 131072
    q = torch.full((T, n), -128, dtype=torch.int8, device=gpu)
    Z = torch.full((m, n), -128, dtype=torch.int8, device=gpu)
    q[1] = 127
    Z[2] = 127
    q[T - 1, n - 1] = -127
    y = ffe.linear_q8(q, torch.ones(T, device=gpu), Z, torch.ones(m, device=gpu))
    rows, cols = torch.full((T,), -128.0, dtype=torch.float64), torch.full((m,), -128.0, dtype=torch.float64)
    rows[1], cols[2] = 127, 127
    want = rows[:, None] * cols * n
    want[T - 1] += cols
    assert torch.equal(y.cpu(), want.to(BF16))


def _calls(gpu):
    """One call of each function that takes a stream."""
    x, W, G = torch.ones(40, 64, dtype=BF16, device=gpu), torch.ones(48, 64, dtype=BF16, device=gpu), torch.eye(20, device=gpu)
    w, dy = torch.ones(64, dtype=BF16, device=gpu), torch.ones(40, 48, dtype=BF16, device=gpu)
    q, Z = torch.ones(40, 64, dtype=torch.int8, device=gpu), torch.ones(48, 64, dtype=torch.int8, device=gpu)
    one, beta = torch.ones(40, device=gpu), torch.ones(48, device=gpu)
    return [lambda **k: ffe.rms_norm(x, w, **k), lambda **k: ffe.rms_norm_q8(x, w, **k), lambda **k: ffe.quantize_rows(x, **k),
            lambda **k: ffe.rms_norm_backward(x, x, w, **k), lambda **k: ffe.linear(x, W, **k),
            lambda **k: ffe.linear_q8(q, one, Z, beta, **k), lambda **k: ffe.linear_backward(dy, x, W, **k),
            lambda **k: ffe.orthogonalize(G, **k)]


@pytest.mark.parametrize("which", range(8))
def test_a_stream_of_another_device(gpu, which):
    call = _calls(gpu)[which]
    with pytest.raises(ValueError, match="stream"):
        call(stream=types.SimpleNamespace(device=torch.device("cuda", 1), cuda_stream=0))
    with pytest.raises(TypeError, match="stream"):
        call(stream=7)


def test_results_outlive_their_use_on_the_callers_stream(gpu):
    """A result of another stream that the caller's stream still reads is not
    handed to the next call on that other stream."""
    x, W = torch.ones(1536, 512, dtype=BF16, device=gpu), torch.ones(1408, 512, dtype=BF16, device=gpu)
    s = torch.cuda.Stream(gpu)
    s.wait_stream(torch.cuda.current_stream(gpu))
    y, _ = ffe.linear(x, W, stream=s)
    torch.cuda.current_stream(gpu).wait_stream(s)
    torch.cuda._sleep(100_000_000)    # some 50 ms
    copy = y.clone()                  # behind it
    taken = y.data_ptr()
    del y
    again, _ = ffe.linear(x, W, stream=s)
    assert again.data_ptr() != taken
    torch.cuda.synchronize()
    assert torch.equal(copy, again)


HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}    # half a unit of a rounded value
SUMS = 2.0 ** -16                                # fp32 sums, relative to the sum of magnitudes
DT = {"bf16": BF16, "f32": torch.float32}


def _rows(gpu, n, dtype, eps):
    """Rows over all of the type's range that eps leaves a norm of any size to."""
    g = torch.Generator().manual_seed(n)
    sizes = torch.tensor([1e-36, 1e-30, 1e-24, 1e-19, 1e-12, 1.0, 1e12, 1e19, 1e24, 1e30, 1e37, 3.0], dtype=torch.float64)
    x = torch.randn(12, n, generator=g, dtype=torch.float64) * sizes[:, None]
    x[11, 0] = 1e30           # one large entry among others
    return x.to(DT[dtype]).to(gpu)


# rows of a wave, of a workgroup of every kind, too long for registers
@pytest.mark.parametrize("n", [5, 700, 1500, 3000, 8192, 9000, 16000, 40000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("eps", [0.0, 1e-70, 1e-6, 1e50])
def test_norms_of_rows_of_any_size(gpu, n, dtype, eps):
    x = _rows(gpu, n, dtype, eps)
    g = torch.Generator().manual_seed(n + 1)
    dy = torch.randn(12, n, generator=g).to(DT[dtype]).to(gpu)
    w = (torch.rand(n, generator=g) + 0.5).to(DT[dtype]).to(gpu)
    x64, w64, u = x.double(), w.double(), dy.double() * w.double()
    i = 1 / torch.sqrt(x64.square().mean(-1, keepdim=True) + eps)
    tiny = 1e-37              # what lies below the normal numbers of both types
    want = x64 * i * w64
    y, _ = ffe.rms_norm(x, w, eps=eps)
    assert bool(((y.double() - want).abs() <= (HALF[dtype] + SUMS) * want.abs() + tiny).all())
    q, scale, _ = ffe.rms_norm_q8(x, w, eps=eps)
    top = want.abs().amax(-1)
    some = top > 1e-35        # (a scale below the normal numbers counts as zeros)
    assert bool((scale.double() - top / 127)[some].abs().le(SUMS * top[some] / 127).all())
    assert bool((q.double() * scale.double()[:, None] - want)[some].abs().le(0.51 * top[some][:, None] / 127).all())
    ds, dw = ffe.rms_norm_backward(dy, x, w, eps=eps)
    mean = (u * x64).mean(-1, keepdim=True)
    want = i * (u - x64 * i * i * mean)
    mag = i * (u.abs() + x64.abs() * i * i * (u * x64).abs().mean(-1, keepdim=True))
    fits = mag.amax(-1) < 1e38
    off = (ds.double() - want).abs() <= HALF[dtype] * want.abs() + SUMS * mag + tiny
    assert bool(off[fits].all())
    share = dy.double() * x64 * i
    assert bool(((dw.double() - share.sum(0)).abs() <= HALF[dtype] * share.sum(0).abs() + SUMS * share.abs().sum(0) + tiny).all())


@pytest.mark.parametrize("n", [64, 700, 40000])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("eps", [1e-300, 1e-50, 1e-30, 1e300])
def test_zero_rows_with_any_eps(gpu, n, dtype, eps):
    """An eps that fp32 does not hold still keeps rows of zeros zeros."""
    x = torch.zeros(7, n, dtype=DT[dtype], device=gpu)
    w = torch.ones(n, dtype=DT[dtype], device=gpu)
    assert not bool(ffe.rms_norm(x, w, eps=eps)[0].any())
    q, scale, _ = ffe.rms_norm_q8(x, w, eps=eps)
    assert not bool(q.any()) and not bool(scale.any())
    ds, dw = ffe.rms_norm_backward(x, x, w, eps=eps)
    assert not bool(ds.any()) and not bool(dw.any())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("m,n", [(40, 50), (128, 128), (300, 200)])
def test_updates_with_any_eps(gpu, m, n, dtype):
    """An eps that fp32 does not hold: zeros stay zeros, tiny updates keep their size beside it."""
    for eps in (1e-300, 1e-50, 1e300):
        assert not bool(ffe.orthogonalize(torch.zeros(m, n, dtype=DT[dtype], device=gpu), eps=eps).any())
    g = torch.Generator().manual_seed(m)
    G = (1e-30 * torch.randn(m, n, generator=g)).to(DT[dtype]).to(gpu)
    assert torch.equal(ffe.orthogonalize(G, eps=1e-60), ffe.orthogonalize(G, eps=0.0))
    assert not bool(ffe.orthogonalize(G, eps=1e300).any())
    with pytest.raises(ffe.FlipFlopError):
        ffe.orthogonalize(G, scale=1e39)


def test_what_is_no_tensor(gpu):
    x, W, dy = (torch.ones(*s, dtype=BF16, device=gpu) for s in ((4, 64), (48, 64), (4, 48)))
    for bad in (7, [1.0], "x", dy.cpu()):
        for call in (lambda: ffe.rms_norm(x, residual=bad), lambda: ffe.rms_norm(x, bad),
                     lambda: ffe.rms_norm_backward(bad, x), lambda: ffe.rms_norm_backward(x, x, dsum=bad),
                     lambda: ffe.linear(x, bad), lambda: ffe.linear(x, W, residual=bad), lambda: ffe.linear(x, W, bias=bad),
                     lambda: ffe.linear_backward(bad, x, W), lambda: ffe.linear_backward(dy, x, bad),
                     lambda: ffe.linear_backward(dy, x, W, preact=bad, activation="silu"), lambda: ffe.orthogonalize(bad)):
            with pytest.raises(TypeError, match="CUDA tensor"):
                call()


@pytest.mark.parametrize("into", ["s", "dy", "dsum"])
@pytest.mark.parametrize("rows,n", [(1100, 40), (1100, 700), (5000, 1500), (600, 3000), (600, 40000)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_gradient_in_place(gpu, rows, n, dtype, into):
    """ds in the place of an input, rows that have to be scaled among rows whose
    gradients are as small or as large as those."""
    g = torch.Generator(gpu).manual_seed(n)
    sizes = torch.tensor([1.0, 1e25, 1e-25, 0.0], device=gpu)[torch.randint(0, 4, (rows, 1), device=gpu, generator=g)]
    x = (torch.randn(rows, n, device=gpu, generator=g) * sizes).to(DT[dtype])
    small = torch.tensor([1e-24, 1.0], device=gpu)[torch.randint(0, 2, (rows, 1), device=gpu, generator=g)]
    dy, dsum = ((torch.randn(rows, n, device=gpu, generator=g) * small).to(DT[dtype]) for _ in range(2))
    w = torch.ones(n, dtype=DT[dtype], device=gpu)
    want, want_dw = ffe.rms_norm_backward(dy, x, w, eps=1e-60, dsum=dsum)
    t = {"s": x.clone(), "dy": dy.clone(), "dsum": dsum.clone()}
    dw = torch.empty_like(w)
    ws = torch.empty(512 * n, dtype=torch.float32, device=gpu)
    a = ffe.ff_norm_grad_args(rows, n, int(dtype == "bf16"), t["s"].data_ptr(), n, t["dy"].data_ptr(), n, t["dsum"].data_ptr(), n,
                              w.data_ptr(), 1e-60, t[into].data_ptr(), n, dw.data_ptr(), ws.data_ptr(), ws.numel() * 4,
                              torch.cuda.current_stream(gpu).cuda_stream)
    assert ffe.load_library().ff_rms_norm_backward(ctypes.byref(a)) == ffe.FF_OK
    assert torch.equal(t[into].nan_to_num(7.0), want.nan_to_num(7.0)) and torch.equal(dw.nan_to_num(7.0), want_dw.nan_to_num(7.0))
