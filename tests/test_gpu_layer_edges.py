"""The layer operators at the ends of what they take."""
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
