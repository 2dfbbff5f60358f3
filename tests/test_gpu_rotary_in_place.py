"""The backward pass in the memory of the incoming gradient: the same bits as elsewhere, whatever the input gradient holds."""
import pytest
import torch

import helpers

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    return helpers.api()


@pytest.mark.parametrize("pairs", [0, 8, 16])
@pytest.mark.parametrize("head", [33, 64, 100])
@pytest.mark.parametrize("shape", [(1, 1), (1, 3), (5, 7), (67, 3), (331, 5)])
def test_gradient_in_place(api, shape, head, pairs):
    """Rows (tokens x heads) that are no multiple of what a CTA takes at a time; the last ones' input gradients are beyond
    f16's range, so that what is stored over dY is infinite, while the weight gradients are finite."""
    T, H = shape
    g = torch.Generator(device="cuda")
    g.manual_seed(T * H + head)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, dy = randn(T, H, head), randn(T, H, head) * 50
    x[-1] *= 1e-4
    x, dy, w = x.half(), dy.half(), (1 + 0.1 * randn(head)).half()
    pos = torch.arange(T, dtype=torch.int32, device="cuda") * 7
    handle = api.Handle()
    info = api.TensorInfo(handle, api.F16, x.shape, x.stride())
    op = api.Rotary(handle, [0.3 / (i + 1) for i in range(pairs)], info, info, norm=True, eps=1e-12)
    ws = torch.empty(op.workspace_size(), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream

    def backward(dx, dy):
        dw = torch.full((head,), float("nan"), device="cuda")
        op.backward(stream, pos.data_ptr(), w.data_ptr(), 0, x.data_ptr(), dy.data_ptr(), dx.data_ptr(), dWq=dw.data_ptr(),
                    workspace=ws.data_ptr(), workspace_bytes=ws.numel())
        torch.cuda.synchronize()
        return dx, dw

    dx, dw = backward(torch.empty_like(dy), dy)
    assert torch.isinf(dx[-1]).any() and torch.isfinite(dw).all()
    for _ in range(5):
        there = dy.clone()
        same, dw_there = backward(there, there)
        assert torch.equal(same.view(torch.int16), dx.view(torch.int16))
        assert torch.equal(dw_there.view(torch.int32), dw.view(torch.int32))
