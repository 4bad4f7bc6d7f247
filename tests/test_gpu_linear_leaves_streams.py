"""Outputs that the leaf and softmax calls make for themselves, on a stream that is not the current one."""
import pytest
import torch

from test_gpu_linear_leaves import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("handle", [False, True])
def test_made_outputs_belong_to_the_calls_stream(handle):
    """The current stream is busy for some 100 ms: what is done there comes long after the call's work on the other."""
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, offs, idx = make(900, [300, 0, 500], 40, 24, "f32", seed=1)
    y = torch.randint(0, 24, (900,), generator=torch.Generator().manual_seed(2), dtype=torch.int32).cuda()

    def calls(stream):
        out = [B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b, stream=stream)]
        out += B.gbdt_leaf_product_grad(dy, x, w, offs, row_idx=idx, stream=stream)
        loss, lse = B.gbdt_softmax_loss(x, w[0, :, :40], y, stream=stream)
        out += [loss, lse, *B.gbdt_softmax_grad(x, w[0], y, lse, stream=stream)]
        return out + list(B.gbdt_softmax_stats(x, w[0], y, lse, 3, 9, stream=stream))
    want = calls(None)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls(None)  # (its memory is there from here on)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    got = calls(side.cuda_stream if handle else side)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, e) for a, e in zip(got, want))
    assert int((want[0] != 0).any(1).sum()) == 800 and int((want[1] != 0).any(1).sum()) == 800


def test_the_default_streams_handle():
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, offs, idx = make(90, [30, 0, 50], 40, 24, "bf16", seed=3)
    want = B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = B.gbdt_leaf_product(x, w, offs, row_idx=idx, bias=b, stream=0)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
