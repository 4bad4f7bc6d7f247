"""The calls of routed rows and of codes on other streams, in captured graphs, with a registered workspace, on tensors of another
device."""
import pytest
import torch

from test_gpu_mixture import made

pytestmark = pytest.mark.gpu


def calls(B, x, dy, w, b, leaves, gates, logits, codes, stream=None):
    k = leaves.shape[1]
    out = list(B.gbdt_route(logits, k, stream=stream))
    out.append(B.gbdt_route_grad(logits, out[0], gates, stream=stream))
    out.append(B.gbdt_mixture_product(x, w, leaves, gates, bias=b, stream=stream))
    out += B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, bias=b, stream=stream)
    c, s = B.gbdt_rows_quantize(x, stream=stream)
    wq, ws = codes
    out += [c, s, B.gbdt_mixture_product_codes(c, s, wq, ws, leaves, gates, dtype=x.dtype, stream=stream)]
    offs = torch.tensor([0, 5, x.shape[0] - 3] + [x.shape[0] - 3] * (w.shape[0] - 2), dtype=torch.int64, device="cuda")
    out.append(B.gbdt_leaf_product_codes(c, s, wq, ws, offs, dtype=x.dtype, stream=stream))
    return out


def inputs(n, dtype="bf16", seed=1, d_out=72):
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, leaves, gates = made(n, 3, 9, 96, d_out, dtype, seed=seed, outside=0.0)
    logits = torch.randn(n, 9, generator=torch.Generator().manual_seed(seed)).cuda()
    wq, ws = B.gbdt_rows_quantize(w.view(-1, 96))
    return x, dy, w, b, leaves, gates, logits, (wq.view(9, d_out, -1), ws.view(9, d_out))


@pytest.mark.parametrize("handle", [False, True])
@pytest.mark.parametrize("n", [3, 900])
def test_another_stream(handle, n):
    """The current stream is busy for some 100 ms: what is done there comes long after the call's work on the other."""
    from paper_1706_08359_amd import binding as B
    data = inputs(n)
    want = calls(B, *data)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        calls(B, *data)  # (its memory is there from here on)
    torch.cuda.synchronize()
    torch.cuda._sleep(200_000_000)
    with torch.cuda.stream(side):
        got = calls(B, *data, stream=side.cuda_stream if handle else side)
    side.synchronize()
    torch.cuda.synchronize()
    assert all(torch.equal(a, e) for a, e in zip(got, want))


@pytest.mark.parametrize("n", [3, 900, 6000])
def test_two_captured_graphs_share_the_scratch(n):
    """Each replayed several times, with eager work between, and on inputs that change in place."""
    from paper_1706_08359_amd import binding as B
    one, two = inputs(n, seed=2), inputs(n + 50, dtype="f32", seed=3)
    calls(B, *two), calls(B, *one)
    torch.cuda.synchronize()
    graphs = []
    for data in (one, two):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = list(B.gbdt_route(data[6], 3))
            out.append(B.gbdt_route_grad(data[6], out[0], data[5]))
            out.append(B.gbdt_mixture_product(data[0], data[2], data[4], data[5], bias=data[3]))
            out += B.gbdt_mixture_product_grad(data[1], data[0], data[2], data[4], data[5], bias=data[3])
            c, s = B.gbdt_rows_quantize(data[0])
            out += [c, s, B.gbdt_mixture_product_codes(c, s, *data[7], data[4], data[5])]
        graphs.append((g, data, out))

    def eager(data):
        out = list(B.gbdt_route(data[6], 3))
        out.append(B.gbdt_route_grad(data[6], out[0], data[5]))
        out.append(B.gbdt_mixture_product(data[0], data[2], data[4], data[5], bias=data[3]))
        out += B.gbdt_mixture_product_grad(data[1], data[0], data[2], data[4], data[5], bias=data[3])
        c, s = B.gbdt_rows_quantize(data[0])
        return out + [c, s, B.gbdt_mixture_product_codes(c, s, *data[7], data[4], data[5])]
    gen = torch.Generator().manual_seed(5)
    for turn in range(4):
        for _, data, _ in graphs:
            data[6].copy_(torch.randn(data[6].shape, generator=gen).cuda())
            data[4].copy_(torch.randint(-1, 9, data[4].shape, generator=gen, dtype=torch.int32).cuda())
            data[5].copy_(torch.rand(data[5].shape, generator=gen).cuda())
        want = [eager(data) for _, data, _ in graphs]
        for g, _, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (_, _, out), w in zip(graphs, want):
            assert all(torch.equal(a, e) for a, e in zip(out, w)), turn


def test_a_registered_workspace():
    from paper_1706_08359_amd import binding as B
    for n, dtype, d_out in ((900, "bf16", 72), (9000, "f32", 40)):
        data = inputs(n, dtype=dtype, seed=4, d_out=d_out)
        want = calls(B, *data)
        size = B.gbdt_mixture_workspace_bytes(n, 3, 9, 96, d_out, data[0].dtype)
        own = torch.zeros(size + 4096, dtype=torch.uint8, device="cuda")
        own[size:] = 77
        B.gbdt_set_workspace(own[:size])
        try:
            got = calls(B, *data)
            torch.cuda.synchronize()
            assert bool((own[size:] == 77).all())
        finally:
            B.gbdt_set_workspace(None)
        assert all(torch.equal(a, e) for a, e in zip(got, want))
        small = torch.zeros(1 << 19, dtype=torch.uint8, device="cuda")
        B.gbdt_set_workspace(small)
        try:
            with pytest.raises(B.GbdtError, match="workspace"):
                B.gbdt_mixture_product_grad(data[1], data[0], data[2], data[4], data[5])
        finally:
            B.gbdt_set_workspace(None)


def test_more_rows_than_are_held_at_once_within_the_stated_scratch():
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, leaves, gates = made(70_000, 4, 6, 40, 520, "bf16", seed=6, outside=0.0)
    want = B.gbdt_mixture_product(x, w, leaves, gates, bias=b)
    size = B.gbdt_mixture_workspace_bytes(70_000, 4, 6, 40, 520, torch.bfloat16)
    assert size < 70_000 * 4 * 520 * 2 + (400 << 20)
    own = torch.zeros(size, dtype=torch.uint8, device="cuda")
    B.gbdt_set_workspace(own)
    try:
        assert torch.equal(B.gbdt_mixture_product(x, w, leaves, gates, bias=b), want)
    finally:
        B.gbdt_set_workspace(None)


def test_wrong_tensors_are_refused():
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, leaves, gates, logits, (wq, ws) = inputs(20)
    c, s = B.gbdt_rows_quantize(x)
    bad = [
        lambda: B.gbdt_route(logits.cpu(), 2), lambda: B.gbdt_route(logits.half(), 2), lambda: B.gbdt_route(logits, 10),
        lambda: B.gbdt_route(logits, 2, score="other"), lambda: B.gbdt_route(logits, 2, choice_bias=logits[0, :8].contiguous()),
        lambda: B.gbdt_route(logits, 2, n_groups=2), lambda: B.gbdt_route(logits.t(), 2),
        lambda: B.gbdt_route(logits, 2, gates_out=torch.zeros(20, 3, device="cuda")), lambda: B.gbdt_route(logits, 2, scale=float("inf")),
        lambda: B.gbdt_route_grad(logits, leaves.long(), gates), lambda: B.gbdt_route_grad(logits, leaves, gates[:19]),
        lambda: B.gbdt_mixture_product(x.float(), w, leaves, gates), lambda: B.gbdt_mixture_product(x, w[:, :, :95], leaves, gates),
        lambda: B.gbdt_mixture_product(x, w, leaves[:19], gates[:19]), lambda: B.gbdt_mixture_product(x, w, leaves, gates.double()),
        lambda: B.gbdt_mixture_product(x, w, leaves, gates, bias=b[:, :71]), lambda: B.gbdt_mixture_product(x, w, leaves.t(), gates.t()),
        lambda: B.gbdt_mixture_product_grad(dy, x, w, leaves, gates, want=("x", "y")),
        lambda: B.gbdt_mixture_product_grad(dy[:, :71], x, w, leaves, gates),
        lambda: B.gbdt_rows_quantize(x, codes_out=torch.zeros(20, 90, dtype=torch.int8, device="cuda")),
        lambda: B.gbdt_rows_quantize(x.cpu()), lambda: B.gbdt_mixture_product_codes(c[:, :80], s, wq, ws, leaves, gates),
        lambda: B.gbdt_mixture_product_codes(c, s, wq[:, :, :95], ws, leaves, gates),
        lambda: B.gbdt_mixture_product_codes(c, s, wq, ws, leaves, gates, dtype=torch.float16),
        lambda: B.gbdt_mixture_product_codes(c, s.double(), wq, ws, leaves, gates),
        lambda: B.gbdt_leaf_product_codes(c, s, wq, ws, torch.zeros(9, dtype=torch.int64, device="cuda")),
    ]
    for i, call in enumerate(bad):
        with pytest.raises((TypeError, B.GbdtError)):
            call()
            pytest.fail(str(i))


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The check itself, without a second device: what counts as current is another number here."""
    from paper_1706_08359_amd import binding as B
    x, dy, w, b, leaves, gates, logits, (wq, ws) = inputs(20)
    c, s = B.gbdt_rows_quantize(x)
    offs = torch.zeros(10, dtype=torch.int64, device="cuda")
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 1)
    for call in (lambda: B.gbdt_route(logits, 2), lambda: B.gbdt_route_grad(logits, leaves, gates),
                 lambda: B.gbdt_mixture_product(x, w, leaves, gates), lambda: B.gbdt_mixture_product_grad(dy, x, w, leaves, gates),
                 lambda: B.gbdt_rows_quantize(x), lambda: B.gbdt_leaf_product_codes(c, s, wq, ws, offs),
                 lambda: B.gbdt_mixture_product_codes(c, s, wq, ws, leaves, gates)):
        with pytest.raises(B.GbdtError, match="current device"):
            call()
