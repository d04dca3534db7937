"""A training step through the differentiable layers, captured: forward and backward pass in
one graph, replayed with other inputs, weights and experts' shares."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    from paper_2202_06819_amd import build, linear
    build.ensure_built()
    return linear


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("tokens", [5, 130])
def test_a_captured_training_step(L, tokens, residual):
    g = torch.Generator(device="cuda").manual_seed(tokens)

    def randn(*shape):
        return torch.randn(*shape, generator=g, device="cuda")
    c, k, experts = 136, 88, 5
    values = {"x": randn(tokens, c).bfloat16(), "h": randn(tokens, c).bfloat16(), "gain": 1 + 0.1 * randn(c),
              "w": randn(c, c) * 0.1, "we": randn(experts, k, c) * 0.1}
    offsets = torch.linspace(0, tokens, experts + 1, device="cuda").to(torch.int32)
    dz, dtotal = randn(tokens, k).bfloat16(), randn(tokens, c).bfloat16()

    def step(leaves):
        h = leaves["h"] if residual else None
        y, total = L.norm_linear_layer(leaves["x"], leaves["gain"], leaves["w"], residual=h)
        z = L.experts_layer(y, leaves["we"], offsets)
        wanted = [t for n, t in leaves.items() if residual or n != "h"]
        grads = torch.autograd.grad([z, total] if residual else [z], wanted, [dz, dtotal] if residual else [dz])
        return [z.detach(), total.detach(), *grads]
    # (the capture has leaves of its own: no other graph of them lives)
    leaves = {n: t.clone().requires_grad_() for n, t in values.items()}
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(leaves)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step(leaves)
    for turn in range(4):
        if turn:
            for n, t in leaves.items():
                values[n] = (randn(*t.shape) * (0.1 if n[0] == "w" else 1.0)).to(t.dtype)
                t.data.copy_(values[n])
            dz.copy_(randn(tokens, k))
            offsets[1:-1] = torch.randint(0, tokens + 1, (experts - 1,), generator=g, device="cuda").sort().values
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        want = step({n: t.clone().requires_grad_() for n, t in values.items()})
        assert len(got) == len(want) and all(torch.equal(a, b) for a, b in zip(got, want))
        assert all(torch.isfinite(t).all() for t in got) and got[-1].any()
