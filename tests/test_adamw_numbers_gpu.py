"""The optimiser's numbers of steps on the device: before, in and after a captured graph."""
import pytest
import torch

from paper_1611_08035_b200.adamw import AdamW

pytestmark = pytest.mark.gpu
U = 2.0**-24
LR = 2.0**-7  # the same in fp32
STATES = ("m", "v", "sm", "sv")


def make(capturable=False):
    g = torch.Generator(device="cuda").manual_seed(3)
    params = [torch.nn.Parameter(0.1 * torch.randn(s, device="cuda", generator=g)) for s in ((300, 130), (7,), (5000,))]
    for p in params:
        p.grad = torch.zeros_like(p)
    return params, AdamW(params, lr=LR, betas=(0.9, 0.99), capturable=capturable)


def alike(a, b, opt_a, opt_b, steps):
    """Moments, whose random rounding goes by the step's number, to the bit; the step's factors come from the host or the device in fp64, rounded to fp32: a last place apart, each step."""
    for p, q in zip(a, b):
        for k in STATES:
            if k in opt_a.state[p]:
                assert torch.equal(opt_a.state[p][k].view(torch.uint8), opt_b.state[q][k].view(torch.uint8)), k
        assert float((p - q).detach().abs().max()) <= steps * 4 * U * float(q.detach().abs().max() + 2 * LR)


def test_set_after_steps_and_taken_back(b2):
    """Two ordinary steps, one with the numbers on the device, three replays, and two ordinary ones: as eight ordinary ones."""
    grads = [[torch.randn(s, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)) for s in ((300, 130), (7,), (5000,))] for i in range(8)]

    def put(params, gs):
        for p, g in zip(params, gs):
            p.grad.copy_(g)

    (a, eager), (b, opt) = make(), make()
    for gs in grads:
        put(a, gs)
        eager.step()
    for gs in grads[:2]:
        put(b, gs)
        opt.step()
    opt.param_groups[0]["capturable"] = True
    torch.cuda.synchronize()
    with pytest.raises(RuntimeError, match="captured"):
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            opt.step()
    put(b, grads[2])
    opt.step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        opt.step()
    for gs in grads[3:6]:
        put(b, gs)
        graph.replay()
    torch.cuda.synchronize()
    opt.param_groups[0]["capturable"] = False
    opt.param_groups[0]["lr"] = LR
    for gs in grads[6:]:
        put(b, gs)
        opt.step()
    torch.cuda.synchronize()
    alike(a, b, eager, opt, 8)
    assert b2.b2_device_status() == 0


@pytest.mark.parametrize("where", ["cpu", "cuda"])
def test_saved_in_between(b2, where):
    """A capturable optimiser after a replay, saved, loaded to the host or the device and captured again: as the one that goes on."""
    import io
    (a, opt), (b, other) = make(capturable=True), make()
    for p in a:
        p.grad.normal_()
    opt.step()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        opt.step()
    graph.replay()
    file = io.BytesIO()
    torch.save(opt.state_dict(), file)
    file.seek(0)
    other.load_state_dict(torch.load(file, map_location=where))
    with torch.no_grad():
        for p, q in zip(a, b):
            q.copy_(p), q.grad.copy_(p.grad)
    graph.replay()
    other.step()
    again = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(again):
        other.step()
    for _ in range(2):
        graph.replay(), again.replay()
    torch.cuda.synchronize()
    assert all(int(st["step"]) == 5 for o in (opt, other) for st in o.state.values())
    assert all(torch.equal(p, q) for p, q in zip(a, b))
    for p, q in zip(a, b):
        assert all(torch.equal(opt.state[p][k].view(torch.uint8), other.state[q][k].view(torch.uint8)) for k in STATES if k in opt.state[p])
