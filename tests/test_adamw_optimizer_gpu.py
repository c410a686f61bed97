"""The optimizer beside captured steps: counts that replays and eager steps both move on."""
import copy

import pytest
import torch

pytestmark = pytest.mark.gpu


def rand(shape, seed, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def make(bits=32, dtype=torch.float32):
    from paper_2505_03983_b200.optim import AdamW
    p = [rand((300,), 1, dtype).requires_grad_(), rand((5, 7), 2, dtype).requires_grad_()]
    for i, q in enumerate(p):
        q.grad = rand(q.shape, 3 + i, dtype)
    return p, AdamW(p, lr=1e-2, weight_decay=0.1, state_bits=bits)


def same(p, opt, q, ref):
    for a, b in zip(p, q):
        assert torch.equal(a, b)
        assert opt.state[a].keys() == ref.state[b].keys()
        for k, v in opt.state[a].items():
            assert torch.equal(v, ref.state[b][k]), k


@pytest.mark.parametrize("bits", [32, 8])
def test_a_captured_step_is_not_split(bits):
    """A replay counts the steps of all that were captured together, so none of them may stand still in an eager step: it is refused, and
    leaves everything as it was.  What else is stepped, eagerly or by replays, counts on."""
    p, opt = make(bits)
    q, ref = make(bits)
    opt.step(), ref.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    graph.replay(), ref.step()
    grad, p[1].grad = p[1].grad, None
    with pytest.raises(RuntimeError, match="captured together"):
        opt.step()
    same(p, opt, q, ref)
    p[1].grad = grad
    graph.replay(), ref.step()
    opt.step(), ref.step()  # all of them together, eagerly
    same(p, opt, q, ref)
    assert opt.state[p[0]]["step"].tolist() == [4, 0] and opt.state[p[0]]["step"] is opt.state[p[1]]["step"]
    # parted from the captured step the optimizer counts them one by one
    opt.load_state_dict(opt.state_dict())
    p[1].grad = q[1].grad = None
    opt.step(), ref.step()
    same(p, opt, q, ref)
    assert int(opt.state[p[0]]["step"][0]) == 5 and int(opt.state[p[1]]["step"][0]) == 4
    # and a step may be captured with the counts apart
    p[1].grad, q[1].grad = grad, grad.clone()
    opt.step(), ref.step()
    second = torch.cuda.CUDAGraph()
    with torch.cuda.graph(second):
        opt.step()
    second.replay(), ref.step()
    same(p, opt, q, ref)
    p[1].grad = q[1].grad = None  # they are counted apart: one of them may stand still
    opt.step(), ref.step()
    p[1].grad, q[1].grad = grad, grad.clone()
    second.replay(), ref.step()
    same(p, opt, q, ref)
    assert int(opt.state[p[0]]["step"][0]) == 9 and int(opt.state[p[1]]["step"][0]) == 7


def test_a_refused_step_changes_nothing():
    """Groups before the one that refuses are not stepped either, and nothing new begins."""
    from paper_2505_03983_b200.optim import AdamW
    p = [rand((20,), i).requires_grad_() for i in range(4)]
    opt = AdamW([{"params": p[:1]}, {"params": p[1:]}], lr=1e-2)
    for q in p[:3]:
        q.grad = torch.ones_like(q)
    opt.step()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        opt.step()
    before = [q.detach().clone() for q in p]
    p[1].grad, p[3].grad = None, torch.ones_like(p[3])
    with pytest.raises(RuntimeError, match="captured together"):
        opt.step()
    assert all(torch.equal(a, b) for a, b in zip(p, before)) and p[3] not in opt.state
    assert int(opt.state[p[0]]["step"][0]) == 1


def test_copies_of_an_optimizer_are_not_captured():
    p, opt = make()
    opt.step()
    with torch.cuda.graph(torch.cuda.CUDAGraph()):
        opt.step()
    for other in (copy.deepcopy(opt), copy.copy(opt).__class__([rand((3,), 1).requires_grad_()])):
        first = other.param_groups[0]["params"]
        first[0].grad = torch.ones_like(first[0])
        for q in first[1:]:
            q.grad = None
        other.step()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_a_parameter_that_is_written_to(dtype):
    """A step begins from what a 16-bit parameter has been set to, and from the master value where it is as the last step left it: against a
    master value that is set beside the parameter."""
    p, opt = make(dtype=dtype)
    q, ref = make(dtype=dtype)
    for _ in range(3):
        opt.step(), ref.step()
    new = rand((150,), 9, dtype)
    nothing = opt.state[p[1]]["master"].clone()
    with torch.no_grad():
        p[0][100:250] = new
        p[1].mul_(1.0)  # written to, and nothing changed: the master's low bits stay
        q[0][100:250] = new
    ref.state[q[0]]["master"][100:250] = new.float()
    opt.step(), ref.step()
    same(p, opt, q, ref)
    assert not torch.equal(nothing, nothing.to(dtype).float())
    assert float((p[0].detach()[100:250] - new).float().abs().max()) <= 2 * 1e-2 * 1.1 + 0.02 * float(new.abs().max())  # one step of lr away
    # a whole network's values at once, as a checkpoint or an average is read in
    net = torch.nn.ParameterList(p)
    values = {k: rand(v.shape, 20, dtype) for k, v in net.state_dict().items()}
    net.load_state_dict(values)
    with torch.no_grad():
        for a, v in zip(q, values.values()):
            a.copy_(v)
            ref.state[a]["master"].copy_(v)
    opt.step(), ref.step()
    same(p, opt, q, ref)
    # through .data no version moves
    for a in (p[0], q[0]):
        a.data.copy_(new.repeat(2))
    opt.refresh_masters()
    ref.state[q[0]]["master"].copy_(new.repeat(2))
    opt.step(), ref.step()
    same(p, opt, q, ref)


def test_a_parameter_that_is_not_a_number():
    """Not a number in the parameter is taken over, and overwritten again."""
    p, opt = make(dtype=torch.bfloat16)
    opt.step()
    with torch.no_grad():
        p[0][3] = float("nan")
    opt.step()
    assert torch.isnan(opt.state[p[0]]["master"][3]) and int(torch.isnan(p[0]).sum()) == 1
    with torch.no_grad():
        p[0][3] = 1.0
    opt.step()
    assert torch.isfinite(p[0]).all() and abs(float(p[0][3]) - 1) < 0.1


def test_values_and_state_are_loaded_in_either_order(tmp_path):
    """The values of a network and the optimizer's state from a checkpoint, one before the other: the same steps; and with the
    values alone steps that begin from them."""
    p, opt = make(dtype=torch.bfloat16)
    for _ in range(3):
        opt.step()
    torch.save([[v.detach() for v in p], opt.state_dict()], tmp_path / "state.pt")
    opt.step()
    for order in (0, 1):
        q, other = make(dtype=torch.bfloat16)
        other.step()
        values, state = torch.load(tmp_path / "state.pt")
        for what in (order, 1 - order):
            if what:
                other.load_state_dict(state)
            else:
                torch.nn.ParameterList(q).load_state_dict({str(i): v for i, v in enumerate(values)})
        other.step()
        same(p, opt, q, other)


def test_a_captured_step_and_a_parameter_that_is_written_to():
    """Replays change parameter and master together; what is written between them is taken over by an eager step."""
    p, opt = make(dtype=torch.bfloat16)
    q, ref = make(dtype=torch.bfloat16)
    opt.step(), ref.step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        opt.step()
    for _ in range(3):
        graph.replay(), ref.step()
    opt.step(), ref.step()
    same(p, opt, q, ref)
    with torch.no_grad():
        for v in (p, q):
            v[0].fill_(0.5)
    opt.step(), ref.step()
    graph.replay(), ref.step()
    same(p, opt, q, ref)
    for a in p:
        assert torch.equal(a, opt.state[a]["master"].to(a.dtype))
