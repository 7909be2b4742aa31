"""The operators run together, as a training step uses them, and the model that does so."""
import types

import numpy as np
import pytest
import torch

import oracle
from paper_2312_08728_b200 import operators as ops
from paper_2312_08728_b200.network import GatedSoftmax
from test_gpu_adamw import Job
from test_gpu_operators import Block, check_residual

pytestmark = pytest.mark.gpu


def sample(N, p, C, dtype, seed=0):
    """Classes around C centres: something to learn."""
    gen = torch.Generator().manual_seed(seed)
    centres = torch.randn(C, p, generator=gen)
    y = torch.randint(0, C, (N,), generator=gen, dtype=torch.int32)
    return (centres[y.long()] + 0.7 * torch.randn(N, p, generator=gen)).to(dtype), y


@pytest.mark.parametrize("p,hidden,C,n,dtype,bits", [(24, 40, 5, 32, torch.bfloat16, 32), (33, 70, 10, 100, torch.float16, 32),
                                                     (64, 128, 16, 256, torch.bfloat16, 8), (200, 301, 10, 300, torch.bfloat16, 32)])
def test_steps_of_a_round_operator_by_operator(p, hidden, C, n, dtype, bits):
    """Three mini-batches: the rows are those of the shuffle, and every operator's result is within its bound of the definition
    on the inputs that it was given."""
    x, y = sample(3 * n - 7, p, C, dtype)
    x, y = x.cuda(), y.cuda()
    net = GatedSoftmax(x.shape[0], p, 1, hidden, C, dtype=dtype, state_bits=bits, weight_decay=0.05, max_norm=0.7, seed=3)
    pi = torch.from_numpy(oracle.perm(9, 0, 0, x.shape[0]).astype(np.int64)).cuda()
    for k in range(3):
        count = min(n, x.shape[0] - k * n)
        bx, by = ops.gather_batch(x, y, 9, 0, 0, k * n, count)
        rows = pi[k * n:k * n + count]
        assert torch.equal(bx, x[rows]) and torch.equal(by, y[rows])
        b = Block.__new__(Block)
        b.x, (b.wg, b.wu, b.wd), b.act, b.dtype = bx, net.weights, net.activation, dtype
        logits, saved = ops.gated_ffn(bx, *net.weights, net.activation, save=True)
        residual, loss = check_residual(logits, by)
        b.dy = residual
        dx, *grads = ops.gated_ffn_backward(residual, bx, *net.weights, saved, net.activation)
        b.check({"y": logits, "dx": dx, "dw_gate": grads[0], "dw_up": grads[1], "dw_down": grads[2]})
        job = Job.__new__(Job)
        job.params, job.masters, job.grads, job.state, job.bits, job.seed, job.t = net.weights, net.masters, grads, net.state, bits, 3, k
        job.decays = [0.05] * 3
        before = job.before()
        norm = float(torch.sqrt(sum(g.double().square().sum() for g in grads)))
        net_loss = net.step(bx, by, 1e-2)
        assert torch.equal(net_loss, loss)
        job.check(before, gscale=min(1.0, 0.7 / (norm + 1e-6)))
    net.sync()


def test_rounds_over_buffers_are_the_steps_in_a_row():
    """run_rounds over two slots, a resident buffer and step by step: the same bits."""
    p, hidden, C, n = 40, 64, 7, 48
    x, y = sample(400, p, C, torch.bfloat16)
    parts = [(x[:200].pin_memory(), y[:200].pin_memory()), (x[200:].pin_memory(), y[200:].pin_memory())]
    nets = [GatedSoftmax(400, p, 2, hidden, C, seed=1) for _ in range(3)]
    copy = torch.cuda.Stream()
    slot = nets[0].load_buffer(*parts[0], stream=copy)
    for k in range(4):  # two passes over two buffers
        following = nets[0].load_buffer(*parts[(k + 1) % 2], stream=copy) if k < 3 else None
        nets[0].run_rounds(slot, 2, n, 1e-2, seed=70 + k)
        slot = following
        dx, dy = (t.cuda() for t in parts[k % 2])
        nets[1].run_rounds_resident(dx, dy, 2, n, 1e-2, seed=70 + k)
        for t in range(2):
            pi = torch.from_numpy(oracle.perm(70 + k, 0, t, 200).astype(np.int64)).cuda()
            for first in range(0, 200, n):
                nets[2].step(dx[pi[first:first + n]], dy[pi[first:first + n]], 1e-2)
    nets[0].sync()
    for a, b, c in zip(*(net.get_theta() for net in nets)):
        assert torch.equal(a, b) and torch.equal(a, c)


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_captured_into_a_graph(bits):
    x, y = sample(128, 48, 6, torch.bfloat16)
    x, y = x.cuda(), y.cuda()
    nets = [GatedSoftmax(128, 48, 1, 96, 6, state_bits=bits, seed=2, max_norm=1.0) for _ in range(2)]
    nets[0].step(x, y, 1e-2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = nets[0].step(x, y, 1e-2)
    for _ in range(4):
        graph.replay()
    for _ in range(5):
        want = nets[1].step(x, y, 1e-2)
    torch.cuda.synchronize()
    assert torch.equal(loss, want)
    for a, b in zip(nets[0].get_theta(), nets[1].get_theta()):
        assert torch.equal(a, b)


def test_refusals():
    net = GatedSoftmax(100, 16, 2, 32, 4)
    x, y = sample(50, 16, 4, torch.bfloat16)
    with pytest.raises(Exception):
        net.run_rounds(0, 1, 10, 1e-3, 0)               # nothing loaded
    with pytest.raises(Exception):
        net.load_buffer(torch.cat([x, x]), torch.cat([y, y]))  # more rows than a slot holds
    for bad_x, bad_y in ((x.float(), y), (x[:, :8], y), (x, y.long()), (x, y[:10])):
        with pytest.raises(ValueError):
            net.load_buffer(bad_x, bad_y)
    with pytest.raises(ValueError):
        net.set_theta([torch.zeros(1)] * 3)


def test_memory_of_a_call_on_another_stream_is_kept():
    """Tensors that the caller drops while a call on another stream is still to run (or outputs of it, while the caller's stream
    still reads them) do not go to the next allocation."""
    here, side = torch.cuda.current_stream(), torch.cuda.Stream()
    bf = dict(dtype=torch.bfloat16, device="cuda")
    weights = [torch.zeros(s, **bf) for s in ((640, 64), (640, 64), (64, 640))]
    labels = torch.zeros(512, dtype=torch.int32, device="cuda")
    calls = [lambda t: ops.gated_ffn(t, *weights, stream=side), lambda t: ops.softmax_residual(t, labels, stream=side)[0],
             lambda t: ops.gather_batch(t, labels, 1, 0, 0, 0, 512, stream=side)[0],
             lambda t: ops.gated_ffn_backward(t, t.clone(), *weights, torch.zeros(512, 5 * 64, **bf), stream=side)[0]]
    for call in calls:
        call(torch.zeros(512, 640, **bf))     # (loads what the call needs, before a kernel holds the stream)
        torch.cuda.synchronize()
        t = torch.zeros(512, 640, **bf)
        at = t.data_ptr()
        side.wait_stream(here)
        with torch.cuda.stream(side):
            torch.cuda._sleep(100_000_000)
        out = call(t)
        del t
        assert torch.empty(512, 640, **bf).data_ptr() != at
        here.wait_stream(side)
        torch.cuda.synchronize()
        torch.cuda._sleep(100_000_000)
        at = out.data_ptr()
        del out
        with torch.cuda.stream(side):
            assert torch.empty(512, 640, **bf).data_ptr() != at
        torch.cuda.synchronize()
    params = [torch.zeros(1 << 20, device="cuda")]
    state = ops.adamw_state(params)
    ops.adamw_step(params, [torch.zeros_like(params[0])], lr=0.1, stream=side, **state)
    torch.cuda.synchronize()
    g = torch.ones_like(params[0])
    at = g.data_ptr()
    side.wait_stream(here)
    with torch.cuda.stream(side):
        torch.cuda._sleep(100_000_000)
    ops.adamw_step(params, [g], lr=0.1, stream=side, **state)
    del g
    assert torch.empty(1 << 20, device="cuda").data_ptr() != at
    torch.cuda.synchronize()


def test_rounds_that_fail_leave_their_slot_in_use(monkeypatch):
    """The steps before the failure still read the buffer: the slot is free behind them, not before."""
    x, y = sample(64, 16, 4, torch.bfloat16)
    net = GatedSoftmax(64, 16, 1, 32, 4)
    slot = net.load_buffer(x.pin_memory(), y.pin_memory())
    torch.cuda.synchronize()

    def step(*_):
        torch.cuda._sleep(100_000_000)
        raise RuntimeError("no memory")
    monkeypatch.setattr(net, "step", step)
    with pytest.raises(RuntimeError, match="no memory"):
        net.run_rounds(slot, 1, 16, 0.1, 0)
    assert not net._freed[slot].query()
    torch.cuda.synchronize()


def test_buffers_are_not_loaded_on_another_device():
    x, y = sample(8, 16, 4, torch.bfloat16)
    net = GatedSoftmax(8, 16, 1, 32, 4)
    with pytest.raises(ValueError, match="stream"):
        net.load_buffer(x.pin_memory(), y.pin_memory(), stream=types.SimpleNamespace(device=torch.device("cuda", 1)))


def known_classes(net, rows, seed=0):
    """Rows close to their class's centre, and output weights that give every row's label odds of about e^9: all residuals are small."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    centres = torch.randn(net.C, net.p, generator=gen, device="cuda")
    y = torch.randint(0, net.C, (rows,), generator=gen, device="cuda", dtype=torch.int32)
    x = (centres[y.long()] + 0.02 * torch.randn(rows, net.p, generator=gen, device="cuda")).half()
    h = hidden(net, centres.double())
    net.set_theta([net.masters[0], net.masters[1], 9.0 * torch.linalg.pinv(h)])
    return x, y


def hidden(net, x):
    g = x @ net.weights[0].double()
    return g * torch.sigmoid(g) * (x @ net.weights[1].double())


@pytest.mark.parametrize("rows,loss_scale", [(100, 64.0), (256, None), (1000, None), (8192, None), (20000, None)])
def test_gradients_in_fp16_of_rows_that_are_known_well(rows, loss_scale):
    """The first moments after one step are (1 - a) times the gradient of the mean loss: each of the three as a whole against 64 bits.

    Logits of up to 16 are rounded to fp16 by at most 2^-8, which moves a probability, odds of two of them, by 2^-7 of itself.  The
    residual, H or dG and dU, and the weights' gradients are rounded by 2^-11 of each value; sums over rows and classes of
    either sign may make the first two count for more: 2^-8 allows seven besides the last.  Values below fp16's
    normal ones are not allowed for.  (Without a scale a restatement has errors of 0.03 at 256 rows to 0.8 at 20,000.)"""
    net = GatedSoftmax(rows, 128, 1, 256, 10, dtype=torch.float16, seed=1, loss_scale=loss_scale)
    x, y = known_classes(net, rows)
    leaves = [w.double().requires_grad_() for w in net.weights]
    xd = x.double()
    g = xd @ leaves[0]
    loss = torch.nn.functional.cross_entropy((g * torch.sigmoid(g) * (xd @ leaves[1])) @ leaves[2], y.long())
    loss.backward()
    assert float(loss.detach()) < 1e-2  # known well, as this test means it
    net.step(x, y, 1e-4)
    assert net.state["control"].tolist()[:2] == [1, 0]
    for m, leaf in zip(net.state["m"], leaves):
        err = float((m.double() / 0.1 - leaf.grad).norm() / leaf.grad.norm())
        assert err < 2.0 ** -7 + 2.0 ** -8, err


def test_scale_in_fp16_falls_where_gradients_overflow():
    """Hidden values of about 2,600 and one label: dWd is -0.75 times their mean at first and S times that, 499,000 with S = 256,
    overflows; so does 125,000 with S = 64, not 31,000 with S = 16.  The first two times eight updates are left out, the others
    taken; the same twice over, whether or not the host waits in between."""
    nets = [GatedSoftmax(256, 32, 1, 64, 4, dtype=torch.float16, activation=ops.ACT_RELU, seed=2) for _ in range(2)]
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = (torch.randn(256, 32, generator=gen, device="cuda").abs() * 40).half()
    y = torch.zeros(256, device="cuda", dtype=torch.int32)
    for net in nets:
        net.set_theta([torch.full_like(net.masters[0], 0.05), torch.full_like(net.masters[1], 0.05), torch.zeros_like(net.masters[2])])
    start = nets[0].get_theta()
    for t in range(60):
        nets[0].step(x, y, 1e-6)
        nets[1].step(x, y, 1e-6)
        torch.cuda.synchronize()
        if t < 8:  # nothing has been looked at yet
            assert nets[1].state["control"].tolist()[:2] == [0, t + 1]
    taken, left_out = nets[0].state["control"].tolist()[:2]
    assert (taken, left_out) == (44, 16)
    assert torch.equal(nets[0].state["control"], nets[1].state["control"])
    for a, b, s in zip(nets[0].get_theta(), nets[1].get_theta(), start):
        assert torch.equal(a, b) and torch.isfinite(a).all()
    assert not torch.equal(nets[0].get_theta()[2], start[2])


def test_loss_scale_is_for_fp16():
    for kw in (dict(loss_scale=2.0), dict(dtype=torch.float16, loss_scale=0.0), dict(dtype=torch.float16, loss_scale=float("inf"))):
        with pytest.raises(ValueError, match="loss_scale"):
            GatedSoftmax(8, 16, 1, 32, 4, **kw)


def test_a_slot_loaded_again_on_another_stream():
    """Three loads without a round in between, on three streams, the first of them held up: the third, into the same slot, is
    behind it, and the slot holds what was loaded last."""
    net = GatedSoftmax(128, 32, 2, 64, 4)
    held, other, last = (torch.cuda.Stream() for _ in range(3))
    parts = [(torch.full((64, 32), k, dtype=torch.bfloat16).pin_memory(), torch.full((64,), k, dtype=torch.int32).pin_memory()) for k in range(3)]
    net.load_buffer(*parts[0]); net.load_buffer(*parts[0])    # (memory for the slots, before a kernel holds a stream)
    torch.cuda.synchronize()
    with torch.cuda.stream(held):
        torch.cuda._sleep(100_000_000)
    slots = [net.load_buffer(*part, stream=s) for part, s in zip(parts, (held, other, last))]
    assert slots == [0, 1, 0]
    assert not net._loaded[0].query()                         # the last copy waits for the one that is held up
    torch.cuda.synchronize()
    x, y = net._slots[0]
    assert bool((x == 2).all()) and bool((y == 2).all())


def test_a_copy_that_fails_is_waited_for(monkeypatch):
    """The labels' copy fails behind the rows': the next load of the slot, on another stream, is behind the rows' copy."""
    net = GatedSoftmax(64, 32, 1, 64, 4)
    x, y = torch.ones(64, 32, dtype=torch.bfloat16).pin_memory(), torch.ones(64, dtype=torch.int32).pin_memory()
    slot = net.load_buffer(x, y)
    net.load_buffer(x, y)
    torch.cuda.synchronize()
    held = torch.cuda.Stream()
    with torch.cuda.stream(held):
        torch.cuda._sleep(100_000_000)
    real = net._slots[slot]
    net._slots[slot] = (real[0], types.SimpleNamespace(__getitem__=None, record_stream=lambda s: None))  # no labels can be copied here
    with pytest.raises(TypeError):
        net.load_buffer(x, y, stream=held)
    assert not net._loaded[slot].query()
    net._slots[slot] = real
    with pytest.raises(Exception):
        net.run_rounds(slot, 1, 16, 0.1, 0)                   # nothing whole to train on
    again = torch.cuda.Stream()
    assert net.load_buffer(x + 1, y, stream=again) == slot
    torch.cuda.synchronize()
    assert bool((net._slots[slot][0] == 2).all())


def test_scale_in_fp16_is_not_lowered_for_rows_with_nan():
    net = GatedSoftmax(256, 32, 1, 64, 4, dtype=torch.float16, seed=2)
    x, y = (t.cuda() for t in sample(256, 32, 4, torch.float16))
    bad = x.clone()
    bad[7, 3] = float("nan")
    for k in range(40):
        net.step(bad if k % 3 == 0 else x, y, 1e-3)
    assert net.state["control"].tolist()[:2] == [26, 14]
    assert net._lowered == 1.0 and all(torch.isfinite(t).all() for t in net.get_theta())


def test_scale_in_fp16_rises_again(monkeypatch):
    """After one mini-batch whose gradients overflow, S is back where it was after as many good updates as are asked for."""
    from paper_2312_08728_b200 import network
    monkeypatch.setattr(network, "_RAISE", 16)
    net = GatedSoftmax(256, 32, 1, 64, 4, dtype=torch.float16, activation=ops.ACT_RELU, seed=2)
    net.set_theta([torch.full_like(net.masters[0], 0.05), torch.full_like(net.masters[1], 0.05), torch.zeros_like(net.masters[2])])
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(256, 32, generator=gen, device="cuda").abs().half()
    y = torch.zeros(256, device="cuda", dtype=torch.int32)
    seen = []
    for k in range(40):
        net.step(x * 40 if k == 3 else x, y, 1e-6)   # (40 x: see the test above)
        seen.append(net._lowered)
    # step 3 is looked at before step 11, the good ones from step 4 on before steps 12 to 27
    assert seen == [1.0] * 11 + [0.25] * 16 + [1.0] * 13
    assert net.state["control"].tolist()[:2] == [39, 1]


def test_a_step_in_fp16_captured_into_a_graph():
    """It keeps the S of its capture and looks at nothing on the host."""
    x, y = (t.cuda() for t in sample(256, 48, 6, torch.float16))
    nets = [GatedSoftmax(256, 48, 1, 96, 6, dtype=torch.float16, seed=2) for _ in range(2)]
    for net in nets:
        net.step(x, y, 1e-2)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        nets[0].step(x, y, 1e-2)
    for _ in range(12):
        graph.replay()
        nets[1].step(x, y, 1e-2)
    nets[0].step(x, y, 1e-2)
    nets[1].step(x, y, 1e-2)
    for a, b in zip(nets[0].get_theta(), nets[1].get_theta()):
        assert torch.equal(a, b)
    assert nets[0].state["control"].tolist()[:2] == [14, 0]
