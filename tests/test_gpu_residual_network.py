"""The operators around the gated block run together: the model of residual blocks, trained and scored, and its copy in 8 bits."""
import pytest
import torch

from paper_2312_08728_b200 import operators as ops
from paper_2312_08728_b200.network import GatedSoftmax, ResidualGatedSoftmax
from test_gpu_dropout import check as check_dropout, kept
from test_gpu_int8_linear import check as check_product
from test_gpu_log_probs import check as check_scores
from test_gpu_network import sample
from test_gpu_norm import activation, check_backward, check_codes, check_norm, gate_error, normed, root_error
from test_gpu_operators import E32, Block, check_residual

pytestmark = pytest.mark.gpu

SIZES = [(24, 40, 5, 32, 1, 0.0, torch.bfloat16), (33, 70, 10, 100, 2, 0.25, torch.bfloat16), (64, 128, 16, 256, 3, 0.1, torch.float16), (200, 301, 10, 60, 2, 0.0, torch.float16)]


def build(p, hidden, C, n, blocks, dropout, dtype, **kw):
    x, y = sample(2 * n, p, C, dtype)
    net = ResidualGatedSoftmax(2 * n, p, 2, hidden, C, blocks=blocks, dropout=dropout, dtype=dtype, seed=4, **kw)
    gen = torch.Generator(device="cuda").manual_seed(1)
    for m, w in zip(net.masters, net.weights):     # norms that are not all ones
        if m.dim() == 1:
            m.add_(0.2 * torch.randn(m.shape, generator=gen, device="cuda"))
            w.copy_(m)
    return net, x.cuda(), y.cuda()


def in_64_bits(net, x, y, step=0):
    """Loss and gradients of the model with its rounded weights, everything else in 64 bits."""
    leaves = [w.double().requires_grad_() for w in net.weights]
    matrices, norms = leaves[:3 * (net.blocks + 1)], leaves[3 * (net.blocks + 1):]
    t = x.double()
    for l in range(net.blocks + 1):
        u = t / torch.sqrt(t.square().mean(dim=1, keepdim=True) + net.norm_eps) * norms[l]
        wg, wu, wd = matrices[3 * l:3 * l + 3]
        f = (torch.nn.functional.silu(u @ wg) * (u @ wu)) @ wd
        if l == net.blocks:
            break
        if net.dropout > 0:
            keep = kept(0, f.numel(), net.dropout, 4, l, step).view(f.shape)
            f = torch.where(keep, f, torch.zeros_like(f)) * (65536.0 / (65536 - round(net.dropout * 65536)))
        t = t + f
    loss = torch.nn.functional.cross_entropy(f, y.long(), reduction="none")
    loss.mean().backward()
    return f.detach(), loss.detach(), [w.grad for w in leaves]


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:6])))
def test_gradients_of_the_whole_model(size):
    net, x, y = build(*size)
    grads, loss = net._gradients(x, y, None)
    logits, want_loss, want = in_64_bits(net, x, y)
    # roundings of 2^-8 (bf16) at each of the values between two operators: about six a block, which add up like random ones; 2^-11 and
    # gradients below the normal numbers in fp16
    bound = (2.0 ** -8 if size[6] == torch.bfloat16 else 2.0 ** -9) * 3 * (net.blocks + 1)
    assert float((loss.double() - want_loss).norm() / want_loss.norm()) < bound
    for k, (g, w) in enumerate(zip(grads, want)):
        assert g.shape == w.shape and float((g.double() - w).norm() / w.norm()) < bound, k
    if net.dropout == 0:
        assert float((net.logits(x).double() - logits).norm() / logits.norm()) < bound


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:6])))
def test_a_step_operator_by_operator(size):
    """Every operator's result is within its bound of the definition on the inputs that it was given."""
    net, x, y = build(*size)
    kept_values, v, total = [], x, None
    for l in range(net.blocks + 1):
        u, total, rstd = check_norm(v, net._norm(l), total)
        b = Block.__new__(Block)
        b.x, (b.wg, b.wu, b.wd), b.act, b.dtype = u, net._block(l), net.activation, net.dtype
        v, saved = ops.gated_ffn(u, *net._block(l), net.activation, save=True)
        kept_values.append((b, v, total, rstd, saved))
        if net.dropout > 0 and l < net.blocks:
            (v, _), total = check_dropout(v, net.dropout, 4, residual=total, layer=l), None
    residual, loss = check_residual(v, y)
    dv, dtotal = residual, None
    for l in reversed(range(net.blocks + 1)):
        b, out, total, rstd, saved = kept_values[l]
        b.dy = dv
        du, *grads = ops.gated_ffn_backward(dv, b.x, *net._block(l), saved, net.activation)
        b.check({"y": out, "dx": du, "dw_gate": grads[0], "dw_up": grads[1], "dw_down": grads[2]})
        check_backward(du, total, net._norm(l), rstd, dtotal)
        dtotal, _ = ops.rms_norm_backward(du, total, net._norm(l), rstd, dtotal)
        if l > 0:
            dv = check_dropout(dtotal, net.dropout, 4, layer=l - 1)[0] if net.dropout > 0 else dtotal


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:6])))
def test_rounds_over_buffers(size):
    """The same bits on slots, on a resident buffer and step by step; the weights move, the masks change with the updates."""
    p, hidden, C, n, blocks, dropout, dtype = size
    nets = [build(*size, weight_decay=0.01, state_bits=32)[0] for _ in range(3)]
    _, x, y = build(*size)
    before = nets[0].get_theta()
    slot = nets[0].load_buffer(x[:n].cpu().pin_memory(), y[:n].cpu().pin_memory())
    nets[0].run_rounds(slot, 3, 16, 1e-2, seed=6)
    nets[1].run_rounds_resident(x[:n].contiguous(), y[:n].contiguous(), 3, 16, 1e-2, seed=6)
    for t in range(3):
        for first in range(0, n, 16):
            nets[2].step(*ops.gather_batch(x[:n].contiguous(), y[:n].contiguous(), 6, 0, t, first, min(16, n - first)), 1e-2)
    nets[0].sync()
    for a, b, c, d in zip(*(net.get_theta() for net in nets), before):
        assert torch.equal(a, b) and torch.equal(a, c) and not torch.equal(a, d) and bool(torch.isfinite(a).all())
    assert nets[0].state["control"][0] == 3 * -(-n // 16)


def test_no_blocks_is_the_layer_behind_a_norm():
    net, x, y = build(24, 40, 5, 32, 0, 0.0, torch.bfloat16)
    u, _ = ops.rms_norm(x, net._norm(0), eps=net.norm_eps)
    assert torch.equal(net.logits(x), ops.gated_ffn(u, *net._block(0)))
    grads, _ = net._gradients(x, y, None)
    assert [tuple(g.shape) for g in grads] == [(24, 40), (24, 40), (40, 5), (24,)]


def test_a_captured_step_draws_new_masks():
    net, x, y = build(33, 70, 10, 100, 2, 0.25, torch.bfloat16)
    twin, _, _ = build(33, 70, 10, 100, 2, 0.25, torch.bfloat16)
    for m in (net, twin):
        m.step(x, y, 0.0)                     # (workspaces, and one update)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        loss = net.step(x, y, 0.0)            # the rate is zero: only the masks change
    losses = []
    for _ in range(3):
        graph.replay()
        losses.append(loss.clone())
        assert torch.equal(loss, twin.step(x, y, 0.0))
    assert not torch.equal(losses[0], losses[1]) and not torch.equal(losses[1], losses[2])


@pytest.mark.parametrize("size", SIZES, ids=lambda s: "x".join(map(str, s[:6])))
def test_scores(size):
    net, x, y = build(*size)
    for model in (net, GatedSoftmax(len(x), size[0], 1, size[1], size[2], dtype=size[6]), net.quantized()):
        got = model.score(x, y, top=3)
        z = model.logits(x)
        assert all(torch.equal(a, b) for a, b in zip(got, ops.log_probs(z, y, top=3)))
        check_scores(z, y, 3)
    assert torch.equal(net.score(x)[1], net.score(x, y)[1]) and not net.score(x)[0].any()


@pytest.mark.parametrize("size", SIZES + [(512, 1024, 300, 4, 1, 0.0, torch.bfloat16)], ids=lambda s: "x".join(map(str, s[:6])))
def test_the_copy_in_8_bits(size):
    """Operator by operator, and the whole against the model in 64 bits."""
    net, x, _ = build(*size)
    scorer = net.quantized()
    v, total = x, None
    for l, (both, both_scale, down, down_scale) in enumerate(scorer.layers):
        wg, wu, wd = net.masters[3 * l:3 * l + 3]
        check_codes(both, both_scale, torch.cat((wg, wu), dim=1).T.double(), 0.0)
        check_codes(down, down_scale, wd.T.double(), 0.0)
        residual = total
        q, scale, total = ops.rms_norm_int8(v, net._norm(l), residual=residual, eps=net.norm_eps)
        check_codes(q, scale, normed_at(total, net._norm(l), net.norm_eps), root_error(size[0]) + 3 * E32)
        h = check_product(q, scale, both, both_scale, dtype=net.dtype)
        gate, up = h[:, :net.hidden], h[:, net.hidden:]
        q, scale = ops.quantize_rows(up, gate=gate, activation=net.activation)
        value, rel = activation(net.activation, gate.double())[0], gate_error(net.activation, gate.double())[0]
        exact = value * up.double()
        top = exact.abs().amax(dim=1, keepdim=True)
        check_codes(q, scale, exact, float((((rel + 2 * E32) * exact.abs()).amax(dim=1, keepdim=True) / top).max()))
        v = check_product(q, scale, down, down_scale, dtype=net.dtype)
    assert torch.equal(v, scorer.logits(x))
    # An operand in 8 bits is off by a scale / sqrt(12) per value, a scale being the largest of its row / 127: for rows of up to a thousand normal
    # values, whose largest is below 4.5 times their norm's share, 1.1 % of that share.  Three such operands a product pair and block, on
    # both sides, and what the gate makes of them (a slope of up to 1.1, two factors): below 5 % a block.
    logits = in_64_bits_without_dropout(net, x)
    assert float((v.double() - logits).norm() / logits.norm()) < 0.05 * (net.blocks + 1)
    before = scorer.logits(x)
    for w in net.masters:
        w.zero_()
    assert torch.equal(scorer.logits(x), before)      # (a copy)


def normed_at(total, w, eps):
    t = total.double()
    return t / torch.sqrt(t.square().mean(dim=1, keepdim=True) + eps) * w.double()


def in_64_bits_without_dropout(net, x):
    t = x.double()
    for l in range(net.blocks + 1):
        u = normed_at(t, net._norm(l), net.norm_eps)
        wg, wu, wd = (w.double() for w in net.masters[3 * l:3 * l + 3])
        f = (torch.nn.functional.silu(u @ wg) * (u @ wu)) @ wd
        t = t + f if l < net.blocks else t
    return f


def test_refusals():
    for kw in (dict(blocks=-1), dict(blocks=65536), dict(dropout=1.0), dict(dropout=-0.1), dict(dropout=float("nan"))):
        with pytest.raises(ValueError):
            ResidualGatedSoftmax(100, 8, 1, 8, 3, **kw)
    net = ResidualGatedSoftmax(100, 8, 1, 8, 3, blocks=1)
    with pytest.raises(ValueError):
        net.set_theta(net.get_theta()[:-1])
    net.set_theta(net.get_theta())
    assert normed(torch.ones(1, 8, device="cuda"), None)[0].shape == (1, 8)


@pytest.mark.parametrize("n", [1, 2, 5, 70])
def test_a_layer_behind_copies_and_other_streams_in_a_graph(n):
    """Launches that start beside the end of the one before them wait for whatever stands there: a copy, a memset, two streams that meet."""
    gen = torch.Generator(device="cuda").manual_seed(n)
    d, f = 520, 1000
    rows = torch.randn(n, d, device="cuda", generator=gen).to(torch.bfloat16)
    w, parts = torch.rand(d, device="cuda", generator=gen) + 0.5, [torch.zeros(n, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    up = ops.quantize_weight(torch.randn(d, 2 * f, device="cuda", generator=gen))
    down = ops.quantize_weight(torch.randn(f, d, device="cuda", generator=gen))
    other = torch.cuda.Stream()

    def layer():
        here = torch.cuda.current_stream()
        other.wait_stream(here)
        with torch.cuda.stream(other):
            parts[1].zero_()
            parts[1].add_(rows)
        parts[0].copy_(rows)
        here.wait_stream(other)
        q, s, total = ops.rms_norm_int8(parts[0], w, residual=parts[1])
        v = ops.int8_linear(q, s, *up)
        q, s = ops.quantize_rows(v[:, f:], gate=v[:, :f])
        return ops.int8_linear(q, s, *down), total

    layer()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer()
    for k in range(20):
        rows.normal_(generator=gen)
        want = [t.clone() for t in layer()]
        for t in (*parts, *got):
            t.zero_()
        graph.replay()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
