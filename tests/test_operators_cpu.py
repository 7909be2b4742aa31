"""What the operators refuse, before any pointer reaches a kernel.  No GPU needed: the Python checks run on tensors' metadata
(the meta device stands in for another one), the C checks on sizes and null pointers."""
import ctypes
import os
import struct

import pytest
import torch

from paper_2312_08728_b200 import binding, operators as ops

L = binding.load_library()
PTR = 1 << 20  # an aligned address that no call here gets as far as reading


def ffn(**kw):
    v = dict(rows=4, inputs=8, hidden=16, outputs=8, type=ops.TYPE_BF16, activation=0, reserved=0, x=PTR, w_gate=PTR, w_up=PTR,
             w_down=PTR, ld_x=8, ld_gate=16, ld_up=16, ld_down=8, y=PTR, ld_y=8, value=0, slope=0, hidden_saved=0, ld_saved=0,
             dy=PTR, ld_dy=8, dx=PTR, dw_gate=PTR, dw_up=PTR, dw_down=PTR)
    v.update(kw)
    return ops._GATED_FFN.pack(*v.values())


def workspace(which=0, **kw):
    need = ctypes.c_int64(-1)
    return L.bmgd_gated_ffn_workspace_bytes(ffn(**kw), which, ctypes.byref(need)), need.value


def test_struct_matches_the_header():
    assert ops._GATED_FFN.size == 192
    assert ctypes.sizeof(ops._AdamwConfig) == 56


def test_workspace_counts_intermediates_and_copies():
    rc, plain = workspace()
    assert rc == 0 and plain >= 4 * 16 * 2
    rc, odd = workspace(inputs=7, ld_x=7)          # rows of 14 bytes: copied
    assert rc == 0 and odd > plain
    rc, moved = workspace(x=PTR + 2)               # rows that start off a 16-byte boundary
    assert rc == 0 and moved > plain
    saved = dict(value=PTR, slope=PTR, hidden_saved=PTR, ld_saved=16)
    rc, kept = workspace(**saved)                  # the hidden rows go to the caller
    assert rc == 0 and kept == 0
    rc, back = workspace(1, **saved)
    assert rc == 0 and back >= 2 * 4 * 16 * 2


@pytest.mark.parametrize("kw,code", [
    (dict(rows=-1), binding.ERR_ARG), (dict(inputs=0), binding.ERR_ARG), (dict(hidden=0), binding.ERR_ARG),
    (dict(outputs=0), binding.ERR_ARG), (dict(rows=2 ** 31), binding.ERR_ARG), (dict(hidden=2 ** 25, ld_gate=2 ** 25, ld_up=2 ** 25), binding.ERR_ARG),
    (dict(type=ops.TYPE_F32), binding.ERR_UNIMPLEMENTED), (dict(type=7), binding.ERR_ARG), (dict(activation=4), binding.ERR_ARG),
    (dict(activation=-1), binding.ERR_ARG), (dict(reserved=1), binding.ERR_ARG), (dict(ld_x=7), binding.ERR_ARG),
    (dict(ld_gate=15), binding.ERR_ARG), (dict(ld_up=15), binding.ERR_ARG), (dict(ld_down=7), binding.ERR_ARG), (dict(ld_y=7), binding.ERR_ARG),
])
def test_gated_ffn_sizes(kw, code):
    assert workspace(**kw)[0] == code
    assert L.bmgd_gated_ffn_forward(ffn(**kw), PTR, 1 << 40, None) == code


@pytest.mark.parametrize("kw", [
    dict(x=0), dict(w_gate=0), dict(w_up=0), dict(w_down=0), dict(y=0), dict(x=PTR + 1), dict(y=PTR + 1), dict(value=PTR, ld_saved=16),
    dict(value=PTR, slope=PTR, hidden_saved=PTR, ld_saved=12), dict(value=PTR + 8, slope=PTR, hidden_saved=PTR, ld_saved=16),
    dict(value=PTR, slope=PTR, hidden_saved=PTR, ld_saved=8),
])
def test_gated_ffn_pointers(kw):
    assert L.bmgd_gated_ffn_forward(ffn(**kw), PTR, 1 << 40, None) == binding.ERR_ARG


def test_gated_ffn_workspace_and_pass():
    assert L.bmgd_gated_ffn_forward(ffn(), None, 1 << 40, None) == binding.ERR_ARG
    assert L.bmgd_gated_ffn_forward(ffn(), PTR + 128, 1 << 40, None) == binding.ERR_ARG
    assert L.bmgd_gated_ffn_forward(ffn(), PTR, 8, None) == binding.ERR_CAPACITY
    assert L.bmgd_gated_ffn_backward(ffn(), PTR, 1 << 40, None) == binding.ERR_ARG       # nothing saved
    saved = dict(value=PTR, slope=PTR, hidden_saved=PTR, ld_saved=16)
    assert L.bmgd_gated_ffn_backward(ffn(**saved, dx=PTR + 1), PTR, 1 << 40, None) == binding.ERR_ARG
    for k in ("dy", "dw_gate", "dw_up", "dw_down"):
        assert L.bmgd_gated_ffn_backward(ffn(**saved, **{k: 0}), PTR, 1 << 40, None) == binding.ERR_ARG
    assert L.bmgd_gated_ffn_backward(ffn(**saved, ld_dy=7), PTR, 1 << 40, None) == binding.ERR_ARG
    need = ctypes.c_int64()
    assert L.bmgd_gated_ffn_workspace_bytes(ffn(), 2, ctypes.byref(need)) == binding.ERR_ARG
    assert L.bmgd_gated_ffn_workspace_bytes(None, 0, ctypes.byref(need)) == binding.ERR_ARG
    assert L.bmgd_gated_ffn_workspace_bytes(ffn(), 0, None) == binding.ERR_ARG
    assert L.bmgd_gated_ffn_forward(ffn(rows=0), None, 0, None) == 0                     # nothing to do


def residual(z=PTR, ldz=10, y=PTR, rows=4, C=10, type=0, scale=1.0, out=2 * PTR, ldo=10, loss=3 * PTR):
    return L.bmgd_softmax_residual(z, ldz, y, rows, C, type, scale, out, ldo, loss, None)


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=2 ** 31), dict(C=0), dict(type=3), dict(type=-1), dict(scale=float("nan")), dict(scale=float("inf")), dict(z=None),
    dict(y=None), dict(out=None), dict(ldz=9), dict(ldo=9), dict(z=PTR + 2), dict(out=2 * PTR + 1), dict(y=PTR + 2), dict(loss=PTR + 2),
    dict(out=PTR), dict(out=PTR + 40), dict(out=PTR - 80),
])
def test_residual_arguments(kw):
    assert residual(**kw) == binding.ERR_ARG


def test_residual_of_nothing():
    assert residual(rows=0, z=None) == 0


@pytest.mark.parametrize("kw", [
    dict(rows=0), dict(rows=2 ** 31), dict(row_bytes=0), dict(first=-1), dict(count=-1), dict(first=90, count=20), dict(first=101, count=0),
    dict(x=None), dict(out_x=None), dict(out_y=None), dict(y=PTR + 1),
])
def test_gather_arguments(kw):
    v = dict(x=PTR, row_bytes=16, y=PTR, rows=100, seed=1, chain=0, round=0, first=0, count=10, out_x=PTR, out_y=PTR)
    v.update(kw)
    assert L.bmgd_gather_batch(*v.values(), None) == binding.ERR_ARG


def adamw(tensors, control=PTR, scratch=8 * PTR, size=1 << 30, **kw):
    """tensors: dicts of bmgd_adamw_tensor members."""
    rows = []
    for i, t in enumerate(tensors):
        v = dict(param=PTR * (16 + 8 * i), grad=PTR * (17 + 8 * i), m=PTR * (18 + 8 * i), v=PTR * (19 + 8 * i), m_scale=0, v_scale=0, master=0,
                 count=100, weight_decay=0.0, param_type=0, grad_type=0, state_bits=32, index=i)
        v.update(t)
        rows.append(struct.pack("=7Qqd4i", *v.values()))
    cfg = ops._AdamwConfig(*[dict(dict(lr=1e-3, a=0.9, b=0.999, eps=1e-8, grad_scale=1.0, max_norm=0.0), **kw)[k]
                             for k in ("lr", "a", "b", "eps", "grad_scale", "max_norm")], 0)
    return L.bmgd_adamw_step(b"".join(rows), len(rows), ctypes.byref(cfg), control, scratch, size, None)


@pytest.mark.parametrize("kw", [
    dict(lr=float("nan")), dict(lr=float("inf")), dict(a=1.0), dict(a=-0.1), dict(b=1.0), dict(b=float("nan")), dict(eps=-1.0), dict(eps=float("inf")),
    dict(grad_scale=float("inf")), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(control=None), dict(control=PTR + 4),
])
def test_adamw_settings(kw):
    assert adamw([{}], **kw) == binding.ERR_ARG


@pytest.mark.parametrize("t,code", [
    (dict(count=-1), binding.ERR_ARG), (dict(count=2 ** 41), binding.ERR_ARG), (dict(param=0), binding.ERR_ARG), (dict(grad=0), binding.ERR_ARG),
    (dict(m=0), binding.ERR_ARG), (dict(v=0), binding.ERR_ARG), (dict(param_type=3), binding.ERR_ARG), (dict(grad_type=-1), binding.ERR_ARG),
    (dict(state_bits=16), binding.ERR_ARG), (dict(state_bits=8), binding.ERR_ARG), (dict(weight_decay=float("nan")), binding.ERR_ARG),
    (dict(param=PTR * 16 + 2), binding.ERR_ARG), (dict(grad=PTR * 17 + 1, grad_type=1), binding.ERR_ARG), (dict(m=PTR * 18 + 2), binding.ERR_ARG),
    (dict(master=PTR * 20), binding.ERR_ARG), (dict(param_type=2), binding.ERR_UNIMPLEMENTED),
    (dict(m=PTR * 19 + 100), binding.ERR_ARG), (dict(grad=PTR * 16), binding.ERR_ARG), (dict(grad=PTR * 18 + 396), binding.ERR_ARG),
])
def test_adamw_tensors(t, code):
    assert adamw([t]) == code and adamw([{}, t]) == code


def test_adamw_the_same_tensor_twice():
    assert adamw([dict(param=PTR * 16), dict(param=PTR * 16)]) == binding.ERR_ARG
    assert adamw([dict(m=PTR * 40), dict(v=PTR * 40)]) == binding.ERR_ARG


def test_host_tensors_are_refused():
    x, w = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(8, 16, dtype=torch.bfloat16)
    for call in (lambda: ops.gated_ffn(x, w, w, w.t().contiguous()), lambda: ops.softmax_residual(x.float(), torch.zeros(4, dtype=torch.int32)),
                 lambda: ops.gather_batch(x, None, 0, 0, 0, 0, 1), lambda: ops.adamw_step([x], [x], [x], [x], torch.zeros(4, dtype=torch.int64), lr=1e-3)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        ops.adamw_step([], [], [], [], None, lr=1e-3)
    with pytest.raises(ValueError):
        ops.adamw_state([])
    with pytest.raises(ValueError):
        ops.adamw_state([x], 16)


@pytest.mark.parametrize("t,args", [
    (torch.zeros(4, 8), (4, 9)), (torch.zeros(4, 8), (5, 8)), (torch.zeros(32), (None, None)), (torch.zeros(4, 8, dtype=torch.float64), (4, 8)),
    (torch.zeros(8, 4).t(), (4, 8)), (torch.zeros(4, 16)[:, ::2], (4, 8)), (torch.zeros(8).expand(4, 8), (4, 8)),
    (torch.zeros(20).as_strided((4, 8), (4, 1)), (4, 8)), (torch.zeros(4, 8, device="meta"), (4, 8)),
])
def test_matrices_are_checked(t, args):
    with pytest.raises(ValueError):
        ops._matrix(t, "x", *args, torch.float32, torch.device("cpu"))


def test_matrix_strides():
    cpu = torch.device("cpu")
    assert ops._matrix(torch.zeros(4, 8), "x", 4, 8, torch.float32, cpu) == (4, 8, 8)
    assert ops._matrix(torch.zeros(4, 16)[:, 3:11], "x", None, 8, torch.float32, cpu) == (4, 8, 16)
    assert ops._matrix(torch.zeros(0, 8), "x", None, None, torch.float32, cpu)[2] == 8
    assert ops._matrix(torch.zeros(16)[3:4].expand(1, 1), "x", None, None, torch.float32, cpu)[2] == 1


def test_columns_are_checked():
    good = [torch.zeros(3), torch.zeros(4, 2)]
    assert ops._column(good, "m", [3, 8], ops._FLOAT, -1) == [t.data_ptr() for t in good]
    for bad in (good[:1], [good[0], torch.zeros(7)], [good[0], torch.zeros(4, 2, dtype=torch.float64)], [good[0], torch.zeros(2, 4).t()],
                [good[0], torch.zeros(4, 2, dtype=torch.float16)]):
        with pytest.raises(ValueError):
            ops._column(bad, "m", [3, 8], ops._FLOAT, -1)
    with pytest.raises(ValueError):
        ops._column(good, "m", [3, 8], ops._FLOAT, 0)


def test_no_cpu_path():
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    from paper_2312_08728_b200.network import GatedSoftmax
    with pytest.raises(RuntimeError):
        GatedSoftmax(100, 8, 2, 16, 4)


@pytest.mark.parametrize("value", [3.5e38, -3.5e38, 1e300])
def test_factors_that_overflow_in_fp32_are_refused(value):
    """They are doubles at the call and fp32 in the kernels: as Inf they would turn every result into NaN."""
    assert residual(scale=value) == binding.ERR_ARG
    assert adamw([{}], lr=value) == binding.ERR_ARG
    assert adamw([{}], grad_scale=value) == binding.ERR_ARG
    assert adamw([dict(weight_decay=value)], lr=1.0) == binding.ERR_ARG
    assert adamw([dict(weight_decay=float("inf"))], lr=0.0) == binding.ERR_ARG


def test_operators_do_not_carry_the_softmax_step_kernel():
    """Its launcher makes the kernel's instances wherever it is included: only where they are launched."""
    csrc = os.path.join(os.path.dirname(binding.__file__), "csrc")
    with_it = [f for f in sorted(os.listdir(csrc)) if '#include "softmax_kernel.cuh"' in open(os.path.join(csrc, f)).read()]
    assert with_it == ["bmgd.cu"]
