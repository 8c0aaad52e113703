"""Host-side checks of the operators around attention (no GPU needed): refusals before
any device work, and the frequencies of rotary positions."""
import ctypes
import inspect
import math
import os
import re
import struct
import subprocess
import sys
import tempfile

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def lib():
    from paper_2205_13542_amd import _binding, _map_binding, build
    if not os.path.exists(_binding.LIB_PATH):
        build.build()
    return _map_binding.load()


@pytest.fixture(scope="module")
def mb(lib):
    from paper_2205_13542_amd import _map_binding
    return _map_binding


P = ctypes.c_void_p(16)     # a pointer that no refused call follows
INVALID, DTYPE, OVERFLOW = -1, -3, -4


def _rms(mb, **over):
    vals = dict(rows=9, channels=12, x_dtype=0, y_dtype=0, weight_dtype=0, x_stride=12, residual_stride=12, eps=1e-6)
    vals.update(over)
    return mb.bevmap_rms(**vals)


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), INVALID), (dict(channels=0), INVALID), (dict(channels=-3), INVALID), (dict(x_stride=11), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=math.nan), INVALID), (dict(eps=math.inf), INVALID), (dict(x_dtype=3), DTYPE),
    (dict(y_dtype=-1), DTYPE), (dict(weight_dtype=9), DTYPE), (dict(rows=1 << 31), OVERFLOW),
    (dict(channels=8193, x_stride=8193, residual_stride=8193), OVERFLOW), (dict(x_stride=1 << 31), OVERFLOW)])
def test_rms_norm_refuses(lib, mb, over, code):
    n = _rms(mb, **over)
    assert lib.bevmap_rms_norm_backward_workspace(n) == code
    assert lib.bevmap_rms_norm(n, P, P, P, P, P, P, None) == code
    assert lib.bevmap_rms_norm_int8(n, P, P, P, P, P, P, None) == code
    assert lib.bevmap_rms_norm_backward(n, P, P, P, P, P, P, P, P, P, 1 << 40, None) == code


def test_rms_norm_refuses_pointers_strides_and_workspaces(lib, mb):
    n = _rms(mb)
    need = lib.bevmap_rms_norm_backward_workspace(n)
    assert need > 0 and need % 48 == 0
    for args in ((None, P, P, P, P, P), (P, P, P, None, P, P), (P, None, P, None, None, P)):
        assert lib.bevmap_rms_norm(n, *args, None) == INVALID
    for args in ((None, P, P, P, P, P), (P, P, P, None, P, P), (P, None, P, None, None, P), (P, None, P, None, P, None)):
        assert lib.bevmap_rms_norm_int8(n, *args, None) == INVALID
    for k in (0, 2, 5, 6):
        args = [P] * 9
        args[k] = None
        assert lib.bevmap_rms_norm_backward(n, *args, need, None) == INVALID
    assert lib.bevmap_rms_norm_backward(n, P, P, P, P, P, P, P, P, P, need - 1, None) == INVALID
    assert lib.bevmap_rms_norm_backward(n, P, P, P, P, P, P, P, P, None, need, None) == INVALID
    assert lib.bevmap_rms_norm_backward(n, P, P, P, P, P, P, P, P, ctypes.c_void_p(8), need, None) == INVALID
    assert lib.bevmap_rms_norm(None, P, P, P, P, P, P, None) == INVALID
    short = _rms(mb, residual_stride=11)
    assert lib.bevmap_rms_norm(short, P, P, P, P, P, P, None) == INVALID
    assert lib.bevmap_rms_norm_backward(short, P, P, P, P, P, P, P, P, P, need, None) == INVALID
    empty = _rms(mb, rows=0)
    assert lib.bevmap_rms_norm_backward_workspace(empty) == 0
    assert lib.bevmap_rms_norm(empty, None, None, None, None, None, None, None) == 0
    assert lib.bevmap_rms_norm_int8(empty, None, None, None, None, None, None, None) == 0
    assert lib.bevmap_rms_norm_backward(empty, None, None, None, None, None, None, None, None, None, 0, None) == 0


def test_rms_norm_workspace_stays_below_the_rows(lib, mb):
    """Parts of the weights' gradient, at most a row of fp32 for each row, and at most 2048 of them."""
    for rows in (1, 3, 600, 5000, 518400, 1 << 30):
        for channels in (1, 80, 1030, 8192):
            n = _rms(mb, rows=rows, channels=channels, x_stride=channels)
            size = lib.bevmap_rms_norm_backward_workspace(n)
            assert 0 < size <= 4 * channels * min(rows, 2048)


@pytest.mark.parametrize("args,code", [
    ((P, 8, P, P, -1, 8, 0), INVALID), ((P, 8, P, P, 4, -8, 0), INVALID), ((P, 7, P, P, 4, 8, 0), INVALID),
    ((None, 8, P, P, 4, 8, 0), INVALID), ((P, 8, None, P, 4, 8, 0), INVALID), ((P, 8, P, None, 4, 8, 0), INVALID),
    ((P, 8, P, P, 4, 8, 3), DTYPE), ((P, 1 << 17, P, P, 4, 1 << 17, 0), OVERFLOW),
    ((P, 1 << 31, P, P, 4, 8, 0), OVERFLOW), ((P, 8, P, P, 1 << 31, 8, 0), OVERFLOW),
    ((None, 8, None, None, 0, 8, 0), 0)])
def test_quantize_refuses(lib, args, code):
    assert lib.bevmap_quantize_int8(*args, None) == code


def _linear(mb, **over):
    vals = dict(rows=5, channels=16, features=7, x_stride=16, w_stride=16, y_dtype=1)
    vals.update(over)
    return mb.bevmap_linear(**vals)


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), INVALID), (dict(features=-1), INVALID), (dict(channels=0), INVALID), (dict(x_stride=15), INVALID),
    (dict(w_stride=15), INVALID), (dict(y_dtype=3), DTYPE), (dict(rows=1 << 30), OVERFLOW),
    (dict(channels=131072, x_stride=131072, w_stride=131072), OVERFLOW), (dict(x_stride=1 << 31), OVERFLOW),
    (dict(w_stride=1 << 31), OVERFLOW), (dict(features=(1 << 20) + 1), OVERFLOW),
    (dict(rows=1 << 20, features=1 << 17), OVERFLOW)])
def test_linear_refuses(lib, mb, over, code):
    assert lib.bevmap_linear_int8(_linear(mb, **over), P, P, P, P, P, P, None) == code


def test_linear_refuses_pointers(lib, mb):
    for k in (0, 1, 2, 3, 5):
        args = [P] * 6
        args[k] = None
        assert lib.bevmap_linear_int8(_linear(mb), *args, None) == INVALID
    assert lib.bevmap_linear_int8(None, P, P, P, P, P, P, None) == INVALID
    for empty in (dict(rows=0), dict(features=0)):
        assert lib.bevmap_linear_int8(_linear(mb, **empty), None, None, None, None, None, None, None) == 0


def _turn(mb, **over):
    vals = dict(batch=2, tokens=3, heads=4, dim=16, pairs=6, axes=2, interleaved=0, positions_type=0, dtype=0,
                amplitude=1.0, x_batch=192, x_row=64, x_head=16)
    vals.update(over)
    return mb.bevmap_turn(**vals)


@pytest.mark.parametrize("over,code", [
    (dict(batch=-1), INVALID), (dict(tokens=-1), INVALID), (dict(heads=0), INVALID), (dict(dim=0), INVALID),
    (dict(pairs=0), INVALID), (dict(axes=0), INVALID), (dict(pairs=9, axes=1), INVALID), (dict(axes=4), INVALID),
    (dict(positions_type=3), INVALID), (dict(positions_type=-1), INVALID), (dict(amplitude=math.inf), INVALID),
    (dict(amplitude=math.nan), INVALID), (dict(x_row=-1), INVALID), (dict(x_batch=-1), INVALID),
    (dict(x_head=-1), INVALID), (dict(dtype=3), DTYPE), (dict(batch=1 << 16, tokens=1 << 15), OVERFLOW),
    (dict(heads=65536), OVERFLOW), (dict(dim=4097), OVERFLOW), (dict(pairs=(1 << 30) + 2, axes=1), INVALID)])
def test_rotary_refuses(lib, mb, over, code):
    for backward in (0, 1):
        assert lib.bevmap_rotary(_turn(mb, **over), P, P, P, P, backward, None) == code


def test_rotary_refuses_pointers(lib, mb):
    for k in range(4):
        args = [P] * 4
        args[k] = None
        assert lib.bevmap_rotary(_turn(mb), *args, 0, None) == INVALID
    assert lib.bevmap_rotary(None, P, P, P, P, 0, None) == INVALID
    assert lib.bevmap_rotary(_turn(mb, tokens=0), None, None, None, None, 0, None) == 0


def _gate(mb, **over):
    vals = dict(rows=5, features=7, act=2, dtype=0, x_stride=14)
    vals.update(over)
    return mb.bevmap_gate(**vals)


@pytest.mark.parametrize("over,code", [
    (dict(rows=-1), INVALID), (dict(features=0), INVALID), (dict(x_stride=13), INVALID), (dict(act=4), INVALID),
    (dict(act=-1), INVALID), (dict(dtype=3), DTYPE), (dict(rows=1 << 31), OVERFLOW), (dict(x_stride=1 << 31), OVERFLOW),
    (dict(features=1 << 24, x_stride=1 << 26), OVERFLOW)])
def test_gated_act_refuses(lib, mb, over, code):
    g = _gate(mb, **over)
    assert lib.bevmap_gated_act(g, P, P, P, P, None) == code
    assert lib.bevmap_gated_act_backward(g, P, P, P, P, P, None) == code


def test_gated_act_refuses_pointers(lib, mb):
    g = _gate(mb)
    for args in ((None, P, P, P), (P, None, P, P), (P, P, None, P), (P, P, P, None)):
        assert lib.bevmap_gated_act(g, *args, None) == INVALID
    for args in ((None, P, P, P, P), (P, None, None, None, P), (P, P, P, P, None), (P, P, P, None, P),
                 (P, P, None, P, P)):
        assert lib.bevmap_gated_act_backward(g, *args, None) == INVALID
    assert lib.bevmap_gated_act(None, P, P, P, P, None) == INVALID
    assert lib.bevmap_gated_act(_gate(mb, rows=0), None, None, None, None, None) == 0
    assert lib.bevmap_gated_act_backward(_gate(mb, rows=0), None, None, None, None, None, None) == 0


def test_python_entries_refuse():
    torch = pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    x, q, s = torch.zeros(2, 8), torch.zeros(2, 8, dtype=torch.int8), torch.zeros(2)
    f = bev.rotary_frequencies(2)
    for call in (lambda: bev.rms_norm(x), lambda: bev.rms_norm_add(x, x), lambda: bev.rms_norm_int8(x),
                 lambda: bev.rms_norm_add_int8(x, x), lambda: bev.quantize_int8(x),
                 lambda: bev.linear_int8(q, s, q, s), lambda: bev.rotary(x.view(1, 2, 2, 4), s.view(1, 2), f),
                 lambda: bev.gated_act(x)):
        with pytest.raises(bev.BevpoolError, match="device tensors"):
            call()
    with pytest.raises(bev.BevpoolError, match="checkpoint"):
        bev.gated_act(x, checkpoint="fp8")


def test_forward_mode_is_refused():
    """An input with a tangent is refused before anything else, with gradients enabled or not; inputs
    without one get as far as the refusal of tensors that no GPU holds."""
    torch = pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    from torch.autograd import forward_ad
    x, f, q, s = torch.ones(2, 8), torch.ones(2, dtype=torch.float64), torch.ones(2, 8, dtype=torch.int8), torch.ones(2)
    with forward_ad.dual_level():
        xd, fd, sd = (forward_ad.make_dual(t, torch.ones_like(t)) for t in (x, f, s))
        for call in (lambda: bev.rms_norm(xd), lambda: bev.rms_norm(x, xd[0]), lambda: bev.rms_norm_add(x, xd),
                     lambda: bev.rotary(xd.view(1, 2, 2, 4), s[None], f),
                     lambda: bev.rotary(x.view(1, 2, 2, 4), s[None], fd), lambda: bev.gated_act(xd),
                     lambda: bev.rms_norm_int8(xd), lambda: bev.rms_norm_add_int8(x, xd), lambda: bev.quantize_int8(xd),
                     lambda: bev.linear_int8(q, s, q, sd)):
            with pytest.raises(NotImplementedError, match="forward mode"):
                call()
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward mode"):
                call()
        for call in (lambda: bev.rms_norm(x), lambda: bev.rms_norm_int8(x), lambda: bev.gated_act(x)):
            with pytest.raises(bev.BevpoolError, match="device tensors"):
                call()


@pytest.mark.parametrize("tracer", ["jit", "real", "symbolic", "pre_dispatch"])
def test_tracing_is_refused(tracer):
    """A tracer does not see these calls and would keep their results as constants: refused before the
    refusal of tensors that no GPU holds, which a call gets again once nothing is traced."""
    torch = pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    from torch.fx.experimental.proxy_tensor import make_fx
    x, q, s = torch.ones(2, 8), torch.ones(2, 8, dtype=torch.int8), torch.ones(2)
    place, f = s.view(1, 2), bev.rotary_frequencies(2)

    def trace(call):
        if tracer == "jit":
            return torch.jit.trace(call, (x,))
        if tracer == "pre_dispatch":
            return make_fx(call, tracing_mode="real", pre_dispatch=True)(x)
        return make_fx(call, tracing_mode=tracer)(x)

    for call in (lambda x: bev.rms_norm(x), lambda x: bev.rms_norm_add(x, x), lambda x: bev.rms_norm_int8(x),
                 lambda x: bev.rms_norm_add_int8(x, x), lambda x: bev.quantize_int8(x),
                 lambda x: bev.linear_int8(q, x[:, 0], q, s), lambda x: bev.rotary(x.view(1, 2, 2, 4), place, f),
                 lambda x: bev.gated_act(x), lambda x: bev.gated_act(x, checkpoint="int8")):
        for enabled in (True, False):
            with torch.set_grad_enabled(enabled), pytest.raises(bev.BevpoolError, match="cannot be traced"):
                trace(call)
        with pytest.raises(bev.BevpoolError, match="device tensors"):
            call(x)


def test_calls_with_other_things_than_tensors():
    torch = pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    x, q, s = torch.zeros(2, 8), torch.zeros(2, 8, dtype=torch.int8), torch.zeros(2)
    for call in (lambda: bev.rms_norm([1.0]), lambda: bev.rms_norm(x, 2.0), lambda: bev.rms_norm(x, eps="small"),
                 lambda: bev.rms_norm(x, out_dtype="bf16"), lambda: bev.rms_norm_add(x, None),
                 lambda: bev.rms_norm_add_int8(x, None), lambda: bev.quantize_int8(None),
                 lambda: bev.linear_int8(q, None, q, s), lambda: bev.linear_int8(q, s, q, s, bias=0.0),
                 lambda: bev.rotary(x, s, None), lambda: bev.gated_act(3)):
        with pytest.raises(bev.BevpoolError, match="must be") as caught:
            call()
        assert caught.value.code == INVALID
    with pytest.raises(RuntimeError, match="has no gradient"):
        bev.quantize_int8(x.clone().requires_grad_())


def test_rotary_frequencies():
    torch = pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    plain = bev.rotary_frequencies(8)
    assert plain.dtype == torch.float64
    assert torch.allclose(plain, torch.tensor([10.0 ** (-i / 2) for i in range(8)], dtype=torch.float64), rtol=1e-14)
    axes = bev.rotary_frequencies(6, base=64.0, axes=2)
    assert torch.allclose(axes, torch.tensor([1, 0.25, 0.0625] * 2, dtype=torch.float64), rtol=1e-14)
    assert torch.allclose(bev.rotary_frequencies(8, scaling="linear", factor=4.0), plain / 4, rtol=1e-15)
    based = bev.rotary_frequencies(8, scaling="base", factor=4.0)
    assert based[0] == 1 and torch.allclose(based[-1], plain[-1] / 4, rtol=1e-13)
    assert ((based <= plain) & (based >= plain / 4 * (1 - 1e-12))).all()
    parts = bev.rotary_frequencies(8, scaling="parts", factor=4.0, context=2000)
    turns = plain * 2000 / (2 * math.pi)
    assert torch.equal(parts[turns >= 32], plain[turns >= 32]) and (turns >= 32).any()
    assert torch.allclose(parts[turns <= 1], plain[turns <= 1] / 4, rtol=1e-15) and (turns <= 1).any()
    middle = (turns > 1) & (turns < 32)
    share = (turns[middle] - 1) / 31
    assert middle.any() and torch.allclose(parts[middle], plain[middle] * (share + (1 - share) / 4), rtol=1e-13)
    for bad in (dict(pairs=0), dict(pairs=5, axes=2), dict(pairs=4, axes=0), dict(pairs=4, base=0.0),
                dict(pairs=4, base=math.inf), dict(pairs=4, factor=0.5), dict(pairs=4, scaling="cubic"),
                dict(pairs=4, scaling="parts"), dict(pairs=4, scaling="parts", context=100, fast=1.0, slow=1.0),
                dict(pairs=2, axes=2, scaling="base", factor=2.0)):
        with pytest.raises(bev.BevpoolError):
            bev.rotary_frequencies(**bad)


def test_star_import_needs_no_torch():
    code = """
import sys
import tempfile
sys.modules["torch"] = None            # an import of torch raises ImportError
from paper_2205_13542_amd import *
for call in (lambda: rms_norm(None), lambda: rms_norm_add(None, None), lambda: rms_norm_int8(None),
             lambda: rms_norm_add_int8(None, None), lambda: quantize_int8(None),
             lambda: linear_int8(None, None, None, None), lambda: rotary(None, None, None),
             lambda: rotary_frequencies(4), lambda: gated_act(None)):
    try:
        call()
    except ImportError:
        continue
    raise SystemExit("an operator ran without torch")
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr


def test_package_names_are_the_operators():
    pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    from paper_2205_13542_amd import layer_ops
    for name in ("rms_norm", "rms_norm_add", "rms_norm_int8", "rms_norm_add_int8", "quantize_int8", "linear_int8",
                 "rotary", "rotary_frequencies", "gated_act"):
        assert name in bev.__all__
        assert inspect.signature(getattr(bev, name)) == inspect.signature(getattr(layer_ops, name))


def _kernels(path):
    """Registers, spills and scratch of the kernels in a library that was built here, from the notes of its
    gfx950 code objects."""
    data = open(path, "rb").read()
    readelf = "/opt/rocm/llvm/bin/llvm-readelf"
    magic, at, out = b"__CLANG_OFFLOAD_BUNDLE__", 0, {}
    while (at := data.find(magic, at)) >= 0:
        count, = struct.unpack_from("<Q", data, at + 24)
        entry = at + 32
        for _ in range(count):
            offset, size, length = struct.unpack_from("<QQQ", data, entry)
            name = data[entry + 24:entry + 24 + length].decode()
            entry += 24 + length
            if "gfx950" not in name or not size:
                continue
            with tempfile.NamedTemporaryFile(suffix=".co") as f:
                f.write(data[at + offset:at + offset + size])
                f.flush()
                notes = subprocess.run([readelf, "--notes", f.name], capture_output=True, text=True, check=True).stdout
            for kernel in re.split(r"\n  - \.", notes)[1:]:
                name = re.search(r"\.name: +(\S+)", kernel)
                if name:
                    out[name.group(1)] = {k: int(v) for k, v in re.findall(r"\.(\w+): +(\d+)\n", kernel)}
        at += len(magic)
    return out


def test_kernels_neither_spill_nor_use_scratch(lib):
    """The kernels of linear_int8 whose rows go through the registers hold up to 240 of them; an earlier
    form of these spilled and had wrong sums. (Scalar registers of other kernels may be kept in lanes of
    vector registers.)"""
    from paper_2205_13542_amd import _binding
    if not os.path.exists("/opt/rocm/llvm/bin/llvm-readelf"):
        pytest.skip("no llvm-readelf")
    kernels = _kernels(_binding.LIB_PATH)
    counts = dict.fromkeys(("k_linear", "k_rms", "k_quantize_long", "k_turn", "k_gate"), 0)
    for name, held in kernels.items():
        for part in counts:
            if part in name:
                counts[part] += 1
                assert held["vgpr_spill_count"] == held["private_segment_fixed_size"] == 0, (name, held)
                assert part != "k_linear" or held["sgpr_spill_count"] == 0, (name, held)
                break
    assert counts["k_linear"] >= 15 and all(counts.values()), counts
