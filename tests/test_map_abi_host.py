"""Host-side checks of the map operators (no GPU needed): the library exports
what include/bevmap.h declares, and refuses bad arguments before any device work."""
import ctypes
import inspect
import os
import re
import subprocess
import sys

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


def test_library_exports_every_declared_symbol(lib, mb):
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "bevmap.h")).read(), flags=re.S)
    names = set(re.findall(r"BEVPOOL_API\s+[\w\s\*]+?\b(bevmap_\w+)\s*\(", text))
    assert names == set(mb.EXPORTED)
    for name in names:
        assert hasattr(lib, name), name


P = ctypes.c_void_p(16)     # a pointer that no refused call follows
INVALID, DTYPE, OVERFLOW = -1, -3, -4


def _norm(mb, **over):
    vals = dict(batch=2, pixels=9, channels=12, groups=3, row_stride=12, eps=1e-5, act=0, x_dtype=0, y_dtype=0,
                weight_dtype=0)
    vals.update(over)
    return mb.bevmap_norm(**vals)


@pytest.mark.parametrize("over,code", [
    (dict(batch=-1), INVALID), (dict(pixels=-1), INVALID), (dict(channels=0), INVALID), (dict(groups=0), INVALID),
    (dict(groups=5), INVALID), (dict(row_stride=11), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(act=4), INVALID), (dict(act=-1), INVALID), (dict(x_dtype=3), DTYPE),
    (dict(y_dtype=-1), DTYPE), (dict(weight_dtype=7), DTYPE), (dict(batch=65536), OVERFLOW),
    (dict(batch=4096, pixels=1 << 20), OVERFLOW), (dict(batch=1, pixels=1 << 30), OVERFLOW), (dict(channels=8193, groups=1, row_stride=8193), OVERFLOW),
    (dict(row_stride=1 << 31), OVERFLOW)])
def test_group_norm_refuses(lib, mb, over, code):
    n = _norm(mb, **over)
    assert lib.bevmap_group_norm_workspace(n, 0) == code
    assert lib.bevmap_group_norm(n, P, P, P, P, P, P, P, 1 << 30, None) == code
    assert lib.bevmap_group_norm_backward(n, P, P, P, P, P, P, P, P, P, P, 1 << 30, None) == code


def test_group_norm_refuses_pointers_and_workspaces(lib, mb):
    n = _norm(mb, pixels=20000)      # small maps need no workspace
    need = lib.bevmap_group_norm_workspace(n, 0)
    assert need > 0 and lib.bevmap_group_norm_workspace(n, 1) > need
    assert lib.bevmap_group_norm(n, None, P, P, P, P, P, P, need, None) == INVALID
    assert lib.bevmap_group_norm(n, P, P, P, None, P, P, P, need, None) == INVALID
    assert lib.bevmap_group_norm(n, P, P, P, P, P, P, P, need - 1, None) == INVALID
    assert lib.bevmap_group_norm(n, P, P, P, P, P, P, None, need, None) == INVALID
    assert lib.bevmap_group_norm(n, P, P, P, P, P, P, ctypes.c_void_p(8), need, None) == INVALID
    assert lib.bevmap_group_norm(None, P, P, P, P, P, P, P, need, None) == INVALID
    assert lib.bevmap_group_norm_backward(n, P, P, P, P, P, P, P, P, P, P, need, None) == INVALID
    assert lib.bevmap_group_norm_backward(n, P, P, P, P, P, P, None, P, P, P, 1 << 30, None) == INVALID
    empty = _norm(mb, pixels=0)
    assert lib.bevmap_group_norm_workspace(empty, 0) == 0
    assert lib.bevmap_group_norm(empty, None, None, None, None, None, None, None, 0, None) == 0


def test_group_norm_of_many_groups_takes_three_kernels(lib, mb):
    """One workgroup to a group reads every cache line of the map once for each group in it: such maps
    need the workspace of the three kernels, small ones with as many groups do not."""
    def workspaces(batch, pixels, channels, groups):
        n = _norm(mb, batch=batch, pixels=pixels, channels=channels, groups=groups, row_stride=channels, x_dtype=1)
        return [lib.bevmap_group_norm_workspace(n, backward) for backward in (0, 1)]

    assert all(size > 0 for size in workspaces(8, 8100, 256, 256))
    assert all(size > 0 for size in workspaces(4, 8100, 32, 32))
    assert all(size > 0 for size in workspaces(64, 16, 1024, 1024))
    assert all(size == 0 for size in workspaces(1, 512, 256, 256))
    assert all(size == 0 for size in workspaces(2, 1073, 66, 11))


def _attend(mb, **over):
    vals = dict(batch=2, queries=5, keys=7, heads=4, key_heads=2, dim=8, dtype=0, scale=0.3, q_batch=160, q_row=32,
                q_head=8, k_batch=112, k_row=16, k_head=8, v_batch=112, v_row=16, v_head=8, mask_batch=7)
    vals.update(over)
    return mb.bevmap_attend(**vals)


@pytest.mark.parametrize("over,code", [
    (dict(batch=-1), INVALID), (dict(queries=-1), INVALID), (dict(keys=-1), INVALID), (dict(heads=0), INVALID),
    (dict(key_heads=0), INVALID), (dict(heads=3), INVALID), (dict(dim=0), INVALID),
    (dict(scale=float("inf")), INVALID), (dict(k_row=-1), INVALID), (dict(q_batch=-1), INVALID),
    (dict(mask_batch=-1), INVALID), (dict(dtype=3), DTYPE), (dict(dim=129), OVERFLOW),
    (dict(batch=40000), OVERFLOW), (dict(keys=1 << 30), OVERFLOW), (dict(queries=1 << 29), OVERFLOW),
    (dict(v_row=1 << 22), OVERFLOW)])
def test_attention_refuses(lib, mb, over, code):
    a = _attend(mb, **over)
    assert lib.bevmap_attention_workspace(a, 0) == code
    assert lib.bevmap_attention(a, P, P, P, None, None, P, None, None, P, 1 << 40, None) == code
    assert lib.bevmap_attention_backward(a, P, P, P, P, None, None, P, P, P, P, P, P, P, 1 << 40, None) == code


@pytest.mark.parametrize("dtype,dim,resident", [
    (0, 32, 1), (0, 64, 1), (1, 32, 2), (1, 64, 2), (2, 96, 1), (1, 128, 1)])
def test_attention_parts_go_by_the_workgroups_that_fit(lib, mb, dtype, dim, resident):
    """One query over many keys is cut into as many parts as workgroups run at once on 256 compute units, or
    half as many again for samples of unequal length, which the workspace has to hold: by the kernel's LDS, of
    160 KB, one or two to a unit."""
    a = _attend(mb, batch=1, queries=1, keys=1 << 20, heads=8, key_heads=2, dim=dim, dtype=dtype, q_row=8 * dim,
                q_head=dim, k_row=2 * dim, k_head=dim, v_row=2 * dim, v_head=dim)
    parts = lib.bevmap_attention_workspace(a, 0) / (8 * (4 * dim + 8))
    assert 0.5 * 256 * resident < 2 * parts <= 1.5 * 256 * resident * 1.01


def test_attention_refuses_more_tiles_than_a_launch_has(lib, mb):
    """By the call that asks for the workspace already: 2048 x 8 problems of 547 tiles each."""
    size = dict(batch=2048, heads=8, key_heads=8, dim=4)
    queries = _attend(mb, **size, queries=70000)
    for backward in (0, 1):
        assert lib.bevmap_attention_workspace(queries, backward) == OVERFLOW
    assert lib.bevmap_attention(queries, P, P, P, None, None, P, None, None, P, 1 << 60, None) == OVERFLOW
    keys = _attend(mb, **size, keys=70000)      # only the backward owns tiles of keys
    assert lib.bevmap_attention_workspace(keys, 0) >= 0
    assert lib.bevmap_attention_workspace(keys, 1) == OVERFLOW
    assert lib.bevmap_attention_backward(keys, P, P, P, P, None, None, P, P, P, P, P, P, P, 1 << 60, None) == OVERFLOW


def test_attention_refuses_pointers_and_workspaces(lib, mb):
    a = _attend(mb)
    need = lib.bevmap_attention_workspace(a, 1)
    assert need > 0
    assert lib.bevmap_attention(a, None, P, P, None, None, P, None, None, P, 1 << 40, None) == INVALID
    assert lib.bevmap_attention(a, P, None, P, None, None, P, None, None, P, 1 << 40, None) == INVALID
    assert lib.bevmap_attention(a, P, P, P, None, None, None, None, None, P, 1 << 40, None) == INVALID
    assert lib.bevmap_attention_backward(a, P, P, P, P, None, None, P, P, P, P, P, P, P, need - 1, None) == INVALID
    assert lib.bevmap_attention_backward(a, P, P, P, P, None, None, P, P, None, P, P, P, P, need, None) == INVALID


@pytest.mark.parametrize("args,code", [
    ((P, 8, P, 8, P, -1, 8, 0, 100, 1, 2), INVALID), ((P, 8, P, 8, P, 4, -8, 0, 100, 1, 2), INVALID),
    ((P, 7, P, 8, P, 4, 8, 0, 100, 1, 2), INVALID), ((P, 8, P, 7, P, 4, 8, 0, 100, 1, 2), INVALID),
    ((P, 8, P, 8, P, 4, 8, 0, -1, 1, 2), INVALID), ((P, 8, P, 8, P, 4, 8, 0, 65537, 1, 2), INVALID),
    ((P, 8, P, 8, P, 4, 8, 3, 100, 1, 2), DTYPE), ((None, 8, P, 8, P, 4, 8, 0, 100, 1, 2), INVALID),
    ((P, 8, P, 8, None, 4, 8, 0, 100, 1, 2), INVALID), ((P, 1 << 31, P, 8, P, 4, 8, 0, 100, 1, 2), OVERFLOW),
    ((P, 1 << 30, None, 0, P, 1 << 12, 1 << 30, 0, 100, 1, 2), OVERFLOW),
    ((None, 0, None, 0, None, 0, 8, 0, 100, 1, 2), 0)])
def test_dropout_refuses(lib, args, code):
    assert lib.bevmap_dropout(*args, None) == code


def test_python_entries_refuse():
    torch = pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    x = torch.zeros(2, 3, 8)
    q = torch.zeros(1, 2, 2, 4)
    for call in (lambda: bev.group_norm_act(x, 2), lambda: bev.cross_attention(q, q, q),
                 lambda: bev.dropout_add(x, 0.1, 3)):
        with pytest.raises(bev.BevpoolError, match="device tensors"):
            call()
    for p, seed, offset in ((-0.1, 0, 0), (1.5, 0, 0), (float("nan"), 0, 0), (0.1, -1, 0), (0.1, 0, 1 << 64)):
        with pytest.raises(bev.BevpoolError, match="outside|must be in"):
            bev.dropout_add(x, p, seed, offset)


def test_forward_mode_is_refused(monkeypatch):
    """An input with a tangent is refused, with gradients enabled or not; the launches are stubs."""
    torch = pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    from paper_2205_13542_amd import map_ops
    from torch.autograd import forward_ad
    monkeypatch.setattr(map_ops, "_norm_forward", lambda x, *a: (x.clone(), x.clone(), None))
    monkeypatch.setattr(map_ops, "_attend_forward", lambda q, *a: (q.clone(), None, q.clone(), None, 0))
    monkeypatch.setattr(map_ops, "_dropout", lambda x, *a: x.clone())
    x, q = torch.ones(2, 3, 8), torch.ones(1, 2, 2, 4)
    with forward_ad.dual_level():
        xd, qd = (forward_ad.make_dual(t, torch.ones_like(t)) for t in (x, q))
        w = forward_ad.make_dual(torch.ones(8), torch.ones(8))
        for call in (lambda: bev.group_norm_act(xd, 2), lambda: bev.group_norm_act(x, 2, w),
                     lambda: bev.cross_attention(qd, q, q), lambda: bev.cross_attention(q, q, qd),
                     lambda: bev.dropout_add(xd, 0.1, 3), lambda: bev.dropout_add(x, 0.1, 3, residual=xd)):
            with pytest.raises(NotImplementedError, match="forward mode"):
                call()
            with torch.no_grad(), pytest.raises(NotImplementedError, match="forward mode"):
                call()
        # inputs without a tangent work
        assert torch.equal(bev.group_norm_act(x, 2), x) and not bev.dropout_add(x, 0.1, 3).requires_grad
    assert torch.equal(bev.cross_attention(q, q, q), q)


def test_star_import_needs_no_torch():
    """Nor does it import torch where there is one; the map operators ask for it when called."""
    code = """
import sys
sys.modules["torch"] = None            # an import of torch raises ImportError
from paper_2205_13542_amd import *
assert bevpool_version() and callable(Plan)
for call in (lambda: group_norm_act(None, 1), lambda: cross_attention(None, None, None),
             lambda: dropout_add(None, 0.1, 3)):
    try:
        call()
    except ImportError:
        continue
    raise SystemExit("a map operator ran without torch")
"""
    done = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert done.returncode == 0, done.stderr


def test_package_names_are_the_map_operators():
    pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    from paper_2205_13542_amd import map_ops
    for name in ("group_norm_act", "cross_attention", "dropout_add"):
        assert name in bev.__all__
        assert inspect.signature(getattr(bev, name)) == inspect.signature(getattr(map_ops, name))


def test_backward_describes_saved_tensors_as_they_come_back(monkeypatch):
    """A hook on saved tensors may bring a strided input back contiguous, or in other rows: what the library
    is told of it then has to be that, or it reads past its end. (Nothing runs here: calls are recorded.)"""
    torch = pytest.importorskip("torch")
    from paper_2205_13542_amd import map_ops
    calls = []
    monkeypatch.setattr(map_ops, "_device", lambda first, *others: 0)
    monkeypatch.setattr(map_ops, "_call", lambda function, index, *args: calls.append(args))

    def spread(t):                                  # each row followed by a row of something else
        room = t.new_zeros((*t.shape[:-1], 2 * t.shape[-1]))
        room[..., :t.shape[-1]] = t
        return room[..., :t.shape[-1]]

    keep = lambda t: t                              # noqa: E731
    hooks = [(keep, keep), (lambda t: t.contiguous().clone(), keep), (spread, keep), (keep, lambda t: t.clone(
        memory_format=torch.contiguous_format))]
    q = torch.zeros(2, 6, 3 * 16)[..., 16:32].unflatten(-1, (2, 8))
    kv = torch.zeros(2, 9, 2, 2, 8)
    mask = torch.ones(2, 20, dtype=torch.bool)[:, :9]
    for pack, unpack in hooks:
        kept = {}

        def back(t, unpack=unpack, kept=kept):
            t = unpack(t)
            kept[t.data_ptr()] = t
            return t

        x, w = torch.zeros(2, 3, 5, 24)[..., 8:16].requires_grad_(), torch.ones(8, requires_grad=True)
        with torch.autograd.graph.saved_tensors_hooks(pack, back):
            y = map_ops.group_norm_act(x, 2, w, w.detach(), act="silu")
            torch.autograd.grad(y, (x, w), torch.zeros_like(y))
        norm, _, at, *rest = calls[-1]
        assert norm.row_stride == kept[at].stride(2) if at in kept else norm.row_stride == 8
        for pointer in rest[:3]:                    # weight, bias, mean
            assert pointer not in kept or kept[pointer].is_contiguous()

        a, k, v = q.detach().requires_grad_(), kv[:, :, 0].requires_grad_(), kv[:, :, 1].requires_grad_()
        kept.clear()
        with torch.autograd.graph.saved_tensors_hooks(pack, back):
            y = map_ops.cross_attention(a, k, v, key_mask=mask)
            torch.autograd.grad(y, (a, k, v), torch.zeros_like(y))
        attend, _, *at = calls[-1]
        for name, pointer in zip("qkv", at):
            got = tuple(getattr(attend, f"{name}_{part}") for part in ("batch", "row", "head"))
            assert got == kept[pointer].stride()[:3] and kept[pointer].stride(3) == 1
        assert at[4] not in kept or attend.mask_batch == kept[at[4]].stride(0)


def test_backward_refuses_saved_tensors_of_another_kind(monkeypatch):
    torch = pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    from paper_2205_13542_amd import map_ops
    monkeypatch.setattr(map_ops, "_device", lambda first, *others: 0)
    monkeypatch.setattr(map_ops, "_call", lambda function, index, *args: None)
    x, q = torch.zeros(2, 5, 8, requires_grad=True), torch.zeros(2, 3, 2, 8, requires_grad=True)
    for change in (lambda t: t[..., :1].clone(), lambda t: t.double()):
        with torch.autograd.graph.saved_tensors_hooks(lambda t: t, change):
            for y, leaf in ((map_ops.group_norm_act(x, 2), x), (map_ops.cross_attention(q, q, q), q)):
                with pytest.raises(bev.BevpoolError, match="saved tensor"):
                    torch.autograd.grad(y, leaf, torch.zeros_like(y))


@pytest.mark.parametrize("tracer", ["jit", "real", "pre_dispatch"])
def test_tracing_is_refused(monkeypatch, tracer):
    """A tracer sees that a result is allocated and not what fills it. (Where a gradient is asked for,
    what torch.jit.trace makes calls the autograd function again.)"""
    torch = pytest.importorskip("torch")
    import paper_2205_13542_amd as bev
    from paper_2205_13542_amd import map_ops
    from torch.fx.experimental.proxy_tensor import make_fx
    monkeypatch.setattr(map_ops, "_device", lambda first, *others: 0)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda index: 0, raising=False)
    ran = []
    for name in ("bevmap_group_norm", "bevmap_attention", "bevmap_dropout"):
        monkeypatch.setattr(map_ops._map_binding, name, lambda *args: ran.append(args))
    x, leaf = torch.ones(1, 4, 2, 8), torch.ones(1, 4, 2, 8, requires_grad=True)

    def trace(call, x=x):
        if tracer == "jit":
            return torch.jit.trace(call, (x,), check_trace=False)
        return make_fx(call, tracing_mode="real", pre_dispatch=tracer == "pre_dispatch")(x)

    for call in (lambda x: map_ops.group_norm_act(x, 2), lambda x: map_ops.cross_attention(x, x, x),
                 lambda x: map_ops.dropout_add(x, 0.1, 3)):
        for enabled in (True, False):
            with torch.set_grad_enabled(enabled), pytest.raises(bev.BevpoolError, match="cannot be traced"):
                trace(call)
        call(x)
        if tracer == "jit":
            again, before = trace(call, leaf), len(ran)
            again(leaf)
            assert len(ran) == before + 1
        else:
            with pytest.raises(bev.BevpoolError, match="cannot be traced"):
                trace(call, leaf)
