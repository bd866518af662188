"""Refusals of the cross-attention branch's calls, by the library and by the binding; no GPU is touched."""
import ctypes

import pytest
import torch

from paper_2607_04461_amd import flashbon as fb

P = 1 << 20      # addresses that no call reaches; each buffer far from the others


def at(i):
    return P + (i << 32)


NORM = dict(dtype=1, M=4, D=8, eps=1e-6, x=at(0), per=2, weight=at(1), modulated=0, bias=at(2), out=at(3), mean=at(4),
            rstd=at(5), stream=None)
NORM_GRAD = dict(dtype=1, M=400, D=8, x=at(0), per=200, weight=at(1), modulated=0, mean=at(2), rstd=at(3), dy=at(4),
                 residual=at(5), dx=at(6), dweight=at(7), dbias=at(8), workspace=at(9), workspace_bytes=1 << 30, stream=None)
CROSS = dict(dtype=1, batch=2, heads=4, kv_heads=2, head_dim=16, tq=3, tk=5, q=at(0), q_bs=192, q_rs=64, k=at(1), v=at(2),
             kv_bs=160, kv_rs=32, kv_index=at(3), n_kv=2, kv_len=at(4), out=at(5), o_bs=192, o_rs=64, lse=at(6),
             workspace=at(7), workspace_bytes=1 << 30, stream=None)
CROSS_GRAD = {k: v for k, v in CROSS.items() if k not in ("workspace", "workspace_bytes", "stream")}
CROSS_GRAD.update(dout=at(8), dq=at(9), dk=at(10), dv=at(11), workspace=at(7), workspace_bytes=1 << 30, stream=None)
ADAPTERS = dict(dtype=1, M=6, N=16, K=24, rank=8, count=2, x=at(0), down=at(1), up=at(2), scales=at(3), index=at(4), per=2,
                epilogue=0, gate=None, base=at(5), out=at(6), u=at(7), stream=None)
ADAPTERS_GRAD = dict(dtype=1, M=6, N=16, K=24, rank=8, count=2, x=at(0), down=at(1), up=at(2), scales=at(3), index=at(4), per=2,
                     u=at(5), dy=at(6), epilogue=0, base=at(7), dx=at(8), d_down=at(9), d_up=at(10), workspace=at(11),
                     workspace_bytes=1 << 30, stream=None)

REFUSED = [
    ("layer_norm", NORM, fb.EINVAL, [{"dtype": 2}, {"x": None}, {"out": None}, {"eps": 0.0}, {"eps": float("inf")},
                                     {"eps": float("nan")}, {"out": at(0) + 64}, {"mean": at(5)}, {"rstd": at(1) + 8},
                                     {"mean": at(3) + 60}]),
    ("layer_norm", NORM, fb.ESHAPE, [{"M": 0}, {"D": 0}, {"D": 6145}, {"per": 0}, {"M": -1}]),
    ("layer_norm_grad", NORM_GRAD, fb.EINVAL, [{"dtype": -1}, {"x": None}, {"mean": None}, {"rstd": None}, {"dy": None},
                                               {"dx": None, "dweight": None, "dbias": None}, {"dx": at(0)}, {"dx": at(4)},
                                               {"dx": at(5) + 4}, {"dweight": at(1)}, {"dweight": at(8)},
                                               {"workspace": at(6)}, {"workspace": at(9) + 8}]),
    ("layer_norm_grad", NORM_GRAD, fb.ESHAPE, [{"M": 0}, {"D": 6145}, {"per": 0}, {"workspace": None}, {"workspace_bytes": 64},
                                               {"M": 1 << 25, "per": 1}]),
    ("cross_attention", CROSS, fb.EINVAL, [{"dtype": 7}, {"q": None}, {"k": None}, {"v": None}, {"out": None}, {"q": at(0) + 8},
                                           {"k": at(1) + 2}, {"out": at(5) + 4}, {"lse": at(6) + 2}, {"q_rs": 60}, {"kv_bs": -160},
                                           {"q_bs": 1 << 36}, {"o_rs": 56}, {"o_bs": 128}, {"o_rs": 0}, {"out": at(0)},
                                           {"lse": at(1)}, {"lse": at(5) + 64}, {"out": at(4)}]),
    ("cross_attention", CROSS, fb.ESHAPE, [{"batch": 0}, {"heads": 0}, {"kv_heads": 0}, {"kv_heads": 3}, {"head_dim": 24},
                                           {"head_dim": 256}, {"tq": 0}, {"tk": 0}, {"n_kv": 0}, {"kv_index": None, "n_kv": 3},
                                           {"tq": (1 << 24) + 1}, {"batch": 1 << 20, "heads": 16}, {"n_kv": 32768}]),
    ("cross_attention_grad", CROSS_GRAD, fb.EINVAL, [{"lse": None}, {"dout": None}, {"dk": None}, {"dv": None},
                                                     {"dq": None, "dk": None, "dv": None}, {"dq": at(9) + 8}, {"q_rs": 56},
                                                     {"q_bs": 0}, {"kv_rs": 24}, {"kv_bs": 0}, {"dq": at(0)}, {"dk": at(1)},
                                                     {"dv": at(10)}, {"dv": at(10) + 32}, {"dv": at(10) + 64},
                                                     {"dv": at(10) - 64}, {"dv": at(10) + 64, "kv_rs": 56},
                                                     {"dv": at(10) + 64, "kv_rs": 64, "kv_bs": 312}, {"dq": at(8)}, {"dk": at(7)},
                                                     {"workspace": at(5)}, {"workspace": at(7) + 4}, {"dv": at(9)}]),
    ("cross_attention_grad", CROSS_GRAD, fb.ESHAPE, [{"batch": 4097}, {"workspace": None}, {"workspace_bytes": 16},
                                                     {"head_dim": 12}, {"kv_index": None, "n_kv": 1}]),
    ("adapters", ADAPTERS, fb.EINVAL, [{"dtype": 3}, {"x": None}, {"down": None}, {"up": None}, {"out": None}, {"u": None},
                                       {"epilogue": 1}, {"epilogue": 4}, {"epilogue": -1}, {"x": at(0) + 8}, {"u": at(7) + 4},
                                       {"index": at(4) + 2}, {"out": at(0)}, {"u": at(6)}, {"out": at(5) + 16}, {"u": at(1)},
                                       {"epilogue": 3, "gate": at(6)}]),
    ("adapters", ADAPTERS, fb.ESHAPE, [{"M": 0}, {"M": (1 << 22) + 1}, {"N": 12}, {"K": 20}, {"N": 0}, {"K": 65544}, {"rank": 4},
                                       {"rank": 136}, {"rank": 12}, {"count": 0}, {"count": 1025}, {"per": 0}]),
    ("adapters_grad", ADAPTERS_GRAD, fb.EINVAL, [{"u": None}, {"dy": None}, {"dx": None, "d_down": None, "d_up": None},
                                                 {"epilogue": 3}, {"epilogue": 1}, {"dx": at(0)}, {"d_down": at(10)},
                                                 {"d_up": at(2)}, {"workspace": at(8)}, {"dx": at(7) + 16}, {"dy": at(6) + 2}]),
    ("adapters_grad", ADAPTERS_GRAD, fb.ESHAPE, [{"workspace": None}, {"workspace_bytes": 256}, {"rank": 0}, {"M": -5}]),
]


@pytest.mark.parametrize("name,call,status,change", [(n, c, s, x) for n, c, s, changes in REFUSED for x in changes])
def test_refused(name, call, status, change):
    args = dict(call, **change)
    got = getattr(fb.load(), "flashbon_op_" + name)(*args.values())
    assert got == status, (got, fb.load().flashbon_last_error())


def test_workspaces():
    lib = fb.load()
    assert lib.flashbon_op_layer_norm_grad_workspace(24960, 1536, 1560) > 0
    assert lib.flashbon_op_layer_norm_grad_workspace(16, 64, 1) == 0          # a group a chunk: none needed
    assert lib.flashbon_op_layer_norm_grad_workspace(0, 64, 1) == 0
    assert lib.flashbon_op_cross_attention_workspace(1, 1, 40, 40, 128, 1, 4096) > 0
    assert lib.flashbon_op_cross_attention_workspace(1, 16, 12, 12, 128, 1560, 512) == 0
    assert lib.flashbon_op_cross_attention_workspace(1, 1, 40, 39, 128, 1, 4096) == 0
    assert lib.flashbon_op_cross_attention_grad_workspace(1, 2, 4, 2, 16, 3, 5, 2) >= 4 * 24
    assert lib.flashbon_op_cross_attention_grad_workspace(1, 5000, 4, 2, 16, 3, 5, 2) == 0
    assert lib.flashbon_op_adapters_grad_workspace(1, 6, 16, 24, 8, 2, 2) > 0
    assert lib.flashbon_op_adapters_grad_workspace(1, 6, 16, 24, 7, 2, 2) == 0


def bf(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16)


def f32(*shape):
    return torch.zeros(shape)


def i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def norm(**change):
    a = dict(dtype=fb.BF16, M=4, D=8, x=f32(4, 8), out=bf(4, 8), weight=f32(2, 8), bias=f32(2, 8), rows_per_group=2, mean=f32(4), rstd=f32(4))
    a.update(change)
    return fb.validate_layer_norm(**a, require_device=False)


def norm_grad(**change):
    a = dict(dtype=fb.BF16, M=4, D=8, x=f32(4, 8), mean=f32(4), rstd=f32(4), dy=bf(4, 8), dx=f32(4, 8), weight=f32(2, 8),
             rows_per_group=2, residual=f32(4, 8), dweight=f32(2, 8), dbias=f32(2, 8), workspace=f32(9))
    a.update(change)
    return fb.validate_layer_norm_grad(**a, require_device=False)


def cross(**change):
    kv = bf(2, 5, 64)
    a = dict(dtype=fb.BF16, batch=2, heads=4, kv_heads=2, head_dim=16, tq=3, tk=5, q=bf(2, 3, 64), q_bs=192, q_rs=64,
             k=kv[:, :, :32], v=kv[:, :, 32:], kv_bs=320, kv_rs=64, kv_index=i32(2), n_kv=2, kv_len=i32(2), out=bf(2, 3, 64),
             o_bs=192, o_rs=64, lse=f32(2, 4, 3))
    a.update(change)
    return fb.validate_cross_attention(**a, require_device=False)


def cross_grad(**change):
    kv, dkv = bf(2, 5, 64), bf(2, 5, 64)
    a = dict(dtype=fb.BF16, batch=2, heads=4, kv_heads=2, head_dim=16, tq=3, tk=5, q=bf(2, 3, 64), q_bs=192, q_rs=64,
             k=kv[:, :, :32], v=kv[:, :, 32:], kv_bs=320, kv_rs=64, kv_index=i32(2), n_kv=2, kv_len=i32(2), out=bf(2, 3, 64),
             o_bs=192, o_rs=64, lse=f32(2, 4, 3), dout=bf(2, 3, 64), dq=bf(2, 3, 64), dk=dkv[:, :, :32], dv=dkv[:, :, 32:])
    a.update(change)
    return fb.validate_cross_attention_grad(**a, require_device=False)


def adapters(**change):
    a = dict(dtype=fb.BF16, M=6, N=16, K=24, rank=8, n_adapters=2, x=bf(6, 24), down=bf(2, 8, 24), up=bf(2, 16, 8), scales=f32(2),
             index=i32(3), rows_per_group=2, epilogue=fb.EPI_STORE, base=bf(6, 16), out=bf(6, 16), u=f32(6, 8))
    a.update(change)
    return fb.validate_adapters(**a, require_device=False)


def adapters_grad(**change):
    a = dict(dtype=fb.BF16, M=6, N=16, K=24, rank=8, n_adapters=2, x=bf(6, 24), down=bf(2, 8, 24), up=bf(2, 16, 8), scales=f32(2),
             index=i32(3), rows_per_group=2, u=f32(6, 8), dy=bf(6, 16), epilogue=fb.EPI_STORE_F32, base=f32(6, 24),
             dx=f32(6, 24), d_down=f32(2, 8, 24), d_up=f32(2, 16, 8), workspace=f32(64))
    a.update(change)
    return fb.validate_adapters_grad(**a, require_device=False)


@pytest.mark.parametrize("check", [norm, norm_grad, cross, cross_grad, adapters, adapters_grad])
def test_binding_takes_what_fits(check):
    assert all(p is None or isinstance(p, int) for p in check())


@pytest.mark.parametrize("check,change", [
    (norm, {"x": None}), (norm, {"x": bf(4, 8)}), (norm, {"out": f32(4, 8)}), (norm, {"out": bf(4, 7)}), (norm, {"weight": f32(1, 8)}),
    (norm, {"rows_per_group": 1}), (norm, {"rows_per_group": 0}), (norm, {"mean": f32(3)}), (norm, {"x": f32(8, 4).t()}),
    (norm, {"M": 1 << 31}),
    (norm_grad, {"dy": f32(4, 8)}), (norm_grad, {"rstd": None}), (norm_grad, {"dbias": f32(1, 8)}), (norm_grad, {"residual": f32(31)}),
    (norm_grad, {"workspace": f32(4, 4)[:, :2]}),
    (cross, {"q": None}), (cross, {"q": f32(2, 3, 64)}), (cross, {"q": bf(2, 3, 63)}), (cross, {"kv_bs": 400}), (cross, {"kv_rs": -64}),
    (cross, {"kv_index": i32(1)}), (cross, {"kv_index": torch.zeros(2, dtype=torch.int64)}), (cross, {"kv_len": i32(1)}),
    (cross, {"lse": f32(23)}), (cross, {"out": bf(383)}), (cross, {"tq": 0}), (cross, {"q_bs": 1 << 40}), (cross, {"heads": 1 << 32}),
    (cross_grad, {"lse": None}), (cross_grad, {"dout": None}), (cross_grad, {"dq": f32(2, 3, 64)}), (cross_grad, {"dv": bf(2, 5, 31)}),
    (cross_grad, {"out": bf(2, 2, 64)}),
    (adapters, {"x": f32(6, 24)}), (adapters, {"index": i32(2)}), (adapters, {"out": f32(6, 16)}), (adapters, {"epilogue": fb.EPI_RESIDUAL}),
    (adapters, {"u": f32(47)}), (adapters, {"scales": f32(1)}), (adapters, {"up": bf(2, 15, 8)}), (adapters, {"down": None}),
    (adapters_grad, {"dx": bf(6, 24)}), (adapters_grad, {"d_up": f32(2, 16, 7)}), (adapters_grad, {"dy": bf(6, 15)}),
    (adapters_grad, {"base": bf(6, 24)}), (adapters_grad, {"u": None}),
])
def test_binding_refuses(check, change):
    with pytest.raises(ValueError):
        check(**change)


def test_binding_refuses_host_tensors():
    if torch.cuda.is_available():
        with pytest.raises(ValueError, match="current device"):
            fb.flashbon_op_layer_norm(fb.BF16, 4, 8, 1e-6, f32(4, 8), bf(4, 8))


def test_arguments_match_the_header():
    lib = fb.load()
    for name, call in (("layer_norm", NORM), ("layer_norm_grad", NORM_GRAD), ("cross_attention", CROSS),
                       ("cross_attention_grad", CROSS_GRAD), ("adapters", ADAPTERS), ("adapters_grad", ADAPTERS_GRAD)):
        assert len(getattr(lib, "flashbon_op_" + name).argtypes) == len(call), name
    assert ctypes.sizeof(ctypes.c_size_t) == 8
