"""Refusals of the embedding, layer-norm, router and gradient-clip calls: every check runs on the host before anything is
launched, so they are tested without a GPU (the addresses are made up and never used)."""
import ctypes as C

import pytest

from paper_2505_20524_b200 import binding

OK_ARGS_STATUS = (-6, -8)          # valid arguments get as far as the device check: no device here, or none that fits
A = 1 << 20                        # a 256-byte aligned address


@pytest.fixture(scope="module")
def lib():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the made-up addresses of this file must not reach a device")
    return binding.load()


EMB_FWD = dict(table=A, fp32=0, V=100, D=64, ids=A, i64=1, T=10, scale=1.0, out=A, amax=None, st=None)
EMB_FWD_Q = dict(table=A, fp32=0, V=100, D=64, ids=A, i64=1, T=10, scale=1.0, qs=A, fmt=0, out=A, out8=A, amax=None, st=None)
EMB_BWD = dict(dy=A, ids=A, i64=0, T=10, V=100, D=64, scale=1.0, dtable=A, fp32=0, acc=0, ws=A, nws=1 << 30, st=None)
LN_FWD = dict(x=A, gamma=A, beta=A, res=None, T=10, D=64, eps=1e-5, out=A, mean=None, rstd=None, amax=None, st=None)
LN_FWD_Q = dict(x=A, gamma=A, beta=A, res=None, T=10, D=64, eps=1e-5, qs=A, fmt=0, out=A, out8=A, mean=None, rstd=None,
                amax=None, st=None)
LN_BWD = dict(dout=A, x=A, gamma=A, mean=A, rstd=A, T=10, D=64, dx=A, dgamma=A, dbeta=A, acc=0, ws=A, nws=1 << 30, st=None)
ROUTE = dict(logits=A, fp32=0, bias=None, T=10, E=8, k=2, norm=0, bal=0.01, z=0.0, expert=A, weight=A, counts=A, offsets=A,
             rows=None, n=A, loss=A, ws=A, nws=1 << 30, st=None)
ROUTE_BWD = dict(logits=A, fp32=0, expert=A, counts=A, n=A, T=10, E=8, k=2, norm=0, bal=0.01, z=0.0, dloss=None, dweight=A,
                 dlogits=A, st=None)
NAN = float("nan")
NULL, ALIGN, SHAPE, ENUM, WORKSPACE = -1, -2, -3, -4, -5

CASES = [
    ("fp8_embedding_fwd", EMB_FWD, {}, None),
    ("fp8_embedding_fwd", EMB_FWD, dict(table=None), NULL),
    ("fp8_embedding_fwd", EMB_FWD, dict(ids=None), NULL),
    ("fp8_embedding_fwd", EMB_FWD, dict(out=None), NULL),
    ("fp8_embedding_fwd", EMB_FWD, dict(D=60), SHAPE),
    ("fp8_embedding_fwd", EMB_FWD, dict(D=0), SHAPE),
    ("fp8_embedding_fwd", EMB_FWD, dict(T=0), SHAPE),
    ("fp8_embedding_fwd", EMB_FWD, dict(V=0), SHAPE),
    ("fp8_embedding_fwd", EMB_FWD, dict(T=(1 << 30) + 1), SHAPE),
    ("fp8_embedding_fwd", EMB_FWD, dict(V=(1 << 30) + 1), SHAPE),
    ("fp8_embedding_fwd", EMB_FWD, dict(table=A + 8), ALIGN),
    ("fp8_embedding_fwd", EMB_FWD, dict(ids=A + 4), ALIGN),
    ("fp8_embedding_fwd", EMB_FWD, dict(ids=A + 8), None),
    ("fp8_embedding_fwd", EMB_FWD, dict(ids=A + 4, i64=0), None),
    ("fp8_embedding_fwd", EMB_FWD, dict(ids=A + 2, i64=0), ALIGN),
    ("fp8_embedding_fwd", EMB_FWD, dict(out=A + 2), ALIGN),
    ("fp8_embedding_fwd_q", EMB_FWD_Q, {}, None),
    ("fp8_embedding_fwd_q", EMB_FWD_Q, dict(out=None), None),
    ("fp8_embedding_fwd_q", EMB_FWD_Q, dict(out8=None), NULL),
    ("fp8_embedding_fwd_q", EMB_FWD_Q, dict(qs=None), NULL),
    ("fp8_embedding_fwd_q", EMB_FWD_Q, dict(fmt=2), ENUM),
    ("fp8_embedding_fwd_q", EMB_FWD_Q, dict(out8=A + 8), ALIGN),
    ("fp8_embedding_bwd", EMB_BWD, {}, None),
    ("fp8_embedding_bwd", EMB_BWD, dict(dy=None), NULL),
    ("fp8_embedding_bwd", EMB_BWD, dict(dtable=None), NULL),
    ("fp8_embedding_bwd", EMB_BWD, dict(D=4), SHAPE),
    ("fp8_embedding_bwd", EMB_BWD, dict(T=0), SHAPE),
    ("fp8_embedding_bwd", EMB_BWD, dict(dy=A + 2), ALIGN),
    ("fp8_embedding_bwd", EMB_BWD, dict(dtable=A + 8), ALIGN),
    ("fp8_embedding_bwd", EMB_BWD, dict(ws=None), WORKSPACE),
    ("fp8_embedding_bwd", EMB_BWD, dict(ws=A + 16), WORKSPACE),
    ("fp8_embedding_bwd", EMB_BWD, dict(nws=16), WORKSPACE),
    ("fp8_layernorm_fwd", LN_FWD, {}, None),
    ("fp8_layernorm_fwd", LN_FWD, dict(x=None), NULL),
    ("fp8_layernorm_fwd", LN_FWD, dict(gamma=None), NULL),
    ("fp8_layernorm_fwd", LN_FWD, dict(beta=None), NULL),
    ("fp8_layernorm_fwd", LN_FWD, dict(D=16392), SHAPE),
    ("fp8_layernorm_fwd", LN_FWD, dict(D=12), SHAPE),
    ("fp8_layernorm_fwd", LN_FWD, dict(T=0), SHAPE),
    ("fp8_layernorm_fwd", LN_FWD, dict(eps=-1.0), SHAPE),
    ("fp8_layernorm_fwd", LN_FWD, dict(eps=NAN), SHAPE),
    ("fp8_layernorm_fwd", LN_FWD, dict(res=A + 2), ALIGN),
    ("fp8_layernorm_fwd", LN_FWD, dict(gamma=A + 4), ALIGN),
    ("fp8_layernorm_fwd_q", LN_FWD_Q, {}, None),
    ("fp8_layernorm_fwd_q", LN_FWD_Q, dict(out8=None), NULL),
    ("fp8_layernorm_fwd_q", LN_FWD_Q, dict(qs=None), NULL),
    ("fp8_layernorm_fwd_q", LN_FWD_Q, dict(fmt=-1), ENUM),
    ("fp8_layernorm_bwd", LN_BWD, {}, None),
    ("fp8_layernorm_bwd", LN_BWD, dict(mean=None), NULL),
    ("fp8_layernorm_bwd", LN_BWD, dict(dbeta=None), NULL),
    ("fp8_layernorm_bwd", LN_BWD, dict(D=16392), SHAPE),
    ("fp8_layernorm_bwd", LN_BWD, dict(dx=A + 8), ALIGN),
    ("fp8_layernorm_bwd", LN_BWD, dict(ws=None), WORKSPACE),
    ("fp8_layernorm_bwd", LN_BWD, dict(nws=256), WORKSPACE),
    ("fp8_moe_route", ROUTE, {}, None),
    ("fp8_moe_route", ROUTE, dict(logits=None), NULL),
    ("fp8_moe_route", ROUTE, dict(loss=None), NULL),
    ("fp8_moe_route", ROUTE, dict(E=257), SHAPE),
    ("fp8_moe_route", ROUTE, dict(E=0), SHAPE),
    ("fp8_moe_route", ROUTE, dict(k=9), SHAPE),
    ("fp8_moe_route", ROUTE, dict(k=0), SHAPE),
    ("fp8_moe_route", ROUTE, dict(E=64, k=17), SHAPE),
    ("fp8_moe_route", ROUTE, dict(T=0), SHAPE),
    ("fp8_moe_route", ROUTE, dict(T=(1 << 26) + 1), SHAPE),
    ("fp8_moe_route", ROUTE, dict(bal=NAN), SHAPE),
    ("fp8_moe_route", ROUTE, dict(weight=A + 4), None),
    ("fp8_moe_route", ROUTE, dict(weight=A + 2), ALIGN),
    ("fp8_moe_route", ROUTE, dict(logits=A + 8), ALIGN),
    ("fp8_moe_route", ROUTE, dict(nws=0), WORKSPACE),
    ("fp8_moe_route_bwd", ROUTE_BWD, {}, None),
    ("fp8_moe_route_bwd", ROUTE_BWD, dict(expert=None), NULL),
    ("fp8_moe_route_bwd", ROUTE_BWD, dict(expert=None, dweight=None), None),
    ("fp8_moe_route_bwd", ROUTE_BWD, dict(counts=None), NULL),
    ("fp8_moe_route_bwd", ROUTE_BWD, dict(dlogits=A + 2), ALIGN),
    ("fp8_moe_route_bwd", ROUTE_BWD, dict(E=300), SHAPE),
]


@pytest.mark.parametrize("call,args,change,status", CASES, ids=[f"{c}-{'-'.join(ch) or 'valid'}-{i}" for i, (c, _, ch, _) in enumerate(CASES)])
def test_refusals(lib, call, args, change, status):
    rc = getattr(lib, call)(*{**args, **change}.values())
    if status is None:
        assert rc in OK_ARGS_STATUS
    else:
        assert rc == status
        assert call.split("_q")[0][:12] in lib.fp8_last_error().decode()


def items(*entries):
    arr = (binding.GradItem * len(entries))()
    for i, e in enumerate(entries):
        arr[i] = binding.GradItem(*e)
    return arr, len(entries)


def test_lists_of_gradients_are_checked():
    import torch
    with pytest.raises(ValueError):
        binding.fp8_grad_items([torch.zeros(8)])                 # not on a GPU
    with pytest.raises(ValueError):
        binding.fp8_grad_items([])


def test_gradient_clip_refusals(lib):
    good = (A, A + 4096, 100, 1, 1)
    n = lib.fp8_grad_norm_workspace_bytes(*items(good))
    assert n >= 8 and n % 256 == 0
    assert lib.fp8_grad_norm(*items(good), A, A, n, None) in OK_ARGS_STATUS
    assert lib.fp8_grad_norm(None, 1, A, A, n, None) == NULL
    assert lib.fp8_grad_norm(*items(good), None, A, n, None) == NULL
    assert lib.fp8_grad_norm(items(good)[0], 0, A, A, n, None) == SHAPE
    assert lib.fp8_grad_norm(*items((None, None, 5, 1, 1)), A, A, n, None) == NULL
    assert lib.fp8_grad_norm(*items((None, None, 0, 1, 1)), A, A, n, None) in OK_ARGS_STATUS       # empty tensors have no address
    assert lib.fp8_grad_norm(*items((A + 4, None, 5, 1, 1)), A, A, n, None) == ALIGN
    assert lib.fp8_grad_norm(*items(good), A, A, n - 1, None) == WORKSPACE
    assert lib.fp8_grad_norm(*items(good), A, A + 8, n, None) == WORKSPACE
    assert lib.fp8_grad_clip(*items(good), A, 1.0, None) in OK_ARGS_STATUS
    assert lib.fp8_grad_clip(*items((A, None, 5, 1, 1)), A, 1.0, None) == NULL
    assert lib.fp8_grad_clip(*items((A, A + 2, 5, 1, 1)), A, 1.0, None) == ALIGN
    assert lib.fp8_grad_clip(*items((A, A, 5, 1, 0)), A, 1.0, None) == SHAPE                          # in place, two types
    for bad in (0.0, -1.0, NAN, float("inf")):
        assert lib.fp8_grad_clip(*items(good), A, bad, None) == SHAPE
    assert lib.fp8_grad_clip(*items(good), None, 1.0, None) == NULL


def test_workspace_sizes_are_host_arithmetic(lib):
    assert lib.fp8_embedding_bwd_workspace_bytes(10, 100, 60) == 0                     # unsupported shape
    assert lib.fp8_layernorm_bwd_workspace_bytes(0, 64) == 0
    assert lib.fp8_moe_route_workspace_bytes(10, 300) == 0
    for T in (1, 31, 33, 8192, 600001, 1 << 24):
        for V in (1, 1000, 1 << 20):
            n = lib.fp8_embedding_bwd_workspace_bytes(T, V, 64)
            assert n >= 16 * T and n % 256 == 0
        assert 0 < lib.fp8_layernorm_bwd_workspace_bytes(T, 4096) <= 148 * 8 * 2 * 4096 * 4
        assert 0 < lib.fp8_moe_route_workspace_bytes(T, 256) < 1 << 20


def test_layouts_of_the_item_structure_match_the_header(tmp_path):
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "layout.c"
    names = [f[0] for f in binding.GradItem._fields_]
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "fp8dpa.h"\nint main(void) { printf("%zu", sizeof(fp8_grad_item));\n'
                   + "".join(f'printf(" %zu", offsetof(fp8_grad_item, {n}));\n' for n in names) + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    out = [int(v) for v in subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()]
    assert out == [C.sizeof(binding.GradItem)] + [getattr(binding.GradItem, n).offset for n in names]
