"""Refusals of the rotary-position, block-joint and AdamW calls: every check runs on the host before anything is launched, so they
are tested without a GPU (the addresses are made up and never used)."""
import ctypes as C
import math

import pytest

from paper_2505_20524_b200 import binding

OK_ARGS_STATUS = (-6, -8)          # valid arguments get as far as the device check: no device here, or none that fits
A = 1 << 20                        # a 256-byte aligned address
NAN, INF = math.nan, math.inf
NULL, ALIGN, SHAPE, ENUM, WORKSPACE = -1, -2, -3, -4, -5


@pytest.fixture(scope="module")
def lib():
    import torch
    if torch.cuda.is_available():
        pytest.skip("the made-up addresses of this file must not reach a device")
    return binding.load()


ROPE = dict(mode=0, alpha=1.0, eps=1e-6, cos=A, sin=A, n_pos=100, rot=64, inter=0, pos=None, i64=0)
TABLE = dict(n_pos=100, rot=64, base=1e4, kind=3, factor=4.0, length=2048.0, low=1.0, high=32.0, mag=1.0, cos=A, sin=A, st=None)
FWD = dict(qkv=A, pitch=512, T=10, Hq=4, Hkv=2, d=64, rope=ROPE, q=A, k=A, v=A, amax=None, st=None)
FWD_Q = dict(qkv=A, pitch=512, T=10, Hq=4, Hkv=2, d=64, rope=ROPE, scales=A, fmt=0, q=None, k=None, v=None, q8=A, k8=A, v8=A, amax=None, st=None)
BWD = dict(dq=A, dk=A, dv=A, qkv=A, pitch=512, T=10, Hq=4, Hkv=2, d=64, rope=ROPE, dqkv=A, opitch=512, amax=None, st=None)
BWD_Q = dict(dq=A, dk=A, dv=A, qkv=A, pitch=512, T=10, Hq=4, Hkv=2, d=64, rope=ROPE, scale=A, fmt=1, dqkv=None, opitch=0, dqkv8=A, amax=None, st=None)
CFG = dict(post=0, gate=1, a=1.0, b=1.0, eps=1e-5)
NORM = dict(x=A, y=A, gate=A, gq=A, gp=A, T=10, D=64, cfg=CFG, h=A, out=A, rq=None, rp=None, amax=None, st=None)
NORM_Q = dict(x=A, y=A, gate=A, gq=A, gp=A, T=10, D=64, cfg=CFG, scale=A, fmt=0, h=A, out=None, out8=A, rq=None, rp=None, amax=None, st=None)
GRAD = dict(dout=A, dh=A, h=A, y=A, gate=A, gq=A, gp=A, rq=A, rp=A, T=10, D=64, cfg=CFG, dx=A, dy=A, dgate=A, dgq=A, dgp=A, acc=0, amax=None,
            ws=A, nws=1 << 30, st=None)
GRAD_Q = dict(dout=A, dh=A, h=A, y=A, gate=A, gq=A, gp=A, rq=A, rp=A, T=10, D=64, cfg=CFG, scale=A, fmt=1, dx=A, dy=None, dy8=A, dgate=A, dgq=A,
              dgp=A, acc=0, amax=None, ws=A, nws=1 << 30, st=None)
rope = lambda **k: dict(rope=ROPE | k)  # noqa: E731
cfg = lambda **k: dict(cfg=CFG | k)  # noqa: E731
NO_PRE = dict(gp=None, out=None)

CASES = [
    ("fp8_rope_table", TABLE, {}, None),
    ("fp8_rope_table", TABLE, dict(cos=None), NULL),
    ("fp8_rope_table", TABLE, dict(sin=A + 4), ALIGN),
    ("fp8_rope_table", TABLE, dict(kind=4), ENUM),
    ("fp8_rope_table", TABLE, dict(n_pos=0), SHAPE),
    ("fp8_rope_table", TABLE, dict(n_pos=1 << 31), SHAPE),
    ("fp8_rope_table", TABLE, dict(rot=0), SHAPE),
    ("fp8_rope_table", TABLE, dict(rot=24), SHAPE),
    ("fp8_rope_table", TABLE, dict(rot=272), SHAPE),
    ("fp8_rope_table", TABLE, dict(rot=256), None),
    ("fp8_rope_table", TABLE, dict(base=0.0), SHAPE),
    ("fp8_rope_table", TABLE, dict(base=NAN), SHAPE),
    ("fp8_rope_table", TABLE, dict(factor=0.0), SHAPE),
    ("fp8_rope_table", TABLE, dict(factor=0.0, kind=0), None),
    ("fp8_rope_table", TABLE, dict(length=-1.0), SHAPE),
    ("fp8_rope_table", TABLE, dict(length=-1.0, kind=2), None),
    ("fp8_rope_table", TABLE, dict(low=32.0), SHAPE),
    ("fp8_rope_table", TABLE, dict(mag=INF), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, {}, None),
    ("fp8_rope_qkv_fwd", FWD, dict(rope=None), NULL),
    ("fp8_rope_qkv_fwd", FWD, dict(qkv=None), NULL),
    ("fp8_rope_qkv_fwd", FWD, dict(q=None, k=None, v=None), NULL),
    ("fp8_rope_qkv_fwd", FWD, dict(q=None, v=None), None),
    ("fp8_rope_qkv_fwd", FWD, rope(cos=None), NULL),
    ("fp8_rope_qkv_fwd", FWD, rope(cos=None, sin=None, rot=0, n_pos=0), None),
    ("fp8_rope_qkv_fwd", FWD, rope(mode=3), ENUM),
    ("fp8_rope_qkv_fwd", FWD, rope(rot=80), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, rope(rot=24), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, rope(n_pos=0), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, rope(eps=-1.0), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, rope(alpha=INF), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, rope(pos=A + 4, i64=0), None),
    ("fp8_rope_qkv_fwd", FWD, rope(pos=A + 4, i64=1), ALIGN),
    ("fp8_rope_qkv_fwd", FWD, rope(sin=A + 8), ALIGN),
    ("fp8_rope_qkv_fwd", FWD, dict(T=0), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(T=1 << 31), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(Hq=0), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(Hkv=-1), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(Hq=65537, pitch=1 << 30), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(d=72, pitch=1024), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(d=272, pitch=4096), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(pitch=504), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(pitch=516), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(pitch=520), None),
    ("fp8_rope_qkv_fwd", FWD, dict(Hkv=0), SHAPE),
    ("fp8_rope_qkv_fwd", FWD, dict(Hkv=0, k=None, v=None), None),
    ("fp8_rope_qkv_fwd", FWD, dict(qkv=A + 8), ALIGN),
    ("fp8_rope_qkv_fwd", FWD, dict(v=A + 2), ALIGN),
    ("fp8_rope_qkv_fwd_q", FWD_Q, {}, None),
    ("fp8_rope_qkv_fwd_q", FWD_Q, dict(scales=None), NULL),
    ("fp8_rope_qkv_fwd_q", FWD_Q, dict(q8=None, k8=None, v8=None, q=A), NULL),
    ("fp8_rope_qkv_fwd_q", FWD_Q, dict(q8=None, v8=None), None),
    ("fp8_rope_qkv_fwd_q", FWD_Q, dict(fmt=2), ENUM),
    ("fp8_rope_qkv_fwd_q", FWD_Q, dict(k8=A + 8), ALIGN),
    ("fp8_rope_qkv_bwd", BWD, {}, None),
    ("fp8_rope_qkv_bwd", BWD, dict(dq=None), NULL),
    ("fp8_rope_qkv_bwd", BWD, dict(dk=None), NULL),
    ("fp8_rope_qkv_bwd", BWD, dict(dk=None, dv=None, Hkv=0), None),
    ("fp8_rope_qkv_bwd", BWD, dict(qkv=None), NULL),
    ("fp8_rope_qkv_bwd", BWD, dict(qkv=None, pitch=0) | rope(mode=2), None),
    ("fp8_rope_qkv_bwd", BWD, dict(dqkv=None), NULL),
    ("fp8_rope_qkv_bwd", BWD, dict(opitch=511), SHAPE),
    ("fp8_rope_qkv_bwd", BWD, dict(pitch=256), SHAPE),
    ("fp8_rope_qkv_bwd", BWD, dict(dv=A + 4), ALIGN),
    ("fp8_rope_qkv_bwd_q", BWD_Q, {}, None),
    ("fp8_rope_qkv_bwd_q", BWD_Q, dict(dqkv8=None), NULL),
    ("fp8_rope_qkv_bwd_q", BWD_Q, dict(scale=None), NULL),
    ("fp8_rope_qkv_bwd_q", BWD_Q, dict(fmt=-1), ENUM),
    ("fp8_rope_qkv_bwd_q", BWD_Q, dict(dqkv=A, opitch=8), SHAPE),
    ("fp8_rope_qkv_bwd_q", BWD_Q, dict(dqkv8=A + 1), ALIGN),
    ("fp8_block_norm_fwd", NORM, {}, None),
    ("fp8_block_norm_fwd", NORM, dict(cfg=None), NULL),
    ("fp8_block_norm_fwd", NORM, dict(x=None), NULL),
    ("fp8_block_norm_fwd", NORM, dict(y=None), NULL),                            # a gate without y
    ("fp8_block_norm_fwd", NORM, dict(y=None, gate=None), None),
    ("fp8_block_norm_fwd", NORM, dict(y=None, gate=None, h=None), None),
    ("fp8_block_norm_fwd", NORM, dict(y=None, gate=None, h=None) | cfg(a=2.0), SHAPE),
    ("fp8_block_norm_fwd", NORM, dict(h=None), SHAPE),
    ("fp8_block_norm_fwd", NORM, dict(gq=None), NULL),
    ("fp8_block_norm_fwd", NORM, dict(gq=None) | cfg(post=2), None),
    ("fp8_block_norm_fwd", NORM, dict(out=None), NULL),
    ("fp8_block_norm_fwd", NORM, NO_PRE, None),
    ("fp8_block_norm_fwd", NORM, NO_PRE | dict(h=None), NULL),
    ("fp8_block_norm_fwd", NORM, dict(gp=None), SHAPE),
    ("fp8_block_norm_fwd", NORM, cfg(post=3), ENUM),
    ("fp8_block_norm_fwd", NORM, cfg(gate=2), ENUM),
    ("fp8_block_norm_fwd", NORM, cfg(eps=-1.0), SHAPE),
    ("fp8_block_norm_fwd", NORM, cfg(eps=NAN), SHAPE),
    ("fp8_block_norm_fwd", NORM, cfg(b=INF), SHAPE),
    ("fp8_block_norm_fwd", NORM, cfg(a=NAN), SHAPE),
    ("fp8_block_norm_fwd", NORM, dict(T=0), SHAPE),
    ("fp8_block_norm_fwd", NORM, dict(D=60), SHAPE),
    ("fp8_block_norm_fwd", NORM, dict(D=16392), SHAPE),
    ("fp8_block_norm_fwd", NORM, dict(gate=A + 8), ALIGN),
    ("fp8_block_norm_fwd", NORM, dict(gp=A + 4), ALIGN),
    ("fp8_block_norm_fwd_q", NORM_Q, {}, None),
    ("fp8_block_norm_fwd_q", NORM_Q, dict(out8=None), NULL),
    ("fp8_block_norm_fwd_q", NORM_Q, dict(scale=None), NULL),
    ("fp8_block_norm_fwd_q", NORM_Q, dict(fmt=3), ENUM),
    ("fp8_block_norm_fwd_q", NORM_Q, NO_PRE, None),
    ("fp8_block_norm_fwd_q", NORM_Q, dict(out8=A + 8), ALIGN),
    ("fp8_block_norm_bwd", GRAD, {}, None),
    ("fp8_block_norm_bwd", GRAD, dict(dh=None), None),
    ("fp8_block_norm_bwd", GRAD, dict(dout=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(h=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(rp=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(rq=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(rq=None) | cfg(post=1), None),
    ("fp8_block_norm_bwd", GRAD, dict(rq=None, gq=None, dgq=None) | cfg(post=2), None),
    ("fp8_block_norm_bwd", GRAD, dict(dgq=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(dgp=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(dgate=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(dx=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(dy=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(gp=None, dout=None), None),
    ("fp8_block_norm_bwd", GRAD, dict(gp=None), SHAPE),
    ("fp8_block_norm_bwd", GRAD, dict(gp=None, dout=None, dh=None), NULL),
    ("fp8_block_norm_bwd", GRAD, dict(y=None, gate=None), SHAPE),
    ("fp8_block_norm_bwd", GRAD, dict(y=None, gate=None, dy=None, dgate=None), None),
    ("fp8_block_norm_bwd", GRAD, dict(D=4), SHAPE),
    ("fp8_block_norm_bwd", GRAD, dict(dgate=A + 8), ALIGN),
    ("fp8_block_norm_bwd", GRAD, dict(ws=None), WORKSPACE),
    ("fp8_block_norm_bwd", GRAD, dict(ws=A + 16), WORKSPACE),
    ("fp8_block_norm_bwd", GRAD, dict(nws=256), WORKSPACE),
    ("fp8_block_norm_bwd_q", GRAD_Q, {}, None),
    ("fp8_block_norm_bwd_q", GRAD_Q, dict(dy=A), None),
    ("fp8_block_norm_bwd_q", GRAD_Q, dict(dy8=None), NULL),
    ("fp8_block_norm_bwd_q", GRAD_Q, dict(scale=None), NULL),
    ("fp8_block_norm_bwd_q", GRAD_Q, dict(fmt=7), ENUM),
    ("fp8_block_norm_bwd_q", GRAD_Q, dict(dy8=A + 2), ALIGN),
]


@pytest.mark.parametrize("i", range(len(CASES)))
def test_refusals_before_any_launch(lib, i):
    name, base, change, status = CASES[i]
    args = base | change
    if isinstance(args.get("rope"), dict):
        args["rope"] = C.byref(binding.Rope(*args["rope"].values()))
    if isinstance(args.get("cfg"), dict):
        args["cfg"] = C.byref(binding.BlockNorm(*args["cfg"].values()))
    rc = getattr(lib, name)(*args.values())
    assert rc in OK_ARGS_STATUS if status is None else rc == status, (name, change, rc, lib.fp8_last_error())
    if status is not None:
        assert name.removesuffix("_q") in lib.fp8_last_error().decode()


ITEM = dict(p=A, g=A, m=A, v=A, me=A, ve=A, p16=A, p8=A, q=A, amax=A, n=300, wd=0.1, f32=0, bits=8, fmt=0)
ADAMW = dict(lr=A, step=A, b1=0.9, b2=0.95, eps=1e-8, norm=A, max_norm=1.0, seed=1, ws=A, nws=256, st=None)
ADAMW_CASES = [
    ({}, {}, None), (dict(p=None), {}, NULL), (dict(g=None), {}, NULL), (dict(m=None), {}, NULL), (dict(v=None), {}, NULL),
    (dict(me=None), {}, NULL), (dict(ve=None), {}, NULL), (dict(me=None, ve=None, bits=32), {}, None), (dict(q=None), {}, NULL),
    (dict(q=None, p8=None, p16=None, amax=None), {}, None), (dict(bits=16), {}, ENUM), (dict(fmt=2), {}, ENUM),
    (dict(p=A + 4), {}, ALIGN), (dict(g=A + 2), {}, ALIGN), (dict(m=A + 8), {}, ALIGN), (dict(p16=A + 2), {}, ALIGN), (dict(p8=A + 8), {}, ALIGN),
    (dict(q=A + 2), {}, ALIGN), (dict(amax=A + 1), {}, ALIGN),
    (dict(me=A + 1, ve=A + 3), {}, None), (dict(wd=-0.1), {}, SHAPE), (dict(wd=NAN), {}, SHAPE), (dict(n=(1 << 40) + 1), {}, SHAPE),
    (dict(n=0, p=None, g=None, bits=5), {}, None),
    ({}, dict(lr=None), NULL), ({}, dict(step=None), NULL), ({}, dict(lr=A + 2), ALIGN), ({}, dict(norm=None, max_norm=NAN), None),
    ({}, dict(max_norm=0.0), SHAPE), ({}, dict(max_norm=INF), SHAPE), ({}, dict(b1=1.0), SHAPE), ({}, dict(b1=-0.1), SHAPE),
    ({}, dict(b2=NAN), SHAPE), ({}, dict(b1=0.0, b2=0.0), None), ({}, dict(eps=0.0), SHAPE), ({}, dict(eps=INF), SHAPE),
    ({}, dict(ws=None), WORKSPACE), ({}, dict(ws=A + 128), WORKSPACE), ({}, dict(nws=255), WORKSPACE),
]


@pytest.mark.parametrize("i", range(len(ADAMW_CASES)))
def test_adamw_refusals(lib, i):
    item, change, status = ADAMW_CASES[i]
    items = (binding.AdamWItem * 2)(binding.AdamWItem(*ITEM.values()), binding.AdamWItem(*(ITEM | item).values()))
    rc = lib.fp8_adamw(items, 2, *(ADAMW | change).values())
    assert rc in OK_ARGS_STATUS if status is None else rc == status, (item, change, rc, lib.fp8_last_error())
    if status is not None:
        assert "fp8_adamw" in lib.fp8_last_error().decode()


def test_adamw_refuses_no_list(lib):
    assert lib.fp8_adamw(None, 1, *ADAMW.values()) == NULL
    assert lib.fp8_adamw((binding.AdamWItem * 1)(), 0, *ADAMW.values()) == SHAPE
    assert lib.fp8_adamw_workspace_bytes(None, 1) == 0 and lib.fp8_adamw_workspace_bytes((binding.AdamWItem * 1)(), 1) == 256
    assert lib.fp8_block_norm_bwd_workspace_bytes(0, 64) == 0 and lib.fp8_block_norm_bwd_workspace_bytes(5, 63) == 0


def test_structures_have_the_header_layout(tmp_path):
    import os
    import re
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    pairs = {"fp8_rope": binding.Rope, "fp8_block_norm": binding.BlockNorm, "fp8_adamw_item": binding.AdamWItem}
    text = open(os.path.join(root, "include", "fp8dpa.h")).read()
    lines = ["#include <stdio.h>", "#include <stddef.h>", '#include "fp8dpa.h"', "int main(void) {"]
    for name, st in pairs.items():
        body = re.search(r"typedef struct \{([^{}]*)\}\s*" + name + r"\s*;", text, re.S).group(1)
        body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
        fields = [re.findall(r"\w+", part)[-1] for d in body.split(";") if d.strip() for part in d.split(",")]
        assert fields == [f[0] for f in st._fields_], (name, fields)
        lines.append(f'printf("%zu", sizeof({name}));')
        lines += [f'printf(" %zu", offsetof({name}, {f}));' for f in fields]
        lines.append('printf("\\n");')
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split("\n")
    for st, line in zip(pairs.values(), out):
        assert [C.sizeof(st)] + [getattr(st, f[0]).offset for f in st._fields_] == [int(v) for v in line.split()]


MANY_TURNS = [  # pairs that turn too often for the table's arithmetic, ones next to them that do not, a magnitude over FP32's range
    (dict(kind=0, base=1e-12, n_pos=1000), SHAPE), (dict(kind=0, base=1e-12, n_pos=1, rot=16), SHAPE), (dict(kind=0, base=1e-300), SHAPE),
    (dict(kind=0, base=1e-7, n_pos=1000), None), (dict(kind=0, base=1e300), None), (dict(kind=1, factor=1e-12, n_pos=10000), SHAPE),
    (dict(kind=1, factor=1e-3, n_pos=10000), None), (dict(kind=2, factor=1e-30), SHAPE), (dict(kind=3, factor=1e-9, n_pos=1000), SHAPE),
    (dict(kind=0, base=1.0, n_pos=(1 << 31) - 1), None), (dict(kind=0, base=5e-324), SHAPE), (dict(kind=1, factor=5e-324), SHAPE),
    (dict(kind=2, factor=5e-324, base=1e308), SHAPE), (dict(kind=0, base=1.7e308, rot=256), None), (dict(kind=3, length=1e308, factor=1e308), None),
    (dict(mag=1e39), SHAPE), (dict(mag=3e38), None),
]


@pytest.mark.parametrize("i", range(len(MANY_TURNS)))
def test_rope_table_refuses_more_turns_than_it_counts(lib, i):
    change, status = MANY_TURNS[i]
    rc = lib.fp8_rope_table(*(TABLE | change).values())
    assert rc in OK_ARGS_STATUS if status is None else rc == status, (change, rc, lib.fp8_last_error())


OUTPUTS_OF_NOTHING = [  # outputs that nothing would be written to
    (dict(y=None, gate=None, dy=None, dgate=None, amax=A), SHAPE), (dict(gate=None), SHAPE), (dict(gate=None, dgate=None), None),
    (dict(gate=None, amax=A), SHAPE), (dict(gate=None, dgate=None, amax=A), None), (dict(y=None, gate=None, dy=None), SHAPE),
]


@pytest.mark.parametrize("i", range(len(OUTPUTS_OF_NOTHING)))
def test_joint_gradient_refuses_outputs_of_what_is_not_there(lib, i):
    change, status = OUTPUTS_OF_NOTHING[i]
    args = GRAD | change
    args["cfg"] = C.byref(binding.BlockNorm(*CFG.values()))
    rc = lib.fp8_block_norm_bwd(*args.values())
    assert rc in OK_ARGS_STATUS if status is None else rc == status, (change, rc, lib.fp8_last_error())


WORDS_OFF_THEIR_TYPE = [
    ("fp8_rope_qkv_fwd", FWD, dict(amax=A + 2)), ("fp8_rope_qkv_fwd_q", FWD_Q, dict(scales=A + 1)), ("fp8_rope_qkv_fwd_q", FWD_Q, dict(amax=A + 3)),
    ("fp8_rope_qkv_bwd", BWD, dict(amax=A + 2)), ("fp8_rope_qkv_bwd_q", BWD_Q, dict(scale=A + 2)),
    ("fp8_block_norm_fwd", NORM, dict(rq=A + 2)), ("fp8_block_norm_fwd", NORM, dict(rp=A + 1)), ("fp8_block_norm_fwd", NORM, dict(amax=A + 2)),
    ("fp8_block_norm_fwd_q", NORM_Q, dict(scale=A + 2)),
    ("fp8_block_norm_bwd", GRAD, dict(rq=A + 2)), ("fp8_block_norm_bwd", GRAD, dict(rp=A + 2)), ("fp8_block_norm_bwd", GRAD, dict(dgq=A + 2)),
    ("fp8_block_norm_bwd", GRAD, dict(dgp=A + 1)), ("fp8_block_norm_bwd", GRAD, dict(amax=A + 2)), ("fp8_block_norm_bwd_q", GRAD_Q, dict(scale=A + 2)),
]


@pytest.mark.parametrize("i", range(len(WORDS_OFF_THEIR_TYPE)))
def test_refuses_words_that_are_not_aligned(lib, i):
    """Scales, maxima, statistics and sums are binary32 words: at 4-byte addresses they are taken, at others refused."""
    name, base, change = WORDS_OFF_THEIR_TYPE[i]
    for args, status in ((base | change, ALIGN), (base | {k: v // 4 * 4 + 4 for k, v in change.items()}, None)):
        args = dict(args)
        if "rope" in args:
            args["rope"] = C.byref(binding.Rope(*args["rope"].values()))
        if "cfg" in args:
            args["cfg"] = C.byref(binding.BlockNorm(*args["cfg"].values()))
        rc = getattr(lib, name)(*args.values())
        assert rc in OK_ARGS_STATUS if status is None else rc == status, (name, change, rc, lib.fp8_last_error())
