"""The block C ABI on the CPU: what include/llblock.h declares is exported and
bound, and bad arguments are refused before any HIP call (no GPU needed)."""
from __future__ import annotations

import ctypes
import os
import re

import pytest

from paper_2607_16100_amd import llblock as lb
from paper_2607_16100_amd import llcoll as ll
from paper_2607_16100_amd import llmoe as lm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
F32, BF16 = ll.LL_F32, ll.LL_BF16
OK, INVALID, UNSUPPORTED, SCRATCH = ll.LL_OK, ll.LL_ERR_INVALID, ll.LL_ERR_UNSUPPORTED, ll.LL_ERR_SCRATCH
# fake device addresses, far apart: never dereferenced
A, B, C, D, E, F, G, H = (k << 40 for k in range(1, 9))


def test_header_and_binding_agree():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "llblock.h")).read(), flags=re.S)
    names = set(re.findall(r"^int (ll_[a-z_0-9]+)\s*\(", text, flags=re.M))
    assert names == set(lb.exported_symbols())
    for n in names:
        assert hasattr(ll.library(), n), n
    for name, value in re.findall(r"#define (LL_[A-Z0-9_]+) (\w+)", text):
        assert getattr(lb, name) == int(value, 0), name


def quantise(x=A, ldx=256, rows=4, end=0, features=200, dt=F32, act=0, q=B, ldq=200, scales=C, lds=4):
    return lb.ll_quantise(x, ldx, rows, end, features, dt, act, q, ldq, scales, lds, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(x=0), INVALID), (dict(q=0), INVALID), (dict(scales=0), INVALID), (dict(x=A + 2), INVALID),
    (dict(ldx=199), INVALID), (dict(ldq=199), INVALID), (dict(lds=1), INVALID), (dict(lds=6), INVALID),
    (dict(scales=C + 2), INVALID), (dict(end=D + 2), INVALID), (dict(act=6), INVALID), (dict(act=-1), INVALID),
    (dict(dt=2), UNSUPPORTED), (dict(act=lm.LL_ACT_SWIGLU), INVALID), (dict(q=A), INVALID), (dict(scales=B), INVALID),
    (dict(scales=A + 1024), INVALID), (dict(end=B), INVALID), (dict(rows=1 << 31), UNSUPPORTED),
    (dict(rows=0, x=0, q=0, scales=0), OK), (dict(features=0, x=0, q=0, scales=0), OK),
])
def test_quantise_refusals(kw, want):
    assert quantise(**kw) == want


def weight(w=A, ldw=200, wstride=40000, groups=2, out=150, in_=200, dt=BF16, transpose=0, q=B, ldq=200, qstride=40000,
           scales=C, lds=4, sstride=8):
    return lb.ll_quantise_weight(w, ldw, wstride, groups, out, in_, dt, transpose, q, ldq, qstride, scales, lds, sstride,
                                 0)


@pytest.mark.parametrize("kw,want", [
    (dict(w=0), INVALID), (dict(q=0), INVALID), (dict(scales=0), INVALID), (dict(w=A + 1), INVALID),
    (dict(ldw=199), INVALID), (dict(ldq=199), INVALID), (dict(lds=5), INVALID), (dict(sstride=4), INVALID),
    (dict(sstride=10), INVALID), (dict(wstride=29999), INVALID), (dict(qstride=29999), INVALID),
    (dict(transpose=1, ldq=149), INVALID), (dict(groups=0), INVALID), (dict(out=0), INVALID), (dict(in_=0), INVALID),
    (dict(groups=1025), UNSUPPORTED), (dict(in_=(1 << 20) + 1, ldw=1 << 21, ldq=1 << 21), UNSUPPORTED),
    (dict(dt=7), UNSUPPORTED), (dict(q=A + 64), INVALID), (dict(scales=B + 1024), INVALID),
])
def test_weight_refusals(kw, want):
    assert weight(**kw) == want


def d(dt=BF16, act=0, groups=2, rows=64, in_=256, out=128, offsets=H, **fields):
    if groups == 1:
        offsets = fields.pop("off", 0)
    return lm.desc(dt, act, groups, rows, in_, out, offsets=offsets, **fields)


def linear8(desc=None, x=A, xs=B, ldxs=4, w=C, ws=D, ldws=4, wsstride=4, bias=0, residual=0, y=E, z=0, ws_at=0,
            ws_bytes=0):
    return lb.ll_linear8(desc if desc is not None else d(), x, xs, ldxs, w, ws, ldws, wsstride, bias, residual, y, z,
                         ws_at, ws_bytes, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(x=0), INVALID), (dict(xs=0), INVALID), (dict(w=0), INVALID), (dict(ws=0), INVALID), (dict(y=0), INVALID),
    (dict(xs=B + 1), INVALID), (dict(ldxs=1), INVALID), (dict(ldxs=6), INVALID), (dict(ldws=2), INVALID),
    (dict(ws=D + 2), INVALID), (dict(wsstride=2), INVALID), (dict(wsstride=1), INVALID),
    (dict(ldxs=(1 << 18) + 4), UNSUPPORTED), (dict(ldws=(1 << 18) + 4), UNSUPPORTED),
    (dict(y=E + 1), INVALID), (dict(bias=F + 1), INVALID), (dict(residual=F + 1), INVALID), (dict(z=F + 1), INVALID),
    (dict(ws_at=F + 8), INVALID), (dict(y=A), INVALID), (dict(y=B), INVALID), (dict(y=C + 1024), INVALID),
    (dict(y=D), INVALID), (dict(z=E + 64), INVALID), (dict(z=A), INVALID), (dict(residual=E + 256), INVALID),
    (dict(bias=E), INVALID),
])
def test_linear8_refusals(kw, want):
    assert linear8(**kw) == want


@pytest.mark.parametrize("fields,want", [
    (dict(ldx=255), INVALID), (dict(ldw=255), INVALID), (dict(wstride=100), INVALID), (dict(ldy=127), INVALID),
    (dict(size=8), INVALID), (dict(groups=1025), UNSUPPORTED), (dict(groups=0), INVALID), (dict(offsets=0), INVALID),
    (dict(act=6), INVALID), (dict(dt=5), UNSUPPORTED), (dict(in_=(1 << 20) + 1), UNSUPPORTED),
    (dict(out=127, act=lm.LL_ACT_SWIGLU), INVALID),
    (dict(out=128256, in_=32768, act=lm.LL_ACT_GEGLU), UNSUPPORTED),
])
def test_linear8_descriptor_refusals(fields, want):
    groups = fields.pop("groups", 2)
    desc = d(**fields)
    desc.groups = groups
    assert linear8(desc) == want
    if want == UNSUPPORTED or "size" in fields:
        assert lb.ll_linear8_bytes(desc)[0] == want


@pytest.mark.parametrize("features,rows", [(8192, 1 << 22), (4096, 1 << 23), (2048, 1 << 24), (1024, 1 << 25), (16384, 1 << 22)])
def test_norm_rows_past_a_launch(features, rows):
    assert norm(nd(rows=rows, features=features, ldy=features), x=0, r=0, h=1 << 50) == UNSUPPORTED


def test_quantise_blocks_past_a_launch():
    assert quantise(rows=1 << 29, features=128, ldx=128, ldq=128, q=1 << 50, scales=1 << 51) == UNSUPPORTED


def test_linear8_of_no_rows():
    assert linear8(d(rows=0), x=0, xs=0, w=0, ws=0, y=0) == OK
    assert lb.ll_linear8_bytes(d(rows=0)) == (OK, 0)


def test_linear8_workspace():
    """Few tiles and a long sum have one, of whole splits; few rows have none."""
    st, few = lb.ll_linear8_bytes(d(groups=1, rows=16, in_=7168, out=256))
    assert (st, few) == (OK, 0)
    st, need = lb.ll_linear8_bytes(d(groups=1, rows=48, in_=7168, out=136))
    assert st == OK and need % (48 * 136 * 4) == 0 and need >= 2 * 48 * 136 * 4


def nd(dt=BF16, wdt=BF16, rows=8, features=200, eps=1e-6, scale=1.0, **fields):
    return lb.norm_desc(dt, wdt, rows, features, eps, scale, **fields)


def norm(desc=None, y=A, x=B, gate=0, post=0, weight=C, r=D, h=E, q=0, scales=0):
    return lb.ll_norm(desc if desc is not None else nd(), y, x, gate, post, weight, r, h, q, scales, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(y=0), INVALID), (dict(weight=0), INVALID), (dict(y=A + 1), INVALID), (dict(x=B + 1), INVALID),
    (dict(gate=F + 2), INVALID), (dict(post=F + 1), INVALID), (dict(weight=C + 1), INVALID), (dict(r=D + 1), INVALID),
    (dict(q=F), INVALID), (dict(q=F, scales=G + 1), INVALID), (dict(q=F, scales=F), INVALID), (dict(h=D), INVALID),
    (dict(h=B), INVALID), (dict(r=A + 400), INVALID), (dict(r=C), INVALID), (dict(q=A, scales=G), INVALID),
    (dict(weight=0, h=0, q=F, scales=G), INVALID), (dict(gate=D), INVALID),
    (dict(r=0, h=0), OK), (dict(weight=0, h=0, r=0), OK),
])
def test_norm_refusals(kw, want):
    assert norm(**kw) == want


@pytest.mark.parametrize("fields,want", [
    (dict(dt=3), UNSUPPORTED), (dict(wdt=3), UNSUPPORTED), (dict(dt=F32, wdt=BF16), UNSUPPORTED), (dict(eps=0.), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(features=0), INVALID), (dict(features=16385), UNSUPPORTED),
    (dict(rows=1 << 31), UNSUPPORTED), (dict(ldy=199), INVALID), (dict(ldx=199), INVALID), (dict(ldr=199), INVALID),
    (dict(ldh=199), INVALID), (dict(size=4), INVALID), (dict(ldy=1 << 31), UNSUPPORTED),
])
def test_norm_descriptor_refusals(fields, want):
    assert norm(nd(**fields)) == want
    if not any(k.startswith("ld") for k in fields) or want == UNSUPPORTED:
        assert lb.ll_norm_bytes(nd(**fields))[0] == want


def grad(desc=None, dh=A, r=B, dr=C, y=D, gate=0, post=0, weight=E, dr_out=F, dy=G, dgate=0, dweight=0, dpost=0,
         flags=0, ws=0, ws_bytes=0):
    return lb.ll_norm_grad(desc if desc is not None else nd(), dh, r, dr, y, gate, post, weight, dr_out, dy, dgate,
                           dweight, dpost, flags, ws, ws_bytes, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(dh=0), INVALID), (dict(r=0), INVALID), (dict(weight=0), INVALID), (dict(weight=0, dh=0, dweight=H), INVALID),
    (dict(dpost=H), INVALID), (dict(post=H, y=0), INVALID), (dict(dgate=H, y=0), INVALID), (dict(flags=1), INVALID),
    (dict(dh=A + 1), INVALID), (dict(dy=G + 1), INVALID), (dict(dgate=H + 2), INVALID), (dict(dweight=H + 2), INVALID),
    (dict(dweight=H), SCRATCH), (dict(dweight=H, ws=9 << 40, ws_bytes=16), SCRATCH),
    (dict(dweight=H, ws=(9 << 40) + 4, ws_bytes=1 << 30), INVALID), (dict(dr_out=A), INVALID), (dict(dr_out=B), INVALID),
    (dict(dy=F), INVALID), (dict(dy=C), INVALID), (dict(dy=E), INVALID), (dict(dr_out=D), INVALID),
    (dict(dweight=H, ws=A, ws_bytes=1 << 30), INVALID), (dict(dr_out=0, dy=0), OK),
])
def test_norm_grad_refusals(kw, want):
    assert grad(**kw) == want


def test_norm_grad_of_no_rows_without_sums():
    assert grad(nd(rows=0), dh=0, r=0, dr=0, y=0, dr_out=0, dy=0) == OK


def adamw(count=1, step=A, work=B, work_bytes=64, lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, decay=0.0, bits=32, size=None,
          lr_ptr=0, scale=0, null=False, **fields):
    t = dict(param=C, grad=D, master=0, m=E, v=F, m_scales=0, v_scales=0, n=100, at=0, dt=F32, gdt=F32)
    t.update(fields)
    table = (lb.LLAdamwTensor * max(count, 1))()
    for i in range(count):
        for k, v in t.items():
            setattr(table[i], k, v)
    desc = lb.LLAdamwDesc(lb.ADAMW_DESC_SIZE if size is None else size, bits, lr, beta1, beta2, eps, decay, 0)
    return lb.ll_adamw(desc, None if null else table, count, step, lr_ptr, scale, work, work_bytes, 0)


@pytest.mark.parametrize("kw,want", [
    (dict(size=8), INVALID), (dict(bits=16), INVALID), (dict(beta1=1.0), INVALID), (dict(beta2=-0.5), INVALID),
    (dict(beta1=float("nan")), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=0.0), INVALID), (dict(eps=1e-50), INVALID),
    (dict(decay=-1.0), INVALID),
    (dict(lr=float("nan")), INVALID), (dict(lr=-1.0), INVALID), (dict(step=0), INVALID), (dict(step=A + 2), INVALID),
    (dict(work=0), INVALID), (dict(work=B + 8), INVALID), (dict(work_bytes=63), SCRATCH), (dict(lr_ptr=G + 1), INVALID),
    (dict(scale=G + 2), INVALID), (dict(null=True), INVALID), (dict(param=0), INVALID), (dict(grad=0), INVALID),
    (dict(m=0), INVALID), (dict(v=0), INVALID), (dict(master=G), INVALID), (dict(dt=BF16), INVALID),
    (dict(m_scales=G), INVALID), (dict(bits=8), INVALID), (dict(bits=8, m_scales=G), INVALID), (dict(param=C + 2), INVALID),
    (dict(grad=D + 1), INVALID), (dict(m=E + 2), INVALID), (dict(dt=BF16, master=G + 2), INVALID),
    (dict(dt=2), UNSUPPORTED), (dict(gdt=2), UNSUPPORTED), (dict(n=(1 << 40) + 1), UNSUPPORTED),
])
def test_adamw_refusals(kw, want):
    assert adamw(**kw) == want


def test_structures_have_the_headers_layout(tmp_path):
    """Sizes and offsets as a C compiler sees them."""
    import subprocess

    fields = {"ll_norm_desc": lb.LLNormDesc, "ll_adamw_tensor": lb.LLAdamwTensor, "ll_adamw_desc": lb.LLAdamwDesc}
    lines = ['#include <stdio.h>', '#include "llblock.h"', "int main(void) {"]
    for name, cls in fields.items():
        lines.append(f'printf("{name} %zu\\n", sizeof({name}));')
        lines += [f'printf("{name}.{f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    lines.append("return 0; }")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)],
                   check=True)
    said = dict(line.split() for line in subprocess.run([str(exe)], capture_output=True, text=True,
                                                        check=True).stdout.splitlines())
    for name, cls in fields.items():
        assert int(said[name]) == ctypes.sizeof(cls)
        for f in cls._fields_:
            assert int(said[f"{name}.{f[0]}"]) == getattr(cls, f[0]).offset, f[0]
