"""What the expert router and the MXFP4 operators refuse, checked on the CPU: every call below returns before anything is launched."""
import ctypes as C
import math
import os
import subprocess
import tempfile

import numpy as np
import pytest
import torch

import focus_inputs as fi
import mx_reference as ref
import paper_2601_23278_amd as pk
from paper_2601_23278_amd import binding
from paper_2601_23278_amd.runner import config_from_workload

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
lib = binding._lib
P = 4096            # an address that no refused call reads


def router(**over):
    d = dict(n_experts=16, experts_per_token=4, score=0, n_groups=4, groups_kept=2, group_top=2, renormalize=1, route_scale=1.0)
    d.update(over)
    return binding.focus_router(**d)


def refused(rc, text=None):
    assert rc == binding.FOCUS_EINVAL, rc
    said = binding._lib.focus_last_error(None).decode()
    assert said and (text is None or text in said), said


def test_struct_layouts_match_the_header():
    prog = r'''
#include <stdio.h>
#include <stddef.h>
#include "focus.h"
int main(void) {
  printf("%zu %zu %zu %zu %zu %d %d %d\n", sizeof(focus_router), offsetof(focus_router, route_scale), sizeof(focus_mx), offsetof(focus_mx, scales),
         sizeof(focus_mx_weights), FOCUS_MX4, FOCUS_SCORE_SOFTMAX, FOCUS_SCORE_SIGMOID);
  return 0;
}'''
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "t.c"), "w").write(prog)
        subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), os.path.join(d, "t.c"), "-o", os.path.join(d, "t")])
        got = [int(x) for x in subprocess.check_output([os.path.join(d, "t")]).decode().split()]
    assert got == [C.sizeof(binding.focus_router), binding.focus_router.route_scale.offset, C.sizeof(binding.focus_mx), binding.focus_mx.scales.offset,
                   C.sizeof(binding.focus_mx_weights), binding.FOCUS_MX4, binding.FOCUS_SCORE_SOFTMAX, binding.FOCUS_SCORE_SIGMOID]


@pytest.mark.parametrize("over", [dict(n_experts=0), dict(n_experts=513, n_groups=1), dict(score=2), dict(n_groups=0), dict(n_groups=5), dict(n_experts=130, n_groups=65),
                                  dict(groups_kept=0), dict(groups_kept=5), dict(group_top=0), dict(group_top=3), dict(experts_per_token=0), dict(experts_per_token=9),
                                  dict(n_experts=256, groups_kept=4, experts_per_token=33), dict(renormalize=2), dict(route_scale=0.0), dict(route_scale=math.nan),
                                  dict(route_scale=math.inf), dict(route_scale=-1.0)])
def test_route_refuses_a_router(over):
    r = router(**over)
    refused(lib.focus_route(C.byref(r), None, 1, 0, P, 1024, None, P, P))


def test_route_refuses_arguments():
    r = router()
    refused(lib.focus_route(None, None, 1, 0, P, 16, None, P, P), "router")
    refused(lib.focus_route(C.byref(r), None, -1, 0, P, 16, None, P, P), "n_rows")
    refused(lib.focus_route(C.byref(r), None, 1 << 26, 0, P, 16, None, P, P), "n_rows")
    refused(lib.focus_route(C.byref(r), None, 1, binding.FOCUS_MX4, P, 16, None, P, P), "dtype")
    refused(lib.focus_route(C.byref(r), None, 1, 0, P, 15, None, P, P), "ld")
    refused(lib.focus_route(C.byref(r), None, 1, 0, None, 16, None, P, P), "null")
    refused(lib.focus_route(C.byref(r), None, 1, 0, P, 16, None, None, P), "null")
    refused(lib.focus_route(C.byref(r), None, 1, 0, P, 16, None, P, None), "null")
    refused(lib.focus_route(C.byref(r), None, 1, 0, P + 2, 16, None, P, P), "aligned")
    refused(lib.focus_route(C.byref(r), None, 1, 1, P + 1, 16, None, P, P), "aligned")
    refused(lib.focus_route(C.byref(r), None, 1, 0, P, 16, P + 1, P, P), "aligned")
    assert lib.focus_route(C.byref(r), None, 0, 0, None, 16, None, None, None) == 0


def test_conversions_refuse():
    mx = binding.focus_mx(P, P)
    for q in (lambda d, r, c, x, ld, co, sc: lib.focus_mx_quantize(None, d, r, c, x, ld, co, sc),
              lambda d, r, c, x, ld, co, sc: lib.focus_mx_dequantize(None, d, r, c, C.byref(binding.focus_mx(co, sc)), x, ld)):
        refused(q(2, 1, 32, P, 32, P, P), "dtype")
        refused(q(0, -1, 32, P, 32, P, P), "negative")
        refused(q(0, 1, -1, P, 32, P, P), "negative")
        refused(q(0, 1, 33, P, 32, P, P), "ldx")
        refused(q(0, 1 << 39, 1, P, 32, P, P), "large")
        refused(q(0, 1 << 36, 32, P, 32, P, P), "large")
        refused(q(0, 1 << 30, 32, P, 32, P, P), "large")
        refused(q(0, 1 << 20, 1 << 15, P, 1 << 15, P, P), "large")
        refused(q(0, 1, 32, None, 32, P, P), "null")
        refused(q(0, 1, 32, P, 32, None, P), "null")
        refused(q(0, 1, 32, P, 32, P, None), "null")
        refused(q(0, 1, 32, P, 32, P + 8, P), "aligned")
        refused(q(0, 1, 32, P + 2, 32, P, P), "aligned")
        refused(q(1, 1, 32, P + 1, 32, P, P), "aligned")
        assert q(0, 0, 32, None, 32, None, None) == 0 and q(0, 5, 0, None, 0, None, None) == 0
    refused(lib.focus_mx_dequantize(None, 0, 1, 32, None, P, 32), "null")


def test_gemm_refuses():
    w, n = binding.focus_mx(P, P), C.c_size_t()

    def call(m=4, n=8, k=64, at=1, a=P, sc=None, lda=64, mw=w, ct=0, c=P, ldc=8, ws=None, wb=0):
        return lib.focus_mx_gemm(None, m, n, k, at, a, sc, lda, None if mw is None else C.byref(mw), ct, c, ldc, ws, wb)
    for bad, text in [(dict(m=-1), "negative"), (dict(n=-1), "negative"), (dict(k=-32), "negative"), (dict(k=48), "multiple"), (dict(at=0), "a_type"), (dict(ct=2), "c_type"),
                      (dict(mw=None), "null"), (dict(ldc=7), "ldc"), (dict(lda=56), "lda"), (dict(lda=68), "lda"), (dict(lda=(1 << 22) + 8), "lda"), (dict(a=None), "null"), (dict(c=None), "null"),
                      (dict(mw=binding.focus_mx(None, P)), "null"), (dict(mw=binding.focus_mx(P, None)), "null"), (dict(at=2), "a_scales"), (dict(sc=P), "a_scales"),
                      (dict(a=P + 8), "aligned"), (dict(mw=binding.focus_mx(P + 8, P)), "aligned"), (dict(ws=P + 8, wb=64), "aligned"), (dict(c=P + 2), "aligned"),
                      (dict(n=1 << 20, k=1 << 13, lda=1 << 13, ldc=1 << 20), "large"),
                      (dict(m=2 ** 31 - 1, n=129, ldc=129), "large"), (dict(m=2 ** 31 - 1, n=129, ldc=129, at=2, sc=P), "large"), (dict(k=(1 << 22) + 32), "k")]:
        refused(call(**bad), text)
    assert call(m=0, a=None, c=None) == 0 and call(n=0, ldc=0, c=None) == 0
    refused(lib.focus_mx_gemm_bytes(4, 8, 64, 1, None))
    refused(lib.focus_mx_gemm_bytes(4, 8, 40, 1, C.byref(n)))
    assert pk.focus_mx_gemm_bytes(0, 8, 64, 1) == 0 and pk.focus_mx_gemm_bytes(8192, 4096, 4096, 1) == 0
    assert pk.focus_mx_gemm_bytes(100, 128, 8192, 2) % (100 * 128 * 4) == 0 and pk.focus_mx_gemm_bytes(100, 128, 8192, 2) > 0


def test_experts_refuse():
    w, n = binding.focus_mx(P, P), C.c_size_t()

    def call(E=8, h=64, f=32, gu=w, dn=w, rows=4, k=2, x=P, ldx=64, e=P, g=P, ot=0, out=P, ldo=64, add=0, ws=P, wb=1 << 30):
        return lib.focus_mx_experts(None, E, h, f, None if gu is None else C.byref(gu), None if dn is None else C.byref(dn), rows, k, x, ldx, e, g, ot, out, ldo, add, ws, wb)
    for bad, text in [(dict(E=0), "n_experts"), (dict(E=513), "n_experts"), (dict(h=48, ldx=48), "multiples"), (dict(f=16), "multiples"), (dict(h=0), "multiples"),
                      (dict(rows=-1), "n_rows"), (dict(k=0), "k in"), (dict(k=33), "k in"), (dict(rows=1 << 24, k=1), "n_rows"), (dict(rows=1 << 18, k=32, h=1 << 14, f=1 << 15, ldx=1 << 14, ldo=1 << 14), "large"), (dict(h=1 << 20, f=1 << 11, ldx=1 << 20, ldo=1 << 20), "large"),
                      (dict(ot=2), "out_type"), (dict(add=2), "add"), (dict(add=1, ot=1), "add"), (dict(ldx=56), "ldx"), (dict(ldx=68), "ldx"), (dict(ldo=63), "ldo"),
                      (dict(rows=1 << 20, ldx=1024), "2^30"), (dict(gu=None), "null"), (dict(dn=binding.focus_mx(P, None)), "null"), (dict(x=None), "null"), (dict(e=None), "null"),
                      (dict(g=None), "null"), (dict(out=None), "null"), (dict(ws=None), "null"), (dict(x=P + 8), "aligned"), (dict(gu=binding.focus_mx(P + 4, P)), "aligned"),
                      (dict(ws=P + 64), "aligned"), (dict(out=P + 2), "aligned")]:
        refused(call(**bad), text)
    assert call(wb=64) == binding.FOCUS_ENOMEM
    assert call(rows=0, x=None, e=None, g=None, out=None, ws=None) == 0
    refused(lib.focus_mx_experts_bytes(8, 64, 32, 4, 2, None))
    refused(lib.focus_mx_experts_bytes(8, 64, 30, 4, 2, C.byref(n)))
    assert pk.focus_mx_experts_bytes(8, 64, 32, 0, 2) <= pk.focus_mx_experts_bytes(8, 64, 32, 4, 2)


def test_context_setters_refuse_a_null_context():
    refused(lib.focus_set_router(None, None, None), "null")
    refused(lib.focus_set_mx_weights(None, None), "null")


def test_python_refuses_tensors_elsewhere_and_wrong_shapes():
    with pytest.raises(pk.FocusError):                              # no GPU tensors here
        pk.focus_route(router(), torch.zeros(2, 16))
    with pytest.raises(pk.FocusError):
        pk.focus_mx_quantize(torch.zeros(2, 64))
    with pytest.raises(pk.FocusError):
        binding._rows_of(torch.zeros(4, 8).t(), "x")                # columns, not rows, are contiguous
    with pytest.raises(pk.FocusError):
        binding._rows_of(torch.zeros(1, 8).expand(3, 8), "x")       # rows overlap
    with pytest.raises(pk.FocusError):
        binding._rows_of(torch.zeros(2, 8, dtype=torch.float16), "x")
    with pytest.raises(pk.FocusError):
        binding._mx_of((torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 2, dtype=torch.uint8)), "w", 4)
    with pytest.raises(pk.FocusError):
        binding._mx_of((torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.int8)), "w", 4)
    mx, k = binding._mx_of((torch.zeros(4, 16, dtype=torch.uint8), torch.zeros(4, 1, dtype=torch.uint8)), "w", 4)
    assert k == 32


def test_reference_pins():
    """The plain forms against values worked out by hand."""
    codes, scales = ref.quantize(np.array([[7.0, -0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 5.01, -0.0] + [0.0] * 22]))
    assert scales.tolist() == [[127]] and codes[0, :10].tolist() == [7, 8, 2, 2, 4, 4, 6, 6, 7, 8]
    codes, scales = ref.quantize(np.array([[2.0 ** -130] * 3, [0.0] * 3, [math.inf, 1.0, 0.0], [2.0 ** 127] * 3]))
    assert scales[:, 0].tolist() == [0, 0, 255, 252] and codes[0, 0] == 0 and codes[2].sum() == 0 and codes[3, 0] == 6
    v = ref.values(torch.tensor([[0x71, 0x08] + [0] * 14], dtype=torch.uint8), torch.tensor([[128]], dtype=torch.uint8))
    assert v[0, :4].tolist() == [1.0, 12.0, 0.0, 0.0]
    e, w = ref.route_row([0.0, 1.0, 1.0, math.nan], [0.0, 0.0, 0.0, 9.0], "softmax", 1, 1, 1, 4, True, 2.0)
    assert e == [1, 2, 0, 3] and abs(sum(w) - 2.0) < 1e-12 and w[3] == 0.0
    e, w = ref.route_row([0.0, 3.0, 2.0, 2.0], None, "sigmoid", 2, 1, 2, 2, False, 1.0)     # groups: 0.5 + 0.953 against 0.881 + 0.881
    assert e == [2, 3] and abs(w[0] - 1 / (1 + math.exp(-2.0))) < 1e-12
