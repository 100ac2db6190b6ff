"""What the operators for branching generation refuse, checked on the CPU: every call below returns before anything is launched."""
import ctypes as C
import math
import os
import subprocess
import tempfile

import pytest
import torch

import paper_2601_23278_amd as pk
from paper_2601_23278_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
lib = binding._lib
P = 4096            # an address that no refused call reads


def kv(**over):
    d = dict(pool=P, dtype=1, n_layers=2, n_pages=9, page_size=16, n_kv_heads=2, head_dim=64)
    d.update(over)
    return binding.focus_kv(**d)


BAD_KV = [(dict(dtype=2), "dtype"), (dict(dtype=-1), "dtype"), (dict(head_dim=32), "head_dim"), (dict(head_dim=256), "head_dim"), (dict(page_size=0), "page_size"),
          (dict(page_size=12), "page_size"), (dict(page_size=1032), "page_size"), (dict(n_kv_heads=0), "n_kv_heads"), (dict(n_kv_heads=257), "n_kv_heads"),
          (dict(n_layers=0), "n_layers"), (dict(n_layers=1025), "n_layers"), (dict(n_pages=0), "n_pages"), (dict(n_pages=2 ** 30 + 1), "n_pages")]


def refused(rc, text=None, code=binding.FOCUS_EINVAL):
    assert rc == code, rc
    said = lib.focus_last_error(None).decode()
    assert said and (text is None or text in said), said


def test_struct_layout_matches_the_header():
    prog = r'''
#include <stdio.h>
#include <stddef.h>
#include "focus.h"
int main(void) { printf("%zu %zu %zu\n", sizeof(focus_kv), offsetof(focus_kv, dtype), offsetof(focus_kv, head_dim)); return 0; }'''
    with tempfile.TemporaryDirectory() as d:
        open(os.path.join(d, "t.c"), "w").write(prog)
        subprocess.check_call(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), os.path.join(d, "t.c"), "-o", os.path.join(d, "t")])
        got = [int(x) for x in subprocess.check_output([os.path.join(d, "t")]).decode().split()]
    assert got == [C.sizeof(binding.focus_kv), binding.focus_kv.dtype.offset, binding.focus_kv.head_dim.offset]


def append(g=None, layer=0, n=3, rows=4, cu=P, lens=P, table=P, stride=5, k=P, ldk=128, v=P, ldv=128):
    return lib.focus_kv_append(C.byref(kv() if g is None else g), None, layer, n, rows, cu, lens, table, stride, k, ldk, v, ldv)


def attend(g=None, layer=0, n=3, rows=4, mr=0, ml=0, cu=P, lens=P, table=P, stride=5, seen=P, words=1, heads=4, scale=0.1, q=P, ldq=256, out=P, ldo=256, ws=None, wb=0):
    return lib.focus_tree_attention(C.byref(kv() if g is None else g), None, layer, n, rows, mr, ml, cu, lens, table, stride, seen, words, heads, scale, q, ldq, out, ldo, ws, wb)


def compact(g=None, n=3, keep_n=4, start=P, cu=P, keep=P, table=P, stride=5, to=P, to_stride=5):
    return lib.focus_kv_compact(C.byref(kv() if g is None else g), None, n, keep_n, start, cu, keep, table, stride, to, to_stride)


def fork(g=None, old=3, new=4, parents=P, lens=P, table=P, stride=5, new_lens=P, new_table=2 * P, refs=P, lacking=P, ws=P, wb=1 << 20):
    return lib.focus_kv_fork(C.byref(kv() if g is None else g), None, old, new, parents, lens, table, stride, new_lens, new_table, refs, lacking, ws, wb)


def reserve(n=3, size=16, pages=9, lens=P, room=1, table=P, stride=5, refs=P, lacking=P, ws=P, wb=1 << 20):
    return lib.focus_kv_reserve(None, n, size, pages, lens, room, table, stride, refs, lacking, ws, wb)


def beam(n=2, beams=3, vocab=100, k=4, dtype=0, logits=P, ld=100, scores=P, done=None, end=0, rows=P, tokens=P, new=P, ws=P, wb=1 << 30):
    return lib.focus_beam_select(None, n, beams, vocab, k, dtype, logits, ld, scores, done, end, rows, tokens, new, ws, wb)


@pytest.mark.parametrize("over,text", BAD_KV)
def test_a_pool_is_refused_everywhere(over, text):
    for call in (append, attend, compact, fork):
        refused(call(kv(**over)), text)
    n = C.c_size_t()
    refused(lib.focus_tree_attention_bytes(C.byref(kv(**over)), 1, 1, 1, 1, 1, 4, C.byref(n)), text)


def test_pools_that_are_not_there():
    for call in (append, attend, compact, fork):
        refused(call(kv(pool=None)), "null")
        refused(call(kv(pool=P + 8)), "aligned")
    refused(lib.focus_kv_append(None, None, 0, 1, 1, P, P, P, 1, P, 128, P, 128), "null")
    refused(lib.focus_kv_compact(None, None, 1, 1, P, P, P, P, 1, P, 1), "null")
    refused(lib.focus_kv_fork(None, None, 1, 1, P, P, P, 1, P, P, P, P, P, 99), "null")
    refused(lib.focus_tree_attention(None, None, 0, 1, 1, 0, 0, P, P, P, 1, None, 0, 4, 1.0, P, 256, P, 256, None, 0), "null")
    refused(lib.focus_tree_attention_bytes(None, 1, 1, 1, 1, 1, 4, C.byref(C.c_size_t())), "null")


@pytest.mark.parametrize("over,text", [(dict(layer=-1), "layer"), (dict(layer=2), "layer"), (dict(n=-1), "n_seq"), (dict(n=1 << 20), "n_seq"), (dict(rows=-1), "n_rows"),
                                       (dict(rows=(1 << 22) + 1), "n_rows"), (dict(stride=0), "stride"), (dict(ldk=127), "ldk"), (dict(ldv=127), "ldv"), (dict(cu=None), "null"),
                                       (dict(lens=None), "null"), (dict(table=None), "null"), (dict(k=None), "null"), (dict(v=None), "null"), (dict(cu=P + 2), "aligned"),
                                       (dict(lens=P + 1), "aligned"), (dict(table=P + 2), "aligned"), (dict(k=P + 1), "aligned"), (dict(v=P + 1), "aligned")])
def test_append_refuses(over, text):
    refused(append(**over), text)


def test_append_of_nothing():
    assert append(n=0, cu=None, lens=None, table=None, k=None, v=None) == 0 and append(rows=0, k=None, v=None) == 0


@pytest.mark.parametrize("over,text", [(dict(layer=-1), "layer"), (dict(layer=2), "layer"), (dict(n=-1), "n_seq"), (dict(n=1 << 20), "n_seq"), (dict(rows=-1), "n_rows"),
                                       (dict(rows=(1 << 22) + 1), "n_rows"), (dict(mr=-1), "max_rows"), (dict(ml=-1), "max_len"), (dict(stride=0), "stride"), (dict(words=0), "seen_words"),
                                       (dict(words=17), "seen_words"), (dict(heads=0), "n_q_heads"), (dict(heads=3), "n_q_heads"), (dict(heads=1026), "n_q_heads"), (dict(rows=1 << 22, heads=512, ldq=1 << 15, ldo=1 << 15), "2^31"),
                                       (dict(scale=math.nan), "scale"), (dict(scale=math.inf), "scale"), (dict(ldq=255), "ldq"), (dict(ldo=255), "ldo"), (dict(cu=None), "null"),
                                       (dict(lens=None), "null"), (dict(table=None), "null"), (dict(q=None), "null"), (dict(out=None), "null"), (dict(cu=P + 2), "aligned"),
                                       (dict(seen=P + 4), "aligned"), (dict(q=P + 1), "aligned"), (dict(out=P + 1), "aligned"), (dict(ws=P + 128, wb=64), "256")])
def test_tree_attention_refuses(over, text):
    refused(attend(**over), text)


def test_tree_attention_of_nothing():
    assert attend(n=0, cu=None, lens=None, table=None, q=None, out=None) == 0 and attend(rows=0, q=None, out=None) == 0
    n = C.c_size_t(5)
    g = kv()
    assert lib.focus_tree_attention_bytes(C.byref(g), 0, 0, 0, 0, 1, 4, C.byref(n)) == 0 and n.value == 0
    refused(lib.focus_tree_attention_bytes(C.byref(g), 1, 1, 1, 1, 1, 4, None), "null")
    for bad in [(-1, 1, 1, 1, 1, 4), (1, -1, 1, 1, 1, 4), (1, 1, -1, 1, 1, 4), (1, 1, 1, -1, 1, 4), (1, 1, 1, 1, 0, 4), (1, 1, 1, 1, 1, 3)]:
        refused(lib.focus_tree_attention_bytes(C.byref(g), *bad, C.byref(n)))


@pytest.mark.parametrize("over,text", [(dict(n=-1), "n_seq"), (dict(n=1 << 20), "n_seq"), (dict(keep_n=-1), "n_keep"), (dict(stride=0), "stride"), (dict(to_stride=0), "to_stride"),
                                       (dict(start=None), "null"), (dict(cu=None), "null"), (dict(keep=None), "null"), (dict(table=None), "null"), (dict(to=None), "null"),
                                       (dict(start=P + 2), "aligned"), (dict(cu=P + 2), "aligned"), (dict(keep=P + 2), "aligned"), (dict(table=P + 2), "aligned"), (dict(to=P + 2), "aligned"),
                                       (dict(n=70000, g=kv(n_kv_heads=256, n_layers=1)), "2^24")])
def test_compact_refuses(over, text):
    refused(compact(**over), text)


def test_compact_of_nothing():
    assert compact(n=0, start=None, cu=None, table=None, to=None) == 0 and compact(keep_n=0, keep=None) == 0


@pytest.mark.parametrize("over,text", [(dict(old=-1), "n_old"), (dict(new=-1), "n_new"), (dict(old=1 << 20), "2^20"), (dict(old=1 << 19, new=1 << 19), "2^20"), (dict(stride=0), "stride"),
                                       (dict(stride=1 << 30), "2^31"), (dict(new=70000, g=kv(n_kv_heads=256, n_layers=1)), "2^24"), (dict(parents=None), "null"), (dict(lens=None), "null"),
                                       (dict(table=None), "null"), (dict(new_lens=None), "null"), (dict(new_table=None), "null"), (dict(refs=None), "null"), (dict(lacking=None), "null"),
                                       (dict(ws=None), "null"), (dict(ws=P + 8), "aligned"), (dict(parents=P + 2), "aligned"), (dict(refs=P + 1), "aligned"), (dict(new_table=P), "new_table")])
def test_fork_refuses(over, text):
    refused(fork(**over), text)


def test_fork_sizes():
    n = C.c_size_t()
    refused(lib.focus_kv_fork_bytes(-1, C.byref(n)), "n_new")
    refused(lib.focus_kv_fork_bytes(1 << 20, C.byref(n)), "n_new")
    refused(lib.focus_kv_fork_bytes(3, None), "null")
    assert lib.focus_kv_fork_bytes(4, C.byref(n)) == 0 and n.value > 0
    refused(fork(wb=n.value - 1), "small", binding.FOCUS_ENOMEM)
    assert fork(old=0, new=0, parents=None, lens=None, table=None, refs=None, ws=None) == 0


@pytest.mark.parametrize("over,text", [(dict(n=-1), "n_seq"), (dict(n=1 << 20), "n_seq"), (dict(size=12), "page_size"), (dict(size=0), "page_size"), (dict(size=2048), "page_size"),
                                       (dict(pages=0), "n_pages"), (dict(pages=2 ** 30 + 1), "n_pages"), (dict(room=-1), "room"), (dict(stride=0), "stride"), (dict(stride=1 << 30), "2^31"),
                                       (dict(lens=None), "null"), (dict(table=None), "null"), (dict(refs=None), "null"), (dict(lacking=None), "null"), (dict(ws=None), "null"),
                                       (dict(ws=P + 8), "aligned"), (dict(lens=P + 2), "aligned"), (dict(table=P + 2), "aligned")])
def test_reserve_refuses(over, text):
    refused(reserve(**over), text)


def test_outputs_over_inputs():
    """Fork: parents, lens and page_table are read by all workgroups while others write.  Beams: a request's scores are read by its own workgroup, before it writes."""
    d = dict(parents=P, lens=2 * P, table=3 * P, new_lens=4 * P, new_table=5 * P, refs=6 * P, lacking=7 * P, ws=8 * P)
    for out in ("new_lens", "new_table", "lacking"):
        for at in (P, P + 4 * 3, 2 * P, 2 * P + 4 * 2, 3 * P + 4 * 14):             # the last words of 4, 3 and 15
            refused(fork(**dict(d, **{out: at})), "overlap")
    refused(fork(**dict(d, new_table=3 * P - 4 * 19)), "overlap")
    refused(fork(**dict(d, new_lens=2 * P - 4 * 3)), "overlap")
    refused(beam(scores=P, new=P), "overlap")                                       # 3 beams, 4 picks
    refused(beam(scores=P, new=P + 4 * 5), "overlap")
    refused(beam(scores=P + 4 * 7, new=P), "overlap")
    refused(beam(scores=P, new=P + 4, beams=4), "overlap")
    refused(compact(keep_n=(1 << 30) + 1), "n_keep")


def test_reserve_sizes():
    n = C.c_size_t()
    refused(lib.focus_kv_reserve_bytes(-1, C.byref(n)), "n_seq")
    refused(lib.focus_kv_reserve_bytes(3, None), "null")
    assert lib.focus_kv_reserve_bytes(3, C.byref(n)) == 0
    refused(reserve(wb=n.value - 1), "small", binding.FOCUS_ENOMEM)
    assert reserve(n=0, lens=None, table=None, refs=None, lacking=None, ws=None) == 0


@pytest.mark.parametrize("over,text", [(dict(n=-1), "n_seq"), (dict(n=1 << 20, beams=2), "2^20"), (dict(beams=0), "n_beams"), (dict(beams=65), "n_beams"), (dict(k=0), "k must"),
                                       (dict(k=65), "k must"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 24) + 1), "vocab"), (dict(dtype=2), "dtype"), (dict(ld=99), "ld"),
                                       (dict(logits=None), "null"), (dict(scores=None), "null"), (dict(rows=None), "null"), (dict(tokens=None), "null"), (dict(new=None), "null"),
                                       (dict(ws=None), "null"), (dict(logits=P + 2), "aligned"), (dict(dtype=1, logits=P + 1), "aligned"), (dict(scores=P + 2), "aligned"),
                                       (dict(rows=P + 2), "aligned"), (dict(tokens=P + 2), "aligned"), (dict(new=P + 2), "aligned"), (dict(ws=P + 64), "aligned")])
def test_beam_select_refuses(over, text):
    refused(beam(**over), text)


def test_beam_select_sizes():
    n = C.c_size_t()
    refused(lib.focus_beam_select_bytes(1, 65, 10, 1, C.byref(n)), "n_beams")
    refused(lib.focus_beam_select_bytes(1, 1, 0, 1, C.byref(n)), "vocab")
    refused(lib.focus_beam_select_bytes(1, 1, 1, 1, None), "null")
    assert lib.focus_beam_select_bytes(2, 3, 100, 4, C.byref(n)) == 0 and n.value > 0
    refused(beam(wb=n.value - 1), "small", binding.FOCUS_ENOMEM)
    assert beam(n=0, logits=None, scores=None, rows=None, tokens=None, new=None, ws=None) == 0


def test_the_binding_refuses_tensors_that_are_not_on_the_current_device():
    pool, q, i = torch.zeros(1, 2, 2, 1, 16, 64), torch.zeros(1, 64), torch.zeros(1, dtype=torch.int32)
    cu, table = torch.zeros(2, dtype=torch.int32), torch.zeros(1, 1, dtype=torch.int32)
    for call in (lambda: pk.focus_kv_append(pool, 0, q, q, cu, i, table), lambda: pk.focus_tree_attention(pool, 0, q, cu, i, table), lambda: pk.focus_kv_compact(pool, i, cu, i, table),
                 lambda: pk.focus_kv_fork(pool, i, i, table, torch.zeros(2, dtype=torch.int32)), lambda: pk.focus_kv_reserve(i, 1, table, i, 16),
                 lambda: pk.focus_beam_select(torch.zeros(2, 5), torch.zeros(1, 2), 1)):
        with pytest.raises(pk.FocusError):
            call()


def test_fork_refuses_lists_that_are_written_over_each_other():
    """The counts change while rows are read and written, and the workspace holds what the launches tell each other."""
    d = dict(parents=P, lens=2 * P, table=3 * P, new_lens=4 * P, new_table=5 * P, refs=6 * P, lacking=7 * P, ws=8 * P)
    words = dict(parents=4, lens=3, table=15, new_lens=4, new_table=20, refs=9, lacking=4, ws=20)
    n = C.c_size_t()
    assert lib.focus_kv_fork_bytes(4, C.byref(n)) == 0 and n.value == 4 * words["ws"]
    written = ("new_lens", "new_table", "refs", "lacking", "ws")
    for x in written:
        for y in words:
            if x == y:
                continue
            refused(fork(**dict(d, **{x: d[y]})), "must")                            # the same address; new_table over page_table has words of its own
            if x != "ws":
                refused(fork(**dict(d, **{x: d[y] + 4 * (words[y] - 1)})), "overlap")    # the last word of the other
                refused(fork(**dict(d, **{x: d[y] - 4 * (words[x] - 1)})), "overlap")    # its last word on the first of the other
    # the workspace is 16-byte aligned
    refused(fork(**dict(d, ws=6 * P + 32)), "overlap")
    refused(fork(**dict(d, ws=7 * P - 64)), "overlap")
    # nothing but the counts is written where no row is new
    for at in (2 * P, 3 * P + 4 * 14):
        refused(fork(new=0, parents=None, lens=2 * P, table=3 * P, new_lens=None, new_table=None, refs=at, lacking=None, ws=None), "overlap")


def test_reserve_refuses_lists_that_are_written_over_each_other():
    d = dict(lens=P, table=2 * P, refs=3 * P, lacking=4 * P, ws=5 * P)
    words = dict(lens=3, table=15, refs=9, lacking=3, ws=13)
    n = C.c_size_t()
    assert lib.focus_kv_reserve_bytes(3, C.byref(n)) == 0 and n.value == 4 * words["ws"]
    for x in ("table", "refs", "lacking", "ws"):
        for y in words:
            if x == y or {x, y} == {"lens", "lacking"}:
                continue
            refused(reserve(**dict(d, **{x: d[y]})), "overlap")
            if x != "ws":
                refused(reserve(**dict(d, **{x: d[y] + 4 * (words[y] - 1)})), "overlap")
                refused(reserve(**dict(d, **{x: d[y] - 4 * (words[x] - 1)})), "overlap")
    refused(reserve(**dict(d, ws=3 * P + 32)), "overlap")
    refused(reserve(**dict(d, ws=P - 48)), "overlap")


def test_beam_select_refuses_lists_that_are_written_over_each_other():
    """2 requests of 3 beams, 4 picks; then of 4 beams, whose scores may be written in place."""
    n = C.c_size_t()
    assert lib.focus_beam_select_bytes(2, 3, 100, 4, C.byref(n)) == 0 and 256 < n.value < P
    d = dict(scores=P, done=2 * P, rows=3 * P, tokens=4 * P, new=5 * P, ws=6 * P)
    size = dict(scores=24, done=6, rows=32, tokens=32, new=32, ws=n.value)
    for x in ("rows", "tokens", "new", "ws"):
        for y in size:
            if x == y:
                continue
            refused(beam(**dict(d, **{x: d[y]})), "overlap")
            if x != "ws":
                refused(beam(**dict(d, **{x: d[y] + (size[y] - 1) // 4 * 4})), "overlap")
                refused(beam(**dict(d, **{x: d[y] - size[x] + 4})), "overlap")
            elif y != "ws":
                refused(beam(**dict(d, ws=d[y] - 256)), "overlap")
    refused(beam(**dict(d, beams=4, new=P + 32 - 4)), "overlap")
    refused(beam(**dict(d, beams=4, new=P, tokens=P)), "overlap")
    refused(beam(**dict(d, beams=4, rows=P, new=P)), "overlap")


def test_a_pool_of_heads_of_no_width_is_refused_like_any_other():
    """Before its width divides the columns of a query."""
    for shape in [(1, 2, 2, 1, 16, 0), (1, 2, 1, 1, 16, 64), (1, 2, 2, 16, 64)]:
        with pytest.raises(pk.FocusError):
            binding._kv_of(torch.zeros(shape))
    assert binding._kv_of(torch.zeros(1, 2, 2, 1, 16, 64)).head_dim == 64
