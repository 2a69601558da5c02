"""What the steps behind the logits refuse, and the host-side checks behind it.  No GPU: every call here is refused, or has
nothing to do."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2609_34645_b200 import binding as B
from paper_2609_34645_b200 import cache as C
from paper_2609_34645_b200 import logits as L

A = 1 << 20               # an address that nothing reads


def code(call, *args):
    try:
        call(*args)
    except B.NereusError as e:
        return e.code
    return B.OK


def logits(rows=6, vocab=100, dtype=B.BF16, base=A):
    v = B.Logits(dtype, 1, rows, vocab, vocab, vocab)
    v.shard[0] = base
    return v


def beams(beams=2, k=4, settle=0, score=A, ended=None, norm=None, reserved=0):
    return B.Beams(beams, k, settle, reserved, score, ended, norm)


def test_beam_select_refuses():
    def select(view=None, how=None, out=(A, A, A), work=A):
        return code(B.beam_select, view or logits(), how or beams(), work, 1 << 30, *out)
    wrong = (beams(beams=0), beams(beams=65), beams(k=0), beams(k=129), beams(settle=2), beams(settle=1, k=4), beams(beams=4), beams(reserved=1))
    for how in wrong:
        assert select(how=how) == code(B.beam_workspace, logits(), how) == B.ERR_ARG
    assert select(how=beams(score=None)) == select(work=None) == B.ERR_ARG and select(work=A + 8) == B.ERR_ALIGN
    assert select(logits(dtype=7)) == B.ERR_UNSUPPORTED
    assert select(logits(vocab=1 << 25)) == B.ERR_TOO_LARGE
    assert select(logits(base=A + 1)) == select(how=beams(score=A + 2)) == select(how=beams(ended=A + 1)) == select(how=beams(norm=A + 3)) == B.ERR_ALIGN
    assert select(out=(A + 1, A, A)) == select(out=(A, A + 2, A)) == select(out=(A, A, A + 3)) == B.ERR_ALIGN
    assert select(out=(None, A, A)) == select(out=(A, None, A)) == select(out=(A, A, None)) == B.ERR_ARG
    assert B._lib.nereus_beam_select(None, beams(), A, 0, A, A, A, None) == B._lib.nereus_beam_select(logits(), None, A, 0, A, A, A, None) == B.ERR_ARG
    assert B._lib.nereus_beam_workspace(logits(), beams(), None) == B.ERR_ARG
    assert select(logits(rows=0)) == B.OK and B.beam_workspace(logits(rows=0), beams()) == 0


def states(rows=6, buffers=2, outer=1, tokens=10, token_bytes=8, row=None, step=0, base=A):
    s = B.States(buffers, rows, outer, tokens, token_bytes, outer * tokens * token_bytes if row is None else row, step)
    for i in range(max(0, min(buffers, B.MAX_BUFFERS))):
        s.buffer[i] = base + i * (1 << 16)
    return s


def test_reorder_refuses():
    def reorder(src=None, dst=None, group=0, parent=A, length=None):
        src = src or states()
        return code(B.states_reorder, src, dst or states(base=1 << 24), group, parent, length)
    for s in (states(buffers=0), states(buffers=257), states(rows=-1), states(outer=0), states(tokens=-1), states(token_bytes=0), states(row=79),
              states(outer=2, step=79), states(outer=3, row=80, step=80), states(base=0, buffers=1)):
        assert reorder(src=s, dst=s, group=2) == B.ERR_ARG
    assert reorder(states(rows=1 << 25)) == reorder(states(token_bytes=1 << 60)) == reorder(states(row=1 << 50)) == B.ERR_TOO_LARGE
    for other in (states(buffers=1, base=1 << 24), states(tokens=9, base=1 << 24), states(token_bytes=4, base=1 << 24), states(outer=2, step=80, base=1 << 24)):
        assert reorder(dst=other) == B.ERR_MISMATCH
    assert reorder(parent=None) == reorder(group=-1) == reorder(group=65) == reorder(group=2) == B.ERR_ARG
    assert reorder(parent=A + 1) == reorder(length=A + 2) == B.ERR_ALIGN
    same = states()
    assert reorder(same, same, 0) == reorder(same, same, 4) == B.ERR_ARG
    assert reorder(same, states(rows=4), 2) == reorder(same, states(row=96), 2) == B.ERR_MISMATCH
    # overlapping, and interleaved without touching
    assert reorder(dst=states(base=A + 80)) == reorder(dst=states(base=A + (1 << 16))) == B.ERR_ALIAS
    assert reorder(states(row=160), states(row=160, base=A + 72)) == B.ERR_ALIAS
    assert reorder(states(rows=0), states(rows=0, base=1 << 24)) == reorder(dst=states(rows=0, base=1 << 24)) == B.OK
    assert reorder(states(tokens=0), states(tokens=0, base=1 << 24)) == B.OK


def pages(pools=2, count=10, size=64, stride=64, base=A):
    p = B.Pages(pools, count, size, stride)
    for i in range(max(0, min(pools, B.MAX_BUFFERS))):
        p.pool[i] = base + i * (1 << 16)
    return p


def book(base, rows=3, columns=4, stride=4, **kw):
    a = dict(table=base, length=base + (1 << 12), refs=base + (2 << 12)) | kw
    return B.PageTable(rows, columns, stride, a["table"], a["length"], a["refs"])


OLD, NEW, REST = 1 << 24, 2 << 24, 3 << 24


def test_fork_refuses():
    def fork(pool=None, old=None, new=None, parent=REST, size=16, room=0, room_of=None, copies=REST + 4096, status=REST + 8192):
        return code(B.cache_fork, pool or pages(), old or book(OLD), new or book(NEW), parent, size, room, room_of, copies, status)
    for p in (pages(pools=-1), pages(pools=257), pages(count=0), pages(size=0), pages(stride=63), pages(base=0, pools=1)):
        assert fork(p) == B.ERR_ARG
    assert fork(pages(count=(1 << 24) + 1)) == fork(pages(size=(1 << 30) + 1, stride=1 << 31)) == fork(pages(stride=1 << 50)) == B.ERR_TOO_LARGE
    for t in (book(NEW, rows=-1), book(NEW, columns=0), book(NEW, stride=3), book(NEW, table=None), book(NEW, length=None), book(NEW, refs=None)):
        assert fork(new=t) == B.ERR_ARG and fork(old=t, new=book(OLD)) == B.ERR_ARG
    assert fork(new=book(NEW, columns=5, stride=5)) == B.ERR_MISMATCH
    assert fork(new=book(NEW, rows=8193)) == fork(size=1 << 30) == B.ERR_TOO_LARGE
    assert fork(new=book(NEW, columns=(1 << 20) + 1, stride=1 << 21)) == B.ERR_TOO_LARGE
    assert fork(size=0) == fork(size=-4) == fork(room=-1) == fork(parent=None) == fork(copies=None) == fork(status=None) == B.ERR_ARG
    assert fork(parent=REST + 1) == fork(room_of=REST + 2) == fork(copies=REST + 4097) == fork(status=REST + 8195) == B.ERR_ALIGN
    assert fork(new=book(NEW, refs=NEW + 2)) == fork(new=book(NEW, table=NEW + 1)) == fork(new=book(NEW, length=NEW + 3)) == B.ERR_ALIGN
    for t in (book(OLD), book(NEW, table=OLD + 8), book(NEW, length=OLD + (1 << 12)), book(NEW, refs=OLD + (2 << 12) + 36), book(NEW, refs=NEW + 8)):
        assert fork(new=t) == B.ERR_ALIAS
    assert fork(copies=NEW) == fork(status=OLD + 4) == fork(parent=NEW) == fork(room_of=NEW + (1 << 12)) == B.ERR_ALIAS
    assert B._lib.nereus_cache_fork(None, book(OLD), book(NEW), REST, 16, 0, None, REST, REST, None) == B.ERR_ARG
    assert B._lib.nereus_cache_fork(pages(), None, book(NEW), REST, 16, 0, None, REST, REST, None) == B.ERR_ARG


def test_compact_refuses():
    def compact(pool=None, old=None, new=None, keep=-1, where=REST, moves=REST + 4096, status=REST + 8192):
        return code(B.cache_compact, pool or pages(), old or book(OLD), new or book(NEW), keep, where, moves, status)
    assert compact(pages(count=0)) == compact(old=book(OLD, refs=None)) == compact(where=None) == compact(moves=None) == compact(status=None) == B.ERR_ARG
    assert compact(new=book(NEW, rows=2)) == compact(new=book(NEW, columns=3)) == B.ERR_MISMATCH
    assert compact(where=REST + 1) == compact(moves=REST + 4100) == compact(status=REST + 2) == B.ERR_ALIGN
    assert compact(new=book(OLD)) == compact(where=OLD) == compact(moves=NEW) == compact(status=REST) == B.ERR_ALIAS


def test_copy_refuses():
    def copy(src=None, dst=None, n=3, a=REST, b=REST + 4096):
        return code(B.cache_copy, src or pages(), dst or pages(base=OLD), n, a, b)
    assert copy(pages(pools=300)) == copy(n=-1) == copy(a=None) == copy(b=None) == B.ERR_ARG
    assert copy(n=1 << 33) == B.ERR_TOO_LARGE
    assert copy(dst=pages(pools=1, base=OLD)) == copy(dst=pages(size=60, base=OLD)) == B.ERR_MISMATCH
    assert copy(a=REST + 1) == copy(b=REST + 2) == B.ERR_ALIGN
    assert copy(dst=pages(base=A + 64)) == copy(dst=pages(base=A + (1 << 16))) == copy(pages(stride=128), pages(stride=128, base=A + 32)) == B.ERR_ALIAS
    assert copy(n=0, a=None, b=None) == copy(pages(pools=0), pages(pools=0)) == copy(n=0) == B.OK


def test_structs_have_the_header_s_layout(tmp_path):
    """sizeof and offsets of the argument structs, from a C program."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    fields = {"nereus_beams_t": B.Beams, "nereus_states_t": B.States, "nereus_pages_t": B.Pages, "nereus_page_table_t": B.PageTable}
    lines = []
    for name, cls in fields.items():
        lines.append(f'printf("%zu\\n", sizeof({name}));')
        lines += [f'printf("%zu\\n", offsetof({name}, {f[0]}));' for f in cls._fields_]
    consts = ["NEREUS_BEAM_MAX", "NEREUS_BEAM_MAX_K", "NEREUS_MAX_BUFFERS", "NEREUS_CACHE_MAX_ROWS", "NEREUS_CACHE_MAX_PAGES"]
    lines += [f'printf("%d\\n", {c});' for c in consts]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "nereus.h"\nint main(void) {' + "\n".join(lines) + "return 0;}")
    exe = tmp_path / "layout"
    subprocess.check_call(["gcc", "-std=c99", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)])
    got = [int(x) for x in subprocess.check_output([str(exe)], text=True).split()]
    want = []
    for cls in fields.values():
        want.append(ctypes.sizeof(cls))
        want += [getattr(cls, f[0]).offset for f in cls._fields_]
    assert got == want + [getattr(B, c.removeprefix("NEREUS_")) for c in consts]


def test_the_torch_layer_refuses_host_tensors_and_wrong_types():
    x, i = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int32)
    for call in (lambda: L.beam_select(x, torch.zeros(4), 2, beams=2), lambda: C.reorder(x, i, beams=2), lambda: C.reorder([], i, beams=2),
                 lambda: C.fork([x], i.view(2, 2), i[:2], i, i[:2], 16), lambda: C.fork([], i.view(2, 2), i[:2], i, i[:2], 16),
                 lambda: C.compact([], i.view(2, 2), i), lambda: C.copy(x, i, i), lambda: C.copy([], i, i)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: C.reorder(3, i), lambda: C.copy(None, i, i)):
        with pytest.raises(TypeError):
            call()
