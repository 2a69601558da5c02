"""A generation stage's states and cache, on torch tensors: ``reorder`` (dense states follow the beams that go on),
``fork`` (a paged cache's sequences are forked, reordered, freed and given room), ``compact`` (the pages in use move to the
front of the pools) and ``copy`` (pages to other pages, or to another cache).

States are one tensor [rows, ...] or a list of them (keys and values of every layer) of one shape; pools are tensors
[pages, ...] of one shape, each page contiguous.  Bytes are moved, so that the element type does not matter.  Books are int32
tensors: table [rows, columns] (the page of every page_size tokens of a sequence, -1 for none), length [rows] (tokens of a
sequence) and refs [pages] (how often a page is held; 0: it is free).

What a call writes shares no memory with anything else that it reads or writes; a pool that is named twice counts as one.

Everything runs in the CUDA library on torch's current stream and synchronises nothing; what is returned was allocated on that
stream unless the caller passed it in.  Wrong types, devices or shapes raise ValueError, everything the library refuses raises
NereusError.  What device arrays say (parents, lengths, page ids) is checked on the device: what is out of range is left
out.  Nothing here has a gradient.
"""
from __future__ import annotations

from . import binding as B
from .logits import _t              # the marshalling, _nereus_torch.so

__all__ = ["reorder", "fork", "compact", "copy", "MAX_BUFFERS"]
MAX_BUFFERS = B.MAX_BUFFERS


def reorder(states, parent, *, beams=None, length=None, dim=1, out=None):
    """Row i of every state becomes row parent[i] (parent int32 [rows]): its first length[parent[i]] tokens along `dim`
    (length int32 [rows]; None: all), what lies behind them stays as it was.  Returns the written states.

    In place, rows come in groups of `beams`: a parent may be any row of the row's own group, and cross others; any other
    value, or the row itself, leaves the row alone.  With `out`, like `states` but for the number of rows, out[i] becomes
    states[parent[i]] for any parent, as when a prompt's states are handed to its beams; a parent that is no row leaves
    out[i] alone."""
    _t.reorder(states, parent, beams, length, dim, out)
    return states if out is None else out


def fork(pools, table, length, refs, parent, page_size, *, room=0, out=None):
    """(table, length, refs, copies, status): every new row i is a fork of row parent[i] (parent int32 [new rows]; -1: an
    empty row).  Full pages are shared; the lowest row that names a parent takes it over whole, the others get copies of its
    begun page in all pools; rows that nothing names are freed; where a row has no pages for `room` more tokens (a number,
    or int32 [new rows]) behind its length it gets fresh ones, the lowest free ids.  pools may be empty: books only.

    copies int32 [new rows, 2]: source and destination of the page copies made, then -1.  status int32 [4]: pages free now,
    pages (or columns of the table) missing, copies made, 0.  Where any are missing nothing is forked: the new books are
    the old ones.  out: (table, length, refs) to write to, none of them an old one."""
    return _t.fork(pools, table, length, refs, parent, page_size, room, out)


def compact(pools, table, refs, *, keep=None, out=None):
    """(table, refs, map, moves, status): the pages in use at or past `keep` (None: as many as are in use) move, in all
    pools, to free ones below, in order, so that the pools' first `keep` pages hold everything.

    map int32 [pages]: where each page is now, -1 for free ones.  moves int32 [pages // 2, 2]: source and destination of
    the first status[2] rows.  status int32 [4]: pages in use; how many they are more than `keep` (nothing is moved then); moves
    made; pages that hold everything now.  out: (table, refs) to write to, none of them an old one."""
    return _t.compact(pools, table, refs, keep, out)


def copy(pools, src, dst, *, to=None):
    """Copies page src[i] to page dst[i] (int32 [n]) in every pool, or of the pools to those of `to`, another cache; pairs
    with an id that is no page are left out.  A page that is written is no other pair's source or destination.  Returns the
    written pools."""
    _t.copy(pools, src, dst, to)
    return pools if to is None else to
