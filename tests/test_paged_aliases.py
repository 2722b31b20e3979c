"""Calls between the linear layers whose arguments are the same memory where each has to have its own: refused, as everything is that a look at the arguments
shows.  No GPU is needed: the context is a page of zeros and the buffers are addresses."""
import ctypes as C

import pytest

import paper_2501_07139_b200 as P
from test_paged_refusals import ARG, ATTENTION, CACHE, CTX, HEADS, KIND, MOVE, PAGE, ROTARY, STORE, Cache, Heads

START = 0x10000


def apart(given):
    """The same arguments, every buffer in a place of its own."""
    n = 0

    def place():
        nonlocal n
        n += 1
        return START + (n << 24)

    out = {}
    for name, v in given.items():
        if isinstance(v, dict):
            whole = {**(CACHE if name in ("cache", "layout") else HEADS), **v}
            out[name] = {f: place() if f in ("dev", "k_dev", "v_dev") else x for f, x in whole.items()}
        else:
            out[name] = place() if v == START else v
    return out


def code(name, args, pointers=()):
    args = dict(args)
    ctx, stream = args.pop("ctx"), args.pop("stream")
    array = (C.c_void_p * max(1, len(pointers)))(*pointers)
    if "caches" in args:
        args["caches"], args["n_caches"] = C.addressof(array), len(pointers)
    made = KIND[name](**{k: (Cache(**v) if k in ("cache", "layout") else Heads(**v)) if isinstance(v, dict) else v for k, v in args.items()})
    got = getattr(P.lib(), name)(ctx, C.addressof(made), stream)
    assert PAGE.raw == bytes(1 << 16) and ctx == CTX
    return got


def far(i):
    return 0x7000_0000_0000 + (i << 24)


@pytest.mark.parametrize("n,first,second", [(2, 0, 1), (64, 0, 63), (64, 30, 31), (128, 3, 127), (300, 0, 299), (300, 150, 160), (65536, 1, 65535)])
def test_a_cache_moved_twice(n, first, second):
    """Twice the same cache would be moved twice at once."""
    pointers = [far((i * 7919) % n) for i in range(n)]
    pointers[second] = pointers[first]
    assert code("fq_cache_move", apart(MOVE), pointers) == ARG


@pytest.mark.parametrize("field", ["lens", "n_kept", "starts", "kept", "table"])
def test_what_is_kept_has_its_own_memory(field):
    """Other parts of the call read these while keep is written."""
    args = apart(MOVE)
    args["keep"] = args[field]
    assert code("fq_cache_move", args, [far(0), far(1)]) == ARG


def test_outputs_in_place_of_queries():
    """A unit's queries are read by several CTAs, which write as they end."""
    args = apart(ATTENTION)
    args["out"]["dev"] = args["q"]["dev"]
    assert code("fq_tree_attention", args) == ARG


@pytest.mark.parametrize("output,other", [("y", "y1"), ("y", "x1"), ("y1", "x")])
def test_turned_tensors_have_their_own_memory(output, other):
    """In place is cell for cell: one tensor's output is not the other's output or source."""
    args = apart(ROTARY)
    args[output]["dev"] = args[other]["dev"]
    assert code("fq_rotary", args) == ARG


@pytest.mark.parametrize("other", ["k", "v", "caches"])
def test_a_step_stores_to_memory_of_its_own(other):
    args = apart(STORE)
    if other == "caches":
        args["cache"]["k_dev"] = args["cache"]["v_dev"]
    else:
        args["q_out"]["dev"] = args[other]["dev"]
    assert code("fq_rotary_cache", args) == ARG
