"""Arguments that the calls between the linear layers refuse.  Every check comes before the context or a pointer is looked into, so that a refused call
needs no GPU: the context here is a page of zeros and the buffers are addresses."""
import ctypes as C
import math

import pytest

import paper_2501_07139_b200 as P


# the structures of include/flexq.h
LL, I, VP = C.c_longlong, C.c_int, C.c_void_p


class Heads(C.Structure):
    _fields_ = [("dev", VP), ("token_stride", LL), ("head_stride", LL), ("heads", I)]


class Cache(C.Structure):
    _fields_ = [("k_dev", VP), ("v_dev", VP), ("block_stride", LL), ("token_stride", LL), ("head_stride", LL), ("blocks", I), ("block_size", I), ("heads", I)]


def fields(text):
    kinds = {"h": Heads, "c": Cache, "p": VP, "l": LL, "i": I, "f": C.c_float}
    return [(name, kinds[k]) for part in text.split() for k, names in [part.split(":")] for name in names.split(",")]


class StepArgs(C.Structure):
    _fields_ = fields("p:lens,keep,new,table l:ld p:free,count,parents,starts,slots,positions,mask i:n,blocks,block,room,tokens,words")


class MoveArgs(C.Structure):
    _fields_ = fields("p:caches c:layout p:table l:ld p:starts,lens,kept l:ld_kept p:n_kept,keep i:n_caches,dtype,dim,n,blocks,most")


class RotaryArgs(C.Structure):
    _fields_ = fields("h:x,x1,y,y1 p:positions,turns i:n,dtype,tokens,dim,rot,id_bytes,interleaved,inverse f:magnitude")


class StoreArgs(C.Structure):
    _fields_ = fields("h:q,q_out,k,v c:cache p:positions,slots,turns i:dtype,tokens,dim,rot,id_bytes,interleaved f:magnitude")


class AttentionArgs(C.Structure):
    _fields_ = fields("h:q,out c:cache p:starts,lens,table l:ld p:mask,lse,scratch l:bytes i:dtype,dim,tokens,n,blocks,words,new f:scale")


KIND = {"fq_cache_step": StepArgs, "fq_cache_move": MoveArgs, "fq_rotary": RotaryArgs, "fq_rotary_cache": StoreArgs, "fq_tree_attention": AttentionArgs}

ARG, SHAPE, ALIGN = -1, -3, -4
PAGE = C.create_string_buffer(1 << 16)
CTX = C.addressof(PAGE)
BUF = 0x10000                # aligned to anything asked for; never read
F16, BF16, F32 = 0, 1, 2

STEP = dict(ctx=CTX, n=4, lens=BUF, keep=BUF, new=BUF, table=BUF, ld=20, blocks=20, block=16, free=BUF, room=100, count=BUF, parents=BUF, tokens=30, starts=BUF,
            slots=BUF, positions=BUF, mask=BUF, words=2, stream=None)
MOVE = dict(ctx=CTX, caches=None, n_caches=2, layout=dict(), dtype=BF16, dim=64, n=4, table=BUF, ld=20, blocks=20, starts=BUF, lens=BUF, kept=BUF, ld_kept=5,
            most=5, n_kept=BUF, keep=BUF, stream=None)
ROTARY = dict(ctx=CTX, x=dict(), x1=dict(), y=dict(), y1=dict(), n=2, dtype=F16, tokens=5, dim=64, rot=32, positions=BUF, id_bytes=4, turns=BUF, interleaved=0, inverse=0, magnitude=1.0,
              stream=None)
STORE = dict(ctx=CTX, q=dict(), q_out=dict(), k=dict(heads=2), v=dict(heads=2), cache=dict(), dtype=F16, tokens=5, dim=64, rot=32, positions=BUF, id_bytes=8, slots=BUF,
             turns=BUF, interleaved=1, magnitude=1.0, stream=None)
ATTENTION = dict(ctx=CTX, q=dict(), out=dict(), cache=dict(), dtype=BF16, dim=64, tokens=5, n=4, starts=BUF, lens=BUF, table=BUF, ld=20, blocks=20, mask=BUF, words=1,
                 new=2, scale=0.1, lse=BUF, scratch=BUF, bytes=1 << 30, stream=None)
HEADS = dict(dev=BUF, token_stride=256, head_stride=64, heads=4)
CACHE = dict(k_dev=BUF, v_dev=BUF, block_stride=2048, token_stride=128, head_stride=64, blocks=9, block_size=16, heads=2)

TABLE = [("n", 0, SHAPE), ("n", 16385, SHAPE), ("table", 0, ARG), ("table", BUF + 2, ALIGN), ("ld", 19, SHAPE), ("blocks", 0, SHAPE), ("blocks", (1 << 20) + 1, SHAPE)]
LAYOUT = [("k_dev", 0, ARG), ("v_dev", 0, ARG), ("k_dev", BUF + 8, ALIGN), ("v_dev", BUF + 2, ALIGN), ("block_stride", 63, SHAPE), ("block_stride", 2052, ALIGN),
          ("token_stride", 60, SHAPE), ("token_stride", 132, ALIGN), ("head_stride", 63, SHAPE), ("head_stride", 65, ALIGN), ("block_stride", -2048, SHAPE), ("blocks", 0, SHAPE), ("block_size", 0, SHAPE),
          ("block_size", 65537, SHAPE), ("heads", 0, SHAPE)]
TURN = [("ctx", None, ARG), ("dtype", 3, ARG), ("tokens", 0, SHAPE), ("tokens", (1 << 20) + 1, SHAPE), ("dim", 1, SHAPE), ("dim", 1025, SHAPE), ("rot", 0, SHAPE), ("rot", 31, SHAPE),
        ("rot", 66, SHAPE), ("positions", 0, ARG), ("positions", BUF + 2, ALIGN), ("id_bytes", 2, ARG), ("turns", 0, ARG), ("turns", BUF + 4, ALIGN), ("magnitude", math.inf, ARG),
        ("magnitude", math.nan, ARG)]
BAD = {
    "fq_cache_step": (STEP, TABLE + [(f, 0, ARG) for f in ("ctx", "args", "lens", "keep", "new", "free", "count", "starts", "slots", "positions", "mask")] + [
        ("tokens", 0, SHAPE), ("tokens", (1 << 20) + 1, SHAPE), ("room", 0, SHAPE), ("words", 0, SHAPE), ("words", 17, SHAPE), ("block", 0, SHAPE), ("block", 65537, SHAPE),
        ("lens", BUF + 1, ALIGN), ("slots", BUF + 4, ALIGN), ("mask", BUF + 4, ALIGN), ("positions", BUF + 2, ALIGN), ("parents", BUF + 1, ALIGN)]),
    "fq_cache_move": (MOVE, TABLE + [(f, 0, ARG) for f in ("ctx", "args", "starts", "lens", "kept", "n_kept", "keep")] + [
        ("n_caches", 0, SHAPE), ("n_caches", 65537, SHAPE), ("dtype", 4, ARG), ("dim", 0, SHAPE), ("dim", 20, SHAPE), ("most", 0, SHAPE), ("most", 1025, SHAPE), ("ld_kept", 4, SHAPE),
        ("kept", BUF + 2, ALIGN), ("caches", 0, ARG)] + [("layout." + f, v, c) for f, v, c in LAYOUT if "dev" not in f] + [("caches", "unaligned", ALIGN), ("caches", "missing", ARG)]),
    "fq_rotary": (ROTARY, TURN + [("n", 0, SHAPE), ("n", 3, SHAPE), ("args", 0, ARG), ("x1.dev", 0, ARG), ("y1.heads", 5, SHAPE), ("x.dev", 0, ARG), ("y.dev", 0, ARG), ("x.dev", BUF + 1, ALIGN), ("x.heads", 0, SHAPE),
                                  ("x.heads", 5, SHAPE), ("x.token_stride", -1, SHAPE), ("y.token_stride", 63, SHAPE), ("y.head_stride", 63, SHAPE), ("y.head_stride", 0, SHAPE),
                                  ("y.token_stride", 128, SHAPE), ("x.head_stride", 72, ARG), ("x.token_stride", 264, ARG)]),
    "fq_rotary_cache": (STORE, TURN + [(f, 0, ARG) for f in ("args", "slots")] + [
        ("slots", BUF + 4, ALIGN), ("k.heads", 3, SHAPE), ("v.heads", 1, SHAPE), ("k.dev", 0, ARG), ("v.dev", BUF + 1, ALIGN), ("q_out.heads", 3, SHAPE), ("q_out.token_stride", 200, SHAPE),
        ("dim", 60, SHAPE)] + [("cache." + f, v, c) for f, v, c in LAYOUT]),
    "fq_tree_attention": (ATTENTION, TABLE + [(f, 0, ARG) for f in ("ctx", "args", "starts", "lens", "scratch")] + [
        ("dtype", F32, ARG), ("dtype", -1, ARG), ("dim", 0, SHAPE), ("dim", 60, SHAPE), ("dim", 264, SHAPE), ("tokens", 0, SHAPE), ("tokens", (1 << 20) + 1, SHAPE), ("words", 0, SHAPE),
        ("words", 17, SHAPE), ("new", 0, SHAPE), ("scale", 0.0, ARG), ("scale", -1.0, ARG), ("scale", math.nan, ARG), ("scale", math.inf, ARG), ("mask", BUF + 4, ALIGN), ("lse", BUF + 2, ALIGN),
        ("scratch", BUF + 8, ALIGN), ("starts", BUF + 2, ALIGN), ("lens", BUF + 1, ALIGN), ("q.dev", 0, ARG), ("out.dev", 0, ARG), ("q.dev", BUF + 8, ALIGN), ("out.dev", BUF + 2, ALIGN),
        ("q.heads", 3, SHAPE), ("q.heads", 1026, SHAPE), ("q.heads", 6, SHAPE), ("q.token_stride", 260, ALIGN), ("q.head_stride", 68, ALIGN), ("q.token_stride", -256, SHAPE),
        ("out.token_stride", 132, SHAPE), ("out.token_stride", 260, ALIGN), ("out.head_stride", 32, SHAPE)] + [("cache." + f, v, c) for f, v, c in LAYOUT]),
}


@pytest.mark.parametrize("name,field,value,code", [(n, f, v, c) for n, (_, bad) in BAD.items() for f, v, c in bad])
def test_refused(name, field, value, code):
    args = {k: dict(v) if isinstance(v, dict) else v for k, v in BAD[name][0].items()}
    if "." in field:
        outer, inner = field.split(".")
        args[outer][inner] = value
    elif not (field == "caches" and value != 0):
        args[field] = value
    pointers = [BUF, BUF]
    if field == "caches" and value == "unaligned":
        pointers[1] += 8
    if field == "caches" and value == "missing":
        pointers[1] = 0
    ctx, stream = args.pop("ctx"), args.pop("stream")
    whole = args.pop("args", 1)
    array = (C.c_void_p * 2)(*pointers)
    if "caches" in args and args["caches"] is None:
        args["caches"] = C.addressof(array)
    made = KIND[name](**{k: (Cache(**{**CACHE, **v}) if k in ("cache", "layout") else Heads(**{**HEADS, **v})) if isinstance(v, dict) else v for k, v in args.items()})
    assert getattr(P.lib(), name)(ctx, C.addressof(made) if whole else None, stream) == code
    assert PAGE.raw == bytes(1 << 16)


@pytest.mark.parametrize("rot,base,factor,context,low,high,code", [(0, 1e4, 1.0, 0, 1.0, 2.0, SHAPE), (3, 1e4, 1.0, 0, 1.0, 2.0, SHAPE), (1026, 1e4, 1.0, 0, 1.0, 2.0, SHAPE), (8, 1.0, 1.0, 0, 1.0, 2.0, ARG),
                                                                  (8, math.nan, 1.0, 0, 1.0, 2.0, ARG), (8, math.inf, 1.0, 0, 1.0, 2.0, ARG), (8, 1e4, 0.5, 0, 1.0, 2.0, ARG), (8, 1e4, math.inf, 0, 1.0, 2.0, ARG),
                                                                  (8, 1e4, 2.0, -1, 1.0, 2.0, ARG), (8, 1e4, 2.0, 10, 2.0, 2.0, ARG), (8, 1e4, 2.0, 10, -1.0, 2.0, ARG), (8, 1e4, 2.0, 10, 1.0, math.inf, ARG)])
def test_tables_refused(rot, base, factor, context, low, high, code):
    with pytest.raises(P.FlexQError) as e:
        P.fq_rotary_table(rot, base, factor, context, low, high, device="cpu")
    assert e.value.code == code


@pytest.mark.parametrize("rot,args", [(128, {}), (2, {}), (1024, dict(base=500000.0)), (64, dict(factor=8.0)), (64, dict(factor=16.0, context=8192, low=1.0, high=32.0))])
def test_table_values(rot, args):
    """Against 60 digits: half a step of 2^-64 of a turn, and the logarithm's and power's error of some 2^-62 of the fraction."""
    from decimal import Decimal, getcontext
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    got = [int(v) % (1 << 64) for v in P.fq_rotary_table(rot, device="cpu", **args)]
    factor, context = Decimal(args.get("factor", 1.0)), args.get("context", 0)
    for i, v in enumerate(got):
        f = Decimal(args.get("base", 10000.0)) ** (Decimal(-2 * i) / rot) / (2 * pi)
        kept = min(Decimal(1), max(Decimal(0), (context * f - 1) / 31)) if context else Decimal(0)
        want = (kept * f + (1 - kept) * f / factor) * 2 ** 64
        assert abs(Decimal(v) - want) <= Decimal(0.5) + want * Decimal(2) ** -59


def test_structures_are_packed_as_c_lays_them_out():
    from paper_2501_07139_b200 import flexq as F
    for made, packed in ((StepArgs, F._STEP_ARGS), (MoveArgs, F._MOVE_ARGS), (RotaryArgs, F._ROTARY_ARGS), (StoreArgs, F._ROTARY_CACHE_ARGS), (AttentionArgs, F._ATTENTION_ARGS)):
        assert C.sizeof(made) == packed.size
        n, values, flat = 0, [], []

        def fill(kind):
            nonlocal n
            s = kind()
            for name, t in kind._fields_:
                if issubclass(t, C.Structure):
                    setattr(s, name, fill(t))
                else:
                    n += 1
                    setattr(s, name, n)
                    flat.append(n)
            return s

        s = fill(made)
        assert packed.unpack(bytes(s)) == tuple(flat)


def test_methods_name_what_does_not_fit():
    """The binding's own checks, on CPU tensors: a context without a device refuses them all."""
    import torch
    fq = P.FlexQ.__new__(P.FlexQ)
    fq._h, fq.device, fq._index = C.c_void_p(), torch.device("cuda", 0), 0
    q, cache = torch.zeros((2, 4, 8), dtype=torch.float16), torch.zeros((3, 4, 2, 8), dtype=torch.float16)
    i32, i64 = torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int64)
    table = torch.zeros((2, 3), dtype=torch.int32)
    for call in (lambda: fq.fq_cache_step(i32, i32, i32, table, i32, i32[:1], 4, 2), lambda: fq.fq_cache_move([cache], table, i32, i32, table, i32), lambda: fq.fq_rotary(q, q, i32, i64),
                 lambda: fq.fq_rotary_cache(q, q, q, i32, i64, i64, cache, cache), lambda: fq.fq_tree_attention(q, cache, cache, table, i32, i32)):
        with pytest.raises(ValueError, match="cuda:0"):
            call()
    with pytest.raises(ValueError, match="none"):
        fq.fq_cache_move([], table, i32, i32, table, i32)


def test_scratch_sizes():
    assert P.lib().fq_tree_attention_scratch(None, 1, 1, 4, 4, 128, 1) == 0
    for args in ((0, 1, 4, 4, 128, 1), (1, 0, 4, 4, 128, 1), (1, 1, 6, 4, 128, 1), (1, 1, 4, 8, 128, 1), (1, 1, 4, 4, 100, 1), (1, 1, 4, 4, 264, 1), (1, 1, 4, 4, 128, 0)):
        assert P.lib().fq_tree_attention_scratch(CTX, *args) == 0
    for code in (-13, -14):
        assert P.fq_strerror(code) != "unknown error"
