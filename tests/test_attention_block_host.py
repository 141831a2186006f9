"""CPU-only checks of the operators around and in attention (embeddings, residual, attention, one token's attention): bad arguments,
arrays that lie over each other and workspaces that are too small are refused before anything reaches a GPU.  A call that passes the checks of its
arrays is seen by the refusal of its workspace, which comes last."""
import ctypes as C

import pytest
import torch

from paper_2509_03110_amd import lsam, ops

MB = 1 << 20
F32, BF16 = ops.DTYPE_FP32, ops.DTYPE_BF16
NAN, INF = float("nan"), float("inf")


def changed(d, over):
    for path, v in over.items():
        *of, name = path.split(".")
        t = d
        for o in of:
            t = getattr(t, o)
        setattr(t, name, v)
    return C.byref(d)


def places(names):
    return {n: 16 * MB * (i + 1) for i, n in enumerate(names)}


def refuses(rc, word, code=lsam.EINVAL):
    assert rc == code and word in lsam.last_error(), (rc, word, lsam.last_error())


# ---- embeddings ---------------------------------------------------------------------------------------

def embedding(**over):
    d = ops.lsam_embedding_desc()
    d.replicas, d.dtype, d.table_dtype, d.scale, d.rows, d.vocab, d.dim = 2, BF16, F32, 1.0, 100, 50, 16
    d.token_replica = 100
    for n, rows in (("table", 50), ("y", 100), ("dy", 100), ("dtable", 50)):
        setattr(d, n + "_stride", 16)
        setattr(d, n + "_replica", 16 * rows)
    return changed(d, over)


LOOKUP = ["tokens", "table", "y"]
SUMS = ["tokens", "dy", "dtable", "ws"]


def lookup(d, **over):
    a = dict(places(LOOKUP), **over)
    return ops._lib().lsam_embedding(d, *(a[n] for n in LOOKUP), None)


def table_gradient(d, need=1, **over):
    a = dict(places(SUMS), **over)
    return ops._lib().lsam_embedding_backward(d, *(a[n] for n in SUMS), need, None)


def test_embeddings():
    need = ops._lib().lsam_embedding_workspace_bytes
    for over, word in ((dict(dtype=7), "dtype"), (dict(table_dtype=-1), "dtype"), (dict(replicas=-1), "replicas"), (dict(replicas=65536), "replicas"),
                       (dict(rows=-1), "rows"), (dict(rows=1 << 31), "rows"), (dict(vocab=0), "vocab"), (dict(vocab=(1 << 22) + 1), "vocab"),
                       (dict(dim=0), "dim"), (dict(dim=(1 << 24) + 1), "dim"), (dict(rows=1 << 30, dim=1 << 14), "too large")):
        refuses(lookup(embedding(**over)), word)
        refuses(table_gradient(embedding(**over)), word)
        assert need(embedding(**over)) == 0 and word in lsam.last_error()
    for over, word in ((dict(table_stride=15), "table"), (dict(table_replica=-1), "table"), (dict(y_stride=15), "y"),
                       (dict(y_replica=1599), "over each other"), (dict(y_replica=0), "over each other"), (dict(token_replica=-1), "tokens"),
                       (dict(table_stride=1 << 62), "table")):
        refuses(lookup(embedding(**over)), word)
    for n in LOOKUP:
        refuses(lookup(embedding(), **{n: None}), n)
        refuses(lookup(embedding(), **{n: places(LOOKUP)[n] + 1}), "aligned")
        if n != "y":
            refuses(lookup(embedding(), y=places(LOOKUP)[n] + 16), "lies over")
    for over in (dict(replicas=0), dict(rows=0)):
        assert lookup(embedding(**over), tokens=None, table=None, y=None) == 0
    assert table_gradient(embedding(replicas=0), tokens=None, dy=None, dtable=None, ws=None) == 0

    for over, word in ((dict(dy_stride=15), "dy"), (dict(dtable_stride=15), "dtable"), (dict(dtable_replica=799), "over each other"),
                       (dict(dtable_replica=0), "over each other"), (dict(token_replica=-1), "tokens")):
        refuses(table_gradient(embedding(**over)), word)
    enough = need(embedding())
    assert enough > 0
    for n in SUMS[:-1]:
        refuses(table_gradient(embedding(), enough, **{n: None}), n)
        refuses(table_gradient(embedding(), enough, ws=places(SUMS)[n]), "lies over")
        if n != "dtable":
            refuses(table_gradient(embedding(), enough, dtable=places(SUMS)[n] + 16), "lies over")
    refuses(table_gradient(embedding(), enough, ws=None), "", lsam.ENOMEM)
    refuses(table_gradient(embedding(), enough - 1), "", lsam.ENOMEM)
    refuses(table_gradient(embedding(), enough, ws=4 * MB + 8), "aligned")
    # shared tokens, rows of one array side by side, and a broadcast gradient are no faults: the workspace is looked at next
    for over in (dict(token_replica=0), dict(token_replica=40), dict(dtable_replica=16, dtable_stride=40), dict(dy_replica=0),
                 dict(replicas=1, dtable_replica=0, dy_replica=0, token_replica=0)):
        refuses(table_gradient(embedding(**over), 1), "", lsam.ENOMEM)


def test_a_table_gradients_workspace_stays_small_beside_what_it_reads():
    need = ops._lib().lsam_embedding_workspace_bytes
    for replicas, rows, vocab, dim in ((4, 4096, 32000, 1024), (1, 131072, 1000, 256), (1, 1 << 20, 1 << 20, 64), (1, 1, 1 << 22, 8)):
        bytes_ = need(embedding(replicas=replicas, rows=rows, vocab=vocab, dim=dim))
        chunks = (rows + 63) // 64
        # an index a row, one a token, partial sums of two rows for each 64, counts that are at most 16 MiB, and roundings
        assert 0 < bytes_ <= replicas * (rows * 4 + vocab * 4 + chunks * 8 * dim + (17 << 20)) + 2048


# ---- residual -----------------------------------------------------------------------------------------

ROWS_OF = ["r", "y", "gate", "r_out", "h", "dr", "dh", "dr_out", "dy", "dgate"]


def residual(**over):
    d = ops.lsam_residual_desc()
    d.replicas, d.dtype, d.rows, d.dim, d.alpha, d.beta, d.eps = 2, BF16, 10, 32, 1.0, 1.0, 1e-6
    for n in ROWS_OF:
        setattr(d, n + "_stride", 32)
        setattr(d, n + "_replica", 320)
    for n in ("w_pre", "w_post", "dw_pre", "dw_post"):
        setattr(d, n + "_replica", 32)
    return changed(d, over)


FORWARD = ["r", "y", "gate", "w_pre", "w_post", "r_out", "h"]
BACKWARD = ["r", "y", "gate", "w_pre", "w_post", "dr", "dh", "dr_out", "dy", "dgate", "dw_pre", "dw_post", "ws"]


def join(d, **over):
    a = dict(places(FORWARD), **over)
    return ops._lib().lsam_residual(d, *(a[n] for n in FORWARD), None)


def join_gradient(d, need=1, **over):
    a = dict(places(BACKWARD), **over)
    return ops._lib().lsam_residual_backward(d, *(a[n] for n in BACKWARD), need, None)


def test_residual():
    need = ops._lib().lsam_residual_workspace_bytes
    for over, word in ((dict(dtype=3), "dtype"), (dict(replicas=-1), "replicas"), (dict(replicas=65536), "replicas"), (dict(rows=-1), "rows"),
                       (dict(rows=1 << 31), "rows"), (dict(dim=0), "dim"), (dict(dim=16385), "dim"), (dict(eps=-1.0), "eps"), (dict(eps=NAN), "eps")):
        refuses(join(residual(**over)), word)
        refuses(join_gradient(residual(**over)), word)
        assert need(residual(**over)) == 0 and word in lsam.last_error()
    for n in FORWARD:
        if n not in ("w_pre", "w_post", "y", "gate"):
            refuses(join(residual(), **{n: None}), n)
        refuses(join(residual(), **{n: places(FORWARD)[n] + 1}), "aligned")
        if not n.startswith("w"):
            refuses(join(residual(**{n + "_stride": 31})), n)
        if n not in ("r_out", "h"):
            for out in ("r_out", "h"):
                refuses(join(residual(), **{out: places(FORWARD)[n] + 4}), "lies over")
    refuses(join(residual(), r_out=places(FORWARD)["h"]), "lies over")
    refuses(join(residual(), y=None, w_pre=None), "nothing to do")
    refuses(join(residual(h_replica=319)), "h")
    refuses(join(residual(r_out_replica=0)), "r_out")
    refuses(join(residual(r_out_stride=64, r_out_replica=640), r_out=places(FORWARD)["r"]), "lies over")      # r itself, but of another stride
    for over in (dict(replicas=0), dict(rows=0)):
        assert join(residual(**over), **{n: None for n in FORWARD}) == 0

    enough = need(residual())
    assert enough > 0
    for n in BACKWARD[:-1]:
        if n in ("r", "dh"):
            refuses(join_gradient(residual(), enough, **{n: None}), n)
        refuses(join_gradient(residual(), enough, ws=places(BACKWARD)[n]), "lies over")
        refuses(join_gradient(residual(), enough, **{n: places(BACKWARD)[n] + 1}), "aligned")
        for out in ("dr_out", "dy", "dgate", "dw_pre", "dw_post"):
            if n != out:
                refuses(join_gradient(residual(), enough, **{out: places(BACKWARD)[n] + 4}), "lies over")
    for over, word in ((dict(dy_stride=31), "dy"), (dict(dgate_replica=319), "dgate"), (dict(dw_pre_replica=31), "dw_pre"), (dict(dw_post_replica=0), "dw_post")):
        refuses(join_gradient(residual(**over), enough), word)
    for fewer in (dict(ws=None), dict(need=enough - 1), dict(need=enough - 1, dw_post=None), dict(need=enough - 1, dw_pre=None)):
        refuses(join_gradient(residual(), **dict(dict(need=enough), **fewer)), "", lsam.ENOMEM)
    # dr's own place, weights' gradients in one array, weights that replicas share, rows of one array side by side: the workspace is looked at next
    at = places(BACKWARD)
    refuses(join_gradient(residual(), dr_out=at["dr"]), "", lsam.ENOMEM)
    refuses(join_gradient(residual(dw_pre_replica=100, dw_post_replica=100), dw_post=at["dw_pre"] + 4 * 32), "", lsam.ENOMEM)
    refuses(join_gradient(residual(dw_pre_replica=100, dw_post_replica=100), dw_post=at["dw_pre"] + 4 * 31), "lies over")
    refuses(join_gradient(residual(w_pre_replica=0, w_post_replica=0)), "", lsam.ENOMEM)
    refuses(join_gradient(residual(dr_out_stride=64, dr_out_replica=640, dy_stride=64, dy_replica=640), dy=at["dr_out"] + 2 * 32), "", lsam.ENOMEM)
    refuses(join_gradient(residual(), y=None, w_pre=None), "nothing to do")
    assert join_gradient(residual(replicas=0), **{n: None for n in BACKWARD}) == 0


# ---- attention ----------------------------------------------------------------------------------------

def attention(**over):
    d = ops.lsam_attention_desc()
    d.rows, d.seqs, d.heads, d.kv_heads, d.dim, d.dtype, d.scale = 100, 3, 4, 2, 16, BF16, 0.25
    for n, heads in (("q", 4), ("k", 2), ("v", 2), ("o", 4), ("d_o", 4), ("dq", 4), ("dk", 2), ("dv", 2)):
        getattr(d, n).stride, getattr(d, n).head = 16 * heads, 16
    return changed(d, over)


ATTEND = ["offsets", "q", "k", "v", "o", "lse"]
ATTEND_BACK = ["offsets", "q", "k", "v", "o", "lse", "d_o", "dq", "dk", "dv", "ws"]


def attend(d, **over):
    a = dict(places(ATTEND), **over)
    return ops._lib().lsam_attention(d, *(a[n] for n in ATTEND), None)


def attend_gradient(d, need=1, **over):
    a = dict(places(ATTEND_BACK), **over)
    return ops._lib().lsam_attention_backward(d, *(a[n] for n in ATTEND_BACK), need, None)


HEADS = ((dict(heads=0), "heads"), (dict(kv_heads=0), "heads"), (dict(kv_heads=3), "heads"), (dict(heads=65538), "heads"), (dict(dim=0), "dim"),
         (dict(dim=129), "dim"), (dict(dtype=2), "dtype"), (dict(scale=-0.5), "scale"), (dict(scale=NAN), "scale"), (dict(scale=INF), "scale"),
         (dict(scale=2.0 ** 101), "scale"))


def test_attention():
    need = ops._lib().lsam_attention_workspace_bytes
    for over, word in HEADS + ((dict(rows=-1), "rows"), (dict(rows=1 << 28), "rows"), (dict(seqs=-1), "seqs"), (dict(seqs=1 << 31), "seqs")):
        refuses(attend(attention(**over)), word)
        refuses(attend_gradient(attention(**over)), word)
        assert need(attention(**over)) == 0 and word in lsam.last_error()
    for n in ATTEND[:-1]:
        refuses(attend(attention(), **{n: None}), n)
    for n in ATTEND:
        refuses(attend(attention(), **{n: places(ATTEND)[n] + 1}), "aligned")
        for out in ("o", "lse"):
            if n != out:
                refuses(attend(attention(), **{out: places(ATTEND)[n] + 8}), "lies over")
    for over, word in (({"q.stride": 15}, "q"), ({"k.stride": -1}, "k"), ({"v.head": -16}, "v"), ({"o.head": 15}, "o"), ({"o.head": 0}, "o"),
                       ({"o.stride": 63}, "o"), ({"q.stride": 1 << 60}, "q")):
        refuses(attend(attention(**over)), word)
    for over in (dict(rows=0), dict(seqs=0)):
        assert attend(attention(**over), **{n: None for n in ATTEND}) == 0
        assert attend_gradient(attention(**over), **{n: None for n in ATTEND_BACK}) == 0
    # the largest sizes have workspaces that are counted in 64 bits
    assert need(attention(rows=(1 << 28) - 1)) >= 4 * ((1 << 28) - 1) * 8

    enough = need(attention())
    assert enough > 0
    for n in ATTEND_BACK[:-1]:
        refuses(attend_gradient(attention(), enough, **{n: None}), n)
        refuses(attend_gradient(attention(), enough, **{n: places(ATTEND_BACK)[n] + 1}), "aligned")
        refuses(attend_gradient(attention(), enough, ws=places(ATTEND_BACK)[n]), "lies over")
        for out in ("dq", "dk", "dv"):
            if n != out:
                refuses(attend_gradient(attention(), enough, **{out: places(ATTEND_BACK)[n] + 8}), "lies over")
    for over, word in (({"dq.stride": 63}, "dq"), ({"dk.head": 0}, "dk"), ({"dv.head": 8}, "dv"), ({"d_o.stride": 1}, "d_o")):
        refuses(attend_gradient(attention(**over), enough), word)
    refuses(attend_gradient(attention(), enough - 1), "", lsam.ENOMEM)
    refuses(attend_gradient(attention(), enough, ws=None), "", lsam.ENOMEM)
    refuses(attend_gradient(attention(), enough, ws=4 * MB + 8), "aligned")
    # q, k and v and their gradients as parts of one array's rows, and heads outside of rows: the workspace is looked at next
    at = places(ATTEND_BACK)
    one = {n + ".stride": 128 for n in ("q", "k", "v", "dq", "dk", "dv")}
    side = dict(k=at["q"] + 128, v=at["q"] + 192, dk=at["dq"] + 128, dv=at["dq"] + 192)
    refuses(attend_gradient(attention(**one), **side), "", lsam.ENOMEM)
    refuses(attend_gradient(attention(**one), **dict(side, dv=at["dq"] + 190)), "lies over")
    outside = {}
    for n in ("q", "k", "v", "o", "d_o", "dq", "dk", "dv"):
        outside[n + ".stride"], outside[n + ".head"] = 16, 1600
    refuses(attend_gradient(attention(**outside)), "", lsam.ENOMEM)
    refuses(attend_gradient(attention(**{"k.head": 0, "v.head": 0})), "", lsam.ENOMEM)          # keys that heads share


# ---- one token's attention ----------------------------------------------------------------------------

def step(**over):
    d = ops.lsam_attention_step_desc()
    d.seqs, d.capacity, d.prefix, d.heads, d.kv_heads, d.dim, d.dtype, d.scale = 3, 500, 300, 4, 2, 16, BF16, 0.25
    for n, heads in (("q", 4), ("o", 4), ("k", 2), ("v", 2), ("prefix_k", 2), ("prefix_v", 2)):
        getattr(d, n).stride, getattr(d, n).head = 16 * heads, 16
    d.k_seq = d.v_seq = 500 * 32
    return changed(d, over)


STEP = ["lengths", "q", "k", "v", "prefix_k", "prefix_v", "o", "ws"]


def one_token(d, need=1, **over):
    a = dict(places(STEP), **over)
    return ops._lib().lsam_attention_step(d, *(a[n] for n in STEP), need, None)


def test_one_tokens_attention():
    need = ops._lib().lsam_attention_step_workspace_bytes
    for over, word in HEADS + ((dict(seqs=-1), "seqs"), (dict(seqs=1 << 21), "seqs"), (dict(capacity=-1), "capacity"), (dict(capacity=1 << 30), "capacity"),
                               (dict(prefix=-1), "prefix"), (dict(prefix=1 << 30), "prefix")):
        refuses(one_token(step(**over)), word)
        assert need(step(**over)) == 0 and word in lsam.last_error()
    enough = need(step())
    assert enough > 0
    for n in STEP[:-1]:
        refuses(one_token(step(), enough, **{n: None}), n)
        refuses(one_token(step(), enough, **{n: places(STEP)[n] + 1}), "aligned")
        refuses(one_token(step(), enough, ws=places(STEP)[n]), "lies over")
        if n != "o":
            refuses(one_token(step(), enough, o=places(STEP)[n] + 8), "lies over")
    for over, word in (({"q.stride": -1}, "q"), ({"k.head": -1}, "k"), ({"v_seq": -1}, "v"), ({"prefix_v.stride": -1}, "prefix_v"), ({"o.head": 15}, "o"),
                       ({"o.stride": 0}, "o"), ({"k_seq": 1 << 60}, "k")):
        refuses(one_token(step(**over), enough), word)
    refuses(one_token(step(), enough - 1), "", lsam.ENOMEM)
    refuses(one_token(step(), enough, ws=None), "", lsam.ENOMEM)
    assert one_token(step(seqs=0), **{n: None for n in STEP}) == 0 and need(step(seqs=0)) == 0
    # what is not there needs no address; caches, prefix and queries may be broadcast: the workspace is looked at next
    refuses(one_token(step(prefix=0), prefix_k=None, prefix_v=None), "", lsam.ENOMEM)
    refuses(one_token(step(capacity=0), k=None, v=None), "", lsam.ENOMEM)
    refuses(one_token(step(**{"k_seq": 0, "k.head": 0, "v.stride": 0, "q.stride": 0, "prefix_k.head": 0})), "", lsam.ENOMEM)
    # one part of one thing to attend to is written by those who read it
    assert need(step(prefix=0, capacity=100)) == 0 and need(step(prefix=0, capacity=100, seqs=50)) == 0
    assert need(step(prefix=0, capacity=0)) == 0


# ---- the binding ----------------------------------------------------------------------------------------

@pytest.mark.parametrize("call, word", [
    (lambda f, i: ops.embedding(i[0], f[0]), "GPU"), (lambda f, i: ops.embedding(i[None], f[0]), "indices"),
    (lambda f, i: ops.embedding_backward(i[0], f, 10), "GPU"), (lambda f, i: ops.embedding_backward(i[None], f, 10), "indices"),
    (lambda f, i: ops.residual(f[0, 0], None, f[0, 0]), "indices"), (lambda f, i: ops.residual_backward(f[0, 0], None, f[0, 0], None, f[0]), "indices"),
    (lambda f, i: ops.residual_backward(f, None, f[0, 0], None, f), "shared"), (lambda f, i: ops.residual_backward(f[0], None, f[0, 0], None, None), "dh"),
    (lambda f, i: ops.attention(f[0], f, f, i), "indices"), (lambda f, i: ops.attention(f, f, f, i), "offsets"),
    (lambda f, i: ops.attention_step(f, f, f, i), "indices"), (lambda f, i: ops.attention_step(f, f[None], f[None], i, prefix_k=f), "missing"),
])
def test_the_binding_refuses_shapes_and_devices(call, word):
    f, i = torch.zeros(2, 3, 4), torch.zeros(2, 3, dtype=torch.int32)
    with pytest.raises(lsam.LsamError) as e:
        call(f, i)
    assert e.value.code == lsam.EINVAL and word in str(e.value)
