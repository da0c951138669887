"""Host-side checks of the layer operators' C boundary that need no GPU: refusals come before
anything is enqueued (the device pointers here are never dereferenced)."""
import pytest

from paper_2609_35481_b200 import binding as B

P = 4096   # stands in for a device pointer


def cfg(**kw):
    a = dict(experts=16, top_k=2, dtype=B.DTYPE_F32, score=B.SCORE_SOFTMAX, normalize=1, scale=1.0)
    a.update(kw)
    return B.RouterConfig(*[a[n] for n, _ in B.RouterConfig._fields_])


def test_router_refuses():
    fwd = lambda c=None, x=P, stride=16, tokens=4, bias=None, mask=None, ids=P, w=P: \
        B.topoep_router_forward(cfg() if c is None else c, x, stride, tokens, bias, mask, ids, w)
    bwd = lambda c=None, x=P, stride=16, tokens=4, ids=P, w=P, dw=P, g=P, gs=16: \
        B.topoep_router_backward(cfg() if c is None else c, x, stride, tokens, ids, w, dw, g, gs)
    assert B.topoep_router_forward(None, P, 16, 4, None, None, P, P) == -1
    for call in (fwd, bwd):
        for kw in (dict(experts=0), dict(experts=16385), dict(top_k=0), dict(top_k=17),
                   dict(experts=64, top_k=33)):
            assert call(cfg(**kw)) == -2
        for kw in (dict(dtype=3), dict(dtype=-1), dict(score=2), dict(normalize=2), dict(scale=0.0),
                   dict(scale=-1.0), dict(scale=float("inf")), dict(scale=float("nan"))):
            assert call(cfg(**kw)) == -10
        assert call(stride=15) == -6 and call(tokens=-1) == -6
        assert call(x=None) == -1 and call(ids=None) == -1 and call(w=None) == -1
        assert call(x=P + 2) == -7 and call(ids=P + 1) == -7 and call(w=P + 2) == -7
        assert call(tokens=0, x=None, ids=None, w=None) == 0
    assert fwd(bias=P) == -10                                        # softmax takes no bias
    assert fwd(cfg(score=B.SCORE_SIGMOID), bias=P + 2) == -7
    assert bwd(gs=15) == -6 and bwd(g=None) == -1 and bwd(dw=None) == -1 and bwd(g=P + 1) == -7


def test_experts_refuse():
    good = dict(ranks=2, experts_per_rank=3, slots_per_rank=1, hidden=64, ffn=32, top_k=2, max_tokens=8)

    def rc(**kw):
        code, h = B.topoep_experts_create(**dict(good, **kw))
        if h is not None:
            B.topoep_experts_destroy(h)
        return code

    assert rc() == 0 and rc(experts_per_rank=0) == 0 and rc(slots_per_rank=0) == 0
    for kw in (dict(ranks=0), dict(experts_per_rank=-1), dict(slots_per_rank=-1), dict(hidden=0),
               dict(hidden=65537), dict(ffn=0), dict(ffn=65537), dict(top_k=0), dict(top_k=17),
               dict(max_tokens=0), dict(max_tokens=129), dict(experts_per_rank=0, slots_per_rank=0),
               dict(ranks=4097), dict(experts_per_rank=8193), dict(ranks=2 ** 30, experts_per_rank=2 ** 30)):
        assert rc(**kw) == -2, kw
    code, h = B.topoep_experts_create(**good)
    assert code == 0
    assert B.topoep_experts_workspace_bytes(h) > 0 and B.topoep_experts_workspace_bytes(h) % 256 == 0
    assert B.topoep_experts_forward(h, P, 64, P, P, 1, P, 64) == -5          # no workspace
    assert B.topoep_experts_read_status(h)[0] == -5
    assert B.topoep_experts_set_workspace(h, None, 1 << 40) == -1
    assert B.topoep_experts_set_workspace(h, P, 16) == -5
    assert B.topoep_experts_set_workspace(h, P + 16, 1 << 40) == -5
    assert B.topoep_experts_set_params(h, None, P) == -1 and B.topoep_experts_set_params(h, P, None) == -1
    assert B.topoep_experts_set_params(h, P + 8, P) == -7 and B.topoep_experts_set_params(h, P, P + 8) == -7
    B.topoep_experts_destroy(h)
    B.topoep_experts_destroy(None)
    assert B.topoep_experts_workspace_bytes(None) == 0
    assert B.topoep_experts_forward(None, P, 64, P, P, 1, P, 64) == -1
    assert B.topoep_experts_set_params(None, P, P) == -1


@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (dict(dst=None), 0), (dict(rows=0), 0), (dict(cols=0), 0), (dict(rows=0, src=None), 0),
    (dict(dtype=3), -10), (dict(rows=-1), -6), (dict(cols=-1), -6), (dict(rows=2 ** 40, cols=2 ** 40), -6),
    (dict(src=None), -1), (dict(src=P + 2), -7), (dict(dst=P + 1), -7), (dict(src_row_stride=7), -6),
    (dict(dst_row_stride=7), -6), (dict(dst=P, dst_row_stride=9), -10), (dict(rows=1, src_row_stride=0), 0),
    (dict(dst=None, dst_row_stride=0), 0)])
def test_clip_refuses(kw, code):
    a = dict(src=P, dst=2 * P, rows=3, cols=8, src_row_stride=8, dst_row_stride=8, dtype=B.DTYPE_F32, reserved=0)
    a.update(kw)
    rc, h = B.topoep_clip_create([B.GradTensor(*[a[n] for n, _ in B.GradTensor._fields_])])
    assert rc == code
    if h is not None:
        assert B.topoep_clip_run(h, 0, 1.0, P) == -5 and B.topoep_clip_norm(h, 0, P) == -5
        assert B.topoep_clip_set_workspace(h, P, 1) == -5 and B.topoep_clip_set_workspace(h, None, 1 << 30) == -1
        B.topoep_clip_destroy(h)


def test_clip_empty_list_and_null_handle():
    rc, h = B.topoep_clip_create([])
    assert rc == 0 and B.topoep_clip_workspace_bytes(h) % 256 == 0
    B.topoep_clip_destroy(h)
    B.topoep_clip_destroy(None)
    assert B.topoep_clip_run(None, 0, 1.0, P) == -1 and B.topoep_clip_workspace_bytes(None) == 0


def test_clip_refuses_a_gradient_listed_twice():
    def rc(*tensors):
        code, h = B.topoep_clip_create([B.GradTensor(src, dst, rows, cols, stride, stride, B.DTYPE_F32, 0)
                                        for src, dst, rows, cols, stride in tensors])
        if h is not None:
            B.topoep_clip_destroy(h)
        return code

    assert rc((P, None, 1, 8, 8), (P + 32, None, 1, 8, 8)) == 0
    assert rc((P, None, 1, 8, 8), (P + 28, None, 1, 8, 8)) == -10
    assert rc((P + 28, None, 1, 8, 8), (P, None, 1, 8, 8)) == -10
    assert rc((P, None, 1, 8, 8), (P, None, 1, 8, 8)) == -10
    assert rc((P, None, 1, 100, 100), (P + 40, None, 1, 2, 2)) == -10
    assert rc((P, 4 * P, 1, 8, 8), (P, 8 * P, 1, 8, 8)) == 0            # one source, two outputs
    assert rc((P, 4 * P, 1, 8, 8), (2 * P, 4 * P, 1, 8, 8)) == -10
    assert rc((P, None, 4, 8, 16), (P + 32, None, 4, 8, 16)) == 0       # two halves of rows
    assert rc((P, None, 4, 8, 16), (P, None, 4, 8, 16)) == -10


def test_router_copies_by_its_arguments():
    import copy
    import pickle
    from paper_2609_35481_b200 import Router
    r = Router(16, 2, score="sigmoid", normalize=False, scale=2.5)
    for c in (copy.deepcopy(r), pickle.loads(pickle.dumps(r))):
        assert (c.experts, c.top_k, c.score, c.normalize, c.scale) == (16, 2, "sigmoid", False, 2.5)
    for bad in (dict(experts=4, top_k=8), dict(experts=4, top_k=2, scale=0.0)):
        with pytest.raises(B.TopoEPError):
            Router(**bad)
    with pytest.raises(ValueError):
        Router(4, 2, score="relu")
