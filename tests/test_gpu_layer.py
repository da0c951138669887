"""Layer operators (router, experts of a few tokens, gradient clipping) on the GPU against plain
64-bit forms; every bound is derived in layer_reference."""
import math

import numpy as np
import pytest
import torch

import layer_reference as ref
from paper_2609_35481_b200 import GradientClip, Router, TokenExperts, binding as B

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
INF, NAN = math.inf, math.nan


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


# ------------------------------------------------------------------------------------- router

def check_router(logits, k, score, normalize, scale, bias=None, mask=None, finite=True):
    E = logits.shape[-1]
    r = Router(E, k, score=score, normalize=normalize, scale=scale)
    ids, w = r.forward(logits, bias=bias, mask=mask)
    want_ids, want_w = ref.router_forward(logits, k, score, normalize, scale, bias, mask)
    assert ids.dtype == torch.int32 and w.dtype == F32
    assert torch.equal(ids.cpu(), want_ids)
    if finite:
        bound = ref.router_weight_bound(logits, want_w, E)
        assert ((w.cpu().double() - want_w).abs() <= bound).all()
    return r, ids, w


def check_router_grad(r, logits, ids, w, seed):
    dw = torch.randn(w.shape, generator=gen(seed), device="cuda")
    got = r.backward(logits, ids, w, dw)
    assert got.dtype == logits.dtype and got.shape == logits.shape
    want, size = ref.router_backward(logits, ids, w, dw, r.score, r.normalize, r.scale)
    bound = ref.router_grad_bound(want, size, logits, logits.dtype, r.experts)
    assert ((got.cpu().double() - want).abs() <= bound).all()


@pytest.mark.parametrize("score,normalize", [("softmax", True), ("softmax", False),
                                             ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("T,E,k", [(1, 256, 8), (5, 1, 1), (7, 2, 2), (33, 8, 3), (130, 60, 6),
                                   (64, 64, 8), (19, 65, 32), (40, 127, 8), (50, 256, 32),
                                   (9, 257, 5), (6, 512, 16), (5, 1000, 8), (3, 1024, 9),
                                   (4, 1025, 8), (3, 4097, 7), (8, 32, 32)])
def test_router_forward_and_backward(T, E, k, dtype, score, normalize):
    logits = (2.0 * torch.randn(T, E, generator=gen(T * 1000 + E), device="cuda")).to(dtype)
    r, ids, w = check_router(logits, k, score, normalize, 2.5)
    check_router_grad(r, logits, ids, w, 3)


@pytest.mark.parametrize("score,normalize,biased", [("softmax", True, False), ("softmax", False, False),
                                                    ("sigmoid", True, True)])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,E,k", [(5001, 100, 8), (5003, 160, 7), (5002, 256, 8), (9601, 256, 8),
                                   (9603, 200, 32), (9700, 257, 8), (5001, 512, 8), (5001, 64, 6),
                                   (5001, 30, 4)])
def test_router_many_tokens_with_special_rows_among_them(T, E, k, dtype, score, normalize, biased):
    """The forms for more tokens than warps; rows with many ties, masked experts and nothing left
    share a warp with ordinary ones."""
    g = gen(T + E)
    logits = (2.0 * torch.randn(T, E, generator=g, device="cuda")).to(dtype)
    logits[::7] = 0.25                                   # all equal
    logits[3::11, ::2] = -INF
    logits[5::13] = -INF                                 # nothing left
    logits[8::17] = torch.randint(0, 3, (E,), generator=g, device="cuda").to(dtype)
    mask = torch.rand(T, generator=g, device="cuda") < 0.9
    bias = 0.2 * torch.randn(E, generator=g, device="cuda") if biased else None
    r = Router(E, k, score=score, normalize=normalize, scale=1.5)
    for rows in (logits, torch.cat([logits, logits[:, :3]], 1)[:, :E]):   # the second one not vectors
        ids, w = r.forward(rows, bias=bias, mask=mask)
        want_ids, want_w = ref.router_forward_many(logits, k, score, normalize, 1.5, bias, mask)
        assert torch.equal(ids.cpu(), want_ids)
        bound = ref.router_weight_bound(logits, want_w, E)
        assert ((w.cpu().double() - want_w).abs() <= bound).all()


@pytest.mark.parametrize("T,E,k,dtype", [(300, 256, 8, F32), (65, 64, 6, BF16), (20, 2000, 8, F32),
                                         (77, 40, 40 - 8, F16)])
def test_router_bias_moves_the_choice_and_not_the_weights(T, E, k, dtype):
    g = gen(5)
    logits = torch.randn(T, E, generator=g, device="cuda").to(dtype)
    bias = 0.3 * torch.randn(E, generator=g, device="cuda")
    bias[E // 2] = -INF
    _, ids, w = check_router(logits, k, "sigmoid", True, 1.0, bias=bias)
    assert not (ids == E // 2).any()
    _, plain, _ = check_router(logits, k, "sigmoid", True, 1.0)
    assert not torch.equal(plain, ids)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("E,k", [(64, 8), (256, 8), (31, 4), (1500, 8)])
def test_router_ties_go_to_the_lowest_id(E, k, dtype):
    logits = torch.zeros(6, E, device="cuda", dtype=dtype)
    logits[1] = -0.0
    logits[1, ::2] = 0.0                                             # +0 and -0 tie
    logits[2] = torch.randint(0, 3, (E,), generator=gen(1), device="cuda").to(dtype)
    logits[3] = torch.randint(0, 2, (E,), generator=gen(2), device="cuda").to(dtype)
    logits[4] = torch.finfo(dtype).min                               # an ordinary, lowest logit
    logits[5] = torch.finfo(dtype).max
    r, ids, w = check_router(logits, k, "softmax", True, 1.0)
    assert ids[0].tolist() == list(range(k)) == ids[4].tolist()
    check_router(logits, k, "softmax", False, 1.0)
    check_router_grad(r, logits[:4].contiguous(), ids[:4].contiguous(), w[:4].contiguous(), 4)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("score,normalize", [("softmax", True), ("softmax", False),
                                             ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("E,k", [(48, 6), (256, 8), (1100, 4)])
def test_router_masked_experts_and_rows_with_nothing_left(E, k, score, normalize, dtype):
    g = gen(9)
    logits = torch.randn(9, E, generator=g, device="cuda").to(dtype)
    logits[0] = -INF                                  # nothing left
    logits[1, 2:] = -INF                              # fewer than k left
    logits[2, torch.randperm(E, generator=g, device="cuda")[:E - k]] = -INF   # exactly k left
    logits[3] = torch.finfo(dtype).min
    logits[3, 5] = -INF
    logits[4, :] = -INF
    logits[4, E - 1] = torch.finfo(dtype).min         # one left, the lowest value
    mask = torch.ones(9, dtype=torch.bool, device="cuda")
    mask[6] = False
    r, ids, w = check_router(logits, k, score, normalize, 1.5, mask=mask)
    assert (ids[0] == -1).all() and (w[0] == 0).all() and (ids[6] == -1).all() and (w[6] == 0).all()
    assert ids[1].tolist() in ([0, 1] + [-1] * (k - 2), [1, 0] + [-1] * (k - 2))
    assert torch.isfinite(w).all()
    check_router_grad(r, logits, ids, w, 6)
    assert (r.backward(logits, ids, w, torch.ones_like(w))[0] == 0).all()


def test_router_nan_is_never_chosen_and_shows_in_the_weights():
    logits = torch.randn(4, 40, generator=gen(2), device="cuda")
    logits[0, 7] = NAN
    logits[1] = NAN
    logits[2, 3] = INF
    for normalize in (True, False):
        _, ids, w = check_router(logits, 4, "softmax", normalize, 1.0, finite=False)
        assert not (ids[0] == 7).any() and (ids[1] == -1).all() and ids[2, 0] == 3
        assert torch.isnan(w[0]).all() == (not normalize)
        assert (w[1] == 0).all() and torch.isfinite(w[3]).all()
    _, ids, w = check_router(logits, 4, "sigmoid", False, 1.0, finite=False)
    assert torch.isfinite(w).all() and w[2, 0] == 1.0


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_router_strides_offsets_and_leading_dimensions(dtype):
    big = torch.randn(2, 3, 10, 300, generator=gen(4), device="cuda").to(dtype)
    cut = big[..., 1:257]                                  # rows 300 apart, odd start
    r = Router(256, 8)
    ids, w = r.forward(cut)
    assert ids.shape == (2, 3, 10, 8)
    want_ids, want_w = r.forward(cut.contiguous())
    assert torch.equal(ids, want_ids) and torch.equal(w, want_w)
    check_router(cut.reshape(-1, 256), 8, "softmax", True, 1.0)
    dw = torch.randn_like(w).transpose(0, 1).contiguous().transpose(0, 1)   # not contiguous
    for kind in ("softmax", "sigmoid"):
        r = Router(256, 8, score=kind, normalize=False)
        ids, w = r.forward(cut)
        a = r.backward(cut, ids, w, dw)
        b = r.backward(cut.contiguous(), ids, w, dw.contiguous())
        assert torch.equal(a, b) and a.is_contiguous()
    flat = torch.randn(7 * 33 + 1, generator=gen(4), device="cuda").to(dtype)
    check_router(flat[1:].view(7, 33), 5, "softmax", True, 1.0)


def test_router_offsets_beyond_32_bits():
    """The last rows of a view whose rows lie far apart start beyond 2^31 elements."""
    stride = 1 << 28
    store = torch.empty(9 * stride, dtype=BF16, device="cuda")
    view = torch.as_strided(store, (9, 64), (stride, 1))
    view.copy_(torch.randn(9, 64, generator=gen(8), device="cuda").to(BF16))
    r, ids, w = check_router(view, 6, "softmax", False, 1.0)
    check_router_grad(r, view, ids, w, 7)


def test_router_gradient_against_differences():
    g = gen(11)
    for score, normalize in (("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)):
        logits = torch.randn(6, 24, generator=g, device="cuda", requires_grad=True)
        r = Router(24, 4, score=score, normalize=normalize, scale=1.5)
        ids, w = r(logits)
        dw = torch.randn(w.shape, generator=g, device="cuda")
        (w * dw).sum().backward()
        assert not ids.requires_grad
        base = logits.detach().double().cpu()

        def loss(z):
            total = 0.0
            for t in range(6):
                ch = ids[t].long().cpu()
                v = z[t][ch]
                if score == "sigmoid":
                    v = torch.special.expit(v)
                    v = v / (v.sum() + 1e-20) if normalize else v
                else:
                    v = torch.exp(v - torch.logsumexp(v if normalize else z[t], 0))
                total += float((1.5 * v * dw[t].double().cpu()).sum())
            return total

        eps = 1e-5
        for t, i in [(0, int(ids[0, 0])), (1, int(ids[1, 3])), (2, 0), (5, 23)]:
            up, down = base.clone(), base.clone()
            up[t, i] += eps
            down[t, i] -= eps
            slope = (loss(up) - loss(down)) / (2 * eps)
            # central difference: eps^2 times a third derivative below 20; results in 32 bits
            assert abs(float(logits.grad[t, i]) - slope) <= 20 * eps ** 2 + 1e-9 / eps * 1e-2 + 4e-6


def test_router_ids_feed_a_plan():
    from gpu_common import make_planner
    import workloads as wl
    w = wl.CONFIGS["tiny"]
    logits = torch.randn(1, w.ranks, w.tokens_per_rank, w.experts, generator=gen(3), device="cuda")
    ids, _ = Router(w.experts, w.top_k).forward(logits)
    pl = make_planner(w)
    out = pl.plan(ids)
    assert pl.status() == 0
    assert int(out.dispatch_counts.sum()) == ids.numel()


def test_router_other_stream_and_graph():
    logits = torch.randn(500, 128, generator=gen(3), device="cuda")
    r = Router(128, 8)
    want = r.forward(logits)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    got = r.forward(logits, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = r.forward(logits)
        grad = r.backward(logits, got[0], got[1], want[1])
    for t in got + (grad,):
        t.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert torch.equal(grad, r.backward(logits, want[0], want[1], want[1]))


def test_router_refusals():
    r = Router(16, 2)
    x = torch.randn(4, 16, device="cuda")
    ids, w = r.forward(x)
    for bad in (lambda: r.forward(x.double()), lambda: r.forward(x[:, :15]), lambda: r.forward(x.cpu()),
                lambda: r.forward(x.t().contiguous().t()), lambda: r.forward(x[0].expand(4, 16)),
                lambda: r.forward(x, mask=torch.ones(3, dtype=torch.bool, device="cuda")),
                lambda: r.forward(x, mask=torch.ones(4, device="cuda")),
                lambda: Router(16, 2, score="sigmoid").forward(x, bias=torch.zeros(15, device="cuda")),
                lambda: r.backward(x, ids.long(), w, w), lambda: r.backward(x, ids, w[:, :1], w),
                lambda: r.backward(x, ids, w, w.double())):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(B.TopoEPError):   # a bias belongs to sigmoid scores
        r.forward(x, bias=torch.zeros(16, device="cuda"))
    assert r.forward(x[:0])[0].shape == (0, 2)
    assert r.backward(x[:0], ids[:0], w[:0], w[:0]).shape == (0, 16)


# ------------------------------------------------------------------------------------ experts

def make_blocks(R, L, N, H, F, seed):
    g = gen(seed)
    out = []
    for n in (L, N):
        b = torch.randn(R, n, 3 * H * F, generator=g, device="cuda")
        b[..., :2 * H * F] *= H ** -0.5
        b[..., 2 * H * F:] *= F ** -0.5
        out.append(b.to(BF16).view(torch.uint8) if n else None)
    return out


def make_ids(T, k, n, g, drop=0.0):
    keys = torch.rand(T, n, generator=g, device="cuda")
    ids = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    m = min(k, n)
    ids[:, :m] = keys.topk(m, dim=1).indices.int()
    ids[torch.rand(T, k, generator=g, device="cuda") < drop] = -1
    return ids


def check_experts(T, k, R, L, N, H, F, seed=0, drop=0.0, ids=None):
    g = gen(seed)
    main, replica = make_blocks(R, L, N, H, F, seed + 1)
    x = torch.randn(T, H, generator=g, device="cuda").to(BF16)
    n = R * (L + N)
    if ids is None:
        ids = make_ids(T, k, n, g, drop)
    w = torch.rand(T, k, generator=g, device="cuda")
    layer = TokenExperts(H, F, k, max(T, 1), L, slots_per_rank=N, ranks=R)
    layer.set_experts(main, replica)
    y = layer.forward(x, ids, w)
    want, bound = ref.experts_forward(x, ids, w, main, replica, L, N, n, H, F)
    assert y.dtype == BF16 and tuple(y.shape) == (T, H)
    worst = ((y.cpu().double() - want).abs() / bound).max() if T else 0.0
    assert worst <= 1.0, float(worst)
    assert torch.equal(y, layer.forward(x, ids, w))        # the same call, the same bits
    assert layer.status() == 0
    return layer, x, ids, w, y


@pytest.mark.parametrize("H,F", [(64, 64), (128, 256), (256, 128), (520, 328), (8, 8), (72, 1000),
                                 (1000, 72), (384, 640), (1, 1), (33, 17), (130, 258), (260, 100)])
@pytest.mark.parametrize("T,k,R,L,N", [(1, 1, 1, 1, 0), (1, 8, 1, 9, 0), (3, 2, 2, 3, 1),
                                       (17, 4, 1, 8, 2)])
def test_experts_sizes(T, k, R, L, N, H, F):
    check_experts(T, k, R, L, N, H, F, seed=T + H)


@pytest.mark.parametrize("T", [1, 2, 15, 16, 17, 31, 33, 64, 65, 100, 127, 128])
def test_experts_token_counts(T):
    check_experts(T, 3, 1, 5, 1, 192, 136, seed=T, drop=0.3)


def test_experts_wide_choice_and_many_instances():
    check_experts(40, 16, 4, 30, 2, 128, 64, seed=1)
    check_experts(128, 16, 1, 20, 0, 64, 128, seed=2)
    check_experts(5, 2, 64, 127, 1, 8, 8, seed=3)          # 8192 instances


def test_experts_all_rows_on_one_instance_and_every_count():
    ids = torch.full((128, 2), -1, dtype=torch.int32, device="cuda")
    ids[:, 1] = 3
    check_experts(128, 2, 1, 4, 0, 256, 192, ids=ids)
    ids = torch.full((128, 4), -1, dtype=torch.int32, device="cuda")
    for t in range(128):                                   # 128, 85, 43 and 1 rows
        ids[t] = torch.tensor([0, 1 if t % 3 else -1, 2 if t % 3 == 0 else -1, 3 if t == 77 else -1])
    check_experts(128, 4, 1, 5, 0, 136, 200, ids=ids, seed=4)


@pytest.mark.parametrize("slots,H,F,T", [(18, 256, 1024, 24), (37, 128, 512, 40), (38, 192, 512, 20),
                                         (60, 128, 640, 33), (75, 72, 520, 128), (148, 64, 256, 40),
                                         (7, 520, 128, 9)])
def test_experts_every_way_of_dealing_out_tiles(slots, H, F, T):
    """On 148 SMs: all tiles whole, exactly one a block, one and a few cut, several rounds and a rest
    cut or whole, a second product with more tiles than the first."""
    g = gen(slots)
    k = -(-slots // T) + 2
    ids = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    ids.view(-1)[torch.randperm(T * k, generator=g, device="cuda")[:slots]] = \
        torch.arange(slots, dtype=torch.int32, device="cuda")            # every instance once
    extra = torch.randint(0, slots, (T,), generator=g, device="cuda", dtype=torch.int32)
    ids[:, -1] = torch.where(ids[:, -1] < 0, extra, ids[:, -1])          # and some again
    check_experts(T, k, 1, slots, 0, H, F, seed=slots, ids=ids)


def test_experts_longer_layers():
    check_experts(2, 2, 1, 3, 1, 4096, 1408, seed=5)
    check_experts(20, 2, 1, 3, 0, 1024, 2048, seed=6)


def test_experts_no_valid_id_and_empty_calls():
    ids = torch.full((6, 3), -1, dtype=torch.int32, device="cuda")
    layer, x, _, w, y = check_experts(6, 3, 1, 4, 0, 64, 64, ids=ids)
    assert (y == 0).all()
    assert layer.forward(x[:0], ids[:0], w[:0]).shape == (0, 64)
    ids[2, 1] = 2                                          # one row of six
    check_experts(6, 3, 1, 4, 0, 64, 64, ids=ids)
    for bad in (4, 1 << 30, -2, -2 ** 31):
        ids[4, 0] = bad
        again = layer.forward(x, ids, w)
        assert layer.status() == B.FLAG_BAD_ID and layer.status() == 0
        assert (again[4] == 0).all()


def test_experts_same_instance_twice_in_a_row():
    ids = torch.tensor([[1, 1, 2], [2, 0, 2], [1, -1, 1]], dtype=torch.int32, device="cuda")
    check_experts(3, 3, 1, 3, 0, 128, 128, ids=ids)


@pytest.mark.parametrize("H,F", [(256, 128), (100, 52)])
def test_experts_bad_values_stay_in_their_rows(H, F):
    """NaN and infinity in another row, in an unnamed block and under an ignored id's weight do not
    reach a row; a block named by one row alone reaches that row alone."""
    main, replica = make_blocks(1, 4, 1, H, F, 3)
    m = main.view(BF16)
    layer = TokenExperts(H, F, 3, 20, 4, slots_per_rank=1)
    layer.set_experts(main, replica)
    g = gen(2)
    x = torch.randn(20, H, generator=g, device="cuda").to(BF16)
    ids = torch.randint(0, 3, (20, 3), generator=g, device="cuda", dtype=torch.int32)
    ids[:, 2] = -1
    w = torch.rand(20, 3, generator=g, device="cuda")
    want = layer.forward(x, ids, w).clone()
    w[:, 2] = NAN                                          # ignored ids' weights
    x[5] = NAN
    x[6, 1] = INF
    replica.view(BF16).fill_(NAN)                          # an unnamed block
    m[0, 3].fill_(INF)                                     # a block that row 9 alone will name
    ids[9, 1] = 3
    got = layer.forward(x, ids, w)
    rows = [t for t in range(20) if t not in (5, 6, 9)]
    assert torch.equal(got[rows], want[rows])
    assert torch.isnan(got[5]).all() and not torch.isfinite(got[9]).any()


@pytest.mark.parametrize("H,F,pad,start", [(128, 64, 8, 0), (128, 64, 8, 8), (128, 64, 3, 1),
                                           (129, 64, 0, 0), (128, 64, 0, 4)])
def test_experts_strided_rows(H, F, pad, start):
    main, replica = make_blocks(1, 4, 0, H, F, 3)
    layer = TokenExperts(H, F, 2, 10, 4)
    layer.set_experts(main)
    g = gen(2)
    store = torch.randn(start + 10 * (H + pad), generator=g, device="cuda").to(BF16)
    x = torch.as_strided(store, (10, H), (H + pad, 1), start)
    ids = make_ids(10, 2, 4, g)
    w = torch.rand(10, 2, generator=g, device="cuda")
    room = torch.full((10, H + 5), 7.0, dtype=BF16, device="cuda")
    want = layer.forward(x.contiguous().clone(), ids, w)
    got = layer.forward(x, ids, w, out=room[:, 3:3 + H])
    ulp = 2.0 ** -7
    # another kernel may serve another alignment: equal but for the rounding of sums
    assert ((got.float() - want.float()).abs() <= ulp * want.float().abs() + 0.02).all()
    assert (room[:, :3] == 7).all() and (room[:, 3 + H:] == 7).all()
    one = x[:1].expand(10, H)                               # one row for every token
    assert torch.equal(layer.forward(one, ids, w), layer.forward(one.contiguous(), ids, w))


def test_experts_on_a_plan_with_replicas():
    """The instances a plan names, on the buffers the replica executor filled."""
    import workloads as wl
    from gpu_common import make_planner
    H, F = 128, 64
    w = wl.CONFIGS["tiny"].replace(tokens_per_rank=64, slots_per_rank=2, hidden=8, ffn=8)
    pl = make_planner(w)
    out = pl.plan(torch.from_numpy(wl.make_topk_ids(w, seed=5)).cuda())
    main = make_blocks(w.ranks, pl.e_loc, 0, H, F, 1)[0]
    slots = torch.zeros(w.ranks, 2, 6 * H * F, dtype=torch.uint8, device="cuda")
    pl.replica_pull(out.replica_map[0], main, slots)
    layer = TokenExperts(H, F, w.top_k, 128, pl.e_loc, slots_per_rank=2, ranks=w.ranks)
    layer.set_experts(main, slots)
    g = gen(1)
    rows = out.token_replica[0].reshape(-1, w.top_k)[:128].contiguous()
    assert ((rows % pl.s_phys) >= pl.e_loc).any()          # some run on replicas
    x = torch.randn(128, H, generator=g, device="cuda").to(BF16)
    wt = torch.rand(128, w.top_k, generator=g, device="cuda")
    y = layer.forward(x, rows, wt)
    want, bound = ref.experts_forward(x, rows, wt, main, slots, pl.e_loc, 2, pl.P, H, F)
    assert ((y.cpu().double() - want).abs() <= bound).all()


def test_experts_other_stream_graph_and_moved_blocks():
    layer, x, ids, w, y = check_experts(12, 3, 1, 6, 0, 256, 128, seed=9)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    other = layer.forward(x, ids, w, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(other, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer.forward(x, ids, w)
    for _ in range(3):
        got.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(got, y)
    main = layer._params[0].clone()
    layer.set_experts(main)
    assert torch.equal(layer.forward(x, ids, w), y)
    ids2 = ids.flip(0).contiguous()                        # other ids, then back: nothing is kept
    layer.forward(x, ids2, w)
    assert torch.equal(layer.forward(x, ids, w), y)
    small = layer.forward(x[:3], ids[:3], w[:3])
    assert ((small.float() - y[:3].float()).abs() <= 0.02 * (1 + y[:3].float().abs())).all()


def test_experts_and_clip_on_two_streams_at_once():
    """Calls on handles of their own overlap freely: each waits for its own blocks alone."""
    g = gen(3)
    sets, streams = [], [torch.cuda.Stream() for _ in range(3)]
    for seed in (1, 2):
        layer, x, ids, w, y = check_experts(9 * seed, 3, 1, 6, 0, 512, 256, seed=seed)
        sets.append((layer, x, ids, w, y))
    t = torch.randn(3_000_000, generator=g, device="cuda")
    out = torch.empty_like(t)
    clip = GradientClip([t], out=[out])
    norm, want = clip.clip(1.0), out.clone()
    wrong = [torch.zeros((), dtype=torch.int64, device="cuda") for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(60):
        for i, (layer, x, ids, w, y) in enumerate(sets):
            with torch.cuda.stream(streams[i]):
                wrong[i] += (layer.forward(x, ids, w) != y).any()
        with torch.cuda.stream(streams[2]):
            wrong[2] += clip.clip(1.0) != norm
    torch.cuda.synchronize()
    assert [int(v) for v in wrong] == [0, 0, 0] and torch.equal(out, want)
    assert all(s[0].status() == 0 for s in sets)


def test_experts_refusals():
    layer, x, ids, w, _ = check_experts(4, 2, 1, 3, 0, 64, 64)
    for bad in (lambda: layer.forward(x.float(), ids, w), lambda: layer.forward(x[:, :32], ids, w),
                lambda: layer.forward(x, ids.long(), w), lambda: layer.forward(x, ids[:3], w),
                lambda: layer.forward(x, ids, w.double()), lambda: layer.forward(x.cpu(), ids, w),
                lambda: layer.forward(torch.cat([x, x]), torch.cat([ids, ids]), torch.cat([w, w])),
                lambda: layer.forward(x, ids, w, out=torch.empty(4, 64, device="cuda")),
                lambda: layer.forward(x.t().contiguous().t(), ids, w),
                lambda: layer.set_experts(torch.zeros(5, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    empty = TokenExperts(64, 64, 2, 4, 3)
    with pytest.raises(B.TopoEPError):                     # no blocks yet
        empty.forward(x, ids, w)


# --------------------------------------------------------------------------------------- clip

def check_clip(tensors, max_norm, norm="l2", out=None):
    kept = [t.clone() for t in tensors]
    want, factor = ref.clip([t for t in kept], max_norm, norm)
    c = GradientClip(tensors, out=out, norm=norm)
    got = c.norm()
    assert got.dtype == F32 and got.dim() == 0
    # squares and short sums in 32 bits, the rest in 64: a few units
    assert abs(float(got) - want) <= 8 * ref.U32 * want + 1e-45
    assert all(torch.equal(a, b) for a, b in zip(tensors, kept))
    again = c.clip(max_norm)
    assert torch.equal(again, got)
    for t, k in zip(tensors if out is None else out, kept):
        exact = k.double() * factor
        bound = exact.abs() * (1.01 * ref.UNIT[t.dtype] + 16 * ref.U32) + ref.TINY[t.dtype]
        assert ((t.double() - exact).abs() <= bound).all()
    if out is not None:
        assert all(torch.equal(a, b) for a, b in zip(tensors, kept))
    return c


@pytest.mark.parametrize("norm", ["l2", "max"])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("sizes", [[1], [7], [1023], [16384], [16385], [100000, 1, 3], [0, 5, 0],
                                   [33, 4097, 250001, 2, 64]])
def test_clip_sizes(sizes, dtype, norm):
    g = gen(len(sizes))
    for max_norm in (0.5, 1e9, 0.0):
        tensors = [torch.randn(n, generator=g, device="cuda").to(dtype) for n in sizes]
        check_clip(tensors, max_norm, norm)
        tensors = [torch.randn(n, generator=g, device="cuda").to(dtype) for n in sizes]
        check_clip(tensors, max_norm, norm, out=[torch.empty_like(t) for t in tensors])


def test_clip_packed_tensors_of_every_alignment_and_type():
    g = gen(3)
    sizes = [1, 2, 3, 5, 8, 13, 100, 1001, 20011, 7, 70001, 1, 9]
    tensors, outs, rooms = [], [], []
    for i, dtype in enumerate((F32, BF16, F16)):
        src = torch.randn(sum(sizes) + 1, generator=g, device="cuda").to(dtype)
        dst = torch.full_like(src, 3.0)
        at = 1
        for n in sizes:
            tensors.append(src[at:at + n])
            outs.append(dst[at:at + n])
            at += n
        rooms.append(dst)
    check_clip(tensors, 2.0, out=outs)
    assert all(float(r[0]) == 3.0 for r in rooms)
    # source and output of different alignment
    src = torch.randn(5001, generator=g, device="cuda").to(BF16)
    dst = torch.zeros(5008, dtype=BF16, device="cuda")
    check_clip([src[1:]], 1.0, out=[dst[4:5004]])
    assert (dst[:4] == 0).all() and (dst[5004:] == 0).all()


def test_clip_strided_and_permuted_tensors():
    g = gen(4)
    a = torch.randn(64, 100, generator=g, device="cuda")
    b = torch.randn(40, 6, 32, generator=g, device="cuda").to(BF16)
    c = torch.randn(31, 17, generator=g, device="cuda").to(F16)
    around = [a.clone(), b.clone(), c.clone()]
    tensors = [a[:, 3:77], a[:, 90].unsqueeze(1), b[:20, 2], b[20:].permute(2, 0, 1), c.t()]
    check_clip(tensors, 1.0)
    assert torch.equal(a[:, :3], around[0][:, :3]) and torch.equal(a[:, 91:], around[0][:, 91:])
    assert torch.equal(b[:20, 3:], around[1][:20, 3:])
    src = torch.randn(12, 50, generator=g, device="cuda")
    room = torch.zeros(12, 64, device="cuda")
    check_clip([src], 1.0, out=[room[:, 5:55]])            # a run into rows
    check_clip([room[:, 5:55]], 0.5, out=[torch.empty(12, 50, device="cuda")])
    check_clip([src[:, ::2]], 1.0)                         # every other element: rows of one
    for bad in (src[:, :30:2], src[0].expand(3, 50), torch.randn(4, 5, 6, device="cuda")[:, 1:3, :2]):
        with pytest.raises(ValueError):
            GradientClip([bad])


@pytest.mark.parametrize("rows,cols,stride", [(5000, 3, 7), (300, 1023, 1030), (2049, 1, 2), (100, 511, 600),
                                              (40, 4097, 5000), (3, 2048, 2049)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_clip_rows_short_and_long(rows, cols, stride, dtype):
    room = torch.randn(rows * stride, generator=gen(rows), device="cuda").to(dtype)
    kept = room.clone()
    view = torch.as_strided(room, (rows, cols), (stride, 1))
    check_clip([view], 0.7)
    gaps = torch.ones(rows * stride, dtype=torch.bool, device="cuda")
    torch.as_strided(gaps, (rows, cols), (stride, 1)).fill_(False)
    assert torch.equal(room[gaps], kept[gaps])
    out = torch.empty(rows, cols, dtype=dtype, device="cuda")
    check_clip([torch.as_strided(kept, (rows, cols), (stride, 1))], 0.7, out=[out])


def test_clip_shared_gradient_is_refused():
    t = torch.randn(100, device="cuda")
    for bad in ([t, t], [t, t[50:]], [t.view(10, 10), t]):
        with pytest.raises(B.TopoEPError):
            GradientClip(bad)


def test_router_is_differentiable_once():
    x = torch.randn(3, 8, device="cuda", requires_grad=True)
    _, w = Router(8, 2)(x)
    (g,) = torch.autograd.grad(w.square().sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def test_clip_very_large_and_very_small_gradients():
    for scale in (1e30, 1e-30, 1e-42):
        t = [scale * torch.randn(100003, generator=gen(5), device="cuda"),
             scale * torch.randn(77, generator=gen(6), device="cuda").to(BF16)]
        check_clip(t, 1e-3)
    mixed = torch.randn(50000, generator=gen(7), device="cuda")
    mixed[::3] *= 1e25
    mixed[1::3] *= 1e-25
    check_clip([mixed], 1.0)


@pytest.mark.parametrize("norm", ["l2", "max"])
def test_clip_infinity_and_nan(norm):
    a, b = torch.randn(70000, generator=gen(1), device="cuda"), torch.randn(50, device="cuda").to(BF16)
    a[69999] = -INF
    c = GradientClip([a, b], norm=norm)
    assert float(c.clip(1.0)) == INF
    assert (a[:69999] == 0).all() and torch.isnan(a[69999]) and (b == 0).all()
    a.normal_(generator=gen(2))
    b.normal_(generator=gen(3))
    a[5] = NAN
    a[6] = INF
    assert math.isnan(float(c.norm()))
    assert math.isnan(float(c.clip(1.0)))
    assert torch.isnan(a).all() and torch.isnan(b).all()


def test_clip_many_tensors_and_a_large_one():
    g = gen(8)
    sizes = np.random.default_rng(1).integers(1, 3000, 2500)
    store = torch.randn(int(sizes.sum()), generator=g, device="cuda")
    tensors = list(torch.split(store, [int(n) for n in sizes]))
    check_clip(tensors, 3.0)
    big = torch.randn(300_000_001, generator=g, device="cuda").to(BF16)
    check_clip([big[1:]], 3.0)


def test_clip_offsets_beyond_32_bits():
    big = torch.zeros(2 ** 31 + 4099, dtype=BF16, device="cuda")
    big[-3:] = torch.tensor([3.0, 4.0, 12.0], dtype=BF16)
    c = GradientClip([big])
    assert float(c.clip(1.0)) == 13.0
    assert big[-1] == torch.tensor(12.0 / 13.0).to(BF16) and int((big != 0).sum()) == 3


def test_clip_repeats_follow_values_graph_and_stream():
    t = torch.randn(300000, generator=gen(8), device="cuda")
    out = torch.empty_like(t)
    c = GradientClip([t], out=[out])
    first = c.clip(1.0).clone()
    want = out.clone()
    for _ in range(4):
        out.zero_()
        assert torch.equal(c.clip(1.0), first) and torch.equal(out, want)
    t.mul_(2.0)
    assert torch.equal(c.norm(), 2 * first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        n = c.clip(1.0)
    t.div_(2.0)
    out.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(n, first) and torch.equal(out, want)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    n = c.clip(1.0, stream=st)
    torch.cuda.synchronize()
    assert torch.equal(n, first)


def test_clip_refusals():
    t = torch.randn(8, device="cuda")
    for bad in (lambda: GradientClip([]), lambda: GradientClip([t.double()]), lambda: GradientClip([t.cpu()]),
                lambda: GradientClip([t], out=[t, t]), lambda: GradientClip([t], out=[t[:4]]),
                lambda: GradientClip([t], out=[t.to(BF16)]), lambda: GradientClip([t], norm="l1"),
                lambda: GradientClip([t.view(2, 4)], out=[torch.empty(4, 2, device="cuda").t()])):
        with pytest.raises(ValueError):
            bad()
    c = GradientClip([t])
    for bad in (-1.0, NAN):
        with pytest.raises(B.TopoEPError):
            c.clip(bad)
