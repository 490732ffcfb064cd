"""Operators for sampled and drafted tokens against their plain 64-bit forms (tests/ref_drafts.py).

Tolerances.  u = eps / 2 of the output's type is the most a rounding is off, relative to the value (bf16 2^-8, fp32 2^-24).
Rotary positions: an output a cos - b sin is off by the roundings of two products and a sum, 3 * 2^-24 (|a| + |b|), and by the
cosine and sine, whose argument is a fraction of a turn below one half rounded to fp32 (2^-26 of a turn = 2^-23.3 of a radian)
and whose values sincospif rounds (2^-23): 2^-22 (|a| + |b|) in all covers both, 2^-21 with the products; plus u |y|.
Attention: a score is a sum of D products in fp32, off by at most (D + 2) 2^-24 sum |q k|, and its product with log2(e) and
the difference to the maximum by 2^-22 of its size; e^x takes the error over as a relative one, in the numerator and the
denominator, so twice; exp2 itself adds 2^-21, sums of T terms T 2^-24 each; with bf16 the probabilities are rounded, 2^-8.  All of
it relative to sum p |v|; plus u |o|.
"""
import math

import numpy as np
import pytest
import torch

import ref_drafts as ref
from gpu_util import library
from paper_2608_12385_b200 import binding

pytestmark = pytest.mark.gpu

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
U = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    library()


def gen(seed):
    return torch.Generator().manual_seed(seed)


def i32(x):
    return torch.as_tensor(x, dtype=torch.int32).cuda()


def assert_within(got, want, bound, what=""):
    err = (got.double().cpu() - want).abs()
    assert torch.isfinite(got.float()).all(), what
    worst = (err - bound).max().item()
    assert worst <= 0, f"{what}: {err.max().item():.3e} off, {worst:.3e} beyond the bound"


# ---- rotary positions ----------------------------------------------------------------------------------------------


def rope_bound(x, freq, scale, interleaved, y, u):
    pairs = freq.numel()
    a, b = (x[..., 0:2 * pairs:2], x[..., 1:2 * pairs:2]) if interleaved else (x[..., :pairs], x[..., pairs:2 * pairs])
    s = scale * (a.abs() + b.abs()) * 2.0 ** -21
    each = torch.stack((s, s), -1).flatten(-2) if interleaved else torch.cat((s, s), -1)
    return torch.nn.functional.pad(each, (0, x.shape[-1] - 2 * pairs)) + u * y.abs()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rows,heads,dim,rot", [(1, 1, 64, 64), (7, 3, 128, 128), (65, 16, 128, 64), (33, 5, 80, 32), (3, 2, 10, 6), (5, 4, 96, 94),
                                                (300, 32, 128, 128), (2, 24, 256, 2)])
@pytest.mark.parametrize("inverse", [False, True])
def test_rope(dtype, interleaved, rows, heads, dim, rot, inverse):
    g = gen(rows * 1000 + dim)
    x = torch.randn(rows, heads, dim, generator=g).to(TYPES[dtype])
    pos = torch.randint(-5, 600000, (rows,), generator=g, dtype=torch.int32)
    pos[0] = 2 ** 31 - 1
    freq, scale = binding.rope_frequencies(rot, 10000.0)
    scale = 1.25
    want = ref.rotate(x.double(), pos, freq, scale, interleaved, inverse)
    got = binding.op_rope(x.cuda(), pos.cuda(), freq.cuda(), scale=scale, interleaved=interleaved, inverse=inverse)
    assert_within(got, want, rope_bound(x.double(), freq, scale, interleaved, want, U[dtype]))
    assert torch.equal(got[..., rot:].cpu(), x[..., rot:])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("shift", [0, 1])
def test_rope_with_strides_in_place_and_unaligned(dtype, interleaved, shift):
    """Heads of a fused projection in place; shift 1 moves every address off the 16 bytes that vectors need."""
    g = gen(5)
    R, H, D, rot = 37, 6, 64, 32
    store = torch.randn(R * (H * D + 40) + 8, generator=g).to(TYPES[dtype])
    pos = torch.randint(0, 5000, (R,), generator=g, dtype=torch.int32)
    freq, _ = binding.rope_frequencies(rot, 500000.0)
    view = lambda t: t[shift:shift + R * (H * D + 40)].view(R, -1)[:, 8:8 + H * D].unflatten(1, (H, D))  # noqa: E731
    want = store.double().clone()
    turned = ref.rotate(view(store).double(), pos, freq, 1.0, interleaved, False)
    bound = torch.zeros_like(want)
    view(bound).copy_(rope_bound(view(store).double(), freq, 1.0, interleaved, turned, U[dtype]))
    view(want).copy_(turned)
    dev = store.cuda()
    binding.op_rope(view(dev), pos.cuda(), freq.cuda(), interleaved=interleaved, out=view(dev))
    assert_within(dev, want, bound)  # the elements between the heads keep their bits (bound 0)
    out = torch.zeros(H, R, D, dtype=TYPES[dtype], device="cuda")  # another order of rows and heads
    binding.op_rope(view(store.cuda()), pos.cuda(), freq.cuda(), interleaved=interleaved, out=out.transpose(0, 1))
    assert torch.equal(out.transpose(0, 1), view(dev))


@pytest.mark.parametrize("interleaved", [False, True])
def test_rope_inverse_is_the_gradient(interleaved):
    """Against the formula (64-bit autograd through the plain form) and against differences: the map is linear in x, so the difference
    of two outputs is the derivative along the step, and its product with dy that of the gradient with the step."""
    g = gen(9)
    R, H, D, rot = 12, 4, 64, 48
    x, dy, h = (torch.randn(R, H, D, generator=g) for _ in range(3))
    pos = torch.randint(0, 90000, (R,), generator=g, dtype=torch.int32)
    freq, scale = binding.rope_frequencies(rot, 10000.0, "ramp", factor=8.0, trained_len=4096)
    xd = x.double().requires_grad_()
    angle = pos.double()[:, None, None] * freq
    a, b = (xd[..., 0:rot:2], xd[..., 1:rot:2]) if interleaved else (xd[..., :rot // 2], xd[..., rot // 2:rot])
    p, q = scale * (a * angle.cos() - b * angle.sin()), scale * (a * angle.sin() + b * angle.cos())
    y = torch.cat((torch.stack((p, q), -1).flatten(-2) if interleaved else torch.cat((p, q), -1), xd[..., rot:]), -1)
    y.backward(dy.double())
    args = (pos.cuda(), freq.cuda())
    kw = dict(scale=scale, interleaved=interleaved)
    grad = binding.op_rope(dy.cuda(), *args, inverse=True, **kw)
    assert_within(grad, xd.grad, rope_bound(dy.double(), freq, scale, interleaved, xd.grad, U["fp32"]))
    up, down = binding.op_rope((x + h).cuda(), *args, **kw).double().cpu(), binding.op_rope((x - h).cuda(), *args, **kw).double().cpu()
    step = ((x + h).double() - (x - h).double())
    lhs, rhs = ((up - down) * dy.double()).sum(), (grad.double().cpu() * step).sum()
    # each output is within 2^-21 * 1.21 (|a| + |b|) of the exact map, with |x +- h| below 9 and at most R H D terms of |dy| below 5
    assert abs(lhs - rhs) <= 2 * R * H * D * 2.0 ** -21 * scale * 2 * 9 * 5


def make_cache(B, N, lens, nkv, D, dtype, g, layers=1, extra=3, order=None):
    pps = max(int(t) + N for t in lens) // 16 + 1 + 1
    pages = B * pps + extra
    pool = torch.randn(layers, 2, pages, nkv, 16, D, generator=g).to(TYPES[dtype])
    table = torch.randperm(pages, generator=g)[:B * pps].view(B, pps).to(torch.int32)
    return pool, table


def slots(table, b, at):
    return int(table[b, at // 16]), at % 16


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D,nq,nkv,rot,interleaved", [(64, 4, 4, 64, False), (128, 16, 8, 128, True), (128, 6, 2, 32, False), (64, 7, 1, 62, True)])
@pytest.mark.parametrize("N,lens,counts", [(1, [0], None), (5, [14, 300, 0], [5, 0, 3]), (64, [33, 16], [64, 1]), (17, [15, 31, 16, 1], None)])
@pytest.mark.parametrize("shift", [0, 1])
def test_rope_append(dtype, D, nq, nkv, rot, interleaved, N, lens, counts, shift):
    g = gen(N + D)
    B = len(lens)
    width = (nq + 2 * nkv) * D + (3 if shift else 0)
    store = torch.randn(B * N * width + shift, generator=g).to(TYPES[dtype])
    qkv = store[shift:].view(B, N, width)[..., :(nq + 2 * nkv) * D]
    pool, table = make_cache(B, N, lens, nkv, D, dtype, g)
    pos = torch.randint(0, 200000, (B, N), generator=g, dtype=torch.int32)
    freq, _ = binding.rope_frequencies(rot, 10000.0)
    n = [N] * B if counts is None else counts
    heads = lambda t: [x.unflatten(-1, (-1, D)) for x in t.split([nq * D, nkv * D, nkv * D], dim=-1)]  # noqa: E731
    q, k, v = heads(qkv)
    dev = store.cuda()
    dq, dk, dv = heads(dev[shift:].view(B, N, width)[..., :(nq + 2 * nkv) * D])
    cache = pool[0].cuda()
    out = torch.full((B, N, nq, D), 7.0, dtype=TYPES[dtype], device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    binding.op_rope_append(dq, dk, dv, pos.cuda(), freq.cuda(), cache, table.cuda(), i32(lens), counts=None if counts is None else i32(counts), scale=0.5,
                           interleaved=interleaved, out=out, status=status)
    binding.check_status(status)
    want_q = torch.full((B, N, nq, D), 7.0, dtype=torch.float64)
    bound_q = torch.zeros_like(want_q)
    want, bound = pool[0].double(), torch.zeros(pool[0].shape, dtype=torch.float64)
    tq, tk = (ref.rotate(x.double(), pos, freq, 0.5, interleaved, False) for x in (q, k))
    for b in range(B):
        for i in range(n[b]):
            want_q[b, i], bound_q[b, i] = tq[b, i], rope_bound(q[b, i].double(), freq, 0.5, interleaved, tq[b, i], U[dtype])
            page, slot = slots(table, b, lens[b] + i)
            want[0, page, :, slot], bound[0, page, :, slot] = tk[b, i], rope_bound(k[b, i].double(), freq, 0.5, interleaved, tk[b, i], U[dtype])
            want[1, page, :, slot] = v[b, i].double()
    assert_within(out, want_q, bound_q, "queries")
    assert_within(cache, want, bound, "cache")  # everything else keeps its bits: bound 0 there


def test_rope_append_reports_bad_pages_and_positions_behind_the_table():
    g = gen(3)
    pool, table = make_cache(2, 4, [20, 20], 2, 64, "fp32", g)
    q, k = torch.randn(2, 4, 2, 64, generator=g).cuda(), torch.randn(2, 4, 2, 64, generator=g).cuda()
    freq = binding.rope_frequencies(64)[0].cuda()
    pos = torch.zeros(2, 4, dtype=torch.int32, device="cuda")
    for lens, tab, detail in (([20, 20], {(1, 1): 999}, 999), ([20, 20], {(1, 1): -3}, -3), ([20, 16 * table.shape[1] - 2], {}, -1), ([-1, 20], {}, -1)):
        t = table.clone()
        for at, page in tab.items():
            t[at] = page
        cache = pool[0].cuda()
        with pytest.raises(binding.DbtError) as e:
            binding.op_rope_append(q, k, k, pos, freq, cache, t.cuda(), i32(lens))
        assert e.value.status == 6 and f"[2, {detail}]" in str(e.value)
        # the sequence with good pages is written, nothing outside the positions that exist is
        changed = (cache.cpu() != pool[0]).flatten(2).any(-1).sum().item()
        assert 0 < changed <= 2 * 2 * 2


# ---- attention of a tree ------------------------------------------------------------------------------------------


def random_parents(B, N, g, kind="random"):
    p = torch.full((B, N), -1, dtype=torch.int32)
    for b in range(B):
        for i in range(1, N):
            p[b, i] = {"random": int(torch.randint(-1, i, (1,), generator=g)), "chain": i - 1, "star": 0, "forest": -1}[kind]
    return p


def attn_bound(out, pv, qk, D, T, dtype):
    p = 2 * ((D + 2) * 2.0 ** -24 * qk + 2.0 ** -21 * (1 + qk)) + 2.0 ** -21 + 2 * T * 2.0 ** -24 + (2.0 ** -8 if dtype == "bf16" else 0.0)
    return p[..., None] * pv + U[dtype] * out.abs() + 1e-30


def run_attention(dtype, D, nq, nkv, N, lens, counts, kind, seed, q_scale=2.0, softmax_scale=0.0, spoil=True, strided=False):
    g = gen(seed)
    B = len(lens)
    pool, table = make_cache(B, N, lens, nkv, D, dtype, g)
    n = [N] * B if counts is None else counts
    q = (torch.randn(B, N, nq, D, generator=g) * q_scale).to(TYPES[dtype])
    parents = random_parents(B, N, g, kind)
    out, pv, qk = ref.tree_attention(q, pool[0], table, lens, parents, n, softmax_scale or D ** -0.5)
    cache = pool[0].clone()
    if spoil:  # what no row may see: slots behind the last node, pages of nobody
        used = torch.zeros(cache.shape[1], 16, dtype=torch.bool)
        for b in range(B):
            for t in range(lens[b] + n[b]):
                used[slots(table, b, t)] = True
        cache.transpose(2, 3)[:, ~used] = math.nan
    dq = q.cuda()
    if strided:
        dq = torch.cat((q, q), dim=-1).transpose(1, 2).contiguous().cuda().transpose(1, 2)[..., D:]
    got = torch.full((B, N, nq, D), 7.0, dtype=TYPES[dtype], device="cuda")
    status = torch.zeros(2, dtype=torch.int32, device="cuda")
    binding.op_attn_tree(dq, cache.cuda(), table.cuda(), i32(lens), parents.cuda(), counts=None if counts is None else i32(counts),
                         softmax_scale=softmax_scale, out=got, status=status)
    binding.check_status(status)
    bound = attn_bound(out, pv, qk, D, max(lens) + N, dtype)
    for b in range(B):
        out[b, n[b]:], bound[b, n[b]:] = 7.0, 0.0  # rows behind the last node stay as they were
    assert_within(got, out, bound)
    return got


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D,nq,nkv", [(64, 4, 4), (128, 4, 2), (128, 8, 2), (64, 6, 2), (128, 16, 1)])
@pytest.mark.parametrize("N,lens,counts,kind", [
    (1, [0], None, "chain"), (1, [1], None, "chain"), (1, [200, 63, 64, 127, 128, 129], None, "chain"), (5, [0, 1, 15, 16, 17], None, "random"),
    (16, [120, 0, 255], [16, 3, 9], "random"), (8, [130, 40, 10], [0, 8, 1], "random"), (33, [100, 31], None, "random"), (64, [70, 192], [64, 41], "random"),
])
def test_attn_tree(dtype, D, nq, nkv, N, lens, counts, kind):
    run_attention(dtype, D, nq, nkv, N, lens, counts, kind, seed=N * 7 + D + nq)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kind", ["chain", "star", "forest"])
def test_attn_tree_shapes_of_trees(dtype, kind):
    run_attention(dtype, 128, 8, 4, 64, [500, 3], None, kind, seed=4)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attn_tree_strided_queries_and_a_given_scale(dtype):
    run_attention(dtype, 64, 8, 4, 7, [90, 17], None, "random", seed=6, softmax_scale=0.31, strided=True)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attn_tree_large_scores(dtype):
    """Scores of some hundred: a softmax without its maximum overflows, one with a stale maximum loses its rows."""
    run_attention(dtype, 128, 4, 2, 9, [700, 300], None, "random", seed=8, q_scale=30.0)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attn_tree_long_ragged_batch(dtype):
    """More units than blocks, items cut between blocks, sequences of one key beside long ones."""
    run_attention(dtype, 64, 4, 2, 6, [4000, 0, 2500, 17, 999, 1, 1024, 60], [6, 1, 4, 6, 0, 2, 5, 6], "random", seed=10)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("B,D,nq,nkv,N,far", [(150, 64, 8, 4, 5, 300), (1000, 128, 2, 1, 2, 40), (70, 128, 64, 4, 21, 400), (40, 64, 32, 2, 64, 200), (333, 64, 4, 4, 1, 700)])
def test_attn_tree_more_items_than_blocks(dtype, B, D, nq, nkv, N, far):
    """Several whole items in a block's run, more sequences than a warp looks through at once, several row blocks an item, sequences without
    nodes between."""
    g = gen(B)
    lens = torch.randint(0, far, (B,), generator=g).tolist()
    counts = torch.randint(0, N + 1, (B,), generator=g).tolist()
    lens[3], counts[3], lens[5], counts[5], counts[7], counts[8] = 0, N, 128, N, 0, 0
    run_attention(dtype, D, nq, nkv, N, lens, counts, "random", seed=B + 1)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
def test_attn_tree_nodes_that_a_row_does_not_see_may_hold_anything(dtype, what):
    """Two branches below the root; the second branch's keys and values are not finite.  Rows of the first do not change."""
    g = gen(12)
    lens, N = [37, 128], 9
    pool, table = make_cache(2, N, lens, 2, 128, dtype, g)
    q = torch.randn(2, N, 8, 128, generator=g).to(TYPES[dtype])
    parents = torch.tensor([[-1, 0, 1, 2, 3, 0, 5, 6, 7]] * 2, dtype=torch.int32)
    cache = pool[0].cuda()
    args = (table.cuda(), i32(lens), parents.cuda())
    clean = binding.op_attn_tree(q.cuda(), cache, *args)
    for b in range(2):
        for node in range(5, 9):
            page, slot = slots(table, b, lens[b] + node)
            for w in range(2):
                cache[w, page, :, slot, node * 3:node * 9] = what
    got = binding.op_attn_tree(q.cuda(), cache, *args)
    assert torch.equal(got[:, :5], clean[:, :5])
    if math.isnan(what):
        assert torch.isnan(got[:, 5:]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_attn_tree_values_that_are_not_finite_reach_the_rows_that_see_them(dtype):
    g = gen(13)
    lens, N = [20], 4
    pool, table = make_cache(1, N, lens, 2, 64, dtype, g)
    parents = torch.tensor([[-1, 0, 0, 1]], dtype=torch.int32)
    q = torch.randn(1, N, 2, 64, generator=g).to(TYPES[dtype])
    cache = pool[0].cuda()
    page, slot = slots(table, 0, 21)  # node 1, seen by nodes 1 and 3
    cache[1, page, :, slot, 5], cache[1, page, :, slot, 6], cache[1, page, :, slot, 7] = math.inf, -math.inf, math.nan
    got = binding.op_attn_tree(q.cuda(), cache, table.cuda(), i32(lens), parents.cuda()).float()
    for node in (1, 3):
        assert (got[0, node, :, 5] == math.inf).all() and (got[0, node, :, 6] == -math.inf).all() and torch.isnan(got[0, node, :, 7]).all()
    assert torch.isfinite(got[0, (0, 2)]).all()
    rest = torch.ones(64, dtype=torch.bool)
    rest[5:8] = False
    assert torch.isfinite(got[..., rest.cuda()]).all()


def test_attn_tree_reports_bad_parents_and_pages():
    g = gen(14)
    pool, table = make_cache(2, 4, [40, 20], 2, 64, "bf16", g)
    q = torch.randn(2, 4, 2, 64, generator=g).to(torch.bfloat16).cuda()
    good = random_parents(2, 4, g)
    for parents, tab, lens, code in (([1, 2], {}, [40, 20], "[4, 2]"), ([1, -2], {}, [40, 20], "[4, -2]"), (None, {(0, 1): 777}, [40, 20], "[2, 777]"),
                                     (None, {}, [40, 16 * table.shape[1]], "[2, -1]"), (None, {}, [-7, 20], "[2, -1]")):
        p, t = good.clone(), table.clone()
        if parents:
            p[0, parents[0]] = parents[1]
        for at, page in tab.items():
            t[at] = page
        with pytest.raises(binding.DbtError) as e:
            binding.op_attn_tree(q, pool[0].cuda(), t.cuda(), i32(lens), p.cuda())
        assert e.value.status == 6 and code in str(e.value), (str(e.value), code)


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_offsets_beyond_32_bits(dtype):
    """A cache layer of more than 2^32 elements, its last pages in use: append, attention and acceptance address them."""
    nkv, D, N = 8, 128, 5
    pages = (2 ** 31 // (nkv * 16 * D)) + 40  # one plane alone passes 2^31 elements
    if torch.cuda.mem_get_info()[0] < 2.2 * pages * nkv * 16 * D * (2 if dtype == "bf16" else 4) + 4e9:
        pytest.skip("not enough free memory")
    g = gen(15)
    cache = torch.zeros(2, pages, nkv, 16, D, dtype=TYPES[dtype], device="cuda")
    lens = [29, 50]
    table = torch.tensor([[pages - 1, pages - 3, 5, 6], [pages - 7, 2, pages - 2, pages - 5]], dtype=torch.int32)
    small = torch.randn(2, 8, nkv, 16, D, generator=g).to(TYPES[dtype])
    local = torch.arange(8, dtype=torch.int32).view(2, 4)
    cache[:, table.flatten().long().cuda()] = small.cuda()
    q, k, v = (torch.randn(2, N, h, D, generator=g).to(TYPES[dtype]).cuda() for h in (16, nkv, nkv))
    freq, pos = binding.rope_frequencies(D)[0].cuda(), i32([[t + i for i in range(N)] for t in lens])
    parents = random_parents(2, N, g, "chain").cuda()
    tokens = i32([[1, 2, 3, 4, 5]] * 2)
    parents[:, 3] = 0  # a second branch: its acceptance moves rows
    drawn = i32([[4, 0, 0, 5, 9], [2, 0, 0, 0, 0]])
    parents[:, 4] = 3
    results = []
    for c, tab in ((cache, table), (small.cuda(), local)):
        dev = tab.cuda()
        rot = binding.op_rope_append(q, k, v, pos, freq, c, dev, i32(lens))
        out = binding.op_attn_tree(rot, c, dev, i32(lens), parents)
        path = binding.op_tree_accept(tokens, parents, drawn, c[None], dev, i32(lens))[0]
        results.append((rot, out, path, c[:, tab.flatten().long().cuda()].clone()))
    for a, b in zip(*results):
        assert torch.equal(a, b)
    assert results[0][2].tolist() == [[0, 3, 4, -1, -1], [0, 1, -1, -1, -1]]


# ---- sampling -----------------------------------------------------------------------------------------------------


def check_sample(z, u, temperature=None, top_k=None, top_p=None, min_p=None, margin=1e-9):
    """Tokens equal the 64-bit form's wherever no decision is closer than `margin` (sums of 2^18 doubles differ by less than
    2^18 * 2^-53 = 3e-11 with their order); log-probabilities within 2^-22 of their size, or 2^-22."""
    R = z.shape[0]
    dev = {k: None if x is None else torch.as_tensor(x, dtype=torch.int32 if k == "top_k" else torch.float32).cuda()
           for k, x in dict(temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p).items()}
    tok, lp = binding.op_sample(z.cuda(), torch.as_tensor(u, dtype=torch.float32).cuda(), **dev)
    tok, lp = tok.cpu().tolist(), lp.cpu().tolist()
    zn = z.float().numpy()
    close = 0
    for r in range(R):
        at = lambda x, d: d if x is None else float(np.float32(x[r]))  # noqa: E731
        want, logp, near = ref.sample_row(zn[r], float(np.float32(u[r])), at(temperature, 1.0), int(at(top_k, 0)), at(top_p, 1.0), at(min_p, 0.0))
        if near < margin and tok[r] != want:
            close += 1
            continue
        assert tok[r] == want, (r, tok[r], want, near)
        assert lp[r] == logp or abs(lp[r] - logp) <= 2.0 ** -22 * max(1.0, abs(logp)), (r, lp[r], logp)
    assert close <= 1
    return tok


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [2, 3, 31, 1000, 1024, 1025, 4096, 4097, 9000, 32000, 128256, 262144])
@pytest.mark.parametrize("filters", ["", "k", "p", "m", "kp", "km", "pm", "kpm"])
def test_sample(dtype, V, filters):
    g = gen(V + len(filters))
    R = 6
    z = torch.randn(R, V, generator=g) * torch.tensor([0.3, 1.0, 2.0, 3.0, 6.0, 0.0])[:, None]
    z[3, torch.randint(0, V, (20,), generator=g)] += 9.0
    u = torch.rand(R, generator=g).tolist()
    pick = lambda xs: [xs[int(i)] for i in torch.randint(0, len(xs), (R,), generator=g)]  # noqa: E731
    check_sample(z.to(TYPES[dtype]), u, pick([0.5, 0.8, 1.0, 1.7]), pick([1, 2, 40, 900, 1500, 5000, 0, V, V + 5]) if "k" in filters else None,
                 pick([0.1, 0.5, 0.9, 0.99, 0.9999, 1.0]) if "p" in filters else None, pick([0.0, 0.001, 0.05, 0.5, 1.0]) if "m" in filters else None)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("R", [160, 700])
@pytest.mark.parametrize("V", [1030, 4000, 9001, 32000, 128256])
def test_sample_many_rows(dtype, R, V):
    """Calls with more blocks than the device holds at once: fourteen rows over and over, each as in a call of its own and as the 64-bit form
    has it.  Narrow rows keep few tokens, wide ones most of the vocabulary; two have few distinct values."""
    g = gen(V + R)
    n = 14
    z = torch.randn(n, V, generator=g) * torch.tensor([0.3, 1.0, 2.0, 3.0, 6.0, 0.0, 2.0, 2.0, 2.0, 2.0, 1.0, 1.0, 4.0, 2.0])[:, None]
    z[3, torch.randint(0, V, (20,), generator=g)] += 9.0
    z[10:12] = torch.randint(0, 5, (2, V), generator=g).float()
    u = torch.rand(n, generator=g)
    settings = dict(temperature=torch.tensor([1.0, 1.0, 0.8, 1.0, 0.0, 1.0, 1.3, 1.3, 1.7, 0.5, 0.9, 0.9, 1.0, 50.0]),
                    top_k=torch.tensor([0, 40, 0, 400, 0, 900, 1500, 0, 0, V // 2, 1025, 0, 50, 0], dtype=torch.int32),
                    top_p=torch.tensor([1.0, 1.0, 0.95, 0.9, 1.0, 0.5, 0.99, 0.7, 0.999, 0.9999, 1.0, 0.6, 0.9, 0.2]),
                    min_p=torch.tensor([0.0, 0.05, 0.0, 0.02, 0.0, 0.0, 0.001, 0.0, 0.0, 0.0, 0.4, 0.0, 0.0, 0.0]))
    z = z.to(TYPES[dtype])
    over = torch.arange(R) % n
    for names in ((), ("temperature",), ("top_k",), ("temperature", "top_p"), tuple(settings)):
        s = {k: settings[k] for k in names}
        check_sample(z, u.tolist(), **{k: v.tolist() for k, v in s.items()})
        few = binding.op_sample(z.cuda(), u.cuda(), **{k: v.cuda() for k, v in s.items()})
        many = binding.op_sample(z.cuda()[over], u.cuda()[over], **{k: v.cuda()[over] for k, v in s.items()})
        for r in range(n):
            assert (many[0][r::n] == few[0][r]).all()
            assert (many[1][r::n] - few[1][r]).abs().nan_to_num(0.0).max() <= 2.0 ** -22 * max(1.0, abs(float(few[1][r])))


@pytest.mark.parametrize("V", [5, 3000, 40000])
def test_sample_edges_of_the_settings(V):
    g = gen(V)
    z = (torch.randn(1, V, generator=g) * 2).repeat(12, 1)
    u = [0.0, 1 - 2.0 ** -24, 0.5, 0.5, 0.5, 0.5, 0.5, 0.5, 0.999, 0.25, 0.75, 0.5]
    check_sample(z, u, [1.0, 1.0, 0.0, -1.0, 1e-6, 50.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1e30], [0] * 6 + [1, -3, 0, 0, 0, 0], [1.0] * 6 + [1.0, 1.0, 0.0, 1.0, 1e-9, 1.0],
                 [0.0] * 9 + [2.0, 1.0, 0.0])


@pytest.mark.parametrize("V", [5, 3000, 40000])
@pytest.mark.parametrize("filters", [dict(), dict(top_k=[3] * 4), dict(top_p=[0.999] * 4), dict(top_k=[2500] * 4)])
def test_sample_numbers_outside_their_range(V, filters):
    """Below zero: the first token that is kept; above one, or not a number: the last.  Ids at both ends weigh nothing."""
    z = (torch.randn(1, V, generator=gen(V)) * 2).repeat(4, 1)
    z[:, : V // 3] = -math.inf
    z[:, V - V // 3 :] = -math.inf
    want = check_sample(z, [0.0, 0.0, 2.0, math.nan], **filters)
    dev = {k: torch.as_tensor(v, dtype=torch.int32 if k == "top_k" else torch.float32).cuda() for k, v in filters.items()}
    assert binding.op_sample(z.cuda(), torch.tensor([-1.0, -math.inf, math.inf, math.nan]).cuda(), **dev)[0].tolist() == want


@pytest.mark.parametrize("V", [6, 2000, 50000])
def test_sample_rows_without_anything_and_with_infinities(V):
    inf, nan = math.inf, math.nan
    z = torch.full((8, V), -inf)
    z[1] = nan
    z[2, V // 2] = 1.0
    z[3, [1, V - 1]] = inf
    z[4, [1, V - 1]] = torch.tensor([3.0, 3.0])
    z[4, 2] = nan
    z[5] = torch.finfo(torch.float32).min
    z[6] = torch.finfo(torch.float32).min
    z[6, V - 2] = -1e30
    z[7] = -0.0
    z[7, 1] = 0.0
    u = [0.3, 0.3, 0.9, 0.6, 0.6, 0.4, 0.4, 0.0]
    for kw in ({}, dict(top_k=[1] * 8), dict(top_p=[0.5] * 8), dict(min_p=[0.1] * 8), dict(top_k=[3] * 8, top_p=[0.9] * 8, min_p=[0.01] * 8),
               dict(temperature=[0.0] * 8)):
        tok = check_sample(z, u, **kw)
        assert tok[:3] == [-1, -1, V // 2]


@pytest.mark.parametrize("V", [1500, 20000, 128256])
@pytest.mark.parametrize("distinct", [1, 2, 7])
def test_sample_ties(V, distinct):
    """Few distinct values: borders fall inside groups of equal logits, of which the lowest ids stay."""
    g = gen(V + distinct)
    z = torch.randint(0, distinct, (9, V), generator=g).float()
    u = torch.rand(9, generator=g).tolist()
    for kw in (dict(top_k=[1, 2, 3, 100, 1024, 1025, 1400, V - 1, V]), dict(top_p=[0.1, 0.2, 0.3, 0.4, 0.5, 0.6, 0.7, 0.8, 0.9]),
               dict(top_k=[V // 2] * 9, top_p=[0.1, 0.25, 0.3, 0.4, 0.5, 0.6, 0.75, 0.8, 0.999]), dict(min_p=[0.4] * 9, top_k=[1200] * 9)):
        # sums of few distinct weights come to the same last bits more often: borders that fall together with a sum are left out
        check_sample(z, u, [0.9] * 9, **kw)


@pytest.mark.parametrize("V", [1100, 2000, 40000, 262144])
@pytest.mark.parametrize("settings", [dict(), dict(top_k=[2000] * 5), dict(top_p=[0.7] * 5), dict(top_k=[5] * 5, top_p=[0.3] * 5, temperature=[0.0, 0.5, 1.0, 3.0, math.inf])])
def test_sample_min_p_above_one_leaves_the_likeliest_also_among_many_equal(V, settings):
    """More equal largest logits than a list holds: the first of them is the only one that stays, whatever `min_p` above one says."""
    z = torch.randn(5, V, generator=gen(V))
    z[0] = 0.25
    z[1, 17:1060] = 9.0
    z[2, 17:1060] = math.inf
    z[3, -1030:] = 9.0
    for m in (float(np.nextafter(np.float32(1), np.float32(2))), 2.0, math.inf):
        tok = check_sample(z, [0.0, 0.5, 1 - 2.0 ** -24, 0.3, 0.9], min_p=[m] * 5, **settings)
        assert tok[:4] == [0, 17, 17, V - 1030]


@pytest.mark.parametrize("V,R", [(4100, 2000), (8200, 1500), (16500, 300), (33000, 1), (70000, 150)])
def test_sample_clusters_whose_blocks_begin_at_different_times(V, R):
    """More clusters of two, four and eight blocks than the device holds, of which many leave at once (rows without a number, temperature 0)
    and make room for others: each row as in a call of its own, call after call."""
    g = gen(V)
    n = 5
    z = torch.randn(n, V, generator=g) * 2
    z[1] = -math.inf
    u, t, k = torch.rand(n, generator=g), torch.tensor([1.0, 1.0, 0.0, 0.8, 1.0]), torch.tensor([0, 0, 0, 40, 1500], dtype=torch.int32)
    want = check_sample(z, u.tolist(), temperature=t.tolist(), top_k=k.tolist())
    over = torch.arange(R) % n
    args = [x.cuda()[over] for x in (z, u, t, k)]
    expected = torch.tensor(want, dtype=torch.int32).cuda()[over]
    for _ in range(20):
        assert torch.equal(binding.op_sample(*args)[0], expected)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [1500, 2207, 40000, 128256])
def test_sample_windows_of_a_few_neighbouring_numbers(dtype, V):
    """Logits so large, or temperatures so low, that the first window of a search holds fewer numbers than it has buckets, while others lie
    more than 2^31 ordered patterns below."""
    g = gen(V)
    z = torch.randn(6, V, generator=g) * torch.tensor([1e6, 1e7, 1e8, 1e12, 3e36, 1e7])[:, None]
    z[5, V // 3 : V // 3 + 1200] = 4e7
    z = z.to(TYPES[dtype])
    u = torch.rand(6, generator=g).tolist()
    for t in (1.0, 1e7, 1e30, 1e37):
        check_sample(z, u, temperature=[t] * 6, top_k=[V - 1, V - 5, V // 2 + 300, 3 * V // 4, V - 2, 1300])
        check_sample(z, u, temperature=[t] * 6, top_k=[V - 1, V - 5, V // 2 + 300, 3 * V // 4, V - 2, 1300], top_p=[0.3, 0.9, 0.5, 0.999, 0.8, 0.7])
        check_sample(z, u, temperature=[t] * 6, top_p=[0.3, 0.9, 0.5, 0.999, 0.8, 0.7])
    y = torch.randn(6, V, generator=g) * 3
    y[:, 100 : 100 + V * 2 // 3] = torch.tensor([4.0, 8.0, 12.0, 16.0, 0.5, 100.0])[:, None]
    y = y.clamp(max=y[:, 100:101]).to(TYPES[dtype])
    for t in (1e-4, 1e-6, 1e-7, 1e-12, 1e-40):
        for kw in (dict(top_p=[0.5, 0.25, 0.75, 0.9, 0.1, 0.6]), dict(top_k=[V - 1, V // 2, 600, 1025, V // 3, 2], top_p=[0.5, 0.25, 0.75, 0.9, 0.1, 0.6]), dict(top_k=[V - 1, V // 2, 600, 1025, V // 3, 2])):
            check_sample(y, u, temperature=[t] * 6, **kw)


def test_sample_strided_and_odd_rows():
    g = gen(21)
    store = torch.randn(5, 1003, generator=g) * 2
    z = store[:, 1:1000]  # rows that begin on odd addresses
    u = torch.rand(5, generator=g)
    want = [ref.sample_row(z[r].numpy(), float(u[r]))[0] for r in range(5)]
    assert binding.op_sample(store.cuda()[:, 1:1000], u.cuda())[0].tolist() == want
    wide = store.to(torch.bfloat16)
    want = [ref.sample_row(wide[r, 3:900].float().numpy(), float(u[r]))[0] for r in range(5)]
    assert binding.op_sample(wide.cuda()[:, 3:900], u.cuda())[0].tolist() == want


def test_sample_follows_the_distribution():
    """Evenly spread numbers give every token its share to within one number at either end."""
    n = 20000
    z = torch.tensor([0.5, -1.0, 2.0, 0.0, 1.0]).repeat(n, 1)
    u = (torch.arange(n) + 0.5) / n
    tok = binding.op_sample(z.cuda(), u.cuda())[0].cpu()
    share = torch.softmax(z[0].double(), 0)
    assert (torch.bincount(tok, minlength=5) - share * n).abs().max() <= 2


# ---- acceptance ---------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("D,nkv,layers", [(64, 4, 2), (128, 1, 3)])
@pytest.mark.parametrize("N,lens,counts,words", [(1, [0, 40], None, 2), (5, [14, 3, 77], [5, 0, 3], 2), (33, [15, 16, 100], [33, 32, 20], 3),
                                                 (64, [31, 63], [64, 63], 2), (64, [5], None, 1)])
def test_tree_accept(dtype, D, nkv, layers, N, lens, counts, words):
    """Tokens of a few words: several children of a node carry the same one, the lowest number is taken."""
    g = gen(N + words)
    B = len(lens)
    pool, table = make_cache(B, N, lens, nkv, D, dtype, g, layers=layers)
    parents = random_parents(B, N, g, "random" if words > 1 else "chain")
    tokens, sampled = (torch.randint(0, words, (B, N), generator=g, dtype=torch.int32) for _ in range(2))
    n = [N] * B if counts is None else counts
    dev = pool.cuda()
    path, count, follows, new = binding.op_tree_accept(tokens.cuda(), parents.cuda(), sampled.cuda(), dev, table.cuda(), i32(lens),
                                                       counts=None if counts is None else i32(counts))
    want = pool.clone()
    for b in range(B):
        walk, nxt = ref.accept(tokens[b], parents[b], sampled[b], n[b])
        assert path[b].tolist() == walk + [-1] * (N - len(walk))
        assert (int(count[b]), int(follows[b]), int(new[b])) == (len(walk), nxt, lens[b] + len(walk))
        for j, c in enumerate(walk):
            (p0, s0), (p1, s1) = slots(table, b, lens[b] + c), slots(table, b, lens[b] + j)
            want[:, :, p1, :, s1] = pool[:, :, p0, :, s0]
    assert torch.equal(dev.cpu(), want)


def test_tree_accept_reports_bad_parents_and_pages():
    g = gen(31)
    pool, table = make_cache(1, 4, [14], 2, 64, "fp32", g)
    tokens, sampled = i32([[9, 1, 2, 3]]), i32([[2, 0, 3, 5]])
    parents = torch.tensor([[-1, 0, 0, 2]], dtype=torch.int32)
    dev = pool.cuda()
    assert binding.op_tree_accept(tokens, parents.cuda(), sampled, dev, table.cuda(), i32([14]))[0].tolist() == [[0, 2, 3, -1]]
    bad = parents.clone()
    bad[0, 3] = 3
    with pytest.raises(binding.DbtError) as e:
        binding.op_tree_accept(tokens, bad.cuda(), sampled, pool.cuda(), table.cuda(), i32([14]))
    assert e.value.status == 6 and "[4, 3]" in str(e.value)
    t = table.clone()
    t[0, 1] = 4711
    dev = pool.cuda()
    with pytest.raises(binding.DbtError) as e:
        binding.op_tree_accept(tokens, parents.cuda(), sampled, dev, t.cuda(), i32([14]))
    assert e.value.status == 6 and "[2, 4711]" in str(e.value)
    assert torch.equal(dev.cpu(), pool)


# ---- together: streams, graphs, a decoding loop ---------------------------------------------------------------------


class Toy:
    """One attention layer between an embedding and an output matrix, in fp32, on the operators: enough to decode with."""

    def __init__(self, seed, vocab=300, nq=4, nkv=2, D=64, pages=64, batch=3):
        g = gen(seed)
        self.vocab, self.nq, self.nkv, self.D, self.B = vocab, nq, nkv, D, batch
        d = 48
        self.embed = torch.randn(vocab, d, generator=g).cuda()
        self.wqkv = (torch.randn((nq + 2 * nkv) * D, d, generator=g) * 0.3).cuda()
        self.wo = (torch.randn(d, nq * D, generator=g) * 0.4).cuda()
        self.head = (torch.randn(vocab, d, generator=g) * 0.5).cuda()
        self.pool = torch.zeros(1, 2, pages, nkv, 16, D, device="cuda")
        self.table = torch.randperm(pages, generator=g)[: batch * (pages // batch)].view(batch, -1).to(torch.int32).cuda()
        f, self.scale = binding.rope_frequencies(D, 10000.0, "bands", factor=4.0, trained_len=32, low=1, high=4)
        self.freq = f.cuda()

    def logits(self, tokens, parents, depth, lens, counts=None):
        """[B, N, vocab] of the nodes; their keys and values are in the cache afterwards."""
        x = self.embed[tokens.long()]
        qkv = (x @ self.wqkv.t()).split([self.nq * self.D, self.nkv * self.D, self.nkv * self.D], dim=-1)
        q, k, v = (t.unflatten(-1, (-1, self.D)) for t in qkv)
        q = binding.op_rope_append(q, k, v, (lens[:, None] + depth).to(torch.int32), self.freq, self.pool[0], self.table, lens, counts=counts, scale=self.scale)
        o = binding.op_attn_tree(q, self.pool[0], self.table, lens, parents, counts=counts)
        return (x + o.flatten(2) @ self.wo.t()) @ self.head.t()


def test_drafted_decoding_gives_the_tokens_of_decoding_one_by_one():
    """Tokens drawn with the same number per position: once node by node, once with trees that hold the true continuation among wrong
    ones.  Every accepted token, and the cache, must be those of the plain loop."""
    steps, B = 24, 3
    uniforms = torch.rand(B, 200, generator=gen(41)).cuda()
    settings = dict(top_k=i32([50] * B), top_p=torch.full((B,), 0.95, device="cuda"), min_p=torch.full((B,), 0.01, device="cuda"))
    start = i32([[5], [77], [123]])
    one = Toy(40)
    lens, tok, plain = i32([0] * B), start.clone(), []
    zero, root = i32([[0]] * B), i32([[-1]] * B)
    for t in range(steps):
        z = one.logits(tok, root, zero, lens)
        nxt, _ = binding.op_sample(z[:, 0], uniforms[torch.arange(B), lens.long()].contiguous(), temperature=torch.full((B,), 0.9, device="cuda"), **settings)
        plain.append(nxt.clone())
        tok, lens = nxt[:, None], lens + 1
    plain = torch.stack(plain, 1)  # [B, steps]: the token after position t

    tree = Toy(40)
    N, g = 8, gen(42)
    lens, tok, out = i32([0] * B), start.clone(), [[] for _ in range(B)]
    rounds = 0
    while min(len(o) for o in out) < steps - 6:
        rounds += 1
        # chain of up to three true tokens below node 0, on numbers with gaps; the others are wrong drafts
        parents, tokens, depth = torch.full((B, N), -1), torch.randint(0, 300, (B, N), generator=g), torch.zeros(B, N, dtype=torch.long)
        tokens[:, 0] = tok[:, 0].cpu()
        for b in range(B):
            for i in range(1, N):
                parents[b, i] = int(torch.randint(0, i, (1,), generator=g))
            cur = 0
            for j, node in enumerate(sorted((torch.randperm(N - 1, generator=g)[: 1 + rounds % 3] + 1).tolist())):
                at = len(out[b]) + j
                parents[b, node], tokens[b, node] = cur, int(plain[b, min(at, steps - 1)])
                cur = node
            for i in range(1, N):
                depth[b, i] = depth[b, parents[b, i]] + 1
        tokens, parents, depth = i32(tokens), i32(parents), i32(depth)
        z = tree.logits(tokens, parents, depth, lens)
        rows = torch.arange(B, device="cuda").repeat_interleave(N)
        u = uniforms[rows, (lens[:, None] + depth).flatten().long()].contiguous()
        drawn, _ = binding.op_sample(z.flatten(0, 1), u, temperature=torch.full((B * N,), 0.9, device="cuda"),
                                     **{k: v.repeat_interleave(N) for k, v in settings.items()})
        path, count, follows, new = binding.op_tree_accept(tokens, parents, drawn.view(B, N), tree.pool, tree.table, lens)
        for b in range(B):
            walk = path[b, : int(count[b])].tolist()
            out[b] += [int(tokens[b, c]) for c in walk[1:]] + [int(follows[b])]
        tok, lens = follows[:, None].contiguous(), new
    assert rounds < steps - 6  # several tokens a round
    for b in range(B):
        n = min(len(out[b]), steps)
        assert out[b][:n] == plain[b, :n].tolist()
        # both caches hold the same rows: the same arithmetic, apart from the shapes of the torch products
        t = min(int(lens[b]), steps)
        for w in range(2):
            a, c = (ref.cache_rows(x.pool[0, w].cpu().double(), x.table[b].cpu(), 0, t) for x in (one, tree))
            assert (a - c).abs().max() <= 48 * 2.0 ** -22 * a.abs().max()


def test_operators_on_a_side_stream_and_in_graphs():
    """Two captured chains replayed together on two streams, each with buffers of its own, and an eager run between: equal bits.  Lengths
    change between replays."""
    g = gen(51)
    B, N, nq, nkv, D = 2, 6, 8, 4, 128
    lens = [300, 45]
    pool, table = make_cache(B, N, [700, 700], nkv, D, "bf16", g)
    freq, parents = binding.rope_frequencies(D)[0].cuda(), random_parents(B, N, g).cuda()
    q, k, v = (torch.randn(B, N, h, D, generator=g).to(torch.bfloat16).cuda() for h in (nq, nkv, nkv))
    z, u = (torch.randn(B * N, 5000, generator=g) * 2).cuda(), torch.rand(B * N, generator=g).cuda()
    p = torch.full((B * N,), 0.9, device="cuda")
    tokens, table = torch.randint(0, 3, (B, N), generator=g, dtype=torch.int32).cuda(), table.cuda()

    class Chain:
        def __init__(self):
            self.pool, self.lens, self.pos = pool.cuda(), i32(lens), i32([[t + i for i in range(N)] for t in lens])
            self.status = torch.zeros(2, dtype=torch.int32, device="cuda")

        def run(self):
            st = dict(status=self.status)
            rot = binding.op_rope_append(q, k, v, self.pos, freq, self.pool[0], table, self.lens, **st)
            o = binding.op_attn_tree(rot, self.pool[0], table, self.lens, parents, **st)
            t, lp = binding.op_sample(z, u, top_p=p)
            self.out = (rot, o, t, lp, *binding.op_tree_accept(tokens, parents, (t % 3).view(B, N), self.pool, table, self.lens, **st))

    eager = Chain()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        eager.run()
    torch.cuda.current_stream().wait_stream(side)
    chains, graphs, streams = [Chain(), Chain()], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in chains:
        c.run()  # (loads the kernels)
        c.pool.copy_(pool)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            c.run()
        graphs.append(graph)
    torch.cuda.synchronize()
    for new in (lens, [17, 600], lens):
        for c in (*chains, eager):
            c.pool.copy_(pool)
            c.lens.copy_(i32(new))
            c.pos.copy_(i32([[t + i for i in range(N)] for t in new]))
        torch.cuda.synchronize()
        for s, graph in zip(streams, graphs):
            with torch.cuda.stream(s):
                graph.replay()
        eager.run()
        torch.cuda.synchronize()
        for c in chains:
            binding.check_status(c.status)
            assert torch.equal(c.pool, eager.pool)
            for a, b in zip(c.out, eager.out):
                assert torch.equal(a, b)


def test_repeated_calls_give_the_same_bits():
    g = gen(61)
    pool, table = make_cache(3, 20, [900, 333, 2000], 2, 128, "bf16", g)
    q = torch.randn(3, 20, 8, 128, generator=g).to(torch.bfloat16).cuda()
    args = (q, pool[0].cuda(), table.cuda(), i32([900, 333, 2000]), random_parents(3, 20, g).cuda())
    z, u = torch.randn(40, 128256, generator=g).cuda(), torch.rand(40, generator=g).cuda()
    first, tok = binding.op_attn_tree(*args), binding.op_sample(z, u, top_p=torch.full((40,), 0.99, device="cuda"))
    for _ in range(5):
        assert torch.equal(binding.op_attn_tree(*args), first)
        for a, b in zip(binding.op_sample(z, u, top_p=torch.full((40,), 0.99, device="cuda")), tok):
            assert torch.equal(a, b)
