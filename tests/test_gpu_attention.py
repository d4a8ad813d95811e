"""Attention on the GPU against its definition in 64 bits (tests/networks_reference.py says how far a kernel may be off)."""
import gc

import pytest
import torch

import networks_reference as R
from activations_reference import assert_close

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def N():
    from paper_2307_05801_amd import networks
    return networks


def rand(shape, seed, dtype=BF16, by=1.0):
    return (torch.randn(*shape, generator=torch.Generator().manual_seed(seed)) * by).to(dtype)


def inputs(batch, queries, keys, heads, kv_heads, width, seed):
    """q, k, v and o's gradient; keys and values with a part that all rows have."""
    q, k, v, g = (rand(s, seed + i) for i, s in enumerate([(batch, queries, heads, width), (batch, keys, kv_heads, width)] + [(batch, keys, kv_heads, width), (batch, queries, heads, width)]))
    return q, k + rand((1, 1, kv_heads, width), seed + 8), v + rand((1, 1, kv_heads, width), seed + 9), g


def run(N, q, k, v, grad, table=None, mask=None, buckets=None, positions=None, scale=None, leaves=None):
    """What the GPU makes of CPU tensors: (o, grad_q, grad_k, grad_v, grad_table or None)."""
    def there(t):
        return t.cuda() if isinstance(t, torch.Tensor) else t

    q, k, v, table = (None if t is None else there(t).detach().requires_grad_(True) for t in (q, k, v, table))
    positions = tuple(None if t is None else there(t) for t in positions) if isinstance(positions, tuple) else there(positions)
    o = N.attention(q, k, v, table=table, mask=there(mask), buckets=there(buckets), positions=positions, scale=scale)
    wanted = [t for t in (q, k, v, table) if t is not None]
    grads = torch.autograd.grad(o, wanted, there(grad))
    return (o.detach(), *grads) + (None,) * (4 - len(grads))


def check(got, r):
    for name, t in zip(("o", "grad_q", "grad_k", "grad_v", "grad_table"), got):
        if t is not None:
            assert_close(t, getattr(r, name), getattr(r, name + "_off"), name)


LENGTHS = [(1, 1, 1), (1, 1, 2), (2, 5, 31), (1, 31, 33), (2, 32, 64), (1, 33, 65), (1, 64, 63), (2, 1, 300), (1, 127, 129), (1, 128, 128), (1, 129, 127), (3, 200, 7), (1, 257, 640)]


@pytest.mark.parametrize("batch,queries,keys", LENGTHS)
@pytest.mark.parametrize("heads,kv_heads,width", [(1, 1, 64), (4, 2, 32), (3, 1, 49), (2, 2, 128)])
def test_lengths(N, batch, queries, keys, heads, kv_heads, width):
    t = inputs(batch, queries, keys, heads, kv_heads, width, 1)
    check(run(N, *t), R.Attention(*t))


@pytest.mark.parametrize("width", [1, 2, 7, 8, 9, 16, 31, 33, 40, 63, 65, 72, 80, 95, 96, 97, 100, 112, 127])
def test_widths(N, width):
    t = inputs(2, 70, 90, 2, 1, width, 11)
    check(run(N, *t), R.Attention(*t))


# keys in parts, put together by a second kernel; heads that share keys side by side: four, two and one at a time
FEW = [(1, 1, 5000, 8, 8, 64), (2, 16, 1500, 8, 2, 64), (1, 33, 1100, 4, 1, 64), (1, 64, 700, 6, 1, 32), (1, 65, 600, 4, 1, 40), (3, 5, 513, 4, 1, 49), (1, 3, 2049, 12, 3, 128), (1, 32, 64, 4, 1, 64),
       (1, 200, 512, 2, 2, 64)]


@pytest.mark.parametrize("batch,queries,keys,heads,kv_heads,width", FEW)
@pytest.mark.parametrize("kind", [None, "late", "scattered", "lengths"])
def test_few_queries_over_many_keys(N, batch, queries, keys, heads, kv_heads, width, kind):
    t = inputs(batch, queries, keys, heads, kv_heads, width, 15)
    mask = masks(batch, keys, kind) if kind else None
    r = R.Attention(*t, mask=mask)
    check(run(N, *t, mask=mask), r)
    with torch.no_grad():
        o = N.attention(*(x.cuda() for x in t[:3]), mask=None if mask is None else mask.cuda())
    r = R.Attention(*t, mask=mask, fine=False)
    assert_close(o, r.o, r.o_off, "o")


@pytest.mark.parametrize("batch,queries,keys,heads,kv_heads,width", FEW)
def test_few_queries_with_a_bias(N, batch, queries, keys, heads, kv_heads, width):
    t = inputs(batch, queries, keys, heads, kv_heads, width, 16)
    _, buckets, many = places(queries, keys, "line")
    table = rand((heads, many), 17, F32)
    check(run(N, *t, table, None, buckets), R.Attention(*t, None, table, buckets))


@pytest.mark.parametrize("batch,queries,keys,heads,kv_heads,width", [(1, 600, 700, 2, 1, 49), (2, 520, 30, 2, 2, 5), (1, 30, 600, 4, 2, 33), (1, 513, 513, 1, 1, 127), (1, 513, 1, 2, 1, 9)])
@pytest.mark.parametrize("kind", [None, "scattered", "lengths"])
def test_rows_that_are_laid_out(N, batch, queries, keys, heads, kv_heads, width, kind):
    """More than 512 of one side, rows that are no multiples of 16 bytes: within a wider array whose other values must not matter."""
    t = inputs(batch, queries, keys, heads, kv_heads, width, 18)
    mask = masks(batch, keys, kind) if kind else None
    r = R.Attention(*t, mask=mask)
    check(run(N, *t, mask=mask), r)
    wide = []
    for x in t:
        room = torch.full(x.shape[:-1] + (width + 6,), float("nan"), dtype=BF16, device="cuda")
        room[..., 5:5 + width] = x.cuda()
        wide.append(room[..., 5:5 + width])
    check(run(N, *wide, mask=mask), r)


@pytest.mark.parametrize("scale", [1e-3, 1.0, 3.0])
def test_scales(N, scale):
    """Probabilities from nearly even to nearly all on one key."""
    t = inputs(1, 100, 150, 2, 2, 40, 21)
    check(run(N, *t, scale=scale), R.Attention(*t, scale=scale))


def test_without_a_backward_pass(N):
    """Of the memory o alone, and its probabilities rounded to bfloat16."""
    t = inputs(2, 300, 200, 4, 2, 64, 31)
    r, (q, k, v) = R.Attention(*t, fine=False), (x.cuda() for x in t[:3])
    q.requires_grad_(True)
    for recording, t in ((False, q), (True, q.detach())):
        gc.collect()
        torch.cuda.reset_peak_memory_stats()
        before = torch.cuda.memory_allocated()
        with torch.set_grad_enabled(recording):
            o = N.attention(t, k, v)
        assert torch.cuda.max_memory_allocated() - before <= o.numel() * 2 + 512
        assert not o.requires_grad
        assert_close(o, r.o, r.o_off, "o")


# ---- masks ----


def masks(batch, keys, kind):
    m = torch.ones(batch, keys, dtype=torch.bool)
    if kind == "lengths":
        for b in range(batch):
            m[b, keys * b // max(1, batch - 1):] = False            # the first item has none
    elif kind == "scattered":
        m = torch.rand(batch, keys, generator=torch.Generator().manual_seed(41)) < 0.5
    elif kind == "late":
        m[:, :keys - 3] = False                                     # whole tiles before the first key
    elif kind == "one":
        m[:] = False
        m[:, keys // 2] = True
    elif kind == "none":
        m[:] = False
    return m


@pytest.mark.parametrize("kind", ["lengths", "scattered", "late", "one", "none"])
@pytest.mark.parametrize("batch,queries,keys,width", [(3, 40, 40, 64), (2, 130, 200, 64), (4, 1, 333, 32), (2, 70, 129, 49), (2, 64, 512, 128)])
def test_masks(N, batch, queries, keys, width, kind):
    t, mask = inputs(batch, queries, keys, 2, 1, width, 42), masks(batch, keys, kind)
    got = run(N, *t, mask=mask)
    check(got, R.Attention(*t, mask=mask))
    gone = ~mask.cuda()
    assert not got[2][gone].any() and not got[3][gone].any()
    none = ~mask.any(1).cuda()
    assert not got[0][none].any() and not got[1][none].any()


@pytest.mark.parametrize("what", [float("nan"), float("inf"), float("-inf"), torch.finfo(BF16).max])
def test_what_a_mask_leaves_out_does_not_matter(N, what):
    q, k, v, g = inputs(2, 70, 150, 2, 1, 64, 51)
    mask = masks(2, 150, "scattered")
    table, buckets = rand((2, 9), 52, F32), torch.randint(0, 9, (299,), generator=torch.Generator().manual_seed(53), dtype=torch.int32)
    want = run(N, q, k, v, g, table, mask, buckets)
    k, v = (torch.where(mask[:, :, None, None], t, what) for t in (k, v))
    assert all(torch.equal(a, b) for a, b in zip(run(N, q, k, v, g, table, mask, buckets), want))


def test_a_value_that_is_not_a_number_reaches_its_own_queries(N):
    q, k, v, g = inputs(2, 40, 70, 2, 2, 64, 54)
    q[1, 7, 0, 3] = float("nan")
    v[0, 5, 1, 2] = float("nan")
    o = run(N, q, k, v, g)[0].cpu()
    bad = torch.zeros(o.shape, dtype=torch.bool)
    bad[1, 7, 0] = True
    bad[0, :, 1, 2] = True
    assert torch.equal(torch.isnan(o), bad)


# ---- the bias ----


def places(queries, keys, kind, seed=61):
    """(positions, buckets, number of buckets)."""
    g = torch.Generator().manual_seed(seed)
    many = 4001 if "many" in kind else 31
    if kind.startswith("line"):
        n = queries + keys - 1 | 1
        return None, torch.randint(0, many, (n,), generator=g, dtype=torch.int32), many
    if kind.startswith("few"):                                      # differences beyond both ends
        return None, torch.randint(0, many, (11,), generator=g, dtype=torch.int32), many
    if kind.startswith("even"):                                     # an even number of them
        return None, torch.randint(0, many, (12,), generator=g, dtype=torch.int32), many
    far = 1 << 29 if "far" in kind else 2000                        # in any order, some more than once
    p = tuple(torch.randint(-far, far + 1, (n,), generator=g, dtype=torch.int32) for n in (queries, keys))
    p[1][keys // 2:] = p[1][:keys - keys // 2].clone()
    return p, torch.randint(0, many, (4001,), generator=g, dtype=torch.int32), many


@pytest.mark.parametrize("kind", ["line", "line many", "few", "even", "anywhere", "anywhere many", "far"])
@pytest.mark.parametrize("batch,queries,keys,heads,kv_heads,width", [(1, 1, 1, 1, 1, 8), (3, 50, 70, 4, 2, 32), (2, 200, 130, 2, 2, 64), (1, 129, 257, 3, 1, 49), (2, 64, 128, 1, 1, 128)])
def test_bias(N, kind, batch, queries, keys, heads, kv_heads, width):
    t = inputs(batch, queries, keys, heads, kv_heads, width, 62)
    positions, buckets, many = places(queries, keys, kind)
    table = rand((heads, many), 63, F32)
    check(run(N, *t, table, None, buckets, positions), R.Attention(*t, None, table, buckets, positions))


@pytest.mark.parametrize("shape,near,codes", [((16,), 16, 16), ((300,), 4, 8), ((12, 11), 12, 12), ((5, 6, 7), 2, 4), ((8, 8, 8), 8, 8), ((1, 40, 3), 1, 3)])
@pytest.mark.parametrize("masked", [False, True])
def test_patches_of_a_grid(N, shape, near, codes, masked):
    positions, buckets = N.relative_buckets(shape, near, codes, device="cpu")
    n, many = len(positions), (2 * codes - 1) ** len(shape)
    t, table = inputs(2, n, n, 2, 2, 32, 71), rand((2, many), 75, F32)
    mask = masks(2, n, "scattered") if masked else None
    check(run(N, *t, table, mask, buckets, positions), R.Attention(*t, mask, table, buckets, positions))


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_types_of_a_table(N, dtype):
    t, (_, buckets, many) = inputs(2, 60, 80, 2, 1, 64, 81), places(60, 80, "line")
    table = rand((2, many), 82, dtype)
    got = run(N, *t, table, None, buckets)
    assert got[4].dtype is dtype
    check(got, R.Attention(*t, None, table, buckets))
    with torch.no_grad():                                           # forward alone
        o = N.attention(*(x.cuda() for x in t[:3]), table=table.cuda(), buckets=buckets.cuda())
    r = R.Attention(*t, None, table, buckets, fine=False)
    assert_close(o, r.o, r.o_off, "o")


def test_a_table_without_a_gradient(N):
    """The gradients of q, k, v with a table that wants none."""
    q, k, v, g = inputs(2, 60, 80, 2, 1, 64, 83)
    _, buckets, many = places(60, 80, "line")
    table = rand((2, many), 84, F32)
    leaves = [t.cuda().requires_grad_(True) for t in (q, k, v)]
    o = N.attention(*leaves, table=table.cuda(), buckets=buckets.cuda())
    r = R.Attention(q, k, v, g, None, table, buckets)
    check((o.detach(), *torch.autograd.grad(o, leaves, g.cuda())), r)


def test_a_table_that_leaves_pairs_out(N):
    """-inf for later keys, and for all keys of the first query: that one's output and gradients are zeros."""
    n = 150
    t, buckets = inputs(1, n, n, 2, 2, 64, 91), torch.zeros(2 * n - 1, dtype=torch.int32)
    buckets[n - 1:] = 2                                             # the key itself and those behind it
    buckets[:n - 20] = 1
    table = torch.tensor([[0.5, -0.5, -torch.inf]]).repeat(2, 1)
    got = run(N, *t, table, None, buckets)
    check(got, R.Attention(*t, None, table, buckets))
    assert not got[0][0, 0].any() and not got[1][0, 0].any() and not got[4][:, 2].any()


@pytest.mark.parametrize("low", [torch.finfo(F32).min, -1e30, -1e4])
def test_a_table_with_a_types_lowest_number(N, low):
    """Where a row has other keys those with the lowest number have no part; where it has none, all the same.  The scores of such a row are the number
    itself to within its rounding, which -1e4's does not hide: they are off by half of 2^-10."""
    n = 140
    q, k, v, g = inputs(1, n, n, 2, 2, 64, 95)
    buckets = torch.zeros(2 * n - 1, dtype=torch.int32)
    buckets[n - 1:] = 1
    table = torch.tensor([[0.25, low]]).repeat(2, 1)
    got = run(N, q, k, v, g, table, None, buckets)
    assert all(torch.isfinite(t).all() for t in got)
    r = R.Attention(q, k, v, g, None, table, buckets)
    for name, t in zip(("o", "grad_q", "grad_v"), got):             # rows with a key before them
        if name != "grad_v":
            assert_close(t[:, 1:], getattr(r, name)[:, 1:], getattr(r, name + "_off")[:, 1:], name)
    if low < -1e20:
        even = v.double().mean(1)
        assert_close(got[0][:, 0], even, v.double().abs().mean(1) * (2 * R.HALF), "o of even probabilities")


def test_precision_of_the_tables_gradient(N):
    """To 32 bits: 1e-5 of its norm (of a bucket's sum of 8000 pairs or so no more than 2^-24 * sqrt(8000) is expected of each roundings' kind)."""
    n = 256
    positions, buckets = N.relative_buckets((16, 16), 4, 6, device="cpu")
    t, table = inputs(4, n, n, 2, 2, 64, 99), rand((2, 121), 98, F32)
    got, r = run(N, *t, table, None, buckets, positions), R.Attention(*t, None, table, buckets, positions)
    assert (got[4].cpu().double() - r.grad_table).norm() <= 1e-5 * r.grad_table.norm()


# ---- layouts ----


def test_heads_of_one_projection(N):
    """q, k, v as slices of rows [3, heads, width], heads before rows, and a gradient that lies otherwise."""
    x = rand((2, 75, 3, 4, 40), 101)
    t = [x[:, :, i] for i in range(3)] + [rand((2, 4, 75, 40), 102).transpose(1, 2)]
    r = R.Attention(*t)
    leaf = x.cuda().requires_grad_(True)
    o = N.attention(*leaf.unbind(2))
    got, = torch.autograd.grad(o, leaf, t[3].cuda().contiguous().transpose(1, 2).contiguous().transpose(1, 2))
    check((o.detach(), *got.unbind(2)), r)
    q, k, v = (s.transpose(1, 2).contiguous().transpose(1, 2) for s in t[:3])
    check(run(N, q, k, v, t[3]), r)


def test_rows_from_any_byte_on(N):
    """Rows that begin at odd multiples of two bytes, a distance of 51 apart."""
    wide = [rand((2, 60, 3, 51), 110 + i) for i in range(4)]
    t = [w[..., 1:50] for w in wide]
    check(run(N, *(w.cuda()[..., 1:50] for w in wide)), R.Attention(*t))


def test_rows_of_one_value_and_tables_of_one_bucket_with_any_last_stride(N):
    q, k, v, g = inputs(2, 5, 37, 3, 3, 1, 313)
    table, buckets = rand((3, 1), 317, F32), torch.zeros(9, dtype=torch.int32)

    def turned(t):
        there = torch.empty(*t.shape[:2], 1, t.shape[2], dtype=t.dtype, device="cuda").transpose(2, 3)
        assert there.stride(3) == 3
        return there.copy_(t)

    line = torch.empty(3, dtype=F32, device="cuda").as_strided((3, 1), (1, 5)).copy_(table)
    assert line.stride(1) == 5
    r = R.Attention(q, k, v, g, table=table, buckets=buckets)
    check(run(N, turned(q), turned(k), turned(v), turned(g), table=line, buckets=buckets), r)


def test_one_item_for_a_batch(N):
    """Keys and values of one item for all (distance 0), heads of one for all: autograd adds the gradients up."""
    q, k, v, g = inputs(1, 50, 90, 2, 2, 32, 121)
    q, g = rand((3, 50, 2, 32), 122), rand((3, 50, 2, 32), 123)
    leaves = [t.cuda().requires_grad_(True) for t in (q, k, v)]
    o = N.attention(leaves[0], leaves[1].expand(3, -1, -1, -1), leaves[2].expand(3, -1, -1, -1))
    got = torch.autograd.grad(o, leaves, g.cuda())
    r = R.Attention(q, k.expand(3, -1, -1, -1), v.expand(3, -1, -1, -1), g)
    assert_close(o, r.o, r.o_off, "o")
    assert_close(got[0], r.grad_q, r.grad_q_off, "grad_q")
    for got_t, name in ((got[1], "grad_k"), (got[2], "grad_v")):        # three roundings and two additions in bfloat16
        want = getattr(r, name)
        assert_close(got_t, want.sum(0, keepdim=True), getattr(r, name + "_off").sum(0, keepdim=True) + 3 * R.HALF * want.abs().sum(0, keepdim=True), name)
    grad = torch.autograd.grad(N.attention(*leaves[:1], leaves[1].expand(3, -1, -1, -1), leaves[2].expand(3, -1, -1, -1)).sum(), leaves[0])[0]      # a gradient of distance 0
    assert torch.isfinite(grad).all() and not torch.equal(grad, got[0])


def test_the_same_tensor_three_times(N):
    x, g = rand((2, 40, 2, 64), 131), rand((2, 40, 2, 64), 132)
    leaf = x.cuda().requires_grad_(True)
    got, = torch.autograd.grad(N.attention(leaf, leaf, leaf), leaf, g.cuda())
    r = R.Attention(x, x, x, g)
    want = r.grad_q + r.grad_k + r.grad_v
    size = r.grad_q.abs() + r.grad_k.abs() + r.grad_v.abs()
    assert_close(got, want, r.grad_q_off + r.grad_k_off + r.grad_v_off + 2 * R.HALF * (size + want.abs()), "grad")


@pytest.mark.parametrize("batch,queries,keys", [(0, 5, 5), (2, 0, 5), (2, 5, 0), (0, 0, 0)])
def test_nothing_to_attend(N, batch, queries, keys):
    t = inputs(batch, queries, keys, 2, 1, 16, 141)
    table, buckets = rand((2, 3), 142, F32), torch.zeros(5, dtype=torch.int32)
    o, gq, gk, gv, gt = run(N, *t, table, None, buckets)
    assert o.shape == t[0].shape and not o.any() and not gq.any() and gk.shape == t[1].shape and not gk.any() and not gv.any() and not gt.any()
    assert not any(x.any() for x in run(N, *t)[:4])


def test_gradients_that_are_wanted(N):
    """Each by itself: the bits of all together."""
    q, k, v, g = inputs(2, 70, 90, 2, 1, 32, 151)
    table, buckets = rand((2, 9), 152, F32), torch.arange(161, dtype=torch.int32) % 9
    every = run(N, q, k, v, g, table, None, buckets)[1:]
    for i in range(4):
        leaves = [t.cuda().requires_grad_(j == i) for j, t in enumerate((q, k, v, table))]
        got, = torch.autograd.grad(N.attention(*leaves[:3], table=leaves[3], buckets=buckets.cuda()), leaves[i], g.cuda())
        assert torch.equal(got, every[i])


@pytest.mark.parametrize("size", [1e-30, 1e-9, 1e6, 1e25])
def test_values_and_gradients_of_any_size(N, size):
    """What o's rounding leaves is kept for numbers of every size: the gradients are as good as for ordinary ones."""
    q, k, v, g = inputs(1, 130, 200, 2, 2, 64, 231)
    v, g = (v.double() * size).to(BF16), (g.double() / size).to(BF16)
    table, buckets = rand((2, 9), 232, F32), torch.arange(329, dtype=torch.int32) % 9
    got, r = run(N, q, k, v, g, table, None, buckets), R.Attention(q, k, v, g, None, table, buckets)
    check(got, r)
    assert (got[4].cpu().double() - r.grad_table).norm() <= 1e-5 * r.grad_table.norm()


def test_buckets_beyond_the_tables_ends(N):
    """They take its ends', and positions may be given for queries or keys alone."""
    t = inputs(1, 70, 90, 2, 2, 64, 241)
    buckets = torch.arange(159, dtype=torch.int32) - 40
    buckets[::7] = torch.iinfo(torch.int32).max
    buckets[1::7] = torch.iinfo(torch.int32).min
    table = rand((2, 60), 242, F32)
    places_ = torch.arange(90, dtype=torch.int32).flip(0)
    for positions in (None, (None, places_), (places_[:70].contiguous(), None)):
        check(run(N, *t, table, None, buckets, positions), R.Attention(*t, None, table, buckets, positions))


def test_keys_and_values_with_a_common_part(N):
    """delta = grad.o has neither o's rounding nor the probabilities': those, alike for all of a query's keys, would add up along the common part.  What is left is
    the rounding of ds, which is as large for a key's common part as for its own, so 2^-8 of (1 + common part) of the norm at most; it was up to 0.34."""
    for common in (1.0, 4.0):
        q, k, v, g = (rand((1, 512, 2, 64), 221 + i) for i in range(4))
        k, v = (t + common * rand((1, 1, 2, 64), 225 + i) for i, t in enumerate((k, v)))
        r, got = R.Attention(q, k, v, g), run(N, q, k, v, g)
        for name, t in zip(("o", "grad_q", "grad_k", "grad_v"), got):
            want = getattr(r, name)
            assert (t.cpu().double() - want).norm() <= R.HALF * (1 + common) * want.norm(), name


# ---- as a program uses it ----


def test_saved_tensors_are_not_packed(N):
    """Within keep_in_8_bits the same gradients: the probabilities are formed again from what made the statistics."""
    from paper_2307_05801_amd import activations as A
    q, k, v, g = (t.cuda() for t in inputs(2, 400, 400, 4, 4, 64, 161))
    table, buckets = rand((4, 799), 162, F32).cuda(), torch.arange(799, dtype=torch.int32).cuda()
    leaves = [t.requires_grad_(True) for t in (q, k, v, table)]

    def step():
        x = leaves[0] * 1.0                                         # no leaf
        return torch.autograd.grad(N.attention(x, *leaves[1:3], table=leaves[3] * 1.0, buckets=buckets), leaves, g)

    want = step()
    with A.keep_in_8_bits(min_values=1):
        got = step()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    with torch.autograd.graph.save_on_cpu():                        # comes back laid out anew
        got = step()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_what_is_kept_is_freed_and_watched(N):
    q, k, v, _ = (t.cuda() for t in inputs(2, 300, 300, 4, 4, 64, 171))
    gc.collect()
    gc.disable()
    try:
        before = torch.cuda.memory_allocated()
        for turn in range(3):
            o = N.attention(q.requires_grad_(True), k, v)           # its backward pass never runs
            del o
        assert torch.cuda.memory_allocated() == before
    finally:
        gc.enable()
    x = q.detach() * 1.0
    o = N.attention(x.requires_grad_(True), k, v)
    with torch.no_grad():
        k.mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        o.sum().backward()


def test_the_same_call_gives_the_same_bits(N):
    t = inputs(4, 500, 500, 4, 2, 64, 181)
    table, buckets = rand((4, 27), 182, F32), torch.arange(999, dtype=torch.int32) // 37
    want = run(N, *t, table, None, buckets)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(run(N, *t, table, None, buckets), want))


def test_another_stream_and_graph_replays(N):
    """Two captured steps that share nothing, replayed in turn with other inputs and eager work between."""
    q, k, v, g = (t.cuda() for t in inputs(2, 300, 300, 2, 2, 64, 191))
    table, buckets = rand((2, 599), 192, F32).cuda(), torch.arange(599, dtype=torch.int32).cuda()
    mask = masks(2, 300, "scattered").cuda()

    def step(q, k, v, g, table):
        leaves = [t.detach().requires_grad_(True) for t in (q, k, v, table)]
        o = N.attention(*leaves[:3], table=leaves[3], buckets=buckets, mask=mask)
        return [o.detach(), *torch.autograd.grad(o, leaves, g)]

    want = step(q, k, v, g, table)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = step(q, k, v, g, table)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del got
    places_, graphs = [[t.clone() for t in (q, k, v, g, table)] for _ in range(2)], []
    for p in places_:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step(*p)
        graphs.append((graph, out))
    for turn in range(4):
        graph, out = graphs[turn % 2]
        new = [t + 0.01 * turn for t in (q, k, v, g, table)]
        new = [n.to(t.dtype) for n, t in zip(new, (q, k, v, g, table))]
        for at, n in zip(places_[turn % 2], new):
            at.copy_(n)
        for t in out:
            t.zero_()
        graph.replay()
        want = step(*new)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), turn


def test_refusals(N):
    x = torch.zeros(2, 5, 4, 16, dtype=BF16, device="cuda")
    table, buckets = torch.zeros(4, 3, device="cuda"), torch.zeros(9, dtype=torch.int32, device="cuda")
    mask = torch.ones(2, 5, dtype=torch.bool, device="cuda")
    bad = [
        dict(q=x.float()), dict(q=x[0]), dict(q=x.half()), dict(k=x[:1]), dict(k=x[..., :8]), dict(v=x[:, :4]), dict(k=x[:, :, :3], v=x[:, :, :3]), dict(k=x.cpu()),
        dict(q=x.transpose(2, 3)), dict(q=torch._neg_view(x)), dict(q=torch.zeros(2, 5, 4, 129, dtype=BF16, device="cuda")),
        dict(mask=mask[:, :4]), dict(mask=mask.int()), dict(mask=mask.cpu()), dict(mask=mask.t().contiguous().t()), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")),
        dict(table=table), dict(buckets=buckets), dict(positions=buckets[:5]), dict(table=table[:3], buckets=buckets), dict(table=table.double(), buckets=buckets),
        dict(table=table[:, :0], buckets=buckets), dict(table=torch.zeros(4, 4097, device="cuda"), buckets=buckets), dict(table=table, buckets=buckets.long()), dict(table=table, buckets=buckets[:0]),
        dict(table=table, buckets=buckets[::2]), dict(table=table, buckets=buckets.cpu()), dict(table=table, buckets=buckets, positions=buckets[:4]),
        dict(table=table, buckets=buckets, positions=(buckets[:5],)), dict(table=table, buckets=buckets, positions=(buckets[:5], buckets[:4])), dict(table=table.t().contiguous().t(), buckets=buckets),
    ]
    good = dict(q=x, k=x, v=x)
    N.attention(**good, table=table, buckets=buckets, positions=buckets[:5], mask=mask)
    for change in bad:
        with pytest.raises(ValueError):
            N.attention(**{**good, **change})


def test_many_queries_and_keys(N):
    """Far more than a tile: 4099 by 4099, rows of both ends against the definition."""
    n, width = 4099, 64
    q, k, v, g = (t.cuda() for t in inputs(1, n, n, 1, 1, width, 201))
    o, gq, gk, gv, _ = run(N, q, k, v, g)
    rows = torch.tensor([0, 1, 63, 64, 2047, 4095, 4096, 4098])
    x = (q.double()[0, :, 0] @ k.double()[0, :, 0].T) / 8.0
    p = torch.softmax(x, 1)
    dp = g.double()[0, :, 0] @ v.double()[0, :, 0].T
    ds = p * (dp - (p * dp).sum(1, keepdim=True))
    for name, got, want in (("o", o, p @ v.double()[0, :, 0]), ("grad_q", gq, ds @ k.double()[0, :, 0] / 8.0), ("grad_k", gk, ds.T @ q.double()[0, :, 0] / 8.0),
                            ("grad_v", gv, p.T @ g.double()[0, :, 0])):
        got, want = got[0, rows.cuda(), 0].double(), want[rows.cuda()]
        # three roundings of half a step at most, of values whose errors do not depend on one another
        assert (got - want).norm() <= 3 ** 0.5 * R.HALF * want.norm(), name


def test_one_of_two_devices_is_enough(N):
    """The tensors' device is what counts: here the current one, as there is no other."""
    t = [x.cuda() for x in inputs(1, 5, 5, 1, 1, 8, 211)]
    with torch.cuda.device(0):
        assert N.attention(*t[:3]).device == t[0].device


@pytest.mark.parametrize("batch,queries,keys", [(2, 0, 300), (1, 0, 5), (0, 5, 5), (2, 0, 0)])
@pytest.mark.parametrize("width", [1, 16, 49])
def test_no_queries_and_a_table_that_wants_no_gradient(N, batch, queries, keys, width):
    """Zeros for keys and values, also where the table is frozen or there is none; each by itself too."""
    q, k, v, _ = (t.cuda() for t in inputs(batch, queries, keys, 2, 1, width, 143))
    table, buckets = rand((2, 9), 144, F32).cuda(), torch.arange(9, dtype=torch.int32).cuda()
    for bias in (dict(), dict(table=table, buckets=buckets)):
        for wanted in ((k, v), (k,), (v,), (q, k)):
            leaves = [t.detach().requires_grad_(any(t is w for w in wanted)) for t in (q, k, v)]
            o = N.attention(*leaves, **bias)
            room = torch.full((1 << 16,), 7.0, device="cuda")       # what memory held before
            del room
            got = torch.autograd.grad(o, [t for t in leaves if t.requires_grad], torch.zeros_like(o))
            assert all(t.shape == w.shape and not t.any() for t, w in zip(got, wanted))


@pytest.mark.parametrize("width", [8, 32, 49, 64, 96, 128])
@pytest.mark.parametrize("seed", [151, 251])
def test_the_gradient_of_keys_does_not_depend_on_what_else_is_wanted(N, width, seed):
    """Its bits, of 17 million pairs: delta is one sum whichever kernel forms it, and a last bit of it that differs shows in one of 2^16 roundings of ds."""
    q, k, v, g = (t.cuda() for t in inputs(4, 1024, 1024, 4, 4, width, seed))
    every = run(N, q, k, v, g)
    leaves = [t.detach().requires_grad_(i > 0) for i, t in enumerate((q, k, v))]
    got = torch.autograd.grad(N.attention(*leaves), leaves[1:], g)
    assert torch.equal(got[0], every[2]) and torch.equal(got[1], every[3])


@pytest.mark.parametrize("what", [float("nan"), float("inf")])
@pytest.mark.parametrize("kind", ["apart", "alike", "anywhere", "anywhere many", "beyond"])
@pytest.mark.parametrize("width", [32, 64, 128])
def test_what_is_not_a_number_reaches_its_own_buckets(N, kind, what, width):
    """A query or a gradient that is not finite: the table's gradient is not a number in the buckets of the query's pairs, in its head, and what it is without it in all others."""
    n = 300
    q, k, v, g = inputs(2, n, n, 2, 2, width, 251)
    positions = None
    if kind == "apart":
        buckets = torch.arange(2 * n - 1, dtype=torch.int32)
    elif kind == "alike":
        buckets = torch.arange(2 * n - 1, dtype=torch.int32) // 3
    elif kind == "beyond":
        buckets = torch.arange(201, dtype=torch.int32)
    else:
        positions = torch.randperm(n, generator=torch.Generator().manual_seed(252)).to(torch.int32)
        buckets = torch.arange(2 * n - 1, dtype=torch.int32) * (6 if "many" in kind else 1)
    table = rand((2, int(buckets.max()) + 1), 253, F32)
    (q if what != what else g)[1, 5 if kind == "beyond" else 130, 1, 3] = what       # (130 has pairs of all differences that are not beyond an end)
    r = R.Attention(q, k, v, g, None, table, buckets, positions)
    lost = ~torch.isfinite(r.grad_table)
    assert lost[1].any() and not lost[1].all() and not lost[0].any()
    got = run(N, q, k, v, g, table, None, buckets, positions)
    assert torch.equal(~torch.isfinite(got[4].cpu()), lost)
    assert_close(got[4].cpu()[~lost], r.grad_table[~lost], r.grad_table_off[~lost], "grad_table")
    fine = torch.isfinite(r.grad_q).all(3)
    assert int((~fine).sum()) == 1
    assert torch.equal(torch.isfinite(got[1].cpu()).all(3), fine)
    assert_close(got[1].cpu()[fine], r.grad_q[fine], r.grad_q_off[fine], "grad_q")


@pytest.mark.parametrize("end", [-(1 << 30), 1 << 30, -(1 << 29) - 150, (1 << 29) - 150])
@pytest.mark.parametrize("order", ["one after the other", "rising", "any"])
@pytest.mark.parametrize("width", [32, 128])
def test_positions_near_their_ends(N, end, order, width):
    """Up to 2^30 either way, side by side so that a tile's differences are read from shared memory: four times a position passes 31 bits, the address does not."""
    n = 300
    t = inputs(2, n, n, 2, 1, width, 261)
    step = {"one after the other": torch.arange(n), "rising": torch.arange(n) // 3 * 4 + torch.arange(n) % 3, "any": torch.randperm(n, generator=torch.Generator().manual_seed(262))}[order]
    places_ = (end + step - (int(step.max()) if end == 1 << 30 else 0)).to(torch.int32)
    assert -(1 << 30) <= int(places_.min()) and int(places_.max()) <= 1 << 30
    buckets = torch.arange(2 * int(step.max()) + 1, dtype=torch.int32)
    table = rand((2, len(buckets)), 263, F32)
    check(run(N, *t, table, None, buckets, places_), R.Attention(*t, None, table, buckets, places_))


def test_negated_positions_and_buckets_are_refused(N):
    x, table = torch.zeros(1, 5, 2, 16, dtype=BF16, device="cuda"), torch.zeros(2, 9, device="cuda")
    t = torch.arange(9, dtype=torch.int32, device="cuda")
    N.attention(x, x, x, table=table, buckets=t, positions=t[:5])
    for bad in (dict(buckets=torch._neg_view(t)), dict(buckets=t, positions=torch._neg_view(t)[:5]), dict(buckets=t, positions=(None, torch._neg_view(t[:5])))):
        with pytest.raises(ValueError):
            N.attention(x, x, x, table=table, **bad)


@pytest.mark.parametrize("kind", ["line", "few", "even", "anywhere", "anywhere many", "far"])
@pytest.mark.parametrize("batch,queries,keys,heads,kv_heads,width", [(1, 1, 20, 8, 2, 100), (1, 4, 837, 8, 2, 49), (2, 200, 130, 2, 2, 64)])
def test_small_sums_of_the_tables_gradient(N, kind, batch, queries, keys, heads, kv_heads, width):
    """Probabilities nearly all on one key, so that buckets' sums differ by many powers of ten: besides the roundings of the scores each pair's ds is held to 2^-46 of its tile's largest: as
    multiples, cut off, of 2^-46 of the power of two that is no more than that."""
    t = inputs(batch, queries, keys, heads, kv_heads, width, 271)
    positions, buckets, many = places(queries, keys, kind)
    table = rand((heads, many), 273, F32)
    r = R.Attention(*t, None, table, buckets, positions, 0.5)
    qp, kp = positions if positions is not None else (torch.arange(queries), torch.arange(keys))
    bias, index = R.bias_of(table, buckets, qp, kp)
    _, _, p = R.attention(*t[:3], None, bias, 0.5)
    group = heads // kv_heads
    dp = t[3].double().transpose(1, 2) @ t[2].double().transpose(1, 2).repeat_interleave(group, 1).transpose(2, 3)
    ds = p * (dp - (p * dp).sum(3, keepdim=True))
    pairs = torch.bincount(index.flatten(), minlength=many) * batch
    got = run(N, *t, table, None, buckets, positions, 0.5)
    assert_close(got[4], r.grad_table, r.grad_table_off + pairs * 2.0 ** -46 * ds.abs().max(), "grad_table")


@pytest.mark.parametrize("batch,heads,width,shape,near,codes", [(6, 3, 64, (1, 8), 2, 4), (17, 4, 128, (29, 1), 3, 6), (57, 1, 128, (2, 9), 2, 3), (22, 4, 64, (3, 1, 8), 1, 3), (57, 6, 11, (23, 3), 2, 4)])
def test_the_tables_gradient_is_that_of_32_bits(N, batch, heads, width, shape, near, codes):
    """Few patches, whose sums hide nothing: of a pair's ds some eight roundings of 2^-24 each (its score's, the exponential's, delta's, dp's), 2^-21 of the norm in all; with probabilities of 16 bits in delta
    it was 2^-20 and more."""
    positions, buckets = N.relative_buckets(shape, near, codes, device="cpu")
    n, many = len(positions), (2 * codes - 1) ** len(shape)
    t = [rand((batch, n, heads, width), 281 + i) for i in range(4)]
    table = rand((heads, many), 285, F32, 0.5)
    got, r = run(N, *t, table, None, buckets, positions), R.Attention(*t, None, table, buckets, positions)
    assert (got[4].cpu().double() - r.grad_table).norm() <= 2.0 ** -21 * r.grad_table.norm()
