"""Operators of networks that are trained through the projector, beside those in 8 bits: what is measured.

"attend": attention over the patches of a volume (or of slices), forward, or a training step with its gradients.  Tensors are bfloat16 [batch,
patches, heads, width]; heads may share keys and values; a mask leaves out patches of a batch's items (outside the field of view).  With
`grid` the patches lie on a grid and every pair of them takes a learned number by the bucket of their relative position, which is added to the pair's
product.
"group": group norm with an activation, channels last, [batch, voxels, channels], forward or a training step.

Relative positions: patch (z, y, x) of a grid has the position ((z (2 ny - 1)) + y) (2 nx - 1) + x, so that differences of positions tell
differences of places apart; `buckets` holds the bucket of every difference, zero in the middle.  On an axis a distance d has a code: d below
`near`, then one more for each doubling, up to `codes` - 1; the two directions differ, and the bucket counts the axes' codes through.
"""
import math

import torch

own = False
DEVICE = "cuda:0"
EPS = 1e-5
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _attend(name, batch, queries, keys, heads, shared, width, grid=None, near=0, codes=0, masked=False, train=True):
    return dict(name=name, op="attend", batch=batch, queries=queries, keys=keys, heads=heads, kv_heads=heads // shared, width=width, type="bf16",
                grid="" if grid is None else "x".join(map(str, grid)), near=near, codes=codes, masked=masked, train=train)


def _group(name, batch, voxels, channels, groups, type="bf16", activation="silu", train=True):
    return dict(name=name, op="group", batch=batch, voxels=voxels, channels=channels, groups=groups, type=type, activation=activation, train=train)


def listed():
    return [
        # one query over a few patches: latency
        _attend("attend_token", 1, 1, 512, 8, 1, 64, train=False),
        # sixteen learned queries that pool the 8^3 patches of a 512^3 volume, in two volumes; four heads share keys
        _attend("attend_pool", 2, 16, 262144, 8, 4, 64, train=False),
        # sixteen stacks of 211 slices, a slice a row; distances along the stack; stacks of different lengths
        _attend("attend_stack", 16, 211, 211, 2, 1, 32, grid=(211,), near=8, codes=14, masked=True),
        # eight slices of 512 x 512 in patches of 16 x 16, those outside the field of view masked
        _attend("attend_slices", 8, 1024, 1024, 4, 1, 64, grid=(32, 32), near=32, codes=32, masked=True),
        # a training batch of eight 256^3 volumes in patches of 8^3, within windows of 8^3 patches
        _attend("attend_windows", 512, 512, 512, 8, 1, 64, grid=(8, 8, 8), near=8, codes=8),
        # two volumes of 128^3 in patches of 8^3, all of a volume's patches
        _attend("attend_volumes", 2, 4096, 4096, 8, 1, 64, grid=(16, 16, 16), near=4, codes=6),
        # a volume of odd size (211 x 187 x 149) in patches of 7^3: no length or width is a multiple of 8
        _attend("attend_ragged", 1, 18414, 18414, 7, 1, 49, grid=(31, 27, 22), near=2, codes=5),
        # the patches of a whole 256^3 volume, four heads share keys: the largest
        _attend("attend_whole", 1, 32768, 32768, 8, 4, 128),
        # a patch of 16 x 16 pixels of features by itself: latency
        _group("group_patch", 1, 256, 64, 8, train=False),
        # eight slices of 256 x 256
        _group("group_slices", 8, 65536, 64, 8),
        # a volume of odd size, float32, groups of five channels, no activation
        _group("group_ragged", 1, 211 * 187 * 149, 20, 4, type="f32", activation=""),
        # eight volumes of 128^3: the largest
        _group("group_volumes", 8, 128 ** 3, 64, 8),
    ]


def draw(rng):
    def spread(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    if rng.random() < 0.35:
        size = rng.choice([1, 2, 4, 5, 7, 8, 16, 24, 32])
        groups = rng.choice([1, 2, 3, 4, 8, 16, 32])
        batch, channels = spread(1, 16), size * groups
        train = rng.random() < 0.7                             # gradients of a value or two that are normed are nothing but rounding
        voxels = min(spread(16 if train else 1, 2 ** 22), 2 ** 29 // (batch * channels))
        return {k: v for k, v in _group("", batch, voxels, channels, groups, rng.choice(["f32", "bf16", "bf16", "f16"]), rng.choice(["", "silu", "silu"]),
                                        train).items() if k != "name"}
    shared = rng.choice([1, 1, 1, 2, 4])
    heads = shared * rng.choice([1, 2, 3, 4, 8])
    width = rng.choice([32, 64, 64, 64, 128, 128, spread(8, 128), spread(8, 128)])
    train = rng.random() < 0.7
    least = 8 if train else 1                                  # (the same of a softmax over one key)
    if rng.random() < 0.6:                                     # patches on a grid
        axes = rng.choice([1, 2, 3])
        grid = tuple(spread(1, {1: 6000, 2: 100, 3: 20}[axes]) for _ in range(axes))
        if math.prod(grid) < least:
            grid = grid[1:] + (least,)
        codes = rng.randint(2, 7)
        near, queries, keys = rng.randint(1, codes), math.prod(grid), math.prod(grid)
    else:
        grid, near, codes, keys = None, 0, 0, spread(least, 16384)
        queries = keys if rng.random() < 0.5 else spread(1, 16384)
    most = 32768 * 32768 * 8 // 2
    batch = max(1, min(spread(1, 64), most // (queries * keys * heads)))
    return {k: v for k, v in _attend("", batch, queries, keys, heads, shared, width, grid, near, codes,
                                     rng.random() < 0.4, train).items() if k != "name"}


# ---- inputs -----------------------------------------------------------------------------------------------------------


def _normal(shape, kind, seed):
    return torch.randn(shape, device=DEVICE, generator=torch.Generator(device=DEVICE).manual_seed(seed), dtype=torch.float32).to(kind)


def _places(case):
    """(positions, buckets) of a grid's patches, int32."""
    sizes = [int(n) for n in case["grid"].split("x")]
    positions, buckets = torch.zeros(1, dtype=torch.int64, device=DEVICE), torch.zeros(1, dtype=torch.int64, device=DEVICE)
    for n in sizes:
        positions = (positions.unsqueeze(1) * (2 * n - 1) + torch.arange(n, device=DEVICE)).flatten()
        d = torch.arange(1 - n, n, device=DEVICE)
        code, far = d.abs().clamp(max=case["near"]), d.abs() // case["near"]
        for k in range(1, 24):
            code = code + (far >= 1 << k)
        code = torch.sign(d) * code.clamp(max=case["codes"] - 1) + case["codes"] - 1
        buckets = (buckets.unsqueeze(1) * (2 * case["codes"] - 1) + code).flatten()
    return positions.int(), buckets.int()


def prepare(case, seed):
    s = {"op": case["op"], "train": case["train"]}
    at, kind, batch = seed * 16, TYPES[case["type"]], case["batch"]
    if case["op"] == "group":
        shape, channels = (batch, case["voxels"], case["channels"]), case["channels"]
        column = torch.exp(0.5 * _normal((channels,), torch.float32, at))
        s["x"] = (_normal(shape, kind, at + 1).mul_(column.to(kind))).add_(_normal((channels,), kind, at + 2))
        s["weight"] = (1.0 + 0.2 * _normal((channels,), torch.float32, at + 3)).to(kind)
        s["bias"] = (0.2 * _normal((channels,), torch.float32, at + 4)).to(kind)
        s["groups"], s["activation"] = case["groups"], case["activation"] or None
        s["grad"] = _normal(shape, kind, at + 5) if case["train"] else None
        s["leaves"] = ("x", "weight", "bias")
    else:
        queries, keys, heads, width = case["queries"], case["keys"], case["heads"], case["width"]
        s["q"] = _normal((batch, queries, heads, width), kind, at)
        s["k"] = _normal((batch, keys, case["kv_heads"], width), kind, at + 1)
        s["v"] = _normal((batch, keys, case["kv_heads"], width), kind, at + 2)
        s["grad"] = _normal((batch, queries, heads, width), kind, at + 3) if case["train"] else None
        s["mask"] = s["table"] = s["positions"] = s["buckets"] = None
        s["leaves"] = ("q", "k", "v")
        if case["masked"]:                                     # the middle part of each item's patches; an item of many has none
            middle = torch.arange(keys, device=DEVICE).sub(0.5 * (keys - 1)).abs()
            reach = torch.rand(batch, 1, device=DEVICE, generator=torch.Generator(device=DEVICE).manual_seed(at + 5)) * 0.4 + 0.2
            if batch > 3:
                reach[batch // 2] = -1.0
            s["mask"] = middle <= reach * keys
        if case["grid"]:
            s["positions"], s["buckets"] = _places(case)
            s["sizes"] = [int(n) for n in case["grid"].split("x")]
            many = (2 * case["codes"] - 1) ** (case["grid"].count("x") + 1)
            s["table"] = 0.5 * _normal((heads, many), torch.float32, at + 4)
            s["leaves"] += ("table",)
    if case["train"]:
        for name in s["leaves"]:
            s[name].requires_grad_(True)
    return s


# ---- the plain form ---------------------------------------------------------------------------------------------------


def _heads_first(t, shared=1):
    """[batch, rows, heads, width] as float32 [batch, heads, rows, width], each head `shared` times."""
    t = t.detach().float().transpose(1, 2)
    return t.repeat_interleave(shared, 1).contiguous() if shared > 1 else t.contiguous()


def _rows_first(t, kind, shared=1):
    """And back, with what `shared` heads have added up."""
    if shared > 1:
        t = t.unflatten(1, (-1, shared)).sum(2)
    return t.transpose(1, 2).to(kind).contiguous()


def _plain_attention(s):
    kind, width = s["q"].dtype, s["q"].shape[-1]
    shared, scale = s["q"].shape[2] // s["k"].shape[2], 1.0 / math.sqrt(width)
    q, k, v = _heads_first(s["q"]), _heads_first(s["k"], shared), _heads_first(s["v"], shared)
    p = torch.matmul(q, k.transpose(2, 3)).mul_(scale)
    index = None
    if s["table"] is not None:
        offset = s["positions"].long().unsqueeze(0) - s["positions"].long().unsqueeze(1) + s["buckets"].numel() // 2
        index = s["buckets"].long()[offset]
        p += s["table"].detach()[:, index]
        del offset
    if s["mask"] is not None:
        p.masked_fill_(~s["mask"][:, None, None, :], -math.inf)
    largest = p.amax(3, keepdim=True)
    p.sub_(torch.where(largest == -math.inf, 0.0, largest)).exp_()
    total = p.sum(3, keepdim=True)
    p.div_(torch.where(total == 0.0, 1.0, total))
    o = torch.matmul(p, v)
    if not s["train"]:
        return _rows_first(o, kind)
    g = _heads_first(s["grad"])
    result = {"o": _rows_first(o, kind), "grad_v": _rows_first(torch.matmul(p.transpose(2, 3), g), kind, shared)}
    ds = torch.matmul(g, v.transpose(2, 3)).sub_((g * o).sum(3, keepdim=True)).mul_(p)
    del p
    result["grad_q"] = _rows_first(torch.matmul(ds, k).mul_(scale), kind)
    result["grad_k"] = _rows_first(torch.matmul(ds.transpose(2, 3), q).mul_(scale), kind, shared)
    if index is not None:
        del index
        table = torch.zeros(s["table"].shape, dtype=torch.float64, device=DEVICE)
        result["grad_table"] = table.index_add_(1, s["buckets"], _by_offset(ds.sum(0).double(), s["sizes"])).float()
    return result


def _by_offset(t, sizes):
    """[heads, patches, patches] of a grid's pairs, added up by the difference of their positions: [heads, differences]."""
    t = t.unsqueeze(3)
    for n in reversed(sizes):                                  # the last axis first: [heads, rest, n, rest, n, done]
        heads, rest, done = t.shape[0], t.shape[1] // n, t.shape[3]
        t = t.reshape(heads, rest, n, rest, n, done).permute(0, 1, 3, 5, 2, 4)
        # with the queries in reverse, rows of 2 n read as rows of 2 n - 1 have every difference in a column
        t = torch.nn.functional.pad(t.flip(4), (0, n)).flatten(4)[..., :n * (2 * n - 1)].unflatten(4, (n, 2 * n - 1)).sum(4)
        t = t.transpose(3, 4).flatten(3)
    return t.view(t.shape[0], -1)


def _plain_group(s):
    x, groups, kind = s["x"].detach().float(), s["groups"], s["x"].dtype
    batch, voxels, channels = x.shape
    x = x.view(batch, voxels, groups, channels // groups)
    weight, bias = s["weight"].detach().float().view(groups, -1), s["bias"].detach().float().view(groups, -1)
    mean = x.mean((1, 3), dtype=torch.float64, keepdim=True).float()
    x = x - mean
    rstd = torch.rsqrt(x.square().mean((1, 3), keepdim=True) + EPS)
    x.mul_(rstd)
    u = x * weight + bias
    gate = torch.sigmoid(u) if s["activation"] else None
    y = u if gate is None else u * gate
    y = y.to(kind).view(batch, voxels, channels)
    if not s["train"]:
        return y
    du = s["grad"].float().view_as(x)
    if gate is not None:
        du = du * (gate * (1.0 + u * (1.0 - gate)))
    result = {"y": y, "grad_bias": du.sum((0, 1), dtype=torch.float64).flatten().to(kind),
              "grad_weight": (du * x).sum((0, 1), dtype=torch.float64).flatten().to(kind)}
    du = du * weight
    dx = (du - du.mean((1, 3), keepdim=True) - x * (du * x).mean((1, 3), keepdim=True)).mul_(rstd)
    return result | {"grad_x": dx.to(kind).view(batch, voxels, channels)}


def _run_plain(s):
    with torch.no_grad():
        return _plain_group(s) if s["op"] == "group" else _plain_attention(s)


# ---- the framework's operators ----------------------------------------------------------------------------------------


def _run_own(s):
    from paper_2307_05801_amd import networks as N
    if s["op"] == "group":
        name = "y"
        y = N.group_norm(s["x"], s["groups"], s["weight"], s["bias"], activation=s["activation"], eps=EPS)
    else:
        name = "o"
        y = N.attention(s["q"], s["k"], s["v"], mask=s["mask"], table=s["table"], buckets=s["buckets"], positions=s["positions"])
    if not s["train"]:
        return y
    grads = torch.autograd.grad(y, [s[n] for n in s["leaves"]], s["grad"])
    return {name: y.detach()} | {"grad_" + n: g for n, g in zip(s["leaves"], grads)}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------------


def work(case):
    size = TYPES[case["type"]].itemsize
    if case["op"] == "group":                      # x read, y written; a step: the gradient read, x's written
        n = case["batch"] * case["voxels"] * case["channels"]
        return {"bytes": n * size * (4 if case["train"] else 2), "flops": n * (30 if case["train"] else 12)}
    pairs = case["batch"] * case["heads"] * case["queries"] * case["keys"]
    rows = case["batch"] * case["queries"] * case["heads"] * case["width"] * size
    kept = case["batch"] * case["keys"] * case["kv_heads"] * case["width"] * size
    if not case["train"]:                          # q, k, v; o: two products
        return {"bytes": 2 * rows + 2 * kept, "flops": 4 * pairs * case["width"]}
    # q, k, v, the gradient of o; o, the gradients of q, k, v: two products and five
    return {"bytes": 4 * rows + 4 * kept, "flops": 14 * pairs * case["width"]}


# ---- the definition in 64 bits ----------------------------------------------------------------------------------------


def _exact_attention(s):
    q, k, v = (s[n].detach().double() for n in ("q", "k", "v"))
    batch, queries, heads, width = q.shape
    keys, shared = k.shape[1], heads // k.shape[2]
    bucket = None
    if s["table"] is not None:
        where = s["positions"].long()
        bucket = s["buckets"].long()[where[None, :] - where[:, None] + (s["buckets"].numel() - 1) // 2]
    o, gq, gk, gv = torch.zeros_like(q), torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(v)
    gt = None if bucket is None else torch.zeros(s["table"].shape, dtype=torch.float64, device=DEVICE)
    step = max(1, 2 ** 28 // (queries * keys))                  # items at once: 2 GiB an array
    for h in range(heads):
        for b in range(0, batch, step):
            i, j = slice(b, b + step), h // shared
            qh, kh, vh = q[i, :, h], k[i, :, j], v[i, :, j]
            logits = torch.matmul(qh, kh.mT) / math.sqrt(width)
            if bucket is not None:
                logits = logits + s["table"].detach()[h].double()[bucket]
            if s["mask"] is not None:
                logits = torch.where(s["mask"][i, None, :], logits, -math.inf)
            p = torch.softmax(logits, 2).nan_to_num(nan=0.0)      # rows without a key
            del logits
            o[i, :, h] = torch.matmul(p, vh)
            if not s["train"]:
                continue
            g = s["grad"][i, :, h].double()
            dp = torch.matmul(g, vh.mT)
            gv[i, :, j] += torch.matmul(p.mT, g)
            dp -= (p * dp).sum(2, keepdim=True)
            dp *= p
            del p
            gq[i, :, h] = torch.matmul(dp, kh) / math.sqrt(width)
            gk[i, :, j] += torch.matmul(dp.mT, qh) / math.sqrt(width)
            if gt is not None:
                every = dp.sum(0)
                part = torch.zeros(queries, gt.shape[1], dtype=torch.float64, device=DEVICE)
                gt[h] += part.scatter_add_(1, bucket, every).sum(0)
    if not s["train"]:
        return o
    result = {"o": o, "grad_q": gq, "grad_k": gk, "grad_v": gv}
    return result if gt is None else result | {"grad_table": gt}


def _exact_group(s):
    x, w, b = s["x"].detach(), s["weight"].detach().double(), s["bias"].detach().double()
    batch, voxels, channels = x.shape
    groups, m = s["groups"], voxels * (channels // s["groups"])
    y, gx = torch.empty(x.shape, dtype=torch.float64, device=DEVICE), torch.empty(x.shape, dtype=torch.float64, device=DEVICE)
    gw, gb = torch.zeros_like(w), torch.zeros_like(b)

    def by_group(t):                               # channels' sums to their groups', for every channel
        return t.view(groups, -1).sum(1).repeat_interleave(channels // groups)

    for n in range(batch):
        v = x[n].double()
        mean = by_group(v.sum(0)) / m
        v = v - mean
        inverse = 1.0 / torch.sqrt(by_group((v * v).sum(0)) / m + EPS)
        v = v * inverse
        u = v * w + b
        if s["activation"]:
            q = 1.0 / (1.0 + torch.exp(-u))
            y[n] = u * q
            slope = q + u * q * (1.0 - q)
        else:
            y[n], slope = u, 1.0
        if s["train"]:
            d = s["grad"][n].double() * slope
            one, two = d.sum(0), (d * v).sum(0)
            gb += one
            gw += two
            gx[n] = inverse * (d * w - by_group(one * w) / m - v * by_group(two * w) / m)
    return {"y": y, "grad_x": gx, "grad_weight": gw, "grad_bias": gb} if s["train"] else y


def exact(case, seed):
    s = prepare(case, seed)
    with torch.no_grad():
        return _exact_group(s) if case["op"] == "group" else _exact_attention(s)
