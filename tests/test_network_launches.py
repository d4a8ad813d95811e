"""What attention and group norm launch, on the CPU (tests/launches.py): how many blocks, of which kernels."""
import pytest

from launches import kernels, record
from paper_2307_05801_amd import binding as B

P = 0x100000


@pytest.fixture(scope="module")
def pack():
    from paper_2307_05801_amd import networks as N
    return lambda *d: N._DESC.pack(*d)


def group(items, voxels, channels, groups, type=1, row=None):
    row = channels if row is None else row
    return "leap_group_norm", (P, type, voxels * row, row, P, P, 0, items, voxels, channels, groups, 1e-5, 2, P, P, P, 0)


def group_backward(items, voxels, channels, groups, type=1, row=None):
    row = channels if row is None else row
    return "leap_group_norm_backward", (P, voxels * row, row, P, type, voxels * row, row, P, P, 0, P, items, voxels, channels, groups, 2, P, P, P, P, 0)


SIZES = [(1, 1, 1, 1), (1, 256, 64, 8), (8, 65536, 64, 8), (8, 1 << 21, 64, 8), (1, 211 * 187 * 149, 20, 4), (1 << 20, 8, 8, 2), (1, 1 << 30, 8, 8), (3, 5, 1 << 20, 1 << 10), (1 << 20, 1, 2047, 1), (1, 1 << 30, 5, 1)]


def test_a_launch_of_group_norm_has_fewer_than_2_32_threads():
    calls = [f(*s) for s in SIZES for f in (group, group_backward)] + [group(2, 1000, 20, 4, row=25), group_backward(2, 1000, 20, 4, row=25)]
    for (name, arguments), (status, launches) in zip(calls, record(calls)):
        assert status == B.LEAP_OK, (name, arguments)
        assert launches[0].kernel in (("k_group_moments", "k_group_small") if name == "leap_group_norm" else ("k_group_sums",))
        for launch in launches:
            across, along, deep = launch.blocks
            assert 0 < across * launch.threads < 1 << 32 and along < 1 << 16 and deep == 1, (name, launch)


def test_items_of_group_norm_are_read_again_before_the_next():
    """Large ones one by one, each read for its sums and again; small ones together."""
    (_, one), (_, many) = record([group(3, 1 << 21, 64, 8), group(3, 1 << 14, 64, 8)])
    assert [launch.kernel for launch in one] == ["k_group_moments", "k_group_stats", "k_group_apply"] * 3
    assert [launch.kernel for launch in many] == ["k_group_moments", "k_group_stats", "k_group_apply"]


@pytest.mark.parametrize("voxels,channels,row", [(1 << 30, 8, None), (1 << 33, 8, None), (1 << 31, 64, None), (1 << 30, 63, None), (1 << 31, 20, 25), (1 << 22, 1 << 13, None), (1 << 20, 1 << 20, None)])
def test_a_thread_of_group_norm_sums_no_more_than_512_values_of_a_channel(voxels, channels, row):
    """As floats: however many there are.  A block has 256 threads, and as many of them have one channel as there is room for a period's eights."""
    for call in (group(1, voxels, channels, 1, row=row), group_backward(1, voxels, channels, 1, row=row)):
        (status, launches), = record([call])
        assert status == B.LEAP_OK
        rows = 1 if row else {0: 1, 1: 8, 2: 4, 3: 8, 4: 2, 5: 8, 6: 4, 7: 8}[channels % 8]
        eights = -(-channels * rows // 8)
        segments, turns = -(-eights // 256), max(1, 256 // eights)
        for launch in launches:
            if launch.kernel in ("k_group_moments", "k_group_apply", "k_group_sums", "k_group_grad"):
                strips = launch.blocks[0] // segments
                assert -(-voxels // rows) <= strips * turns * 512, launch


def test_few_values_take_one_launch():
    small = [group(1, 256, 64, 8), group(1, 16384 // 8, 64, 8), group(1, 1, 16384, 1), group(64, 256, 64, 8, row=70)]
    large = [group(1, 16384 // 8 + 1, 64, 8), group(1, 256, 60, 8 - 2), group(65, 256, 64, 8), group(1, 2, 16384, 1)]
    assert all([launch.kernel for launch in launches] == ["k_group_small"] for _, launches in record(small))
    assert all(launches[0].kernel == "k_group_moments" for _, launches in record(large))
    (status, launches), = record([(group(1, 256, 64, 8)[0], group(1, 256, 64, 8)[1][:15] + (None, 0))])
    assert status == B.LEAP_OK and launches[0].blocks[0] == 8              # needs no workspace


def test_every_kernel_of_group_norm_is_reached():
    calls = [f(2, 1000, channels, 4, type, row) for f in (group, group_backward) for type in (0, 1, 2) for channels, row in ((20, 25), (20, 20), (32, 32))]
    calls += [(name, a[:12] + (activation,) + a[13:] if name == "leap_group_norm" else a[:15] + (activation,) + a[16:]) for name, a in calls for activation in (0, 1)]
    calls += [(name, a[:9] + (a[4],) + a[10:]) for name, a in calls if name == "leap_group_norm_backward"]                # weights of x's type
    taken = {(launch.kernel, launch.parameters) for _, launches in record(calls) for launch in launches if launch.kernel.startswith("k_group")}
    assert taken == {k for k in kernels() if k[0].startswith("k_group")}


# ---- attention: its description goes as bytes, which launches.record does not hand on ----

RECORD = """
import ctypes as C, json, struct, sys
sys.path[:0] = [{root!r}, {here!r}]
import launches
recorder = C.CDLL(launches.LIB, mode=C.RTLD_GLOBAL)
from paper_2307_05801_amd import binding as B
lib, room, out = B.load_activations(), C.create_string_buffer(1 << 20), []
for name, desc, arguments in json.load(sys.stdin):
    status = getattr(lib, name)(struct.pack("<18q5Qif", *desc), *arguments)
    recorder.recorded_launches(room, len(room))
    out.append((status, room.value.decode()))
print(json.dumps(out))
"""


def record_attention(calls):
    import json
    import os
    import subprocess
    import sys

    import launches
    launches._build()
    here = os.path.dirname(os.path.abspath(__file__))
    done = subprocess.run([sys.executable, "-c", RECORD.format(root=os.path.dirname(here), here=here)], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr
    out = []
    for status, text in json.loads(done.stdout):
        lines = [line.split() for line in text.splitlines()]
        out.append((status, [launches.Launch(*launches._name(n), tuple(map(int, s[:3])), int(s[3]) * int(s[4]) * int(s[5])) for n, *s in lines]))
    return out


def attention(batch, queries, keys, heads, kv_heads, width, buckets=0, offsets=1, base=P, stats=True):
    desc = [batch, queries, keys, heads, kv_heads, width] + [queries * heads * width, heads * width, width] + [keys * kv_heads * width, kv_heads * width, width] * 2
    desc += [0, offsets, buckets, 0, P if buckets else 0, P, 0, 0, 0, 0.125]
    kept = P if stats else 0
    forward = ("leap_attention", desc, [base, base, base, P, kept, kept, P, 0])
    return forward, ("leap_attention_backward", desc, [base, queries * heads * width, heads * width, width, base, base, base, P, P, P, P, P, P, P if buckets else 0, P, 0])


def test_launches_of_attention():
    """Queries, keys and parts are covered, and few of anything still fills blocks."""
    sizes = [(1, 1, 512, 8, 8, 64), (2, 16, 262144, 8, 2, 64), (512, 512, 512, 8, 8, 64, 3375, 3375), (1, 32768, 32768, 8, 2, 128), (1, 1, 1, 1, 1, 1), (1, 33, 100, 4, 1, 32), (1, 64, 100, 4, 1, 32),
             (3, 129, 70, 6, 2, 49, 4096, 1 << 20), ((1 << 20) - 1, 1, 1, 1, 1, 8), (1, 1 << 30, 1, 1, 1, 8), (1, 1, 1 << 30, 1, 1, 8)]
    calls = [c for s in sizes for c in attention(*s)]
    for (name, desc, _), (status, launches) in zip(calls, record_attention(calls)):
        batch, queries, keys, heads, kv_heads = desc[:5]
        assert status == B.LEAP_OK, (name, desc)
        by = {launch.kernel: launch for launch in launches}
        for launch in launches:
            across, along, deep = launch.blocks
            assert 0 < across * launch.threads < 1 << 32 and along < 1 << 16 and deep == 1, (name, launch)
        if name == "leap_attention":
            units = [batch * (heads // abreast) * -(-queries // (128 // abreast)) for abreast in (1, 2, 4)]
            assert any(by["k_attention"].blocks[0] % u == 0 for u in units)
            assert ("k_join" in by) == (by["k_attention"].blocks[0] not in units)
        else:
            assert by["k_grad_key"].blocks[0] == batch * kv_heads * -(-keys // 128)
            if desc[17]:
                assert by["k_grad_query"].blocks[0] <= 2048 and by["k_join_table"].blocks[1] == heads
            else:
                assert by["k_grad_query"].blocks[0] == batch * heads * -(-queries // 128)
    status, launches = record_attention([attention(2, 16, 262144, 8, 2, 64)[0]])[0]
    assert launches[0].blocks[0] == 512                       # four heads abreast, 128 parts of 2048 keys


def test_rows_that_are_no_multiples_of_16_bytes_are_laid_out():
    """Keys and values where more than 512 queries read them; and, backward, queries and gradients where more than 512 keys do."""
    for queries, keys, forward, backward in ((513, 9, 2, 2), (9, 513, 0, 2), (513, 513, 2, 4), (512, 512, 0, 0)):
        got = [sum(launch.kernel == "k_lay_rows" for launch in launches) for _, launches in record_attention(attention(1, queries, keys, 2, 1, 49))]
        assert got == [forward, backward], (queries, keys)
        assert not any(launch.kernel == "k_lay_rows" for _, launches in record_attention(attention(1, queries, keys, 2, 1, 48)) for launch in launches)


def test_every_kernel_of_attention_is_reached():
    calls = []
    for width in (32, 64, 96, 128):
        for base in (P, P + 2):                               # rows of whole aligned 16 bytes, and not
            for buckets in (0, 1024, 1025):
                for stats in (True, False):
                    calls += attention(1, 9, 5000, 2, 2, width, buckets, 9, base, stats)[:2 if stats else 1]
                name, desc, a = attention(1, 9, 300, 2, 2, width, buckets, 9, base)[1]
                calls.append((name, desc, a[:13] + [0] + a[14:]))                     # a table without a gradient
                calls.append((name, desc, a[:10] + [0] + a[11:13] + [0] + a[14:]))    # of keys and values alone
    taken = {(launch.kernel, launch.parameters) for status, launches in record_attention(calls) for launch in launches if status == B.LEAP_OK}
    mine = ("k_attention", "k_grad_query", "k_grad_key", "k_delta", "k_lines", "k_join", "k_join_table")
    names = {k for k in kernels() if k[0] in mine and k != ("k_join", (0,)) and k != ("k_join", (1,)) and k != ("k_join", (2,))}       # (the norm's weights' gradient has a k_join too)
    assert {k for k in taken if k[0] in mine} == names


@pytest.mark.parametrize("batch", [0, 2])
def test_no_kernel_reads_lines_that_are_not_written(batch):
    """With a table every kernel that takes a number for a pair comes after the one that writes those, whichever gradients are wanted; without queries nothing is read at all."""
    calls = []
    for queries in (0, 1, 5, 130):
        for keys in (0, 300):
            for wanted in range(1, 16):
                for buckets in (0, 9):
                    name, desc, a = attention(batch, queries, keys, 2, 1, 64, buckets, 9)[1]
                    calls.append((name, desc, a[:10] + [P if wanted >> i & 1 and (buckets or i < 3) else 0 for i in range(4)] + a[14:]))
                calls.append((name, desc, a))
            calls.append(attention(batch, queries, keys, 2, 1, 64, 9, 9)[0])
    for (name, desc, a), (status, launches) in zip(calls, record_attention(calls)):
        assert status == B.LEAP_OK
        names = [launch.kernel for launch in launches]
        for i, launch in enumerate(launches):
            biased = launch.kernel in ("k_attention", "k_grad_query", "k_grad_key") and launch.parameters[2]
            assert not biased or "k_lines" in names[:i], (desc, a)
        if name == "leap_attention_backward" and not (batch and desc[1]):
            keys = batch and desc[2]
            assert names == ["k_zeros"] * (bool(a[11] and keys) + bool(a[12] and keys) + bool(a[13])), (desc, a)


def test_gradients_without_queries_need_no_memory_but_their_own():
    name, desc, a = attention(2, 0, 300, 2, 1, 64, 9, 9)[1]
    (status, launches), = record_attention([(name, desc, [0] + a[1:4] + [0] * 6 + a[10:14] + [0, 0])])
    assert status == B.LEAP_OK and [launch.kernel for launch in launches] == ["k_zeros"] * 3
