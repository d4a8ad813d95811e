"""What the operators on activations in 8 bits launch, without a GPU: tests/host/launch_recorder.cpp stands in for the HIP runtime.

    record([("leap_pack8", (...)), ...]) -> [(status, [Launch(kernel, parameters, blocks, threads), ...]), ...]
    kernels() -> {(kernel, parameters), ...}, all that the library has

Arguments are those of include/leap_activations.h; addresses are never touched."""
import json
import os
import re
import subprocess
import sys
from typing import NamedTuple, Tuple

HERE = os.path.dirname(os.path.abspath(__file__))
SRC, LIB = os.path.join(HERE, "host", "launch_recorder.cpp"), os.path.join(HERE, "host", "liblaunch_recorder.so")


class Launch(NamedTuple):
    kernel: str                          # k_product, ...
    parameters: Tuple[int, ...]          # its template's numbers
    blocks: Tuple[int, int, int]
    threads: int                         # of a block


def _build():
    from paper_2307_05801_amd import binding as B
    if not os.path.exists(B.LIB_PATH):
        from paper_2307_05801_amd.build import build_library
        build_library()
    if not os.path.exists(LIB) or os.path.getmtime(LIB) < os.path.getmtime(SRC):
        tmp = f"{LIB}.{os.getpid()}.tmp"
        subprocess.run(["g++", "-O1", "-std=c++17", "-fPIC", "-shared", "-o", tmp, SRC], check=True, capture_output=True)
        os.replace(tmp, LIB)


def _run(calls):
    """In a process of its own, which must not have loaded the runtime (nor torch)."""
    _build()
    done = subprocess.run([sys.executable, os.path.abspath(__file__)], input=json.dumps(calls), capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stderr
    return json.loads(done.stdout)


def _name(mangled):
    found = re.search(r"\d(k_[a-z_]+?)(I(?:L[ib]\d+E)+E)?(?=E|v|P|N|S|$)", mangled)
    return (found.group(1), tuple(int(v) for v in re.findall(r"L[ib](\d+)E", found.group(2) or ""))) if found else None


def record(calls):
    out = []
    for status, text in _run(calls)[1:]:
        lines = [line.split() for line in text.splitlines()]
        out.append((status, [Launch(*_name(name), tuple(map(int, n[:3])), int(n[3]) * int(n[4]) * int(n[5])) for name, *n in lines]))
    return out


def kernels():
    return set(filter(None, map(_name, _run([])[0].splitlines())))


def _main():
    import ctypes as C
    sys.path.insert(0, os.path.dirname(HERE))
    recorder = C.CDLL(LIB, mode=C.RTLD_GLOBAL)
    from paper_2307_05801_amd import binding as B
    lib = B.load_activations()
    room = C.create_string_buffer(1 << 20)
    assert recorder.registered_kernels(room, len(room)) < len(room)
    out = [room.value.decode()]
    for name, arguments in json.load(sys.stdin):
        status = getattr(lib, name)(*arguments)
        assert recorder.recorded_launches(room, len(room)) < len(room)
        out.append((status, room.value.decode()))
    print(json.dumps(out))


if __name__ == "__main__":
    _main()
