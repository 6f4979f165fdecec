"""Kernels compiled for the CPU (host_lanes/lanes.h) and arrays beside unmapped pages, for the tests
that run them there."""
import ctypes
import mmap
import multiprocessing
import os
import re
import subprocess

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_1911_05063_amd", "csrc")
CLANG = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++")
F32, BF16, F16 = 0, 1, 2
PAGE = mmap.PAGESIZE


def launches_as_calls(source: str) -> str:
    """name<..><<<grid, threads, 0, stream>>>(args)  ->  lanes::launch(grid, threads, [&] { name<..>(args); })"""
    out, n = source, 0
    while "<<<" in out:
        at = out.index("<<<")
        name = re.search(r"(\w+(?:<[^<>]*>)?)\s*$", out[:at])
        end = out.index(">>>(", at)
        close, depth = end + 4, 1
        while depth:
            depth += {"(": 1, ")": -1}.get(out[close], 0)
            close += 1
        parts, depth = [""], 0
        for c in out[at + 3:end]:
            depth += {"(": 1, ")": -1}.get(c, 0)
            if c == "," and depth == 0:
                parts.append("")
            else:
                parts[-1] += c
        assert len(parts) == 4
        out = (out[:name.start()] + f"lanes::launch({parts[0]}, {parts[1]}, [&] {{ {name.group(1)}"
               f"{out[end + 3:close]}; }})" + out[close:])
        n += 1
    assert n > 0
    return out


def build(folder: str, unit: str, source: str, flags=()) -> str:
    """host_lanes/<unit>.cpp with the kernels of `source`, as a library in `folder`."""
    os.makedirs(os.path.join(folder, "hip"), exist_ok=True)
    with open(os.path.join(folder, "hip", "hip_runtime.h"), "w") as f:
        f.write(f'#include "{HERE}/host_lanes/lanes.h"\n')
    with open(source) as f:
        text = launches_as_calls(f.read())
    kernels, so = os.path.join(folder, unit + ".inc"), os.path.join(folder, unit + ".so")
    with open(kernels, "w") as f:
        f.write(text)
    subprocess.run([CLANG, "-std=c++17", "-O2", "-g1", "-fPIC", "-shared", "-mf16c", "-ffp-contract=off", "-w",
                    *flags, f"-I{folder}", f"-I{CSRC}", f"-I{ROOT}/include",
                    f'-D{unit.upper()}_LOSS="{kernels}"', os.path.join(HERE, "host_lanes", unit + ".cpp"),
                    "-o", so], check=True)
    return so


libc = ctypes.CDLL(None, use_errno=True)
libc.mmap.restype = ctypes.c_void_p
libc.mmap.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_long]
libc.mprotect.argtypes = [ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int]


def place(a: np.ndarray, at_end: bool):
    """A copy of `a` whose last (first) byte has an unmapped page behind (before) it."""
    n = -(-max(a.nbytes, 1) // PAGE) * PAGE
    base = libc.mmap(None, n + 2 * PAGE, 3, 0x22, -1, 0)        # read and write, private and anonymous
    assert base not in (None, ctypes.c_void_p(-1).value)
    assert libc.mprotect(base, PAGE, 0) == 0 and libc.mprotect(base + PAGE + n, PAGE, 0) == 0
    start = base + PAGE + (n - a.nbytes if at_end else 0)
    out = np.frombuffer((ctypes.c_char * a.nbytes).from_address(start), a.dtype).reshape(a.shape)
    out[...] = a
    return out


def ptr(a):
    return None if a is None else ctypes.c_void_p(a.ctypes.data)


def stored(x: np.ndarray, dtype: int):
    """x as it is stored in dtype, and its values."""
    if dtype == F32:
        return x.astype(np.float32), x.astype(np.float32).astype(np.float64)
    if dtype == F16:
        return x.astype(np.float16), x.astype(np.float16).astype(np.float64)
    b = x.astype(np.float32).view(np.uint32).astype(np.uint64)
    b = ((b + 0x7FFF + (b >> 16 & 1)) >> 16).astype(np.uint16)
    return b, values(b, BF16)


def values(a: np.ndarray, dtype: int):
    if dtype == BF16:
        return (a.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return a.astype(np.float64)


def in_child(target, *args):
    """In a process of its own: an access outside a buffer ends it with a signal."""
    p = multiprocessing.get_context("fork").Process(target=target, args=args)
    p.start()
    p.join(300)
    if p.exitcode is None:
        p.kill()
        p.join()
    assert p.exitcode == 0, f"exit code {p.exitcode}"
