"""The serving step's kernels, their own source compiled for the host (tests/on_host/hip_on_host.h), under the address and
undefined-behaviour sanitizers: results against the definitions, and every access within buffers of the size that a caller owes.
Among the cases are those whose run on the GPU once ended with an illegal memory access, with the kernel that is
there now and with the one that was taken out (four row tiles of 16 for 128 dims)."""
import os
import re
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
CSRC = os.path.join(ROOT, "paper_2606_30391_amd", "csrc")
CLANG = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "clang++")
FLAGS = ["-O1", "-std=c++17", "-mf16c", "-mfma", "-w", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
         "-I", os.path.join(HERE, "on_host"), "-I", os.path.join(ROOT, "include"), "-I", CSRC]
ENV = {**os.environ, "ASAN_OPTIONS": "detect_leaks=0:detect_stack_use_after_return=0"}

pytestmark = pytest.mark.skipif(not os.path.exists(CLANG), reason="needs clang++ with vector types")


def _build(name, to, *changes):
    """The source as host C++ (launches become calls), with its driver: the program's path."""
    s = open(os.path.join(CSRC, name + ".hip")).read().replace("#include <hip/hip_runtime.h>", '#include "hip_on_host.h"')
    for old, new in changes:
        assert s.count(old) == 1, old
        s = s.replace(old, new)
    s, n = re.subn(r"(\w+(?:<[^<>;]*>)?)<<<(.*), ([^,]+), 0, st>>>\((.*)\);", r"emu::launch([=] { \1(\4); }, dim3(\2), \3);", s)
    assert n >= 3 and "<<<" not in s
    src, exe = to / (name + ".kernels.cpp"), to / name
    src.write_text(s)
    proc = subprocess.run([CLANG, *FLAGS, str(src), os.path.join(HERE, "on_host", name + ".cpp"), "-o", str(exe)],
                          stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    assert proc.returncode == 0, proc.stdout.decode()[-3000:]
    return str(exe)


def _run(exe, args, **env):
    proc = subprocess.run([exe, *args.split()], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, env={**ENV, **env})
    return proc.returncode, proc.stdout.decode()


def _check(exe, args):
    rc, said = _run(exe, args)
    assert rc == 0, said[-3000:]


# the other head sizes' kernels differ in numbers only, and take long to compile
OF_64_AND_128 = (("    case 96: run<T, 96>(a, s, plan, st); break;\n", ""),
                 ("    default: run<T, 256>(a, s, plan, st); break;\n", ""))


@pytest.fixture(scope="module")
def attend(tmp_path_factory):
    return _build("attend", tmp_path_factory.mktemp("attend"), *OF_64_AND_128)


@pytest.fixture(scope="module")
def attend_of_four(tmp_path_factory):
    return _build("attend", tmp_path_factory.mktemp("attend_of_four"), *OF_64_AND_128,
                  ("D <= 96 ? 4 : D <= 128 ? 2 : 1", "4"))


@pytest.fixture(scope="module")
def blocks(tmp_path_factory):
    return _build("blocks", tmp_path_factory.mktemp("blocks"))


@pytest.fixture(scope="module")
def cache(tmp_path_factory):
    return _build("cache", tmp_path_factory.mktemp("cache"))


FAULTED = ["128 2 4 32 bf16 0 0 0 0 0 13:13 700:13 1:1 65:5 0:0", "128 2 4 32 f16 0 0 0 0 0 16:16 700:16 1:1 65:5 0:0"]


@pytest.mark.parametrize("args", FAULTED + [
    "128 1 1 32 bf16 0 0 0 0 0 40:40 700:33 1:1",                       # 33 to 64 rows of 128 dims
    "128 2 4 64 f16 0 0 0 3 0 300:1 17:1 64:1",                         # one launch; rows of no request
    "128 1 8 16 bf16 0 0 0 0 0 520:4 9:2",                              # two row tiles, cut
    "64 1 4 16 bf16 0 0 0 0 0 520:13 1:1",                              # four row tiles, cut
    "64 2 2 128 bf16 100 0 0 0 0 700:1 130:1 0:1 513:1",                # windows, a row without keys
    "64 1 2 16 bf16 0 300 60 0 0 30:1x20 0:0x15 1300:60 7:1x5",         # single tokens and idle requests beside a chunk, split
    "64 1 2 16 f16 0 80 0 0 0 30:1x520 1000:40",                        # more requests than a workgroup sums
    "64 1 1 64 f16 150 0 0 0 0 300:130", "64 1 4 64 f16 0 0 0 0 18 600:2 300:40"])
def test_attention(attend, args):
    _check(attend, args)


@pytest.mark.parametrize("args", FAULTED)
def test_attention_with_the_kernel_that_was_taken_out(attend_of_four, args):
    _check(attend_of_four, args)


def test_a_buffer_that_is_too_short_is_noticed(attend):
    rc, said = _run(attend, "64 1 2 32 f16 0 0 0 0 0 300:1 65:1", ON_HOST_SHORT="1")
    assert rc and "AddressSanitizer" in said


@pytest.mark.parametrize("args", ["40 16 100 50 0 0 0", "64 16 40 50 0 1 0", "65 16 40 50 0 1 0", "3000 32 100 50 1 1 0",
                                  "16385 16 2 90 2 1 0", "33000 16 3 50 2 0 3", "9000 64 900 10 0 1 1000"])
def test_blocks(blocks, args):
    _check(blocks, args)


@pytest.mark.parametrize("args", ["700 12 64 32 0 90", "300 40 64 16 1 20", "150 60 96 32 0 70", "90 250 64 16 0 3",
                                  "120 2 256 128 2 200", "130 33 128 64 1 150"])
def test_cache(cache, args):
    _check(cache, args)
