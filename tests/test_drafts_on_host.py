"""The kernels of a step of drafted tokens, their own source compiled for the host (tests/on_host) under the address and
undefined-behaviour sanitizers: results against loops, and every access within buffers of the size that a caller owes, with
trees, paths, tables and lengths that no caller should bring among them."""
import os
import re
import subprocess

import pytest

from test_device_code_on_host import CLANG, CSRC, FLAGS, HERE, OF_64_AND_128, _check

pytestmark = pytest.mark.skipif(not os.path.exists(CLANG), reason="needs clang++ with vector types")


def _build(source, driver, to, *changes):
    s = open(os.path.join(CSRC, source + ".hip")).read().replace("#include <hip/hip_runtime.h>", '#include "more_on_host.h"')
    for old, new in changes:
        assert s.count(old) == 1, old
        s = s.replace(old, new)
    s, n = re.subn(r"(\w+(?:<[^<>;]*>)?)<<<(.*), ([^,]+), 0, st>>>\((.*)\);", r"emu::launch([=] { \1(\4); }, dim3(\2), \3);", s)
    assert n >= 3 and "<<<" not in s
    src, exe = to / (driver + ".kernels.cpp"), to / driver
    src.write_text(s)
    proc = subprocess.run([CLANG, *FLAGS, str(src), os.path.join(HERE, "on_host", driver + ".cpp"), "-o", str(exe)],
                          stdout=subprocess.PIPE, stderr=subprocess.STDOUT)
    assert proc.returncode == 0, proc.stdout.decode()[-3000:]
    return str(exe)


@pytest.fixture(scope="module")
def drafts(tmp_path_factory):
    return _build("drafts", "drafts", tmp_path_factory.mktemp("drafts"))


@pytest.fixture(scope="module")
def rotate(tmp_path_factory):
    return _build("rotate", "rotate", tmp_path_factory.mktemp("rotate"))


@pytest.fixture(scope="module")
def attend(tmp_path_factory):
    return _build("attend", "attend_drafts", tmp_path_factory.mktemp("attend_drafts"), *OF_64_AND_128)


@pytest.fixture(scope="module")
def attend_in_pieces(tmp_path_factory):
    """As for very many keys: all tiles on one line that is cut into equal pieces."""
    return _build("attend", "attend_drafts", tmp_path_factory.mktemp("attend_in_pieces"), *OF_64_AND_128, ("kFew = 8,", "kFew = 0,"))


@pytest.mark.parametrize("odd", [0, 1])
@pytest.mark.parametrize("args", ["40 8 64 2 16 2 1", "30 64 64 1 16 1 2", "25 64 128 2 32 1 3", "20 33 96 2 64 2 4",
                                  "12 64 256 1 256 1 5", "30 5 64 3 128 1 6"])
def test_trees_paths_and_moves(drafts, args, odd):
    _check(drafts, f"{args} {odd}")


@pytest.mark.parametrize("args", [
    "9 8 2 128 128 0 bf16 1 0 0", "5 14 7 64 32 1 f16 1 8 0", "7 3 1 96 96 0 f32 1 0 1", "6 5 2 256 128 0 bf16 0 1 0",
    "4 9 3 96 48 1 f32 0 3 1", "3 1 1 64 0 0 f16 1 0 0", "5 4 4 256 256 1 f16 1 16 1", "2 0 3 128 64 0 bf16 1 0 0",
    "2051 2 1 64 64 0 bf16 1 0 0"])
def test_norm_and_rotation(rotate, args):
    _check(rotate, args)


TREES = [
    "128 2 4 64 bf16 0 0 0 3 1 300:8 17:3 64:1 0:0 9:9",                # short tables: one launch
    "128 1 4 32 f16 0 0 0 0 1 700:16 1:1 65:5 600:64",                  # 128 rows a tile, trees across units
    "128 1 4 32 bf16 0 0 0 0 1 700:16 1:1 65:5 600:12",                 # 64 rows, their keys in halves
    "128 2 4 64 bf16 0 0 0 0 1 900:4 17:3 64:1 0:0 600:4",              # up to 16 rows, cut
    "64 1 4 16 bf16 0 0 0 0 1 520:13 130:64 1:1 40:40",
    "64 1 1 16 f16 0 0 0 0 1 100:90 300:31 64:64",                      # a run in a short table
    "128 1 4 64 bf16 0 0 0 0 1 500:32 77:20 30:30",                     # eight row tiles of one launch
    "64 2 2 128 f16 100 0 0 0 1 700:30 130:1 0:1 513:64",               # windows, a row without keys
    "64 1 1 32 bf16 5 0 0 0 2 700:40 30:30 64:64 3:2",                  # windows shorter than the paths
    "64 1 2 16 bf16 0 300 70 0 1 30:1x20 0:0x15 1300:70 7:1x5 900:31",  # trees beside a run
    "64 1 2 16 f16 0 80 0 0 1 30:1x520 1000:40",                        # more requests than a workgroup sums
    "64 1 2 16 bf16 0 0 0 0 1 30:1x60 200:33 0:0x9 400:20",             # more than a wave has lanes
    "64 1 4 32 bf16 0 0 0 2 3 600:20 300:64 20:30",                     # words that are no trees; fewer held than new
    "128 1 1 64 f16 33 0 0 0 3 300:64 64:64 700:16", "128 1 8 16 bf16 0 0 0 0 2 520:4 9:2 1:1"]


@pytest.mark.parametrize("args", TREES)
def test_attention_over_trees(attend, args):
    _check(attend, args)


@pytest.mark.parametrize("args", TREES[1:])
def test_attention_over_trees_in_pieces(attend_in_pieces, args):
    _check(attend_in_pieces, args)


NO_TREES = [
    "64 1 1 16 f16 0 0 0 0 1 300:90",                                   # a run alone
    "128 1 4 32 bf16 40 0 0 2 1 700:70 900:65",                         # runs alone, rows of no request
    "64 2 1 16 bf16 0 0 80 3 1 300:0 40:0",                             # no request has new tokens
    "64 1 2 16 bf16 0 300 70 5 1 30:0x20 600:0"]


@pytest.mark.parametrize("args", NO_TREES)
def test_steps_without_trees(attend, args):
    _check(attend, args)


@pytest.mark.parametrize("args", NO_TREES)
def test_steps_without_trees_in_pieces(attend_in_pieces, args):
    _check(attend_in_pieces, args)


FAR_WINDOWS = [
    "64 1 4 32 bf16 2147483647 0 0 2 3 600:20 300:64 20:30",            # windows past all positions, fewer held than new
    "128 1 1 64 f16 2147483647 0 0 0 1 40:64 700:16 2:9", "64 1 1 16 f16 1073741824 0 0 0 1 100:40 600:33 7:20",
    "64 1 2 16 bf16 2147483600 0 0 0 1 900:4 3:6 1:1"]


@pytest.mark.parametrize("args", FAR_WINDOWS)
def test_windows_past_all_positions(attend, args):
    _check(attend, args)
