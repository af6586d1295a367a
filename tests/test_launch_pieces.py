"""Launches of more workgroups than a grid takes: every workgroup once, in order, no piece of 2^32 threads or more."""
import os
import subprocess

import pytest

from paper_2103_07454_amd import build

SOURCE = r"""
#include <stdio.h>
#include <stdlib.h>
#include "launch_pieces.h"
int main(int argc, char** argv) {
  const uint64_t groups = strtoull(argv[1], 0, 10);
  const uint32_t threads = (uint32_t)atoi(argv[2]);
  uint64_t next = 0;
  int pieces = 0;
  evg::launch_pieces(groups, threads, [&](uint32_t first, uint32_t count) {
    if (first != next || !count || (uint64_t)count * threads >> 32) exit(1);
    if (next + count < groups && count % 8) exit(2);
    next += count;
    ++pieces;
  });
  if (next != groups) return 3;
  printf("%d\n", pieces);
  return 0;
}
"""


@pytest.fixture(scope="module")
def pieces(tmp_path_factory):
    d = tmp_path_factory.mktemp("pieces")
    (d / "main.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", build.CSRC, "-o", str(d / "pieces"), str(d / "main.cpp")], check=True)
    return d / "pieces"


@pytest.mark.parametrize("groups,threads,count", [
    (0, 256, 0), (1, 64, 1), (7, 1024, 1), (2 ** 22 - 8, 1024, 1), (2 ** 22, 1024, 2), (2 ** 24 - 1, 256, 2), (2 ** 24, 256, 2), (2 ** 24 - 8, 256, 1),
    (2 ** 31 - 1, 64, 33), (2 ** 31 - 1, 1024, 513), (20_480_000, 256, 2)])
def test_pieces(pieces, groups, threads, count):
    out = subprocess.run([str(pieces), str(groups), str(threads)], capture_output=True, text=True, timeout=20)
    assert out.returncode == 0 and int(out.stdout) == count, out
