"""The arithmetic that deals out an attention call of one token (csrc/decode_split.h), compiled for the host."""
import ctypes
import os
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2607_25291_amd", "csrc")

SOURCE = r"""
#include "decode_split.h"
#include <string.h>
// How often the join of `units` units of a group of G heads, `rows` heads a unit, stores each head of the group, summed
// over the group's units. Returns the number of stores to heads that the storing unit does not have.
extern "C" int join_stores(long long units, int G, int rows, int* stores) {
  const cosa::JoinShape s = cosa::join_shape(units, G, rows);
  int foreign = 0;
  memset(stores, 0, sizeof(int) * G);
  for (int qg = 0; qg * rows < G; ++qg)
    for (int y = 0; y < s.groups; ++y)
      for (int group = 0; group < cosa::kJoinGroups; ++group) {
        const int head = cosa::join_head(s.heads, s.log2_per_head, cosa::unit_heads(G, rows, qg), y, group);
        if (head < 0 || (group & ((1 << s.log2_per_head) - 1))) continue;  // one lane group of a head stores it
        if (head >= rows || qg * rows + head >= G) ++foreign;
        else ++stores[qg * rows + head];
      }
  return foreign;
}
"""


@pytest.fixture(scope="module")
def split(tmp_path_factory):
    d = tmp_path_factory.mktemp("split")
    (d / "split.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-shared", "-fPIC", "-O1", "-Wall", "-Werror", f"-I{CSRC}", "-o", str(d / "split.so"),
                    str(d / "split.cpp")], check=True)
    lib = ctypes.CDLL(str(d / "split.so"))
    lib.join_stores.argtypes = [ctypes.c_longlong, ctypes.c_int, ctypes.c_int, ctypes.POINTER(ctypes.c_int)]
    return lib


@pytest.mark.parametrize("rows", [16, 32])
def test_every_head_is_joined_once_by_its_own_unit(split, rows):
    for G in list(range(1, 100)) + [128, 255, 1024]:
        units_per_group = -(-G // rows)
        stores = (ctypes.c_int * G)()
        for units in range(units_per_group, 700 * units_per_group, units_per_group):
            foreign = split.join_stores(units, G, rows, stores)
            assert foreign == 0, f"{foreign} stores outside their unit: {units} units, {G} heads, {rows} a unit"
            assert list(stores) == [1] * G, f"{units} units, {G} heads, {rows} a unit"
