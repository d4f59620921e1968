"""The two-part sums of the histograms' bins, on the host: exact up to the longest
slice for any mass, whatever its low bits."""
import os
import subprocess

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), 'paper_2606_00722_gb300', 'csrc')

PROGRAM = r'''
#include <stdio.h>
#include "mass_parts.h"
using namespace epic;
static long long wrong = 0, seen = 0;
static void same(uint32_t q) {  // a bin of kSliceElems elements of mass q
  const MassParts one = mass_parts(q);
  uint32_t high = 0, low = 0;
  for (int i = 0; i < kSliceElems; ++i) high += one.high, low += one.low;
  const int32_t s = (int32_t)one.low;
  ++seen;
  wrong += one.value() != q || s > 16384 || s < -16384 || one.high > 32768 ||
           MassParts{high, low}.value() != (uint64_t)q * kSliceElems;
}
int main() {
  const uint32_t top = 1u << 30;
  for (uint32_t r = 0; r < 32768; r += 37) same(r), same(top - r), same((r << 15) + 12345), same((1000u << 15) + r);
  for (uint32_t r = 16000; r < 16800; ++r) same(r), same((32767u << 15) + r);
  same(32767), same(16383), same(16384), same(16385), same(top), same(top - 1), same(0);
  // a mixture
  uint32_t high = 0, low = 0, x = 1;
  uint64_t all = 0;
  for (int i = 0; i < kSliceElems; ++i) {
    x = x * 1664525u + 1013904223u;
    const uint32_t q = (x >> 2 & ~0x7fffu) + 16383;
    const MassParts p = mass_parts(q);
    high += p.high, low += p.low, all += q;
  }
  wrong += MassParts{high, low}.value() != all;
  printf("%lld %lld\n", seen, wrong);
}
'''


def test_sums_of_the_longest_slice_are_exact(tmp_path):
    source, program = tmp_path / 'sums.cpp', tmp_path / 'sums'
    source.write_text(PROGRAM)
    subprocess.check_call(['g++', '-std=c++17', '-O2', '-I', CSRC, str(source), '-o', str(program)])
    seen, wrong = map(int, subprocess.check_output([str(program)]).split())
    assert seen > 5000 and wrong == 0
