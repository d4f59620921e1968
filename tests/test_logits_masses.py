"""The two-part sums of the histograms' bins, on the host: exact up to the longest
slice for any mass, whatever its low bits; and the search of a target in a
list's running total, which always ends at one of its elements."""
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


SEARCH = r'''
#include <stdio.h>
#include <initializer_list>
#include "mass_parts.h"
using namespace epic;
int main() {
  long long wrong = 0, seen = 0;
  uint32_t x = 7;
  for (int n = 1; n < 40; ++n)
    for (int round = 0; round < 20; ++round) {
      uint64_t q[40], total = 0;
      for (int i = 0; i < n; ++i) {
        x = x * 1664525u + 1013904223u;
        total += q[i] = round == 0 ? 0 : x >> 28 & 7;  // some of them nothing
      }
      for (uint64_t t : {uint64_t(0), total / 2, total - 1, total, total + 1, total + 1000000, ~uint64_t(0)}) {
        int first = n - 1, hits = 0, at = -1;
        uint64_t upto = 0;
        for (int i = n; i--;) upto += q[i];
        for (int i = n; i--; upto -= q[i])
          if (upto > t) first = i;
        upto = 0;
        for (int i = 0; i < n; upto += q[i++])
          if (passes(upto, q[i], t, i == n - 1)) ++hits, at = i;
        ++seen;
        wrong += hits != 1 || at != first;
      }
    }
  printf("%lld %lld\n", seen, wrong);
}
'''


def test_a_target_past_the_end_is_the_last_element(tmp_path):
    source, program = tmp_path / 'search.cpp', tmp_path / 'search'
    source.write_text(SEARCH)
    subprocess.check_call(['g++', '-std=c++17', '-O2', '-I', CSRC, str(source), '-o', str(program)])
    seen, wrong = map(int, subprocess.check_output([str(program)]).split())
    assert seen > 5000 and wrong == 0
