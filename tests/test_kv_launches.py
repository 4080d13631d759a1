"""The launches of the paged cache's calls, on the CPU: a program with a HIP runtime of its own (launches are only noted) loads the
built library and calls the entry points with sizes up to their limits.  A launch takes fewer than 2^32 lanes."""
import subprocess

import pytest

import paper_2605_30010_amd as et
from paper_2605_30010_amd.build import LIB, ROOT

PROGRAM = r"""
#include <dlfcn.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>
#include "earlytom.h"
struct Dim3 { uint32_t x, y, z; };
static Dim3 pushed[2];
static size_t pushed_lds;
static void *pushed_stream;
static uint64_t lanes;                                           // of the largest launch
static int launches;
extern "C" {
// Handles are passed through; nothing is registered or launched.
void **__hipRegisterFatBinary(const void *) { static void *h; return &h; }
void __hipUnregisterFatBinary(void **) {}
void __hipRegisterFunction(void **, const void *, char *, const char *, unsigned, void *, void *, void *, void *, int *) {}
void __hipRegisterVar(void **, void *, char *, char *, int, size_t, int, int) {}
int __hipPushCallConfiguration(Dim3 grid, Dim3 block, size_t lds, void *stream) {
  pushed[0] = grid; pushed[1] = block; pushed_lds = lds; pushed_stream = stream;
  return 0;
}
int __hipPopCallConfiguration(Dim3 *grid, Dim3 *block, size_t *lds, void **stream) {
  *grid = pushed[0]; *block = pushed[1]; *lds = pushed_lds; *stream = pushed_stream;
  return 0;
}
int hipLaunchKernel(const void *, Dim3 grid, Dim3 block, void **, size_t, void *) {
  const uint64_t n = (uint64_t)grid.x * block.x;
  if (n > lanes) lanes = n;
  ++launches;
  return 0;
}
int hipGetLastError() { return 0; }
}
int main(int, char **argv) {
  void *lib = dlopen(argv[1], RTLD_NOW);
  if (!lib) { fprintf(stderr, "%s\n", dlerror()); return 2; }
  auto rows_call = (decltype(&et_kv_append))dlsym(lib, "et_kv_append");
  auto read_call = (decltype(&et_kv_read))dlsym(lib, "et_kv_read");
  auto need = (decltype(&et_attention_paged_workspace_bytes))dlsym(lib, "et_attention_paged_workspace_bytes");
  auto attend = (decltype(&et_attention_paged))dlsym(lib, "et_attention_paged");
  int32_t *ints = (int32_t *)4096;                               // (nothing is looked into)
  uint16_t *data = (uint16_t *)4096;
  char line[256];
  // "rows KV HEAD_DIM FORMAT ROWS" | "attend KV HEADS HEAD_DIM SEQS BOUND WINDOW" -> "code lanes launches workspace"
  while (fgets(line, sizeof line, stdin)) {
    int a[6];
    char what[16];
    if (sscanf(line, "%15s %d %d %d %d %d %d", what, a, a + 1, a + 2, a + 3, a + 4, a + 5) < 5) return 3;
    lanes = launches = 0;
    size_t bytes = 0;
    int rc;
    if (!strcmp(what, "attend")) {
      const et_kv_cache c{data, 8, 256, a[0], a[2], ET_KV_BF16};
      const et_kv_seqs s{ints, 1 << 22, 1 << 22, ints, a[3]};
      bytes = need(&c, &s, a[1], a[4], a[5]);
      rc = attend(&c, &s, data, (int64_t)a[1] * a[2], a[1], a[4], a[5], 0.1f, data, bytes, data, nullptr);
    } else {
      const et_kv_cache c{data, 8, 64, a[0], a[1], a[2]};
      const et_kv_seqs s{ints, 8, 8, ints, 3};
      const int64_t width = (int64_t)a[0] * a[1];
      rc = rows_call(&c, &s, ints, a[3], data, width, data, width, nullptr);
      const int again = read_call(&c, &s, ints, a[3], data, width, data, width, nullptr);
      if (again != rc) return 4;
    }
    printf("%d %llu %d %llu\n", rc, (unsigned long long)lanes, launches, (unsigned long long)bytes);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """Calls (lists of words) -> [(code, lanes of the largest launch, launches, workspace bytes)]."""
    et.load_library()
    d = tmp_path_factory.mktemp("kv_launches")
    src, exe = str(d / "launches.cpp"), str(d / "launches")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-O1", "-std=c++17", "-rdynamic", "-I", ROOT + "/include", src, "-o", exe, "-ldl"], check=True)

    def call(calls):
        run = subprocess.run([exe, LIB], input="".join(" ".join(map(str, c)) + "\n" for c in calls), capture_output=True, text=True,
                             cwd=ROOT, timeout=120)
        assert run.returncode == 0, run.stderr
        return [tuple(map(int, line.split())) for line in run.stdout.splitlines()]
    return call


def test_attention_launches_what_it_accepts(ask):
    """Up to n_seqs * n_heads = 2^24, with every grouping of the heads, as one part for each sequence and shared out."""
    calls = []
    for heads in (1, 2, 8, 32, 64, 1024):
        for group in (1, 2, 8, 17, 64):
            kv = heads
            if kv * group > 65536:
                continue
            most = 2 ** 24 // (kv * group)
            for seqs in {1, 3, 63, most // 300 + 1, most // 2, most - 1, most, most + 1}:
                for bound, window in ((64, 0), (600, 0), (2000, 0), (4000, 0), (4000, 100)):
                    if seqs >= 1 and seqs * bound <= 2 ** 36:
                        calls.append(("attend", kv, kv * group, 64, seqs, bound, window))
    results = ask(calls)
    assert len(results) == len(calls) > 600
    for c, (code, lanes, launches, _) in zip(calls, results):
        kv, heads, seqs = c[1], c[2], c[4]
        assert (code == 0 and 0 < lanes < 2 ** 32 and launches in (1, 2)) or (code == -1 and launches == 0), c
        if seqs * heads <= 2 ** 24 - 2 ** 19 or (kv < heads and seqs * heads <= 2 ** 24):
            assert code == 0, c
        if seqs * heads > 2 ** 24:
            assert code == -1, c


def test_rows_launch_what_they_accept(ask):
    most = 2 ** 30 - 64
    calls = [("rows", kv, d, fmt, rows) for kv in (1, 2, 16, 33, 1024) for d in (64, 256) for fmt in (0, 1, 2)
             for rows in (1, 63, 4999, 2 ** 20, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, 2 ** 29 + 5, most, most + 1, 2 ** 30, 2 ** 31 - 1)]
    for c, (code, lanes, launches, _) in zip(calls, ask(calls)):
        if c[4] <= most:
            assert code == 0 and 0 < lanes < 2 ** 32 and launches == 2, c
        else:
            assert code == -1 and launches == 0, c


def test_many_sequences_are_one_part_each(ask):
    """Where a call is shared out, every workgroup looks at all lengths: not with any number of sequences."""
    calls = [("attend", kv, heads, 64, seqs, bound, 0) for kv, heads in ((1, 1), (1, 8), (8, 32)) for seqs in (4097, 2 ** 16, 2 ** 19)
             for bound in (2049, 2 ** 17)]
    for c, (code, lanes, launches, bytes) in zip(calls, ask(calls)):
        assert code == 0 and launches == 1 and bytes == 0 and lanes == c[1] * c[4] * 256, c
    assert all(r[2] == 2 and r[3] > 0 for r in ask([("attend", 1, 8, 64, seqs, 4000, 0) for seqs in (2, 1000, 4096)]))
