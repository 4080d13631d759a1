"""Launches of the 4-bit cache, the page pool and the rotary positions, on the CPU: a program with a HIP runtime of its own (launches are only
noted) calls the entry points with sizes up to their limits.  A launch takes fewer than 2^32 lanes."""
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
static size_t pushed_lds, lds;
static void *pushed_stream;
static uint64_t lanes;                                           // of the largest launch
static int launches, threads;
extern "C" {
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
int hipLaunchKernel(const void *, Dim3 grid, Dim3 block, void **, size_t l, void *) {
  const uint64_t n = (uint64_t)grid.x * block.x;
  if (n > lanes) lanes = n;
  if (!launches) threads = block.x;
  if (l > lds) lds = l;
  ++launches;
  return 0;
}
int hipGetLastError() { return 0; }
}
int main(int, char **argv) {
  void *lib = dlopen(argv[1], RTLD_NOW);
  if (!lib) { fprintf(stderr, "%s\n", dlerror()); return 2; }
#define F(name) auto name = (decltype(&et_##name))dlsym(lib, "et_" #name)
  F(kv_append); F(kv_append_slots); F(kv_read); F(attention_paged_workspace_bytes); F(attention_paged); F(rotary_apply); F(kv_resize); F(kv_resize_workspace_bytes);
  int32_t *ints = (int32_t *)4096;                               // (nothing is looked into)
  uint16_t *data = (uint16_t *)4096;
  char line[256];
  // "attend KV HEADS HEAD_DIM SEQS BOUND WINDOW" | "rows KV HEAD_DIM ROWS" | "rotary HEADS HEAD_DIM ROT_DIM ROWS" | "resize SEQS PAGES ROWS APART"
  // -> "code lanes launches threads-of-the-first lds workspace"
  while (fgets(line, sizeof line, stdin)) {
    int a[6];
    char what[16];
    if (sscanf(line, "%15s %d %d %d %d %d %d", what, a, a + 1, a + 2, a + 3, a + 4, a + 5) < 4) return 3;
    lanes = launches = threads = 0;
    lds = 0;
    size_t bytes = 0;
    int rc;
    if (!strcmp(what, "attend")) {
      const et_kv_cache c{data, 8, 256, a[0], a[2], ET_KV_MXFP4};
      const et_kv_seqs s{ints, 1 << 22, 1 << 22, ints, a[3]};
      bytes = attention_paged_workspace_bytes(&c, &s, a[1], a[4], a[5]);
      rc = attention_paged(&c, &s, data, (int64_t)a[1] * a[2], a[1], a[4], a[5], 0.1f, data, bytes, data, nullptr);
    } else if (!strcmp(what, "rows")) {
      const et_kv_cache c{data, 8, 64, a[0], a[1], ET_KV_MXFP4};
      const et_kv_seqs s{ints, 8, 8, ints, 3};
      const int64_t width = (int64_t)a[0] * a[1];
      rc = kv_append(&c, &s, ints, a[2], data, width, data, width, nullptr);
      if (kv_read(&c, &s, ints, a[2], data, width, data, width, nullptr) != rc) return 4;
      if (kv_append_slots(&c, (int64_t *)ints, a[2], data, width, data, width, nullptr) != rc) return 4;
    } else if (!strcmp(what, "rotary")) {
      const et_rotary r{(uint64_t *)data, a[1], a[2], ET_ROTARY_HALF, 1.f};
      const int64_t width = (int64_t)a[0] * a[1];
      const et_rotary_rows x{data, width, data, width, a[0]};
      rc = rotary_apply(&r, ints, a[3], &x, nullptr, 0, nullptr);
    } else {
      const et_kv_pool p{ints, 8, 64};
      bytes = kv_resize_workspace_bytes(a[0]);
      rc = kv_resize(&p, ints, ints + (a[3] ? 4 : 0), ints, a[1], a[1], ints, ints, a[0], a[2], ints, ints, (int64_t *)ints, data, bytes, nullptr);
    }
    printf("%d %llu %d %d %llu %llu\n", rc, (unsigned long long)lanes, launches, threads, (unsigned long long)lds, (unsigned long long)bytes);
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def ask(tmp_path_factory):
    """Calls (lists of words) -> [(code, lanes of the largest launch, launches, lanes of a workgroup, LDS, workspace bytes)]."""
    et.load_library()
    d = tmp_path_factory.mktemp("decoding_launches")
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
    for kv in (1, 2, 8, 32, 64, 1024):
        for group in (1, 2, 8, 17, 64):
            if kv * group > 65536:
                continue
            most = 2 ** 24 // (kv * group)
            for seqs in {1, 3, 9, 63, most // 300 + 1, most // 2, most - 1, most, most + 1}:
                for bound, window in ((64, 0), (600, 0), (2000, 0), (4000, 0), (4000, 100), (9000, 2047)):
                    if seqs >= 1 and seqs * bound <= 2 ** 36:
                        calls.append(("attend", kv, kv * group, 64, seqs, bound, window))
    results = ask(calls)
    assert len(results) == len(calls) > 600
    for c, (code, lanes, launches, threads, _, _) in zip(calls, results):
        kv, heads, seqs = c[1], c[2], c[4]
        assert (code == 0 and 0 < lanes < 2 ** 32 and launches in (1, 2) and threads in (256, 512)) or (code == -1 and launches == 0), c
        if seqs * heads <= 2 ** 24 - 2 ** 19 or (kv < heads and seqs * heads <= 2 ** 24):
            assert code == 0, c
        if seqs * heads > 2 ** 24:
            assert code == -1, c


def test_attention_is_one_part_each_or_shared_out_by_its_rule(ask):
    """(sequences, key-value heads, bound, window) -> launches, lanes of a workgroup."""
    rule = [(1, 2, 512, 0, 1, 256), (1, 2, 513, 0, 2, 256), (8, 8, 1024, 0, 1, 512), (7, 8, 1024, 0, 2, 256), (32, 8, 1024, 0, 1, 512), (33, 8, 1024, 0, 1, 256),
            (24, 8, 2048, 0, 1, 512), (23, 8, 2048, 0, 2, 256), (24, 8, 9000, 2048, 1, 512), (24, 8, 9000, 2049, 2, 256), (64, 8, 2048, 0, 1, 256),
            (64, 8, 2064, 0, 2, 256), (4097, 1, 10 ** 6, 0, 1, 256), (4096, 1, 10 ** 6, 0, 2, 256), (64, 8, 400, 0, 1, 256)]
    for r, (code, _, launches, threads, _, bytes) in zip(rule, ask([("attend", r[1], r[1], 128, r[0], r[2], r[3]) for r in rule])):
        assert code == 0 and (launches, threads) == r[4:] and (bytes > 0) == (launches == 2), r


def test_rows_launch_what_they_accept(ask):
    most = 2 ** 30 - 64
    calls = [("rows", kv, d, rows) for kv in (1, 2, 16, 33, 1024) for d in (64, 80, 256)
             for rows in (1, 63, 4999, 2 ** 20, 2 ** 24 - 1, 2 ** 24, 2 ** 24 + 1, 2 ** 29 + 5, most, most + 1, 2 ** 30, 2 ** 31 - 1)]
    for c, (code, lanes, launches, _, _, _) in zip(calls, ask(calls)):
        if c[3] <= most:
            assert code == 0 and 0 < lanes < 2 ** 32 and launches == 3, c
        else:
            assert code == -1 and launches == 0, c


def test_rotary_launches_what_it_accepts(ask):
    most = 2 ** 27 - 8
    calls = [("rotary", heads, d, rot, rows) for heads in (1, 40, 65536) for d, rot in ((128, 128), (64, 2), (512, 512), (510, 510), (2, 2))
             for rows in (1, 511, 512, 4096, 2 ** 24, most, most + 1, 2 ** 31 - 1)]
    for c, (code, lanes, launches, threads, lds, _) in zip(calls, ask(calls)):
        if c[4] <= most:
            assert code == 0 and 0 < lanes < 2 ** 32 and launches == 1 and threads == 256 and 0 < lds <= 64 * 1024, c
        else:
            assert code == -1 and launches == 0, c


def test_resize_launches_what_it_accepts(ask):
    """One launch for a step; for thousands of rows a second one where the new state takes the old one's place; two beyond 4096 sequences."""
    for seqs in (0, 1, 256, 1024, 1025, 4096, 4097, 2 ** 20, 2 ** 20 + 1):
        for rows in (0, 1, 1024, 1025, 6144, 6145, 10 ** 6, 2 ** 31 - 1):
            for apart in (0, 1):
                (code, lanes, launches, _, _, bytes), = ask([("resize", seqs, 3, rows, apart)])
                if seqs > 2 ** 20:
                    assert code == -1 and launches == 0
                    continue
                several = max(rows, seqs) > 6144
                assert code == 0 and 0 < lanes < 2 ** 32 and (bytes > 0) == (seqs > 4096)
                assert launches == (2 if seqs > 4096 or (several and not apart) else 1), (seqs, rows, apart)
