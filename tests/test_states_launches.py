"""Launches of the state operators as the runtime is asked for them: a host program calls libuf.so, and has the runtime's launch
functions itself, which write down what would be launched."""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <vector>
#include "ufs.h"

struct Dim { uint32_t x, y, z; };
static Dim grid, block;
static int launched = 0, fails_at = 0, error = 0;
extern "C" {
int __hipPushCallConfiguration(Dim g, Dim b, size_t, void*) { grid = g, block = b; return 0; }
int __hipPopCallConfiguration(Dim* g, Dim* b, size_t* shared, void** stream) {
  *g = grid, *b = block, *shared = 0, *stream = nullptr;
  return 0;
}
int hipLaunchKernel(const void*, Dim g, Dim b, void**, size_t, void*) {
  if (++launched == fails_at) return error = 719;
  printf("launch %u %u %u %u\n", g.x, g.y, g.z, b.x * b.y * b.z);
  return 0;
}
int hipGetLastError() { const int e = error; error = 0; return e; }
}

int main(int c, char** v) {
  auto arg = [&](int i) { return i < c ? atoi(v[i]) : 0; };
  char* const p = reinterpret_cast<char*>(uintptr_t(1) << 32);   // (never read: nothing runs)
  float* const f = reinterpret_cast<float*>(p);
  int32_t* const words = reinterpret_cast<int32_t*>(p);
  if (!strcmp(v[1], "whole")) {                                  // batch, tokens, key heads, group
    const int64_t H = int64_t(arg(4)) * arg(5), D = 128;
    const uft_stride s{H * D * arg(3), H * D, D}, t{int64_t(arg(4)) * D * arg(3), arg(4) * D, D};
    const ufs_linear_desc d{arg(2), arg(3), int32_t(H), arg(4), int32_t(D), 1.f, s, t, t};
    for (int back = 0; back < 2; ++back) {
      size_t need = 0;
      int rc = back ? ufs_linear_bwd_work_bytes(&d, &need) : ufs_linear_work_bytes(&d, &need);
      printf("size %d %zu\n", rc, need);
      rc = back ? ufs_linear_bwd(&d, p, p, p, p, f, nullptr, f, f, p, p, p, f, p, need, nullptr)
                : ufs_linear_fwd(&d, p, p, p, f, nullptr, f, p, f, p, need, nullptr);
      printf("call %d\n", rc);
    }
  }
  if (!strcmp(v[1], "step")) {                                   // key heads, group, sequences, tokens of each
    const int n = arg(4);
    std::vector<int32_t> seqs(n), counts(n, arg(5));
    for (int i = 0; i < n; ++i) seqs[i] = i;
    const ufs_desc d{1, arg(2), 128, n, 0};
    ufs_cache* cache;
    size_t pool, table;
    if (ufs_pool_bytes(&d, &pool) || ufs_table_bytes(&d, &table) || ufs_create(&d, p, pool, p, table, &cache)) return 1;
    ufs_extend(cache, n, seqs.data(), counts.data(), nullptr);
    const uft_stride s{0, 128 * arg(2), 128}, t{0, 128 * arg(2) * arg(3), 128};
    const ufs_attn_desc a{arg(2) * arg(3), 1.f, t, s, s};
    printf("size %d\n", ufs_attn_work_bytes(cache, &pool));
    printf("call %d %zu\n", ufs_attn(cache, 0, &a, p, p, p, f, p, p, 1 << 30, nullptr), pool);
  }
  if (!strcmp(v[1], "fails")) {                                  // which call, and which of its launches fails
    const int n = 1200, beams = 4;
    std::vector<int32_t> seqs(n), more(n), counts(n, 7);
    for (int i = 0; i < n; ++i) seqs[i] = i, more[i] = n + i;
    const ufs_desc d{2, 1, 128, 2 * n, 0};
    ufs_cache* cache;
    size_t pool, table;
    if (ufs_pool_bytes(&d, &pool) || ufs_table_bytes(&d, &table) || ufs_create(&d, p, pool, p, table, &cache) ||
        ufs_extend(cache, n, seqs.data(), counts.data(), nullptr))
      return 1;
    launched = 0, fails_at = arg(3);
    for (int i = 0; i < n; ++i) counts[i] = 5 + i % 2;
    auto call = [&] {
      return !strcmp(v[2], "extend")    ? ufs_extend(cache, n, seqs.data(), counts.data(), nullptr)
             : !strcmp(v[2], "reorder") ? ufs_reorder(cache, n / beams, beams, seqs.data(), words, nullptr)
                                        : ufs_fork(cache, n, seqs.data(), more.data(), nullptr);
    };
    auto tell = [&](int rc) {
      ufs_info info;
      int32_t held[2];
      ufs_get_info(cache, &info);
      ufs_seq_tokens(cache, 0, held);
      ufs_seq_tokens(cache, n, held + 1);
      const uft_stride s{0, 128, 128};
      const ufs_attn_desc a{1, 1.f, s, s, s};
      const int attn = ufs_attn(cache, 0, &a, p, p, p, f, p, p, 1 << 30, nullptr);
      printf("after %d %d %d %d %d\n", rc, info.step_tokens, held[0], held[1], attn);
    };
    tell(call());
    fails_at = 0;
    tell(call());
  }
  return 0;
}
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    import paper_2606_09150_amd._lib as L
    L.load()
    d = tmp_path_factory.mktemp("launches")
    (d / "launches.cpp").write_text(PROGRAM)
    exe, where = str(d / "launches"), os.path.dirname(L.LIB_PATH)
    rocm = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "lib")
    subprocess.run(["g++", "-std=c++17", "-rdynamic", f"-I{ROOT}/include", str(d / "launches.cpp"), L.LIB_PATH, "-o", exe, f"-Wl,-rpath,{where}",
                    f"-Wl,-rpath,{rocm}", f"-Wl,-rpath-link,{rocm}", "-Wl,--allow-shlib-undefined"], check=True)

    def call(*args):
        lines = subprocess.check_output([exe, *map(str, args)], text=True).splitlines()
        return [(x.split()[0], *map(int, x.split()[1:])) for x in lines]

    return call


OK, BAD, EMPTY, HIP = 0, -1, -4, -5                 # status codes
THREADS = 2 ** 32 - 1                                # of a launch


def launches(lines):
    return [x[1:] for x in lines if x[0] == "launch"]


@pytest.mark.parametrize("batch,tokens,heads,group", [
    (1, 1, 1, 1), (3, 5000, 7, 2),
    (43690, 1, 64, 1),                               # 2,796,160 places: the backward's walks in one launch
    (43691, 1, 64, 1), (50000, 32, 64, 1), (65535, 1, 64, 1), (65535, 1, 64, 3),   # in two
    (131071, 1, 64, 1),                              # the most places of a launch of walks, but for 63
])
def test_every_call_that_is_accepted_fits_its_launches(run, batch, tokens, heads, group):
    lines = run("whole", batch, tokens, heads, group)
    back = max(i for i, x in enumerate(lines) if x[0] == "size")
    assert lines[0][1] == lines[back][1] == OK
    assert [x for x in lines if x[0] == "call"] == [("call", OK)] * 2
    for x, y, z, threads in launches(lines):
        assert x * threads <= THREADS and y == z == 1
    if lines[back][2] == 0:                                    # each place once, and three walks of each backwards, of eight places together
        places = batch * heads
        assert launches(lines[:back]) == [(places, 1, 1, 512)]
        walks = [x for x, _, _, _ in launches(lines[back:])]
        assert sum(walks) == -(-places // 8) * 24 and all(x % 24 == 0 for x in walks)


@pytest.mark.parametrize("batch,tokens,heads,group", [(131072, 1, 64, 1), (2 ** 23, 1, 1, 1), (2 ** 24, 40, 1, 1), (2 ** 30, 1, 4, 1)])
def test_calls_of_more_places_than_a_launch_has_are_refused(run, batch, tokens, heads, group):
    lines = run("whole", batch, tokens, heads, group)
    bad = [x[1] for x in lines if x[0] in ("size", "call")]
    assert len(bad) == 4 and set(bad) == {BAD} and not launches(lines)


@pytest.mark.parametrize("heads,few,many", [(128, OK, OK), (129, OK, BAD), (256, OK, BAD), (257, BAD, BAD)])
def test_steps_of_more_places_than_a_launch_has_are_refused(heads, few, many):
    """Token by token a place has 256 threads, in chunks 512."""
    import paper_2606_09150_amd as P
    n = 65535
    cache = P.StateCache(1, heads, n, flags=P._lib.UF_F_DRYRUN)
    for count, status in ((4, few), (5, many)):
        held = cache.tokens(0)
        if status == OK:
            cache.extend(range(n), [count] * n)
            assert cache.step_tokens() == n * count
        else:
            with pytest.raises(P.UfError) as e:
                cache.extend(range(n), [count] * n)
            assert e.value.status == BAD and cache.tokens(0) == held


@pytest.mark.parametrize("what,at,step,after", [
    # tokens of the step that holds, those of a sequence and of its fork, when the launch fails and when the call is made again
    ("extend", 1, 8400, (6600, 12, 0)), ("extend", 2, 0, (6600, 12, 0)),
    ("reorder", 1, 8400, (0, 7, 0)), ("reorder", 2, 0, (0, 7, 0)),
    ("fork", 1, 8400, (8400, 7, 7)), ("fork", 2, 8400, (8400, 7, 7)),
])
def test_a_launch_that_fails_leaves_no_step_over_what_others_changed(run, what, at, step, after):
    lines = [x[1:] for x in run("fails", what, at) if x[0] == "after"]
    assert lines[0] == (HIP, step, 7, 0, OK if step else EMPTY)
    assert lines[1] == (OK, *after, OK if after[0] else EMPTY)


@pytest.mark.parametrize("heads,group,seqs,tokens,launch", [
    # token by token, the columns of a state in four workgroups, or all in one (workgroups, threads); and in chunks
    (2, 1, 1, 4, (8, 256)), (2, 1, 1, 5, (2, 512)), (1, 16, 2, 4, (8, 256)), (1, 17, 2, 4, (2, 256)), (1, 16, 2, 5, (2, 512)),
    (3, 21, 2, 3, (24, 256)), (3, 22, 2, 3, (6, 256)), (255, 1, 1, 1, (1020, 256)), (256, 1, 1, 1, (256, 256)), (64, 1, 4, 4, (256, 256)),
])
def test_steps_of_few_tokens(run, heads, group, seqs, tokens, launch):
    lines = run("step", heads, group, seqs, tokens)
    at = lines.index(("size", OK))
    assert lines[-1] == ("call", OK, 0)
    assert [(x, threads) for x, _, _, threads in launches(lines[at:])] == [launch]
