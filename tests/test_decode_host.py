"""The host side of the decode entry points on a device that is not there (fake_hip.cpp): what they allocate, what they do while a stream
captures, and that every launch of the largest calls stays within the runtime's limits."""
import os
import random
import subprocess

from test_workspace_host import ROOT, run

CALLS = """
def attend(h, rows, N, group, T, D=128, dtype=0, weight=True):
    return lib.proxykv_attend(h, P, P, P, P, dtype, rows, N, group, T, D, P, P if weight else None, None)

def shared(h, batch, heads, Pn, N, group, T, D=128, dtype=0, weights=True):
    w = P if weights else None
    return lib.proxykv_attend_shared(h, P, P, P, P, P, P, P, dtype, batch, heads, Pn, N, group, T, D, P, w, w, None)

def evict(h, rows, N, budget, recent, D=128):
    return lib.proxykv_evict(h, P, P, P, P, P, None, rows, N, budget, recent, D, None)
"""


def test_one_call_makes_room_for_all_that_are_no_larger():
    """Fewer rows are split more often, and a smaller batch keeps its logits: neither takes more workspace than the largest call left."""
    rng = random.Random(3)
    largest = [("attend", (256, 4000, 4, 1)), ("attend", (64, 9000, 7, 5)), ("attend", (8, 9000, 4, 100)), ("shared", (64, 8, 9000, 700, 4, 1)),
               ("shared", (9, 4, 40000, 300, 2, 3)), ("evict", (300, 5000))]
    plan = []
    for name, sizes in largest:
        less = []
        for _ in range(200):
            if name == "attend":
                T = sizes[3]
                less.append((rng.randint(1, sizes[0]), rng.randint(T, sizes[1]), *sizes[2:]))
            elif name == "shared":
                b, h, Pn, N, g, T = sizes
                less.append((rng.randint(1, b), rng.randint(1, h), rng.randint(1, Pn), rng.choice([0, rng.randint(T, N)]), g, T))
            else:
                N = rng.randint(2, sizes[1])
                b = rng.randint(1, N)
                less.append((rng.randint(1, sizes[0]), N, b, rng.randint(0, b)))
        plan.append((name, (*sizes, 4000, 64) if name == "evict" else sizes, less))
    out = run(CALLS + f"""
out = []
for name, sizes, less in {plan!r}:
    h = context(LLAMA)
    assert globals()[name](h, *sizes) == 0
    before = fake.fake_mallocs()
    fake.fake_capturing(1)
    out.append([sum(globals()[name](h, *s) != 0 for s in less), fake.fake_mallocs() - before])
    fake.fake_capturing(0)
""")
    assert out == [[0, 0]] * len(plan)


def test_nothing_is_allocated_while_the_stream_captures():
    out = run(CALLS + """
        out = []
        for name, small, large in (("attend", (8, 1000, 4, 1), (8, 20000, 4, 1)), ("shared", (4, 8, 1000, 64, 4, 1), (4, 8, 20000, 64, 4, 1)),
                                   ("evict", (8, 1000, 900, 64), (8, 20000, 900, 64))):
            h = context(LLAMA)
            f = globals()[name]
            fake.fake_capturing(1)
            before = fake.fake_mallocs()
            launches()
            got = [f(h, *small), len(launches()), fake.fake_mallocs() - before]
            fake.fake_capturing(0)
            got.append(f(h, *small))
            fake.fake_capturing(1)
            before = fake.fake_mallocs()
            launches()
            got += [f(h, *small), len(launches()) > 0, f(h, *large), len(launches()), fake.fake_mallocs() - before]
            fake.fake_capturing(0)
            out.append(got)
    """.replace("\n        ", "\n"))
    estate = -4
    assert out == [[estate, 0, 0, 0, 0, True, estate, 0, 0]] * 3


def test_workspace_is_a_part_of_the_cache():
    """At most half of what a large cache of 16-bit keys and values takes, and a context gives it back."""
    out = run(CALLS + """
        out = []
        for name, sizes, cache in (("attend", (8, 10343, 4, 1), 8 * 10343 * 512), ("attend", (256, 4352, 4, 1), 256 * 4352 * 512), ("attend", (8, 32768, 8, 4), 8 * 32768 * 512),
                                   ("shared", (64, 8, 32768, 512, 4, 1), (64 * 512 + 32768) * 8 * 512), ("evict", (256, 4352, 4096, 64), 256 * 4352 * 512)):
            used = fake.fake_used()
            h = context(LLAMA)
            assert globals()[name](h, *sizes) == 0
            out.append((fake.fake_used() - used) / cache)
            kept.clear()
            out.append(fake.fake_used() - used)
    """.replace("\n        ", "\n"))
    assert all(x <= 0.5 for x in out[::2]) and not any(out[1::2])


def test_memory_that_is_not_there():
    out = run(CALLS + """
        h = context(LLAMA)
        fake.fake_budget(fake.fake_used() + (1 << 20))
        out = [attend(h, 8, 10343, 4, 1), shared(h, 4, 8, 10343, 64, 4, 1), evict(h, 256, 4352, 4096, 64), len(launches())]
        fake.fake_budget(1 << 40)
        out += [attend(h, 8, 10343, 4, 1), shared(h, 4, 8, 10343, 64, 4, 1), evict(h, 256, 4352, 4096, 64)]
    """.replace("\n        ", "\n"))
    assert out == [-3, -3, -3, 0, 0, 0, 0]


def test_the_largest_calls_are_launched():
    largest = [
        ("attend", (2**22 - 1, 511, 1, 1)), ("attend", (2**22 - 1, 1, 1, 1)), ("attend", (1, 2**31 - 4097, 32, 1)), ("attend", (1, 2**31 - 4097, 1, 2**21)),
        ("attend", (2**17 - 1, 16383, 31, 1)), ("attend", (2**17 - 1, 16383, 11, 2)), ("attend", (63549, 33790, 33, 2)), ("attend", (2**20, 2047, 1, 3)),
        ("shared", (1, 2**22 - 1, 511, 511, 1, 1)), ("shared", (2**22 - 1, 1, 2**31 - 4097, 511, 1, 1)), ("shared", (2**21, 1, 2**31 - 4097, 0, 1, 1)),
        ("shared", (17, 2**17 - 1, 16383, 900, 1, 1)), ("shared", (32, 63549, 33790, 1000, 2, 1)),
        ("evict", (2**21 - 1, 1000, 500, 10)), ("evict", (1, 2**31 - 4097, 2**30, 2**29)), ("evict", (1, 2**31 - 4097, 1, 0))]
    out = run(CALLS + f"""
out = []
for name, sizes in {largest!r}:
    for D in (64, 128):
        h = context(LLAMA)
        rc = globals()[name](h, *sizes, D)
        log = fake.fake_launches().decode()
        out.append([rc, "REFUSED" in log, len(log.splitlines()) > 1])
""")
    assert out == [[0, False, True]] * (2 * len(largest))


def test_sizes_behind_the_largest_are_refused():
    out = run(CALLS + """
        h = context(LLAMA)
        out = [attend(h, 2**22, 1, 1, 1), attend(h, 1, 2**30, 1, 2**22), attend(h, 2**16, 2**15, 1, 1), shared(h, 2**11, 2**11, 8, 8, 1, 1),
               shared(h, 1, 2**16, 2**15, 8, 1, 1), shared(h, 2**8, 2**8, 8, 2**15, 1, 1), evict(h, 2**21, 10, 5, 1), len(launches())]
    """.replace("\n        ", "\n"))
    assert out == [-1] * 7 + [0]


def test_workspace_of_many_short_rows():
    """Two shares of D + 2 fp32 words a query at most, its logits by whole tiles and what it leaves, and 64 MB, however many rows there are: with one query
    a row it is not that of 32."""
    sizes = [("attend", (2**20, 16, 1, 1), 2**20, 32), ("attend", (2**18, 16, 4, 1), 2**20, 32), ("attend", (2**16, 100, 8, 2), 2**20, 128),
             ("shared", (2**12, 2**6, 100, 16, 1, 1), 2**18, 32)]
    out = run(CALLS + f"""
out = []
for name, sizes, queries, logits in {sizes!r}:
    used = fake.fake_used()
    h = context(LLAMA)
    assert globals()[name](h, *sizes) == 0
    out.append((fake.fake_used() - used) / (queries * (2 * 130 + logits + 6) * 4 + (1 << 26)))
    kept.clear()
""")
    assert all(x <= 1 for x in out), out


def test_threads_without_a_piece_store_nothing_in_the_longest_row(tmp_path):
    """A step of eviction's moves has 1024 pieces of 16 bytes; of those that are no whole token no thread may take part, however many entries are left."""
    (tmp_path / "t.cpp").write_text("""
#include "kernels.hpp"
#include <cstdio>
int main() {
  const int most = 2147483647 - 4096;  // entries of a row
  int bad = 0;
  for (int cps = 1; cps <= 32; ++cps)
    for (int step = 1024 / cps, piece = 0; piece < 1024; ++piece) {
      const int t = pkv::evict_token(piece, step, cps);
      bad += piece < step * cps ? t != piece / cps : t < most;
    }
  printf("%d", bad);
}
""")
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "paper_2605_16360_amd", "csrc"),
                    str(tmp_path / "t.cpp"), "-o", str(tmp_path / "t")], check=True)
    assert subprocess.run([str(tmp_path / "t")], capture_output=True, text=True, check=True).stdout == "0"
