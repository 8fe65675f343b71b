"""The host side of the paged cache's calls under UndefinedBehaviorSanitizer (host code only, no GPU): compiled with a runtime
that registers nothing and launches nothing, so that every call runs up to its last launch."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")
CLANG, NM = "/opt/rocm/llvm/bin/clang++", "nm"

RUNTIME = r"""
#include <cstdint>
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include "mx.h"
extern "C" {
struct dim { unsigned x, y, z; };
static dim grid, block;
static size_t lds;
static void* on;
static uint64_t threads;   // of the largest launch
void** __hipRegisterFatBinary(const void*) { static void* handle; return &handle; }
void __hipUnregisterFatBinary(void**) {}
void __hipRegisterFunction(void**, const void*, char*, const char*, unsigned, void*, void*, void*, void*, int*) {}
int __hipPushCallConfiguration(dim g, dim b, size_t n, void* s) { grid = g; block = b; lds = n; on = s; return 0; }
int __hipPopCallConfiguration(dim* g, dim* b, size_t* n, void** s) { *g = grid; *b = block; *n = lds; *s = on; return 0; }
int hipLaunchKernel(const void*, dim g, dim b, void**, size_t, void*) {
    if ((uint64_t)g.x * b.x > threads) threads = (uint64_t)g.x * b.x;
    return 0;
}
int hipGetLastError() { return 0; }
int hipGetDevice(int* d) { *d = 0; return 0; }
int hipFuncSetAttribute(const void*, int, int) { return 0; }
}
static char at[1 << 12] __attribute__((aligned(256)));
static mx_status append(const mx_cache& c, int64_t tokens) {
    const int64_t row = (int64_t)c.heads * c.dim;
    return mx_cache_append(at, at, MX_F32, tokens, row, row, c, at, (uint8_t*)at, at, (uint8_t*)at, (int32_t*)at, nullptr);
}
static mx_status attend(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new, int64_t max_len, int64_t width) {
    const int64_t row = (int64_t)heads_q * c.dim;
    return mx_cache_attention(at, MX_BF16, tokens, row, heads_q, c, at, (uint8_t*)at, at, (uint8_t*)at, (int32_t*)at, width, (int32_t*)at,
                              (int32_t*)at, requests, max_new, max_len, 0.125f, at, at, row, nullptr);
}
"""


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    """Builds a program of the library's host code, the runtime above and a main(), and gives what it prints."""
    if not (os.path.exists(HIPCC) and os.path.exists(CLANG) and shutil.which(NM)):
        pytest.skip("no hipcc")
    where = tmp_path_factory.mktemp("host")
    include = ["-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2307_15517_amd", "csrc")]
    objects, fatbins = [], ""
    for name in ("mx_cache", "mx_cache_attention"):
        objects.append(str(where / (name + ".o")))
        cmd = [HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-w", *include, "-Xarch_host",
               "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all", "-Xarch_host", "-fno-sanitize=vptr,function",
               "-c", os.path.join(ROOT, "paper_2307_15517_amd", "csrc", name + ".hip"), "-o", objects[-1]]
        made = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert made.returncode == 0, made.stdout[-4000:]
        names = subprocess.run([NM, "-u", objects[-1]], stdout=subprocess.PIPE, text=True, check=True).stdout
        fatbins += "".join('extern "C" { char %s[64]; }\n' % n for n in re.findall(r"__hip_fatbin\w*", names))

    def program(body):
        source = where / "main.cpp"
        source.write_text(RUNTIME + fatbins + "int main() {\n" + body + "\nreturn 0;\n}\n")
        cmd = [CLANG, "-O1", "-std=c++17", "-w", *include, "-fsanitize=undefined", "-fno-sanitize-recover=all",
               "-fno-sanitize=vptr,function", str(source), *objects, "-o", str(where / "main")]
        made = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert made.returncode == 0, made.stdout[-4000:]
        ran = subprocess.run([str(where / "main")], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=60)
        assert ran.returncode == 0, ran.stdout[-4000:]
        return ran.stdout.split()
    return program


def test_a_bfloat16_cache_needs_no_format(run):
    """A format of zeros, as a C program leaves it for bfloat16 elements, and one of nonsense: block 0 is all that is read."""
    assert run("""
        mx_cache c{};
        c.pages = 4; c.page = 16; c.heads = 2; c.dim = 64;
        for (int bits : {0, -5, 40}) {
            c.f.exp_bits = bits;
            printf("%d ", append(c, 8));
            printf("%d ", append(c, 0));
            printf("%d ", attend(c, 8, 2, 4, 1, 64, 4));
            printf("%d ", attend(c, 80, 2, 4, 60, 64, 4));
        }""") == ["0"] * 12


def test_lengths_near_the_end_of_32_bits_are_refused(run):
    """A table row or packed rows so long that a kernel's key or row number, a tile past the last, would leave 32 bits."""
    got = run("""
        mx_cache c{};
        c.pages = 4; c.heads = 1; c.dim = 64;
        for (int page : {16, 128, 1024}) {
            c.page = page;
            for (int64_t room : {0, 127, 8192, 65535}) printf("%d ", attend(c, 1, 1, 1, 1, 1 << 20, (2147483647 - room) / page));
            printf("%d ", attend(c, 1, 1, 1, 1, 1 << 20, (2147483647 - 65536) / page));
        }
        c.page = 16;
        for (int heads_q : {1, 2, 7}) {
            printf("%d ", attend(c, 2147483647 / heads_q, 1, heads_q, 1, 64, 4));
            printf("%d ", attend(c, (2147483647 - 65536) / heads_q, 1, heads_q, 1, 64, 4));
        }""")
    assert got == ["2", "2", "2", "2", "0"] * 3 + ["2", "0"] * 3


def test_launches_of_many_tokens_stay_below_32_bits(run):
    """The threads of a launch are counted in 32 bits: padding tokens of a step without requests, as many as a call takes."""
    got = run("""
        mx_cache c{};
        c.pages = 4; c.page = 16; c.heads = 1; c.dim = 16;
        for (int64_t tokens : {(int64_t)1, (int64_t)1 << 24, (int64_t)1 << 25, (int64_t)2147483647 - 65536}) {
            threads = 0;
            printf("%d ", attend(c, tokens, 0, 1, 1, 1, 4));
            printf("%d ", threads > 0 && threads < (1ull << 32));
        }""")
    assert got == ["0", "1"] * 4


def test_batches_of_more_workgroups_than_a_launch_can_have_are_refused(run):
    """Requests times heads near 2^24 with as many row tiles again: refused, not launched in part."""
    got = run("""
        mx_cache c{};
        c.pages = 4; c.page = 16; c.dim = 16;
        for (int heads : {8, 300, 600, 1000}) {
            c.heads = heads;
            threads = 0;
            printf("%d ", attend(c, 16384 * 20, 16384, heads, 20, 64, 4));
            printf("%d ", threads < (1ull << 32));
        }
        c.heads = 1;
        printf("%d ", attend(c, 2147483647 - 65536, 16384, 1, 1 << 20, 64, 4));""")
    assert got == ["0", "1", "0", "1", "2", "1", "2", "1", "2"]
