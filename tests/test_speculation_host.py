"""The host side of the calls that check drafted tokens under UndefinedBehaviorSanitizer (host code only, no GPU): compiled with a
runtime that registers nothing and launches nothing, so that every call runs up to its last launch."""
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
static int32_t* ints() { return (int32_t*)at; }
static uint8_t* bytes() { return (uint8_t*)at; }
static mx_status plan(int64_t requests, int64_t tokens, int32_t words) {
    return mx_tree_plan(ints(), ints(), ints(), requests, tokens, words, (uint64_t*)at, ints(), nullptr);
}
static mx_status attend(const mx_cache& c, int64_t tokens, int64_t requests, int32_t heads_q, int64_t max_new, int64_t max_len, int64_t width,
                        int32_t type = MX_BF16, int32_t words = 1) {
    const int64_t row = (int64_t)heads_q * c.dim;
    return mx_cache_tree_attention(at, type, tokens, row, heads_q, c, at, bytes(), at, bytes(), ints(), width, ints(), ints(), (uint64_t*)at,
                                   words, requests, max_new, max_len, 0.125f, at, at, row, nullptr);
}
static mx_status verify(int64_t tokens, int64_t requests, int64_t vocab, int64_t width = 4, bool draft = true) {
    return mx_verify(at, draft ? at : nullptr, MX_F32, tokens, vocab, vocab, vocab, ints(), ints(), ints(), requests, (float*)at, (float*)at,
                     (float*)at, vocab, at, ints(), width, ints(), ints(), nullptr);
}
static mx_status move(const mx_cache& c, int64_t width, int64_t path_width, int64_t requests) {
    return mx_cache_move(c, at, bytes(), at, bytes(), ints(), width, ints(), ints(), path_width, ints(), requests, nullptr);
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
    for name, *flags in (("mx_tree",), ("mx_verify",), ("mx_cache_attention", "-DMX_CACHE_TREE=1")):
        objects.append(str(where / (name + ".o")))
        cmd = [HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-w", *flags, *include, "-Xarch_host",
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


def test_largest_arguments(run):
    """The largest of each argument alone and together: taken or refused, and nothing on the way leaves its type."""
    got = run("""
        const int64_t most = INT64_MAX;
        printf("%d %d %d ", plan(16384, 2147483647, 16), plan(16385, 8, 1), plan(1, most, 1));
        printf("%d %d ", plan(1, 8, 17), plan(1, 8, INT32_MAX));
        printf("%d %d %d ", verify(2147483647, 16384, 1 << 28, 2147483647), verify(8, 16385, 100), verify(most, 1, 100));
        printf("%d %d %d ", verify(8, 1, (1 << 28) + 1), verify(8, 1, most), verify(8, 1, 100, most));
        mx_cache c{};
        c.pages = 4; c.page = 1024; c.heads = 128; c.dim = 128;
        printf("%d %d %d ", move(c, 2147483647, 2147483647, 16384), move(c, most, 4, 1), move(c, 4, most, 1));
        c.heads = 1;
        printf("%d %d %d ", move(c, 4, 4, 16385), attend(c, 8, 1, 1, most, most, 4), attend(c, 2147483647 - 65536, 16384, 1, most, most, 4));
        printf("%d ", threads < (1ull << 32));""")
    assert got == ["0", "2", "2", "2", "2", "0", "2", "2", "2", "2", "2", "0", "2", "2", "2", "0", "2", "1"]


def test_trees_by_the_thousand_launch_in_bounds(run):
    """Requests times heads near 2^24 with as many row tiles again: refused, not launched in part; every launch counts its threads in 32 bits."""
    got = run("""
        mx_cache c{};
        c.pages = 4; c.page = 16; c.dim = 16;
        for (int type : {MX_F32, MX_BF16})
            for (int heads : {8, 300, 600, 1000}) {
                c.heads = heads;
                threads = 0;
                printf("%d ", attend(c, 16384 * 20, 16384, heads, 20, 64, 4, type));
                printf("%d ", threads < (1ull << 32));
            }""")
    # (2560 row tiles and a request each, 16384, in every head: 11.4 million of 600 heads, 18.9 of 1000)
    assert got == ["0", "1"] * 3 + ["2", "1"] + ["0", "1"] * 3 + ["2", "1"]


def test_workspaces_of_many_batches(run):
    """Arguments that a call takes have a workspace, and its size grows with them."""
    got = run("""
        uint64_t x = 12345;
        auto draw = [&](int64_t hi) { x = x * 6364136223846793005ull + 1442695040888963407ull; return 1 + (int64_t)((x >> 33) % (uint64_t)hi); };
        int bad = 0;
        for (int i = 0; i < 20000; ++i) {
            mx_cache c{};
            c.pages = 4; c.page = 16; c.heads = (int)draw(64); c.dim = 16 * (int)draw(8);
            const int group = (int)draw(8);
            const int64_t requests = draw(1 << draw(14)), tokens = draw(1 << draw(20)), most = draw(1 << draw(11)), len = draw(1ll << draw(30));
            const size_t n = mx_cache_tree_attention_workspace_bytes(c, tokens, requests, c.heads * group, most, len);
            const mx_status st = attend(c, tokens, requests, c.heads * group, most, len, 4, i & 1 ? MX_F32 : MX_BF16);
            bad += n == 0 ? st != MX_ERR_UNSUPPORTED : n < 65536;
            if (n == 0) continue;
            bad += mx_cache_tree_attention_workspace_bytes(c, tokens, requests, c.heads * group, most + 1, len + 1) < n;
            const size_t v = mx_verify_workspace_bytes(tokens, requests, len > 1 << 28 ? 1 << 28 : len);
            bad += v < 65536 || mx_verify_workspace_bytes(tokens + 1, requests + (requests < 16384), 1 << 28) < v;
            bad += verify(tokens, requests, len > 1 << 28 ? 1 << 28 : len, 4, i & 2) != MX_OK;
        }
        printf("%d", bad);""")
    assert got == ["0"]
