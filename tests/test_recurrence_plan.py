"""How the recurrence deals out an utterance's frames (csrc/layer_block_internal.h), compiled for the host: every frame is somebody's, launches and workspaces
fit what the kernels assume."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = r'''
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <initializer_list>
#include <vector>
#include "layer_block_internal.h"
using namespace layer;
static unsigned long long seed = 12345;
static unsigned rnd() { seed = seed * 6364136223846793005ull + 1442695040888963407ull; return static_cast<unsigned>(seed >> 33); }
static void fail(const char* what, int T, int B, int H, int F, int V) { std::printf("%s: T %d B %d H %d forward %d V %d\n", what, T, B, H, F, V); std::exit(1); }
static void look(int T, int B, int H, int F)
{
    const int back = H - F;
    const int V = (F == 0 || F >= 2) && (back == 0 || back >= 2) ? 2 : 1, tile = 64 * V;
    const int64_t tiles = (F + tile - 1) / tile + (back + tile - 1) / tile;
    for (int run : {kRun, kRunBack}) {
        const RecurrencePlan p = recurrence_plan(T, tiles * B, run);
        if (p.waves != 1 && p.waves != 4 && p.waves != kRecurrenceWaves) fail("waves", T, B, H, F, V);
        if (p.waves * run < T && p.waves != kRecurrenceWaves) fail("too few wavefronts", T, B, H, F, V);
        if (p.stretches < 1 || static_cast<int64_t>(p.steps) * p.stretches < T) fail("frames left over", T, B, H, F, V);
        if (p.stretches > 1 && (p.waves != kRecurrenceWaves || p.steps % (run * p.waves))) fail("a stretch of no whole rounds", T, B, H, F, V);
        if (p.stretches > 1 && static_cast<int64_t>(p.steps) * (p.stretches - 1) >= T) fail("an empty stretch", T, B, H, F, V);
        if (tiles * B * p.stretches > 0x7fffffffll) fail("groups", T, B, H, F, V);
        if (p.stretches > 1 && static_cast<size_t>(p.stretches + 1) * B * H * 16 > recurrence_bytes(T, B, H)) fail("workspace", T, B, H, F, V);
        if (p.stretches > 1 && recurrence_bytes(T, B, H) == 0) fail("no workspace", T, B, H, F, V);
        if (p.stretches > 1 && p.stretches * (tiles * B) > 512) fail("more than fill the compute units", T, B, H, F, V);
    }
}
int main()
{
    for (int T : {1, 2, 4, 5, 16, 17, 32, 33, 64, 65, 127, 128, 129, 191, 192, 193, 224, 255, 256, 257, 1000, 40000, 1 << 20, 1 << 30})
        for (int B : {1, 2, 3, 31, 64, 512, 65535})
            for (int H : {1, 2, 3, 63, 64, 65, 127, 128, 129, 1999, 2048, 16383, 16384})
                for (int F : {0, 1, H / 2, H - 1, H})
                    if (F >= 0 && static_cast<int64_t>(T) * B <= 1 << 30) look(T, B, H, F);
    for (int i = 0; i < 300000; ++i) {
        const int T = 1 + rnd() % (1u << rnd() % 22), B = 1 + rnd() % (1u << rnd() % 10), H = 1 + rnd() % 16384;
        look(T, B, H, static_cast<int>(rnd() % (H + 1)));
    }
    for (int H = 1; H <= 16384; ++H) {
        const RowTeam t = row_team(H);
        if (t.lanes * t.elements < H || t.lanes > 1024 || (t.lanes > 64 && t.lanes % 64)) fail("a row's team", 0, 0, H, 0, 0);
        if (t.lanes <= 64 && t.rows * t.lanes != 256) fail("teams of a workgroup", 0, 0, H, 0, 0);
        int last = 0;
        for (int rows : {1, 2, 7, 8, 31, 33, 255, 1000, 5000, 100000, 1 << 30}) {
            const int g = block_norm_groups(rows, H);
            if (g < 1 || g < last || g > 2048 || (g - 1) * static_cast<int64_t>(t.rows) >= rows) fail("groups", rows, 0, H, 0, 0);
            last = g;
        }
    }
    // Each unit of each utterance is one workgroup's, and no die has many more than another.
    for (unsigned B : {1, 2, 5, 7, 8, 9, 15, 16, 17, 27, 63, 64, 65, 200})
        for (unsigned units : {1, 2, 3, 4, 7, 8, 9, 13, 16, 17, 31, 128, 257, 512}) {
            const unsigned each = units_of_a_die(units, B);
            std::vector<int> seen(static_cast<size_t>(B) * units, 0);
            int64_t count = 0;
            for (unsigned number = 0; number < 8 * each + 1000; ++number) {
                const Unit u = unit_of(number, units, B);
                if (u.utterance >= B) continue;
                if (u.unit >= units) fail("no such unit", 0, B, units, 0, 0);
                if (number >= 8 * each) fail("behind the grid", 0, B, units, 0, 0);
                if (seen[static_cast<size_t>(u.utterance) * units + u.unit]++) fail("twice", 0, B, units, 0, 0);
                ++count;
            }
            if (count != static_cast<int64_t>(B) * units) fail("nobody's", 0, B, units, 0, 0);
            if (8ll * each > count + 7) fail("idle workgroups", 0, B, units, 0, 0);
        }
    std::puts("ok");
}
'''


def test_every_frame_is_somebodys(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PROGRAM)
    include = ["-I", str(tmp_path), "-I", os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_1512_02595_amd", "csrc")]
    subprocess.run(["g++", "-std=c++17", "-O2", *include, str(src), "-o", str(exe)], check=True)
    assert subprocess.run([str(exe)], capture_output=True, text=True).stdout.strip() == "ok"
