"""What hsadmm_softmax_loss writes lies inside the regions of its workspace: the host arithmetic that cuts the products into tiles
(csrc/loss_plan.hpp), compiled by itself and swept over sizes, types and pieces of the vocabulary."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SWEEP = r"""
#include <cstdio>
#include <vector>
#include "loss_plan.hpp"

static long long cases = 0, wrong = 0;
static int64_t up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

static void say(const char* what, int64_t size, bool gradients, int64_t n, int64_t D, int64_t V, int64_t held, int64_t a, int64_t b)
{
    if (++wrong <= 20)
        std::printf("%s: size %lld gradients %d n %lld D %lld V %lld held %lld: %lld for %lld\n", what, (long long)size, (int)gradients,
                    (long long)n, (long long)D, (long long)V, (long long)held, (long long)a, (long long)b);
}

static void check(int64_t size, bool gradients, int64_t n, int32_t D, int32_t V, int64_t off, int64_t held)
{
    const LossScratch s = loss_scratch(held, V, D, off, n, size, gradients);
    ++cases;
    const auto fits = [&](const char* what, int64_t needs, int64_t has) { if (needs > has) say(what, size, gradients, n, D, V, held, needs, has); };
    // rows and columns that a product's tiles cover, and those that its outputs have room for
    const auto rows = [&](const ProductPlan& p) { return up(n, p.b); };
    const auto across = [](const ProductPlan& p, int64_t out) { return up(out, p.b == kNarrow ? kNarrowTile : p.b); };
    fits("rows of the logits", rows(s.logits), s.Np);
    fits("rows of the logits' gradients", up(n, s.logits.b == kNarrow ? 128 : s.logits.b), s.Np);
    if (gradients) fits("rows of the inputs' sums", rows(s.inputs), s.Np);
    if (!s.small) {
        const int waves = s.logits.b == kNarrow ? 4 : 2;
        if (s.slab_elems * waves != (s.logits.b == kNarrow ? kNarrowTile : s.logits.b)) say("classes of a slab", size, gradients, n, D, V, held, s.slab_elems, s.logits.b);
        fits("slabs", across(s.logits, V) / s.slab_elems, s.slabs);
    }
    fits("classes", V, s.pieces * s.Vc);
    fits("a piece too many", (s.pieces - 1) * s.Vc + 1, V);
    if (s.small) fits("pieces of small logits", s.pieces, 1);
    // the k axis is covered once, by parts that begin at a multiple of a tile's length
    const auto covered = [&](const char* what, const ProductPlan& p, int64_t k) {
        fits(what, k, p.splits * p.k_part);
        fits(what, (p.splits - 1) * p.k_part + 1, std::max<int64_t>(k, 1));
        fits(what, p.k_part % 64, 0);
    };
    covered("k of the logits", s.logits, s.Dp);
    covered("k of the inputs' gradients", s.inputs, s.Vc);
    // regions: in this order, each as long as what is written there
    const int64_t each = s.rest_inputs || s.rest_weights ? 2 : 1;
    const struct { const char* what; size_t at; int64_t bytes; } all[] = {
        {"head", s.head, kLossHeadBytes}, {"row", s.row, 4 * n}, {"label", s.label, 4 * n}, {"place", s.place, 4 * n},
        {"held_loss", s.held_loss, 4 * n}, {"picked", s.picked, 4 * n}, {"own", s.own, gradients ? 4 * n : 0}, {"rounded", s.rounded, gradients ? 4 * s.Np : 0}, {"stat", s.stat, 8 * n}, {"slab", s.slab, 8 * s.slabs * s.Np},
        {"rows", s.rows, size * s.Np * s.Dp}, {"packed", s.packed, s.pack ? size * std::min<int64_t>(V, s.Vc) * s.Dp : 0},
        {"parts", s.parts, s.small ? 4 * s.logits.splits * s.Np * s.Vc : 0}, {"grads", s.grads, gradients ? each * size * s.Np * s.Vc : 0},
        {"sums", s.sums, gradients ? 4 * s.inputs.splits * s.Np * s.Dp : 0}, {"total", s.total, 0}};
    for (size_t i = 0; i + 1 < sizeof all / sizeof *all; ++i) {
        fits(all[i].what, (int64_t)all[i].at + all[i].bytes, (int64_t)all[i + 1].at);
        fits(all[i].what, (int64_t)(all[i].at % 256), 0);
    }
}

int main()
{
    const int64_t ns[] = {0, 1, 2, 31, 32, 33, 48, 64, 65, 100, 127, 128, 129, 192, 255, 256, 257, 300, 511, 513, 1000, 1024, 1537, 4095, 4096, 8191, 16384, 65536, 1000003, 1 << 21};
    const int32_t Ds[] = {1, 5, 8, 24, 63, 64, 65, 72, 128, 255, 256, 512, 1000, 1024, 1441, 2048, 4096, 4104, 8192, 16384};
    const int32_t Vs[] = {1, 3, 10, 64, 127, 128, 129, 255, 256, 257, 700, 1000, 4096, 4100, 8192, 16383, 16384, 20011, 32000, 32768, 65280, 65281, 65536, 70000,
                          131072, 151936, 262144, 1 << 20};
    const int64_t helds[] = {kLossHeld, 1ll << 28, 1ll << 22, 1};
    for (int64_t size : {2, 4})
        for (int gradients = 0; gradients < 2; ++gradients)
            for (int64_t off : {0, 4})
                for (int64_t n : ns)
                    for (int32_t D : Ds)
                        for (int32_t V : Vs)
                            for (int64_t held : helds) check(size, gradients != 0, n, D, V, off, held);
    std::printf("%lld of %lld\n", wrong, cases);
    return wrong != 0;
}
"""


def test_what_the_products_write_lies_inside_the_workspaces_regions(tmp_path):
    src, exe = tmp_path / "sweep.cpp", tmp_path / "sweep"
    src.write_text(SWEEP)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused-function", "-Werror", "-I", os.path.join(ROOT, "paper_2512_14628_amd", "csrc"),
                           str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout
    assert r.stdout.startswith("0 of ")
