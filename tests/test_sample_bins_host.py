"""Borders in the running sums of a row's histogram, `csrc/sample_bins.h` compiled with the host C++ compiler (no GPU):
whatever the sums and the target, one thread of the row has the border, and it is the bin that one running sum over
all bins finds.  The threads' sums are made as the kernel makes them, a scan in a warp and a butterfly over the warps'
totals; with sums in fp32 made so, some targets have two such threads or none."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36452_gb300", "csrc")

DRIVER = r"""
#include "sample_bins.h"
#include <cmath>
#include <cstdio>
#include <random>
#include <vector>
constexpr int kBins = 4096, kThreads = 512;

// Sums before and behind every thread's bins, as the kernel adds them up.
template <typename Sum>
void running(const std::vector<Sum> &bins, int ranks, std::vector<Sum> &before, std::vector<Sum> &behind) {
    const int per = kBins / ranks / kThreads, threads = ranks * kThreads, warps = threads / 32;
    std::vector<Sum> upto(threads), own(threads);
    for (int t = 0; t < threads; ++t) {
        Sum m = 0;
        for (int i = 0; i < per; ++i) m += bins[t * per + i];
        own[t] = upto[t] = m;
    }
    for (int o = 1; o < 32; o <<= 1) {
        const std::vector<Sum> old = upto;
        for (int t = 0; t < threads; ++t)
            if (t % 32 >= o) upto[t] += old[t - o];
    }
    before.resize(threads);
    behind.resize(threads);
    for (int w = 0; w < warps; ++w) {
        Sum lane[32] = {};
        for (int i = 0; i < warps; ++i)  // lane l looks at the totals l, l + 32, ...
            if (i < w) lane[i % 32] += upto[i * 32 + 31];
        for (int o = 16; o; o >>= 1) {
            Sum other[32];
            for (int l = 0; l < 32; ++l) other[l] = lane[l ^ o];
            for (int l = 0; l < 32; ++l) lane[l] += other[l];
        }
        for (int l = 0; l < 32; ++l) behind[w * 32 + l] = lane[0] + upto[w * 32 + l];
        for (int l = 0; l < 32; ++l) before[w * 32 + l] = l ? behind[w * 32 + l - 1] : lane[0];
    }
}

int main() {
    std::mt19937 rng(5);
    long long bad = 0, bad_floats = 0, asked = 0;
    double worst = 0;
    for (int kind = 0; kind < 6; ++kind)
        for (int ranks = 1; ranks <= 8; ranks *= 2) {
            std::normal_distribution<double> normal;
            std::vector<int> count(kBins);
            const double width = kind < 3 ? 64.0 / kBins : 12.0 / kBins;  // of a bin, in octaves
            double middle = kind % 3 == 0 ? 14 : kind % 3 == 1 ? 4 : 30;
            for (int i = 0; i < 152064; ++i) {
                const int b = static_cast<int>((middle + 2.5 * normal(rng)) / width);
                if (b >= 0 && b < kBins) ++count[b];
            }
            count[0] += 1;
            std::vector<float> weight(kBins);
            double sum = 0;
            for (int b = 0; b < kBins; ++b) {
                weight[b] = static_cast<float>(count[b] * std::exp2(-(b + 0.5) * width));
                sum += weight[b];
            }
            const float about = static_cast<float>(sum * (1 + 1e-5 * normal(rng))), units = rpd::kBinUnits / about;
            std::vector<uint32_t> bins(kBins), before, behind;
            std::vector<int> tokens, tokens0, tokens1;
            double off = 0;
            for (int b = 0; b < kBins; ++b) {
                bins[b] = rpd::bin_units(weight[b], units);
                off += std::fabs(bins[b] * static_cast<double>(about) / rpd::kBinUnits - weight[b]);
                tokens.push_back(count[b]);
            }
            worst = std::fmax(worst, off / about);
            running(bins, ranks, before, behind);
            running(tokens, ranks, tokens0, tokens1);
            std::vector<float> float0, float1;
            running(weight, ranks, float0, float1);
            const int threads = ranks * kThreads, per = kBins / threads;
            rpd::BinBorder border{false, false, 0.f, about / rpd::kBinUnits};
            const auto ask = [&](float least, bool more, bool by_count) {
                border.least = least;
                border.more = more;
                border.by_count = by_count;
                int holders = 0, found = kBins, first = kBins, n = 0;
                uint32_t m = 0;
                for (int b = 0; b < kBins; ++b) {
                    m += bins[b];
                    n += count[b];
                    if (border.holds(n, m)) {
                        first = b;
                        break;
                    }
                }
                for (int t = 0; t < threads; ++t)
                    if (border.within(t == 0, tokens0[t], before[t], tokens1[t], behind[t])) {
                        ++holders;
                        n = tokens0[t];
                        m = before[t];
                        for (int i = 0; i < per; ++i) {
                            n += count[t * per + i];
                            m += bins[t * per + i];
                            if (i == per - 1 || border.holds(n, m)) {
                                found = t * per + i;
                                break;
                            }
                        }
                    }
                bad += holders != (first < kBins) || found != first;
                ++asked;
                if (by_count) return;
                holders = 0;
                for (int t = 0; t < threads; ++t) {
                    const auto f = [&](float x) { return more ? x > least : x >= least; };
                    holders += (t == 0 || !f(float0[t])) && f(float1[t]);
                }
                bad_floats += holders > 1;
            };
            for (int i = 0; i < 150; ++i) {
                const int t = static_cast<int>(rng() % threads), w = t / 32 * 32;
                for (float x : {border.weight(behind[t]), border.weight(before[w]), float0[t], float1[t], float0[w]})
                    for (float y : {std::nextafterf(x, 0.f), x, std::nextafterf(x, 1e9f)})
                        for (int more = 0; more < 2; ++more) ask(y, more, false);
                ask(static_cast<float>(rng() % 160000), false, true);
                ask(about * (rng() % 100000) * 1e-5f, i & 1, false);
            }
            for (float x : {-1.f, 0.f, about * 2.f}) ask(x, false, false), ask(x, true, false);
        }
    std::printf("%lld %lld %lld %.9g\n", asked, bad, bad_floats, worst);
    return 0;
}
"""


def test_one_thread_has_the_border(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if not cxx:
        pytest.skip("no host C++ compiler")
    src, exe = tmp_path / "bins.cpp", tmp_path / "bins"
    src.write_text(DRIVER)
    subprocess.run([cxx, "-std=c++17", "-O1", "-Wall", "-Werror", "-I", CSRC, "-o", str(exe), str(src)], check=True)
    asked, bad, bad_floats, worst = subprocess.run([str(exe)], check=True, capture_output=True, text=True).stdout.split()
    assert int(asked) > 10000
    assert int(bad) == 0
    assert int(bad_floats) > 0  # what fp32 sums would do with the same targets
    # 4096 bins, half a unit of 2^-30 of the sum each; quotient and product are an fp32 rounding off, 2^-23 of the sum
    assert float(worst) <= 4096 * 2.0 ** -31 + 2.0 ** -22
