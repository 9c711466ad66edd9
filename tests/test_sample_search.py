"""The threshold search of the draw (csrc/sample.cu), walked through on the host with the kernel's own key arithmetic
(csrc/sample_keys.h): every entry that a round counts has a bin of the histogram, and the key that comes out is the
wanted one in the sorted row.  Rows with zeros of both signs beside the smallest negative values are the hard ones: the
key between those of zero and of the largest negative value is that of -0, which no entry has."""
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CUDA = os.environ.get("CUDA_HOME", "/usr/local/cuda")

PROGRAM = r"""
#include <algorithm>
#include <cstdio>
#include <vector>
#include "sample_keys.h"
using namespace gala;

// the wanted-th largest of the entries above `floor`, as the kernel finds it; 1: a bin outside the histogram, 2: no end
template <typename T>
int search(const std::vector<uint32_t>& bits, float temp, uint32_t floor, long long wanted, uint32_t& key, long long& ahead) {
    uint32_t top = 0;
    for (uint32_t u : bits) top = std::max(top, key_of<T>(u));
    const float most = logit_of<T>(top), inv = 1.0f / temp;
    const int last = kBins - 1;
    auto step = [&](float l) { return (int)std::fmin((most - l) * inv * kFirstBins, (float)last); };
    std::vector<long long> bins(kBins, 0);
    long long tail = 0;
    const float least = logit_of<T>(floor);
    for (uint32_t u : bits) {
        const float x = value_of<T>(u);
        if (x > least) {
            const int b = step(x);
            if (b < last) bins[b]++;
            else tail++;
        }
    }
    ahead = 0;
    int b1 = -1;
    long long c = 0;
    for (int b = 0; b < kBins && b1 < 0; b++) {
        if (c + bins[b] >= wanted) b1 = b, ahead = c;
        c += bins[b];
    }
    KeyRange<T> range = {floor + 1, top};
    if (b1 >= 0) {
        uint32_t a = floor + 1, b = top;
        while (a < b) {
            const uint32_t m = a + (b - a) / 2;
            if (step(logit_of<T>(m)) <= b1) b = m;
            else a = m + 1;
        }
        range.lo = a;
        b = top;
        while (a < b) {
            const uint32_t m = a + (b - a + 1) / 2;
            if (step(logit_of<T>(m)) >= b1) a = m;
            else b = m - 1;
        }
        range.hi = a;
    }
    for (int rounds = 0; range.lo < range.hi; rounds++) {
        if (rounds > 8) return 2;
        const int shift = range.shift();
        std::fill(bins.begin(), bins.end(), 0);
        const float from = range.from(), to = range.to();
        for (uint32_t u : bits) {
            const float x = value_of<T>(u);
            if (x >= from && x <= to) {
                const uint32_t b = range.bin(u, shift);
                if (b >= (uint32_t)kBins) return 1;
                bins[b]++;
            }
        }
        int at = -1;
        c = ahead;
        for (int b = 0; b < kBins && at < 0; b++) {
            if (c + bins[b] >= wanted) at = b;
            else c += bins[b];
        }
        if (at < 0) return 2;
        ahead = c;
        range.narrow(at, shift);
    }
    key = range.hi;
    return 0;
}

template <typename T>
int row(const std::vector<uint32_t>& bits, float temp, long long k, long long k2) {
    std::vector<uint32_t> sorted;
    for (uint32_t u : bits) sorted.push_back(key_of<T>(u));
    std::sort(sorted.rbegin(), sorted.rend());
    uint32_t cut = 0;
    long long ahead = 0;
    int rc = search<T>(bits, temp, key_bottom<T>(), k, cut, ahead);
    if (rc) return rc;
    if (cut != sorted[k - 1] || ahead != std::lower_bound(sorted.begin(), sorted.end(), cut, [](uint32_t a, uint32_t b) { return a > b; }) - sorted.begin()) return 3;
    // a second search among what lies above that cut, as top-p's after top-k's
    if (ahead >= k2 && k2 > 0) {
        const uint32_t floor = cut;
        if ((rc = search<T>(bits, temp, floor, k2, cut, ahead))) return 10 + rc;
        if (cut != sorted[k2 - 1]) return 13;
    }
    return 0;
}

int main(int, char** argv) {
    FILE* f = fopen(argv[1], "rb");
    int head[4];
    float temp;
    int n = 0, bad = 0;
    while (fread(head, 4, 4, f) == 4 && fread(&temp, 4, 1, f) == 1) {
        std::vector<uint32_t> bits(head[1]);
        if (fread(bits.data(), 4, bits.size(), f) != bits.size()) return 9;
        const int rc = head[0] == 0 ? row<float>(bits, temp, head[2], head[3])
                       : head[0] == 1 ? row<__nv_bfloat16>(bits, temp, head[2], head[3])
                                      : row<__half>(bits, temp, head[2], head[3]);
        if (rc && bad++ < 5) printf("row %d: type %d, %d entries, T %g, wanted %d then %d: %d\n", n, head[0], head[1], temp, head[2], head[3], rc);
        n++;
    }
    printf("%d rows, %d bad\n", n, bad);
    return bad ? 1 : 0;
}
"""


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    if not shutil.which("g++") or not os.path.isdir(os.path.join(CUDA, "include")):
        pytest.skip("needs g++ and the CUDA headers")
    at = tmp_path_factory.mktemp("search")
    src, exe = at / "search.cpp", at / "search"
    src.write_text(PROGRAM)
    subprocess.run(["g++", "-O2", "-std=c++17", "-I", os.path.join(CUDA, "include"), "-I", os.path.join(ROOT, "paper_1906_04585_b200", "csrc"), str(src), "-o", str(exe)],
                   check=True)

    def go(rows):
        """rows: (type, stored bits, temperature, first wanted rank, second)"""
        with open(at / "rows", "wb") as f:
            for kind, bits, temp, k, k2 in rows:
                np.array([kind, len(bits), k, k2], np.int32).tofile(f)
                np.array([temp], np.float32).tofile(f)
                np.asarray(bits).astype(np.uint32).tofile(f)
        r = subprocess.run([str(exe), str(at / "rows")], capture_output=True, text=True)
        assert r.returncode == 0, r.stdout

    return go


F32, BF16, F16 = 0, 1, 2
SIGN = {F32: 1 << 31, BF16: 1 << 15, F16: 1 << 15}


def stored(kind, values):
    v = np.asarray(values, np.float32)
    if kind == F16:
        return v.astype(np.float16).view(np.uint16).astype(np.uint32)
    return v.view(np.uint32) >> (16 if kind == BF16 else 0)


def around_zero(kind, top, zeros, below, step=1):
    """One entry of the bits `top`, zeros of both signs, and `below` entries `step` units below zero."""
    z = np.where(np.arange(zeros) % 3 == 2, SIGN[kind], 0)
    return np.concatenate([[top], z, np.full(below, SIGN[kind] + step)])


def test_zeros_beside_the_smallest_negative_values(walk):
    rows = [(F16, around_zero(F16, 7, 100, 300), 1.0, 150, 20),
            (F16, around_zero(F16, int(stored(F16, [0.0664673])[0]), 99, 900), 1.7, 500, 50),
            (F32, around_zero(F32, 0x0007ffff, 100, 300), 1.0, 150, 20),
            (F32, around_zero(F32, int(stored(F32, [0.99999994])[0]), 100, 300), 200.0, 150, 20)]
    rng = np.random.default_rng(1)
    for kind, most in ((F16, 0x7c00), (BF16, 0x7f80), (F32, 0x7f800000)):
        for _ in range(400):
            top = int(np.exp(rng.uniform(0, np.log(most - 1))))
            zeros, below = int(rng.integers(1, 120)), int(rng.integers(200, 700))
            row = around_zero(kind, top, zeros, below, int(np.exp(rng.uniform(0, 6))))
            row = np.concatenate([row, SIGN[kind] + rng.integers(1, 900, 50), rng.integers(0, top + 1, 30)])
            rng.shuffle(row)
            k = int(rng.integers(1, len(row) + 1))
            rows.append((kind, row, float(np.exp(rng.uniform(-4, 6))), k, int(rng.integers(0, k))))
    walk(rows)


def test_every_threshold_of_mixed_rows(walk):
    rng = np.random.default_rng(2)
    rows = []
    for kind in (F16, BF16, F32):
        for scale in (2.5, 1e-3, 1e-7, 30.0):
            v = stored(kind, rng.standard_normal(400) * scale)
            v[::40] = 0
            v[1::40] = SIGN[kind]
            for k in range(1, 400, 7):
                rows.append((kind, v, float(np.exp(rng.uniform(-2, 2))), k, int(rng.integers(0, k))))
    walk(rows)
