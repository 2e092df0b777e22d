"""The weight gradient's layout on the host: every kept weight is the product of its own row of G and row of X, once, and
what the kernel reads lies inside the arrays.  The builder is compiled with gcc and its sanitizers into a driver program."""
import os
import shutil
import subprocess

import pytest

import paper_2407_19644_amd as ubp

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2407_19644_amd", "csrc")

DRIVER = r"""
#include <cstdio>
#include <cstdlib>
#include <vector>
#include "ubp_internal.h"

namespace ubp {
ubp_status upload(ubp_packed *) { return UBP_ERR_DEVICE; }
void release_device(ubp_packed *) {}
}

#define CHECK(c) do { if (!(c)) { std::fprintf(stderr, "line %d: %s\n", __LINE__, #c); return 1; } } while (0)

int main(int argc, char **argv) {
    CHECK(argc == 8);
    const int M = atoi(argv[1]), K = atoi(argv[2]), bh = atoi(argv[3]), bw = atoi(argv[4]), mode = atoi(argv[6]);
    const double density = atof(argv[5]);
    const ubp_dtype dt = (ubp_dtype)atoi(argv[7]);
    int64_t nb = ubp_target_block_count(M, K, bh, bw, density);
    std::vector<ubp_block> blocks((size_t)nb + 1);
    int64_t got = 0;
    CHECK(ubp_select_reference(M, K, bh, bw, density, 7, mode, 1.1, blocks.data(), nb, &got) == UBP_OK && got == nb);
    std::vector<unsigned char> W((size_t)M * K * (dt == UBP_F32 ? 4 : 2), 1);
    ubp_packed *p = nullptr;
    CHECK(ubp_pack(W.data(), dt, M, K, K, bh, bw, blocks.data(), nb, UBP_HOST_ONLY, &p) == UBP_OK);
    const ubp::GradLayout &L = ubp::get_grad_layout(p);
    CHECK(L.usable && L.built);
    CHECK((int64_t)L.ops.size() == L.n_tiles * 16 && (int64_t)L.inv.size() == L.n_tiles * 256 && (int)L.regions.size() == 4 * L.n_regions);
    const ubp::GradShape S = ubp::kGradShapes[L.shape];
    CHECK(L.max_tiles <= S.tiles && L.max_g <= S.g_slots && L.max_x <= S.x_slots);
    std::vector<int32_t> start((size_t)nb);
    for (int r = 0; r + bh <= M; ++r)
        for (int32_t b = p->indptr[(size_t)r]; b < p->indptr[(size_t)r + 1]; ++b) start[(size_t)b] = r;
    std::vector<char> seen((size_t)(nb * bh * bw), 0);
    int64_t next_tile = 0;
    CHECK((int64_t)L.rows.size() == (int64_t)L.n_regions * (L.max_g + L.max_x));
    for (int g = 0; g < L.n_regions; ++g) {
        const int32_t *R = &L.regions[(size_t)g * 4], *rows_g = L.rows.data() + (size_t)g * (L.max_g + L.max_x), *rows_x = rows_g + L.max_g;
        const int64_t first = R[0], tiles = R[1], g_slots = R[2], x_slots = R[3];
        CHECK(first == next_tile && tiles >= 1);
        next_tile += tiles;
        CHECK(g_slots > 0 && x_slots > 0 && g_slots % 16 == 0 && x_slots % 16 == 0 && g_slots <= L.max_g && x_slots <= L.max_x);
        CHECK((tiles + ubp::kGradWaves - 1) / ubp::kGradWaves <= L.max_tiles);
        for (int s = 0; s < L.max_g; ++s) CHECK(rows_g[s] >= 0 && rows_g[s] < M);
        for (int s = 0; s < L.max_x; ++s) CHECK(rows_x[s] >= 0 && rows_x[s] < K);
        for (int64_t t = first; t < first + tiles; ++t) {
            int32_t gr[16], xr[16];
            for (int k = 0; k < 16; ++k) {
                const uint32_t o = L.ops[(size_t)(t * 16 + k)];
                CHECK((int64_t)(o & 0xffff) < g_slots && (int64_t)(o >> 16) < x_slots);
                gr[k] = rows_g[o & 0xffff];
                xr[k] = rows_x[o >> 16];
            }
            for (int i = 0; i < 16; ++i)
                for (int j = 0; j < 16; ++j) {
                    const int32_t v = L.inv[(size_t)(t * 256 + (16 * (i / 4) + j) * 4 + i % 4)];
                    CHECK(v >= -1 && v < nb * bh * bw);
                    if (v < 0) continue;
                    CHECK(!seen[(size_t)v]);
                    seen[(size_t)v] = 1;
                    const int64_t b = v / (bh * bw);
                    const int q = v / bh % bw, s = v % bh;
                    const int row = start[(size_t)b] + ((s - start[(size_t)b]) % bh + bh) % bh;
                    CHECK(gr[i] == row && xr[j] == p->indices[(size_t)b] + q);
                }
        }
    }
    CHECK(next_tile == L.n_tiles);
    for (char c : seen) CHECK(c);
    for (int64_t n : {0, 1, 63, 64, 65, 127, 128, 129, 1567, 4096, 8192, 12543, 1 << 20, 0x7fffffff}) {
        const ubp::GradRanges r = ubp::grad_ranges(L, n, dt == UBP_F32 ? 32 : 64);
        CHECK(r.splits >= 1 && r.splits <= 256 && r.tokens >= 64 && r.tokens % 64 == 0);
        CHECK(r.splits == 1 || (int64_t)(r.splits - 1) * r.tokens < n);
        CHECK((int64_t)r.splits * r.tokens + 63 >= n);
    }
    std::printf("%lld tiles %d regions %d of a wavefront %d + %d rows\n", (long long)L.n_tiles, L.n_regions, L.max_tiles, L.max_g, L.max_x);
    ubp_packed_free(p);
    return 0;
}
"""

LAYERS = [  # M, K, bh, bw, density, mode, dtype
    (64, 64, 4, 4, 0.5, 0, 0), (960, 160, 4, 4, 0.3, 0, 1), (256, 2304, 4, 4, 0.25, 0, 2), (512, 512, 4, 1, 0.2, 0, 1),
    (1024, 1024, 16, 16, 0.1, 1, 2), (100, 300, 8, 8, 0.2, 0, 2), (70, 45, 3, 1, 0.4, 0, 0), (33, 40, 5, 3, 0.3, 0, 1),
    (256, 256, 2, 1, 0.3, 0, 1), (256, 256, 1, 1, 0.5, 0, 1), (64, 900, 1, 7, 0.3, 0, 2), (130, 90, 20, 4, 0.3, 0, 1),
    (300, 64, 33, 2, 0.2, 0, 0), (16, 16, 16, 16, 1.0, 0, 1), (40, 50, 40, 50, 1.0, 0, 2), (17, 19, 1, 1, 1.0, 0, 2),
    (96, 3000, 2, 2, 0.9, 0, 2)[:4] + (0.5, 0, 2), (8, 8, 4, 4, 0.0, 0, 1), (1, 1, 1, 1, 1.0, 0, 0), (4096, 4096, 16, 16, 0.1, 1, 2),
]


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("grad_layout")
    src = d / "driver.cpp"
    src.write_text(DRIVER)
    exe = d / "driver"
    cmd = [gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-I", os.path.join(ROOT, "include"), "-I", CSRC, str(src)]
    cmd += [os.path.join(CSRC, s) for s in ("ubp_host.cpp", "ubp_layouts.cpp", "ubp_grad_layout.cpp")] + ["-o", str(exe), "-lpthread"]
    r = subprocess.run(cmd, stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
    assert r.returncode == 0, r.stdout
    return str(exe)


@pytest.mark.parametrize("args", LAYERS, ids=lambda a: "x".join(map(str, a)))
def test_layout(driver, args):
    r = subprocess.run([driver] + [str(a) for a in args], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    print(r.stdout)
    assert r.returncode == 0, r.stdout


def test_refusals_without_a_device():
    """A handle without a device: sizes of workspaces, and refused calls."""
    import numpy as np
    from layer_util import layer
    blocks, W, _ = layer(64, 48, 4, 4, 0.3, "f16", 1)
    p = ubp.pack(W, "f16", 4, 4, blocks)
    assert ubp.weight_grad_workspace(p, 0) == 0 and ubp.weight_grad_workspace(p, 255) == 0
    assert ubp.weight_grad_workspace(p, 100000) > 0 and ubp.weight_grad_workspace(p, 100000) % 1024 == 0
    assert ubp.linear_grad_workspace(p, 8192) == 0 and ubp.linear_grad_workspace(p, 8193) == 64 * 2 * 4
    for call in (lambda: ubp.weight_grad_workspace(p, -1), lambda: ubp.linear_grad_workspace(p, -1)):
        with pytest.raises(ubp.UBPError):
            call()
    for call in (lambda: ubp.weight_grad(p, 64, 8, 64, 8, 8, 64), lambda: ubp.weight_grad_checkpoint(p, 64, 8, 64, 8, 64, 1, 8, 64),
                 lambda: ubp.weight_grad_prepare(p), lambda: ubp.linear_grad(p, 64, 8, 64, 8, 8, 64, 8, activation="silu"),
                 lambda: ubp.checkpoint_save(p, 64, 8, 8, 64, 8, 64, 1), lambda: ubp.checkpoint_load(p, 64, 8, 64, 1, 8, 64, 8)):
        with pytest.raises(ubp.UBPError) as e:
            call()
        assert e.value.code == 1
    with pytest.raises(KeyError):
        ubp.linear_grad(p, 64, 8, 64, 8, 8, 64, 8, activation="swish")


def test_more_tokens_than_columns_can_be_counted():
    """The kernels count columns in 32 bits, past the last one: refused before anything else about the call."""
    from layer_util import layer
    blocks, W, _ = layer(64, 48, 4, 4, 0.3, "f16", 1)
    p = ubp.pack(W, "f16", 4, 4, blocks)
    N = 2**31 - 2**16
    assert ubp.weight_grad_workspace(p, N) > 0 and ubp.linear_grad_workspace(p, N) > 0
    for n in (N + 1, 2**31 - 1):
        for call in (lambda: ubp.weight_grad_workspace(p, n), lambda: ubp.linear_grad_workspace(p, n)):
            with pytest.raises(ubp.UBPError):
                call()
        for call in (lambda: ubp.weight_grad(p, 64, n, 64, n, n, 64), lambda: ubp.weight_grad_checkpoint(p, 64, n, 64, n, 64, n, n, 64),
                     lambda: ubp.linear_grad(p, 64, n, 64, n, n, 64, n, activation="silu"),
                     lambda: ubp.checkpoint_save(p, 64, n, n, 64, n, 64, n), lambda: ubp.checkpoint_load(p, 64, n, 64, n, n, 64, n)):
            with pytest.raises(ubp.UBPError) as e:
                call()
            assert e.value.code == 4
