/* Replays the cut of shared-prefix decode calls on the host, for many sizes: every prefix and own block belongs to exactly one worker;
 * the partial results of the workers lie in slots of their own, inside the ranges that the plan reserves; the slots that the merge
 * reads for a row are those that were written for it; and the plan fits the workspace that the library asks for. */
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>

#include "decode_shared.cuh"

using namespace loma;

#define CHECK(c)                                                                                                          \
    do {                                                                                                                  \
        if (!(c)) {                                                                                                       \
            std::printf("line %d: %s (B %d Hq %d Hkv %d D %d P %d max %d pages %d cuda cores %d)\n", __LINE__, #c, B, Hq,  \
                        Hkv, D, P, mx, pages, (int)cores);                                                                \
            std::exit(1);                                                                                                 \
        }                                                                                                                 \
    } while (0)

static void replay(int B, int Hq, int Hkv, int D, int P, int mx, int pages, bool cores, std::mt19937& rng) {
    const SharedPlan p = make_shared_plan(B, Hq, Hkv, D, P, mx, pages, cores);
    CHECK((size_t)p.total * 4 <= loma_decode_shared_workspace_bytes(B, Hq, Hkv, D, P, mx));
    const int64_t g = Hq / Hkv;
    CHECK((int64_t)p.m_tiles * SHP_ROWS >= B * g && (int64_t)p.g_tiles * p.g_rows >= g);
    // prefix
    const int64_t p_room = p.p_lse - p.p_o;
    CHECK(p.own_o - p.p_lse >= p_room / D);
    if (p.p_blocks) {
        const int64_t all = (int64_t)Hkv * p.p_blocks;
        CHECK(p.p_workers >= 1 && p.p_workers <= all && first_block(0, all, p.p_workers) == 0 && first_block(p.p_workers, all, p.p_workers) == all);
        std::vector<int> head_of(p.p_workers + Hkv, -1);   // by slot, before the tiles
        for (int64_t w = 0; w < p.p_workers; ++w) {
            const int64_t t0 = first_block(w, all, p.p_workers), t1 = first_block(w + 1, all, p.p_workers);
            CHECK(t0 < t1 && block_worker(t0, all, p.p_workers) == w && block_worker(t1 - 1, all, p.p_workers) == w);
            for (int64_t h = t0 / p.p_blocks; h * p.p_blocks < t1; ++h) {
                const int64_t last = (w + h) * p.m_tiles + p.m_tiles - 1;
                CHECK(head_of[w + h] == -1 && (last + 1) * SHP_ROWS * D <= p_room && (last + 1) * SHP_ROWS <= p.own_o - p.p_lse);
                head_of[w + h] = (int)h;
            }
        }
        for (int64_t h = 0; h < Hkv; ++h) {
            const int64_t w0 = block_worker(h * p.p_blocks, all, p.p_workers), w1 = block_worker((h + 1) * p.p_blocks - 1, all, p.p_workers);
            for (int64_t s = 0; s < p.p_workers + Hkv; ++s) CHECK((head_of[s] == h) == (s >= w0 + h && s <= w1 + h));
        }
    }
    // own entries of ragged sequences
    std::vector<int64_t> cum(B + 1, 0);
    for (int b = 0; b < B; ++b) {
        const int kind = (int)(rng() % 4), len = kind == 0 ? -1 : kind == 1 ? mx : (int)(rng() % ((unsigned)mx + 1));
        cum[b + 1] = cum[b] + own_blocks(b == 0 && rng() % 2 ? mx : len);
    }
    const int64_t units = (int64_t)Hkv * p.g_tiles, T = cum[B] * units, W = own_workers(T, p.workers);
    const int64_t own_room = p.own_lse - p.own_o;
    if (p.whole) {
        CHECK(units * B * p.g_rows * D <= own_room && units * B * p.g_rows <= p.cum - p.own_lse);
        return;
    }
    CHECK(p.total - p.cum >= 2 * ((int64_t)B + 1));
    if (T == 0) return;
    CHECK(W >= 1 && first_block(0, T, W) == 0 && first_block(W, T, W) == T);
    std::vector<int64_t> unit_of(W + units * B, -1);
    for (int64_t w = 0; w < W; ++w) {
        const int64_t t0 = first_block(w, T, W), t1 = first_block(w + 1, T, W);
        CHECK(t0 < t1 && block_worker(t0, T, W) == w && block_worker(t1 - 1, T, W) == w);
        int64_t hh = t0 / cum[B], rem = t0 - hh * cum[B];
        int b = 0;
        while (cum[b + 1] <= rem) ++b;
        for (int64_t t = t0; t < t1;) {                      // the worker's stay in (hh, b)
            const int64_t slot = w + hh * B + b;
            CHECK(unit_of[slot] == -1 && (slot + 1) * p.g_rows * D <= own_room && (slot + 1) * p.g_rows <= p.cum - p.own_lse);
            unit_of[slot] = hh * B + b;
            t = std::min(t1, hh * cum[B] + cum[b + 1]);
            do {
                if (++b == B) { b = 0; ++hh; }
            } while (t < t1 && cum[b + 1] == cum[b]);
        }
    }
    for (int64_t hh = 0; hh < units; ++hh)
        for (int b = 0; b < B; ++b) {
            if (cum[b + 1] == cum[b]) continue;
            const int64_t w0 = block_worker(hh * cum[B] + cum[b], T, W), w1 = block_worker(hh * cum[B] + cum[b + 1] - 1, T, W), u = hh * B + b;
            for (int64_t s = w0; s <= w1; ++s) CHECK(unit_of[s + u] == u);
            if (w0 + u > 0) CHECK(unit_of[w0 + u - 1] != u);
            if (w1 + u + 1 < W + units * B) CHECK(unit_of[w1 + u + 1] != u);
        }
}

int main() {
    std::mt19937 rng(7);
    const int heads[][2] = {{1, 1}, {2, 1}, {3, 1}, {8, 8}, {32, 8}, {32, 32}, {64, 8}, {40, 2}, {100, 100}, {9, 1}, {64, 4}};
    const int batches[] = {1, 2, 3, 7, 16, 33, 64, 130, 300}, prefixes[] = {0, 1, 33, 64, 700, 2304, 2400, 9000, 65537}, bounds[] = {0, 5, 111, 127, 128, 400, 5000};
    long n = 0;
    for (const auto& h : heads)
        for (int B : batches)
            for (int P : prefixes)
                for (int mx : bounds) {
                    const int D = rng() % 2 ? 64 : 128, pages[] = {0, 4, 16, 64, 256};
                    for (bool cores : {false, true}) replay(B, h[0], h[1], D, P, mx, pages[rng() % 5], cores, rng), ++n;
                }
    for (int i = 0; i < 3000; ++i) {
        const auto& h = heads[rng() % 11];
        const int P = (int)(rng() % (1u << (1 + rng() % 17))), mx = (int)(rng() % (1u << (1 + rng() % 13)));
        replay(1 + (int)(rng() % (1u << (1 + rng() % 8))), h[0], h[1], rng() % 2 ? 64 : 128, P, mx, rng() % 2 ? 16 : 0, rng() % 2, rng), ++n;
    }
    std::printf("%ld shared plans ok\n", n);
    return 0;
}
