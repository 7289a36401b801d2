// CPU check of the arithmetic that attention calls are cut by (attention_plan.h): the few-rows kernel's line of units, its slots and
// what join looks up, over batches of all kinds; the workspace's parts; and every status of the argument checks.  Runs under the
// sanitizers (tests/test_attention_host.py).
#include <stdio.h>
#include <stdlib.h>

#include <map>
#include <random>
#include <set>
#include <vector>

#include "attention_plan.h"

using namespace wht;

#define CHECK(c) do { if (!(c)) { printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #c); exit(1); } } while (0)

// Walks the line as the workers do, and compares what each item leaves with what item_slots says.
static void walk(const std::vector<int>& lengths, int heads, int front, int rows, int gang_log2) {
    const int gang = 1 << gang_log2;
    heads = (heads + gang - 1) / gang * gang;
    const int B = (int)lengths.size(), W = kWorkers / gang, groups = heads / gang;
    std::vector<int> units(B), cum(B + 1, 0);
    for (int b = 0; b < B; ++b) {
        units[b] = ceil_div(front, kBlockKeys) + ceil_div(lengths[b], kBlockKeys);
        cum[b + 1] = cum[b] + units[b];
    }
    const int total = cum[B] * groups, per = line_share(total, rows, gang_log2);
    std::map<int, std::vector<int64_t>> of;             // item -> slots, in order
    std::set<int64_t> used;
    int covered = 0;
    for (int w = 0; w < W; ++w) {
        int u = w * per, end = total < u + per ? total : u + per, b = 0;
        while (u < end) {
            if (u >= cum[b + 1] * groups) { ++b; continue; }
            const int n = units[b], within = u - cum[b] * groups, group = within / n, u0 = within - group * n;
            const int u1 = n < u0 + (end - u) ? n : u0 + (end - u);
            const int64_t slot = (int64_t)b * groups + group + w;
            CHECK(used.insert(slot).second);
            CHECK(slot >= 0 && (slot + 1) * gang <= (int64_t)B * heads + kWorkers);
            of[b * groups + group].push_back(slot);
            covered += u1 - u0;
            u += u1 - u0;
        }
    }
    CHECK(covered == total);
    for (int b = 0; b < B; ++b)
        for (int h = 0; h < groups; ++h) {
            const Slots s = item_slots(b * groups + h, cum[b] * groups + h * units[b], units[b], total, rows, gang_log2);
            const auto& got = of[b * groups + h];
            CHECK(s.count == (int)got.size());
            for (int i = 0; i < s.count; ++i) CHECK(got[i] == s.first + i);
        }
}

// Every tile of every group is some die's, once, and within the workgroups that a die has.
static void deal(const std::vector<int>& queries, int heads, int splits, int G) {
    const int B = (int)queries.size(), per = heads * splits;
    int64_t T = 0, max_q = 1;
    for (int q : queries) { T += q; max_q = q > max_q ? q : max_q; }
    const int64_t most = die_blocks(T, B, G, max_q, per);
    std::set<std::pair<int, int>> seen;
    for (int x = 0; x < kDies; ++x) {
        int64_t blocks = 0;
        for (int b = 0; b < B; ++b) {
            const int n = die_groups(b, per, x);
            CHECK(n >= 0);
            for (int k = 0; k < n; ++k) {
                const int g = die_group(b, per, x, k);
                CHECK(g >= 0 && g < per && (b * per + g) % kDies == x && seen.insert({b, g}).second);
                blocks += ceil_div64((int64_t)queries[b] * G, kTileRows);
            }
        }
        CHECK(blocks <= most);
    }
    CHECK((int64_t)seen.size() == (int64_t)B * per);
    int64_t tiles = 0;
    for (int q : queries) tiles += ceil_div64((int64_t)q * G, kTileRows);
    CHECK(tiles <= most_tiles(T, B, G, max_q));
}

// Starts that do not ascend give many sequences all of T: the many-rows kernel's look-up still ends at one of the batch that has tiles.
static void deal_to_overlapping(int B, int64_t T, int heads, int G) {
    const int splits = splits_for(most_tiles(T, B, G, T) * heads, 1 << 20), per = heads * splits, run = ceil_div(B, 64);
    auto tiles_at = [&](int i, int x) { return die_groups(i, per, x) * (i % 2 ? 0 : (int)ceil_div64(T * G, kTileRows)); };
    const int64_t most = die_blocks(T, B, G, T, per);
    CHECK(most <= kMostWorkgroups / kDies);
    for (int x = 0; x < 8; x += 7) {
        int upto[64], last = 0;
        for (int lane = 0; lane < 64; ++lane) {
            int mine = 0;
            for (int i = lane * run; i < B && i < (lane + 1) * run; ++i) mine = add_tiles(mine, tiles_at(i, x));
            last = upto[lane] = last + mine;
        }
        for (int64_t y = 0; y <= most; y = y * 5 / 4 + 1) {
            if (y >= upto[63]) continue;
            int from = 0;
            while (upto[from] <= y) ++from;
            int b = from * run;
            int64_t cum = from ? upto[from - 1] : 0;
            for (; b < B && y >= cum + tiles_at(b, x); ++b) cum += tiles_at(b, x);
            CHECK(b < B && tiles_at(b, x) > 0);
        }
    }
}

static void plans() {
    std::mt19937 rng(7);
    auto upto = [&](int n) { return (int)(rng() % (unsigned)n); };
    for (int i = 0; i < 20000; ++i) {
        const int heads = 1 + upto(32), G = 1 + upto(16), B = upto(300), dim = 64 + 32 * upto(3), max_q = i % 2 ? 1 : 1 + upto(5000);
        const int64_t T = 1 + upto(9000), prefix = i % 3 ? upto(40000) : 0, most = upto(100000);
        const AttentionPlan p = plan_attention(T, B, heads * G, heads, dim, max_q, most, prefix);
        CHECK(p.own_few == (max_q * G <= kFewRows));
        CHECK(p.front_splits >= 1 && p.own_splits >= 1 && p.front_splits <= kWorkgroups && p.own_splits <= kWorkgroups);
        if (p.own_few) CHECK(p.own_rows == (((size_t)B + 1) * heads + kWorkers) * (size_t)p.own_cap && p.own_cap >= max_q * G);
        if (p.front && p.front_few) CHECK(p.own_cap == T * G && p.own_cap <= kFewRows);
        if (p.front && !p.front_few) CHECK(p.front_rows == (size_t)p.front_splits * (size_t)T * (size_t)(heads * G));
        if (!p.combine) CHECK(!p.front && !p.own_few && p.own_rows == 0);
        const size_t at[] = {p.front_at, p.own_at, p.front_sums_at, p.own_sums_at, p.cum_at, p.bytes};
        const size_t need[] = {p.front_rows * dim * 4, p.own_rows * dim * 4, p.front_rows * 8, p.own_rows * 8, p.own_few ? ((size_t)B + 2) * 4 : 0};
        for (int k = 0; k < 5; ++k) CHECK(at[k] % 256 == 0 && at[k] + need[k] <= at[k + 1]);
    }
}

static void statuses() {
    void* P = reinterpret_cast<void*>((uintptr_t)0x1000);
    const int32_t* I = static_cast<const int32_t*>(P);
    const wht_attention_cache_t c0{P, P, 8 * 64 * 128, 64 * 128, 128, 10, 8, 64, 128};
    const wht_attention_batch_t b0{I, I, nullptr, 4, 3, 4};
    const wht_attention_rows_t r0{P, 48 * 128, 128}, none{nullptr, 0, 0};
    const float* F = static_cast<const float*>(P);
    auto append = [&](wht_attention_cache_t c, wht_attention_batch_t b, wht_attention_rows_t q, wht_attention_rows_t k, const float* rope, int64_t rope_rows,
                      int32_t rotary, int64_t position, int32_t dtype, int64_t T = 3, int32_t q_heads = 32) {
        return check_append(&q, &k, &k, &q, T, q_heads, &c, &b, rope, rope_rows, rotary, position, dtype);
    };
    auto cache = [&](auto f) { wht_attention_cache_t c = c0; f(c); return append(c, b0, r0, r0, F, 100, 128, 0, 1); };
    auto batch = [&](auto f) { wht_attention_batch_t b = b0; f(b); return append(c0, b, r0, r0, F, 100, 128, 0, 1); };
    auto rows = [&](auto f) { wht_attention_rows_t r = r0; f(r); return append(c0, b0, r0, r, F, 100, 128, 0, 1); };
    CHECK(append(c0, b0, r0, r0, F, 100, 128, 0, 1) == WHT_OK);
    CHECK(append(c0, b0, none, r0, F, 100, 64, 0, 1) == WHT_OK);                 // no queries
    CHECK(append(c0, b0, r0, r0, nullptr, 0, 0, 0, 1) == WHT_OK);                // no rotation
    CHECK(append(c0, b0, r0, none, F, 100, 128, 0, 1) == WHT_ERR_NULL_PTR);
    CHECK(append(c0, b0, r0, r0, nullptr, 100, 128, 0, 1) == WHT_ERR_NULL_PTR);
    CHECK(append(c0, b0, r0, r0, F, 100, 128, 0, 2) == WHT_ERR_BAD_DTYPE);
    CHECK(append(c0, b0, r0, r0, F, 100, 136, 0, 1) == WHT_ERR_BAD_DIM);
    CHECK(append(c0, b0, r0, r0, F, 100, 24, 0, 1) == WHT_ERR_BAD_DIM);
    CHECK(append(c0, b0, r0, r0, F, 100, -16, 0, 1) == WHT_ERR_BAD_DIM);
    CHECK(append(c0, b0, r0, r0, F, -1, 128, 0, 1) == WHT_ERR_BAD_DIM);
    CHECK(append(c0, b0, r0, r0, F, 100, 128, -1, 1) == WHT_ERR_BAD_DIM);
    CHECK(append(c0, b0, r0, r0, F, 100, 128, 0, 1, -1) == WHT_ERR_BAD_DIM);
    CHECK(append(c0, b0, r0, r0, F, 100, 128, 0, 1, 3, 0) == WHT_ERR_BAD_DIM);
    CHECK(cache([](auto& c) { c.k = nullptr; }) == WHT_ERR_NULL_PTR);
    CHECK(cache([](auto& c) { c.head_dim = 80; }) == WHT_ERR_BAD_DIM);
    CHECK(cache([](auto& c) { c.page_size = 48; }) == WHT_ERR_BAD_DIM);
    CHECK(cache([](auto& c) { c.page_size = 4; }) == WHT_ERR_BAD_DIM);
    CHECK(cache([](auto& c) { c.page_size = 2048; }) == WHT_ERR_BAD_DIM);
    CHECK(cache([](auto& c) { c.heads = 0; }) == WHT_ERR_BAD_DIM);
    CHECK(cache([](auto& c) { c.pages = 0; }) == WHT_ERR_BAD_DIM);
    CHECK(cache([](auto& c) { c.token_stride = 64; }) == WHT_ERR_BAD_DIM);       // tokens over one another
    CHECK(cache([](auto& c) { c.page_stride = (int64_t)1 << 31; }) == WHT_ERR_BAD_DIM);
    CHECK(cache([](auto& c) { c.token_stride = (int64_t)1 << 25; }) == WHT_ERR_BAD_DIM);
    CHECK(cache([](auto& c) { c.token_stride = 132; }) == WHT_ERR_MISALIGNED);
    CHECK(cache([](auto& c) { c.v = reinterpret_cast<void*>((uintptr_t)0x1008); }) == WHT_ERR_MISALIGNED);
    CHECK(batch([](auto& b) { b.table = nullptr; }) == WHT_ERR_NULL_PTR);
    CHECK(batch([](auto& b) { b.lengths = nullptr; }) == WHT_ERR_NULL_PTR);
    CHECK(batch([](auto& b) { b.width = 0; }) == WHT_ERR_BAD_DIM);
    CHECK(batch([](auto& b) { b.B = -1; }) == WHT_ERR_BAD_DIM);
    CHECK(batch([](auto& b) { b.width = 1 << 25; }) == WHT_ERR_BAD_DIM);
    CHECK(batch([](auto& b) { b.q_starts = reinterpret_cast<const int32_t*>((uintptr_t)0x1002); }) == WHT_ERR_MISALIGNED);
    CHECK(rows([](auto& r) { r.token_stride = 48 * 128 + 4; }) == WHT_ERR_MISALIGNED);
    CHECK(rows([](auto& r) { r.head_stride = 64; }) == WHT_ERR_MISALIGNED);
    CHECK(rows([](auto& r) { r.data = reinterpret_cast<void*>((uintptr_t)0x1004); }) == WHT_ERR_MISALIGNED);

    auto paged = [&](wht_attention_rows_t q, int32_t q_heads, const int32_t* prefix_table, int64_t prefix, int32_t max_q, int64_t most, float scale, int32_t dtype) {
        return check_paged(&q, &q, nullptr, 3, q_heads, &c0, &b0, prefix_table, prefix, max_q, most, scale, dtype);
    };
    CHECK(paged(r0, 32, nullptr, 0, 1, 256, 1.0f, 1) == WHT_OK);
    CHECK(paged(r0, 32, I, 100, 7, 0, 1e-3f, 1) == WHT_OK);
    CHECK(paged(none, 32, I, 100, 1, 256, 1.0f, 1) == WHT_ERR_NULL_PTR);
    CHECK(paged(r0, 32, nullptr, 100, 1, 256, 1.0f, 1) == WHT_ERR_NULL_PTR);
    CHECK(paged(r0, 32, I, 100, 1, 256, 1.0f, 3) == WHT_ERR_BAD_DTYPE);
    CHECK(paged(r0, 20, I, 100, 1, 256, 1.0f, 1) == WHT_ERR_BAD_DIM);            // heads do not divide
    CHECK(paged(r0, 32, I, -1, 1, 256, 1.0f, 1) == WHT_ERR_BAD_DIM);
    CHECK(paged(r0, 32, I, 100, 0, 256, 1.0f, 1) == WHT_ERR_BAD_DIM);
    CHECK(paged(r0, 32, I, 100, 1, -1, 1.0f, 1) == WHT_ERR_BAD_DIM);
    {
        wht_attention_cache_t c = c0;
        wht_attention_batch_t b = b0;
        b.B = 1 << 16; b.width = 1 << 14;                                        // 64 Ki sequences of 1 Mi tokens: more blocks than the line counts
        CHECK(check_paged(&r0, &r0, nullptr, 3, 32, &c, &b, nullptr, 0, 1, (int64_t)1 << 20, 1.0f, 1) == WHT_ERR_BAD_DIM);
        CHECK(check_paged(&r0, &r0, nullptr, 3, 32, &c, &b, nullptr, 0, 1, 1 << 12, 1.0f, 1) == WHT_OK);
    }
    // outputs over themselves: rows or heads at one place, one inside the other's
    auto written = [&](int64_t T, int64_t token_stride, int64_t head_stride) {
        const wht_attention_rows_t o{P, token_stride, head_stride};
        return check_paged(&r0, &o, nullptr, T, 32, &c0, &b0, nullptr, 0, 1, 256, 1.0f, 1);
    };
    CHECK(written(3, 48 * 128, 128) == WHT_OK && written(3, 128, 3 * 128) == WHT_OK && written(3, 32 * 128, 128) == WHT_OK && written(1, 0, 128) == WHT_OK);
    CHECK(written(3, 0, 128) == WHT_ERR_MISALIGNED && written(3, 128, 128) == WHT_ERR_MISALIGNED && written(3, 31 * 128, 128) == WHT_ERR_MISALIGNED);
    CHECK(written(3, 128, 2 * 128) == WHT_ERR_MISALIGNED && written(3, 64, 3 * 128) == WHT_ERR_MISALIGNED);
    {
        const wht_attention_rows_t o{P, 0, 128};
        CHECK(check_append(&r0, &r0, &r0, &o, 3, 32, &c0, &b0, F, 100, 128, 0, 1) == WHT_ERR_MISALIGNED);
        CHECK(check_append(&none, &r0, &r0, &o, 3, 32, &c0, &b0, F, 100, 128, 0, 1) == WHT_OK);
    }
    CHECK(cache([](auto& c) { c.page_stride = 0; }) == WHT_ERR_MISALIGNED);
    CHECK(cache([](auto& c) { c.page_stride = 0; c.pages = 1; }) == WHT_OK);
    CHECK(cache([](auto& c) { c.head_stride = 0; }) == WHT_ERR_MISALIGNED);
    CHECK(cache([](auto& c) { c.page_stride -= 128; }) == WHT_ERR_MISALIGNED);
    CHECK(cache([](auto& c) { c.token_stride = 8 * 128; c.head_stride = 128; }) == WHT_OK);                                     // [pages][slots][heads]
    CHECK(cache([](auto& c) { c.page_stride = 64 * 128; c.head_stride = 10 * 64 * 128; }) == WHT_OK);                            // [heads][pages][slots]
    CHECK(cache([](auto& c) { c.page_stride = 64 * 128; c.head_stride = (int64_t)1 << 61; }) == WHT_OK);
    // a scale whose product with log2(e) is infinite would make NaN of every score of zero
    for (float s : {1e-45f, 1e-38f, 1.0f, 1e38f, 2.3e38f}) CHECK(paged(r0, 32, I, 100, 1, 256, s, 1) == WHT_OK && base2_scale(s) > 0.0f && base2_scale(s) < __builtin_inff());
    for (float s : {2.4e38f, 3.0e38f, 3.4e38f}) CHECK(paged(r0, 32, I, 100, 1, 256, s, 1) == WHT_ERR_BAD_DIM);
    for (float s : {0.0f, -1.0f, __builtin_nanf(""), __builtin_inff()}) CHECK(paged(r0, 32, I, 100, 1, 256, s, 1) == WHT_ERR_BAD_DIM);
}

int main() {
    std::mt19937 rng(3);
    for (int i = 0; i < 300; ++i) {
        std::vector<int> lengths(rng() % 200);
        const int most = 1 << (rng() % 16);
        for (int& n : lengths) n = (int)(rng() % (unsigned)most) * (rng() % 5 != 0);
        walk(lengths, 1 + (int)(rng() % 40), i % 3 ? 0 : (int)(rng() % 5000), 1 + (int)(rng() % 32), i % 2 ? 0 : kGangLog2);
    }
    for (int i = 0; i < 300; ++i) {
        std::vector<int> queries(rng() % 60);
        const int most = 1 + (1 << (rng() % 12));
        for (int& n : queries) n = (int)(rng() % (unsigned)most) * (rng() % 5 != 0);
        deal(queries, 1 + (int)(rng() % 40), 1 + (int)(rng() % 9), 1 + (int)(rng() % 17));
    }
    deal_to_overlapping(1 << 20, 1 << 19, 8, 128);
    deal_to_overlapping(8192, 1 << 20, 8, 128);
    deal_to_overlapping(70, 5000, 8, 4);
    walk({}, 8, 0, 4, 0);
    walk({0, 0}, 8, 0, 4, kGangLog2);
    walk({1}, 1, 0, 1, 0);
    CHECK(gang_log2_of(16, 192, 192) == kGangLog2 && gang_log2_of(16, 192, 64 * 192) == 0 && gang_log2_of(6, 192, 192) == 0 && gang_log2_of(16, 256, 256) == 0);
    // 400 sequences of 10 tokens behind 100, 8 heads of 128: 16.8 MB, though every sequence reads the prefix's 0.4 MB; of 100 tokens 164 MB
    CHECK(!streams(400, 8, 128, 2, 10, 100, 0) && streams(400, 8, 128, 2, 100, 100, 0) && !streams(400, 8, 128, 2, 100, 100, kGangLog2));
    CHECK(streams(1, 8, 128, 2, 0, 1 << 20, 0));
    plans();
    statuses();
    printf("attention_selftest: ok\n");
    return 0;
}
