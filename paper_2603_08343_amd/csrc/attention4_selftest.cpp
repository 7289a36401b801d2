// CPU check of the arithmetic that calls over the cache in 4 bits are cut by (attention4_plan.h): the line with its own number of workers, what join looks up,
// which items are taken whole, and the workspace's parts.  Runs under the sanitizers (tests/test_attention4_host.py).
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <map>
#include <random>
#include <set>
#include <vector>

#include "attention4_plan.h"

using namespace wht;

#define CHECK(c) do { if (!(c)) { printf("FAILED %s:%d: %s\n", __FILE__, __LINE__, #c); exit(1); } } while (0)

// Walks the line as the workers do, and compares what each item leaves with what item_slots says; blocks: of each sequence.
template <int WORKERS>
static void walk(const std::vector<int>& blocks, int heads, int rows, int gang_log2) {
    const int gang = 1 << gang_log2;
    heads = (heads + gang - 1) / gang * gang;
    const int B = (int)blocks.size(), groups = heads / gang;
    std::vector<int> cum(B + 1, 0);
    for (int b = 0; b < B; ++b) cum[b + 1] = cum[b] + blocks[b];
    const int total = cum[B] * groups, per = line_share<WORKERS>(total, rows, gang_log2);
    CHECK(per >= 1 && (int64_t)per * (WORKERS / gang) >= total);
    std::map<int, std::vector<int64_t>> of;             // item -> slots, in order
    std::set<int64_t> used;
    int64_t covered = 0;
    for (int w = 0; w < WORKERS / gang; ++w) {
        int u = (int)std::min((int64_t)total, (int64_t)w * per), b = 0;
        const int end = (int)std::min((int64_t)total, (int64_t)u + per);
        while (u < end) {
            if (u >= cum[b + 1] * groups) { ++b; continue; }
            const int n = blocks[b], within = u - cum[b] * groups, group = within / n, u0 = within - group * n;
            const int u1 = std::min(n, u0 + (end - u));
            const int64_t slot = (int64_t)b * groups + group + w;
            CHECK(used.insert(slot).second);
            CHECK(slot >= 0 && (slot + 1) * gang <= (int64_t)B * heads + kMostWorkers4);                // what the plan has room for
            of[b * groups + group].push_back(slot);
            covered += u1 - u0;
            u += u1 - u0;
        }
    }
    CHECK(covered == total);
    for (int b = 0; b < B; ++b)
        for (int h = 0; h < groups; ++h) {
            const Slots s = item_slots<WORKERS>(b * groups + h, cum[b] * groups + h * blocks[b], blocks[b], total, rows, gang_log2);
            const auto& got = of[b * groups + h];
            CHECK(s.count == (int)got.size());
            for (int i = 0; i < s.count; ++i) CHECK(got[i] == s.first + i);
        }
}

// The longest lines that are taken: no sum passes 31 bits, and every block is some worker's.
template <int WORKERS>
static void longest(int gang_log2) {
    const wht_attention_cache4_t c{(void*)16, (void*)16, (uint8_t*)16, (uint8_t*)16, 1024 * 64, 1 << 20, 64, 4096, 4096, 4, 1, gang_log2 ? 4 : 1, 1024, 128};
    const wht_attention_rows_t q{(void*)16, 512, 128};
    for (int64_t B : {1, 7, 1000, 1 << 15, 1 << 20}) {
        int64_t most = 1 << 30;
        auto takes = [&](int64_t length) {
            const wht_attention_batch_t b{(const int32_t*)16, (const int32_t*)16, nullptr, 0, (int32_t)B, 1 << 20};
            return check_paged4(&q, &q, nullptr, 1, c.heads, &c, &b, nullptr, 0, 1, length, 1.0f, WHT_DTYPE_BF16) == WHT_OK;
        };
        while (!takes(most)) most -= most / 64 + 1;
        const int64_t total = B * ceil_div64(most, kBlockKeys) * (c.heads >> gang_log2);
        CHECK(total + WORKERS < INT32_MAX);
        const int per = line_share<WORKERS>((int)total, 1, gang_log2);
        CHECK((int64_t)per * (WORKERS >> gang_log2) >= total && (int64_t)per * (WORKERS >> gang_log2) <= INT32_MAX);
    }
}

static void plans() {
    std::mt19937 rng(11);
    auto upto = [&](int n) { return (int)(rng() % (unsigned)n); };
    int whole = 0;
    for (int i = 0; i < 20000; ++i) {
        const int heads = 1 + upto(32), G = 1 + upto(16), B = upto(i % 4 ? 300 : 20), dim = 64 + 32 * upto(3), max_q = i % 3 ? 1 + upto(3) : 1 + upto(5000);
        const int64_t T = 1 + upto(9000), prefix = i % 3 ? 0 : upto(4000), most = i % 5 ? upto(3000) : upto(100000);
        const AttentionPlan4 p = plan_attention4(T, B, heads * G, heads, dim, max_q, most, prefix);
        const AttentionPlan q = plan_attention(T, B, heads * G, heads, dim, max_q, most, prefix);
        CHECK(p.own_few == q.own_few && p.front == q.front && p.front_few == q.front_few && p.own_cap == q.own_cap && p.own_splits == q.own_splits);
        whole += p.whole;
        if (p.whole) {
            CHECK(p.own_few && !p.front && !p.combine && p.bytes == 0 && B > 0 && p.own_cap <= 2 * kSmallTile);
            CHECK((int64_t)B * heads <= (dim == 64 ? 512 : 256) && most + prefix <= 2560);
            continue;
        }
        if (p.own_few) CHECK(p.own_rows == (((size_t)B + 1) * heads + kMostWorkers4) * (size_t)p.own_cap);
        const size_t at[] = {p.front_at, p.own_at, p.front_sums_at, p.own_sums_at, p.cum_at, p.bytes};
        const size_t need[] = {p.front_rows * dim * 4, p.own_rows * dim * 4, p.front_rows * 8, p.own_rows * 8, p.own_few ? ((size_t)B + 2) * 4 : 0};
        for (int k = 0; k < 5; ++k) CHECK(at[k] % 256 == 0 && at[k] + need[k] <= at[k + 1]);
    }
    CHECK(whole > 500);
    for (bool f32 : {false, true})
        for (int dim : {64, 96, 128})
            for (int tiles : {1, 2})
                for (bool front : {false, true}) CHECK(4 * workgroups4(f32, dim, tiles, front) == (f32 || dim == 128 || tiles == 2 || front ? kWorkers : kMostWorkers4));
    CHECK(tiles4(8, 1) == 2 && tiles4(16, 16) == 1 && tiles4(16, 17) == 2 && tiles4(1024, kFewRows) == 2);
}

// The search for a token's sequence adds to their number in 32 bits.
static void sequences() {
    const wht_attention_rows_t r{(void*)16, 1024, 128}, none{nullptr, 0, 0};
    for (int32_t B : {0, 3, 1 << 30, (1 << 30) + 1, INT32_MAX - 62, INT32_MAX}) {
        const wht_attention_batch_t b{(const int32_t*)16, (const int32_t*)16, (const int32_t*)16, 1, B, 1};
        const wht_attention_cache_t c{(void*)16, (void*)16, 8 * 16 * 128, 16 * 128, 128, 4, 8, 16, 128};
        const wht_attention_cache4_t c4{(void*)16, (void*)16, (uint8_t*)16, (uint8_t*)16, 8 * 16 * 64, 16 * 64, 64, 8 * 16 * 4, 16 * 4, 4, 4, 8, 16, 128};
        const int want = B <= 1 << 30 ? WHT_OK : WHT_ERR_BAD_DIM;
        CHECK(check_append(&none, &r, &r, &none, 3, 0, &c, &b, nullptr, 0, 0, 0, WHT_DTYPE_BF16) == want);
        CHECK(check_append4(&none, &r, &r, &none, &none, &none, 3, 0, &c4, &b, nullptr, 0, 0, 0, nullptr, 1, nullptr, WHT_DTYPE_BF16) == want);
    }
}

// Heads may be any distance apart: their offsets are 64 bits.
static void heads_apart() {
    const wht_attention_rows_t r{(void*)16, 1024, 128};
    const wht_attention_batch_t b{(const int32_t*)16, (const int32_t*)16, nullptr, 1, 3, 1};
    for (int64_t head : {(int64_t)16, (int64_t)4 * 16 * 64, (int64_t)1 << 31, (int64_t)70000 << 16, (int64_t)1 << 60}) {
        const wht_attention_cache4_t c{(void*)16, (void*)16, (uint8_t*)16, (uint8_t*)16, 16 * 64, head, 64, 16 * 4, head / 16, 4, 4, 8, 16, 128};
        CHECK(check_paged4(&r, &r, nullptr, 3, 8, &c, &b, nullptr, 0, 1, 16, 1.0f, WHT_DTYPE_BF16) == WHT_OK);
        CHECK(check_append4(&r, &r, &r, &r, &r, &r, 3, 8, &c, &b, nullptr, 0, 0, 0, nullptr, 1, nullptr, WHT_DTYPE_BF16) == (head == 16 ? WHT_ERR_MISALIGNED : WHT_OK));
    }
}

int main() {
    sequences();
    heads_apart();
    std::mt19937 rng(5);
    for (int i = 0; i < 300; ++i) {
        std::vector<int> blocks(rng() % 200);
        const int most = 1 << (rng() % 12), front = i % 3 ? 0 : (int)(rng() % 150);
        for (int& n : blocks) n = front + (int)(rng() % (unsigned)most) * (rng() % 5 != 0);
        const int heads = 1 + (int)(rng() % 40), rows = 1 + (int)(rng() % 32), gang = i % 2 ? 0 : kGangLog2;
        walk<kMostWorkers4>(blocks, heads, rows, gang);
        walk<kWorkers>(blocks, heads, rows, gang);
    }
    walk<kMostWorkers4>({}, 8, 4, 0);
    walk<kMostWorkers4>({0, 0}, 8, 4, kGangLog2);
    walk<kMostWorkers4>({kMostWorkers4}, 1, 1, 0);
    walk<kMostWorkers4>({kMostWorkers4 + 1}, 1, 1, 0);
    for (int gang : {0, kGangLog2}) { longest<kWorkers>(gang); longest<kMostWorkers4>(gang); }
    plans();
    printf("attention4_selftest: ok\n");
    return 0;
}
