// The plan of a batch over a paged cache, looked over on the host: every key tile of every row tile and head is dealt exactly once, every
// token's keys are those it should see, partial results lie side by side without overlap, and every offset stays inside its array.
//   cache_plan_check <seed> <rounds>      prints "ok" or the first fault
#include <cstdio>
#include <cstdlib>
#include <map>
#include <random>
#include <set>
#include <tuple>

#include "../paper_2511_21317_b200/csrc/httm_batch_plan.h"

using namespace httm;

static std::mt19937 rng;
static int pick(int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(rng); }
#define NEED(c)                                                     \
    do {                                                            \
        if (!(c)) {                                                 \
            printf("line %d: %s does not hold\n", __LINE__, #c);    \
            return false;                                           \
        }                                                           \
    } while (0)

static bool one_round() {
    httm_batch_config c{};
    const int groups[] = {1, 1, 2, 3, 4, 5, 8, 16, 17, 40, 65, 128};
    c.kv_heads = pick(1, 8);
    const int group = groups[pick(0, 11)];
    c.heads = c.kv_heads * group;
    c.head_dim = pick(0, 1) ? 64 : 128;
    c.page_size = 16 << pick(0, 4);
    c.causal = pick(0, 1);
    const int n_seq = pick(0, 3) ? pick(0, 12) : pick(0, 200), sms = pick(0, 3) ? 148 : pick(1, 20);
    const int prefix = pick(0, 3) ? pick(0, 6000) : 0;
    std::vector<int32_t> lengths(n_seq), queries(n_seq);
    const int kind = pick(0, 3);
    for (int i = 0; i < n_seq; ++i) {
        queries[i] = kind == 0 ? 1 : kind == 1 ? pick(0, 9) : kind == 2 ? pick(0, 600) : (pick(0, 2) ? pick(0, 3) : pick(0, 700));
        lengths[i] = pick(0, 5) ? queries[i] + pick(0, 900) : pick(0, 300);
    }
    int stride = 0;
    for (int n : lengths) stride = std::max(stride, pages_of(n, c.page_size));
    stride += pick(0, 2);
    std::vector<int32_t> tables((size_t)n_seq * stride, -7), pre(pages_of(prefix, c.page_size));
    int next = 0;
    for (auto& p : pre) p = next++;
    for (int i = 0; i < n_seq; ++i)
        for (int j = 0; j < pages_of(lengths[i], c.page_size); ++j) tables[(size_t)i * stride + j] = next++;
    c.n_pages = next + 1;
    const BatchInput in{n_seq, lengths.data(), queries.data(), tables.data(), stride, pre.data(), prefix};
    std::string why;
    NEED(check_batch(c, in, &why) == HTTM_OK);
    BatchPlan p;
    make_batch_plan(c, in, sms, &p);
    int tokens = 0;
    for (int q : queries) tokens += q;
    NEED(p.n_tokens == tokens && (int)p.prefix_seg.size() == tokens && (int)p.own_seg.size() == tokens);
    NEED((int)p.slots.size() == tokens && (int)p.positions.size() == tokens && p.parts.size() == p.segs.size() * c.kv_heads);
    // row tiles: what every token sees
    int t = 0;
    bool append = true;
    for (int i = 0; i < n_seq; ++i) {
        append &= queries[i] <= lengths[i];
        for (int j = 0; j < queries[i]; ++j, ++t) {
            const int sees = c.causal ? std::max(0, std::min(lengths[i], lengths[i] - queries[i] + j + 1)) : lengths[i];
            int own = 0, shared = 0;
            for (int which : {p.prefix_seg[t], p.own_seg[t]}) {
                if (which < 0) continue;
                NEED(which < (int)p.segs.size());
                const RowTile& s = p.segs[which];
                NEED(t >= s.token0 && t < s.token0 + s.tokens && s.tokens * group <= s.tile_rows);
                NEED(s.tile_rows == 16 || s.tile_rows == 32 || s.tile_rows == 64 || s.tile_rows == kWideRows);
                NEED(s.prefix_keys == 0 || s.prefix_keys == prefix);
                shared += s.prefix_keys;
                if (s.own_keys > 0) {
                    own += std::max(0, std::min(s.own_keys, s.seen0 + (c.causal ? t - s.token0 : 0)));
                    for (int k = 0; k < pages_of(s.own_keys, c.page_size); ++k) {
                        NEED(s.own_table + k < (int)p.table.size());
                        NEED(p.table[s.own_table + k] == tables[(size_t)i * stride + k]);
                    }
                }
            }
            NEED(own == sees && shared == prefix);
            if (queries[i] <= lengths[i]) {
                const int place = lengths[i] - queries[i] + j;
                NEED(p.slots[t] == tables[(size_t)i * stride + place / c.page_size] * c.page_size + place % c.page_size);
                NEED(p.positions[t] == prefix + place);
            }
        }
    }
    NEED(append == p.can_append && !p.same_place);
    for (size_t i = 0; i < pre.size(); ++i) NEED(p.table[i] == pre[i]);
    // jobs
    std::map<std::tuple<int, int>, std::map<int, std::pair<int, int>>> dealt;   // (row tile, head) -> first key tile -> (last, part)
    for (int wide = 0; wide < 2; ++wide) {
        const auto& jobs = wide ? p.wide_jobs : p.narrow_jobs;
        const auto& start = wide ? p.wide_start : p.narrow_start;
        if (jobs.empty()) continue;
        NEED((int)start.size() - 1 <= (wide ? 1 : narrow_ctas_per_sm(c.head_dim)) * sms && start[0] == 0 && start.back() == (int)jobs.size());
        for (size_t i = 1; i < start.size(); ++i) NEED(start[i] > start[i - 1]);
        for (const CacheJob& j : jobs) {
            NEED(j.head >= 0 && j.head < c.kv_heads && j.pair >= 0 && j.pair <= wide);
            NEED(j.tile0 >= 0 && j.tile1 > j.tile0 && (j.tile_rows == kWideRows) == (wide == 1));
            int token = j.token0;
            for (int k = 0; k <= j.pair; ++k) {   // the record holds what its row tiles are
                NEED(token >= 0 && token < tokens);
                const int at[2] = {p.prefix_seg[token], p.own_seg[token]};
                const int s = j.own_keys[k] > 0 ? at[1] : at[0] >= 0 ? at[0] : at[1];
                NEED(s >= 0);
                const RowTile& seg = p.segs[s];
                NEED(seg.token0 == token && seg.tokens == j.tokens[k] && seg.tile_rows == j.tile_rows && seg.prefix_keys == j.prefix_keys);
                NEED(seg.own_keys == j.own_keys[k] && (seg.own_keys == 0 || (seg.own_table == j.own_table && seg.seen0 == j.seen0[k])));
                auto& of = dealt[std::make_tuple(s, j.head)];
                NEED(of.count(j.tile0) == 0);
                of[j.tile0] = {j.tile1, j.part[k]};
                token += j.tokens[k];
            }
        }
    }
    std::set<std::pair<int, int>> ranges;   // of partial results
    for (int s = 0; s < (int)p.segs.size(); ++s)
        for (int h = 0; h < c.kv_heads; ++h) {
            const RowTile& seg = p.segs[s];
            const int keys = seg.tile_rows == kWideRows ? kWideKeys : kNarrowKeys, units = seg.tile_rows / kPartUnit;
            const int2 parts = p.parts[(size_t)s * c.kv_heads + h];
            int at = 0, n = 0, end = 0;
            for (const auto& d : dealt[std::make_tuple(s, h)]) {
                NEED(d.first == at);
                at = d.second.first;
                if (parts.y < 0) {
                    NEED(d.second.second == -1);
                } else {
                    NEED(d.second.second == parts.x + n * units);
                    end = d.second.second + units;
                    NEED(end <= p.part_units);
                    ++n;
                }
            }
            // a pair walks the key tiles of its second row tile, which sees at least as many
            const int least = (seg.prefix_keys + keys - 1) / keys + (seg.own_keys + keys - 1) / keys;
            NEED(at >= least && (seg.tile_rows == kWideRows || at == least));
            NEED(parts.y == -1 || (parts.y == n && n > 0));
            if (parts.y > 0) ranges.insert({parts.x, end});
            if (parts.y < 0)
                for (int k = seg.token0; k < seg.token0 + seg.tokens; ++k) NEED((p.prefix_seg[k] < 0) != (p.own_seg[k] < 0));
        }
    int last = 0;
    for (const auto& r : ranges) {
        NEED(r.first >= last);
        last = r.second;
    }
    // rows that are written by a job, and rows whose partial results are added up: every row exactly once
    std::vector<int> written((size_t)tokens * c.heads, 0);   // (token, query head)
    for (const CombineTask& k : p.combine_tasks) {
        NEED(k.rows > 0 && k.rows <= k.room && (k.room == kCombineRows || k.room == kCombineFewRows));
        NEED(k.first_head >= 0 && k.first_head < group && k.head >= 0 && k.head < c.kv_heads && k.token0 >= 0);
        for (int r = 0; r < k.rows; ++r) {
            const int i = k.token0 + (k.first_head + r) / group, g = (k.first_head + r) % group;
            NEED(i < tokens);
            for (int w = 0; w < 2; ++w) {
                const int s = w ? p.own_seg[i] : p.prefix_seg[i];
                NEED((s < 0) == (k.parts[w] == 0));
                if (s < 0) continue;
                const int2 parts = p.parts[(size_t)s * c.kv_heads + k.head];
                NEED(k.unit[w] == parts.x && k.parts[w] == parts.y && parts.y > 0 && k.tile_rows[w] == p.segs[s].tile_rows);
                NEED(k.row[w] + r == (i - p.segs[s].token0) * group + g && k.row[w] + r < k.tile_rows[w]);
            }
            ++written[(size_t)i * c.heads + k.head * group + g];
        }
    }
    for (int s = 0; s < (int)p.segs.size(); ++s)
        for (int h = 0; h < c.heads; ++h)
            if (p.parts[(size_t)s * c.kv_heads + h / group].y < 0)
                for (int i = p.segs[s].token0; i < p.segs[s].token0 + p.segs[s].tokens; ++i) ++written[(size_t)i * c.heads + h];
    for (int w : written) NEED(w == 1);
    // the block of memory
    const BatchLayout at(p);
    std::vector<unsigned char> block(at.bytes, 0);
    at.write(p, block.data());
    NEED(p.wide_jobs.empty() || memcmp(block.data() + at.wide_jobs, p.wide_jobs.data(), p.wide_jobs.size() * sizeof(CacheJob)) == 0);
    NEED(p.positions.empty() || memcmp(block.data() + at.positions, p.positions.data(), p.positions.size() * 4) == 0);
    return true;
}

int main(int argc, char** argv) {
    const int seed = argc > 1 ? atoi(argv[1]) : 0, rounds = argc > 2 ? atoi(argv[2]) : 200;
    for (int i = 0; i < rounds; ++i) {
        rng.seed(seed * 100003 + i);
        if (!one_round()) {
            printf("round %d\n", i);
            return 1;
        }
    }
    printf("ok\n");
    return 0;
}
