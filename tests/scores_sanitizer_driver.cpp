// Feeds the planner seeded random batches with changed scores, valid and invalid ones, and checks of each accepted plan that
// items and units stay inside what their rows see.  Built with the address and undefined-behaviour sanitizers by
// tests/test_scores_sanitizers.py.
#include <algorithm>
#include <cmath>
#include <cstdio>
#include <cstdlib>
#include <random>
#include <string>
#include <vector>

#include "../paper_2410_18038_amd/csrc/pod_planner.h"

static void require(bool ok, const char *what, int seed)
{
    if (ok) return;
    std::fprintf(stderr, "seed %d: %s\n", seed, what);
    std::exit(1);
}

int main(int argc, char **argv)
{
    const int n_seeds = argc > 1 ? std::atoi(argv[1]) : 100;
    int n_ok = 0, n_refused = 0;
    for (int seed = 0; seed < n_seeds; ++seed) {
        std::mt19937 rng((unsigned)seed);
        auto pick = [&](int lo, int hi) { return lo + (int)(rng() % (unsigned)(hi - lo + 1)); };
        const int heads[5][3] = {{8, 2, 128}, {4, 4, 64}, {9, 3, 128}, {16, 1, 64}, {8, 1, 256}};
        const int *h = heads[pick(0, 4)];
        pod_attn_params prm = {};
        prm.n_prefill = pick(0, 3); prm.n_decode = pick(0, 20);
        prm.n_q_heads = h[0]; prm.n_kv_heads = h[1]; prm.head_dim = h[2];
        prm.dtype = pick(0, 1); prm.softmax_scale = 0.1f;
        prm.block_size = pick(0, 2) == 0 ? 0 : 16; prm.max_blocks_per_seq = 400; prm.n_cache_rows = 64; prm.n_blocks = 30000;
        prm.kv_seq_stride = (int64_t)6400 * h[1] * h[2];
        prm.n_compute_units = 256;
        if (pick(0, 2) == 0) { prm.decode_chunk = pick(1, 300); prm.prefill_split_len = pick(1, 300); prm.max_prefill_waves = 64; }
        std::vector<int32_t> meta;
        int at = 0;
        for (int r = 0; r < prm.n_prefill; ++r) {
            const int q = pick(1, 400), kv = q + pick(0, 3000);
            meta.insert(meta.end(), {at, q, kv, r});
            at += q;
        }
        for (int r = 0; r < prm.n_decode; ++r) meta.insert(meta.end(), {r, 1, pick(1, 6000), prm.n_prefill + r});
        const int n_rows = at + prm.n_decode, n_req = prm.n_prefill + prm.n_decode;
        std::vector<float> slopes((size_t)prm.n_q_heads);
        for (float &s : slopes) s = (float)pick(-10, 100) / 50.f;
        std::vector<int32_t> docs((size_t)n_rows), prefix((size_t)n_req);
        const bool nothing = pick(0, 9) == 0;
        for (int32_t &d : docs) d = nothing || pick(0, 9) == 0 ? 1 << 30 : pick(0, 3000);
        for (int32_t &p : prefix) p = pick(0, 7000);
        pod_attn_scores sc = {};
        if (pick(0, 1)) sc.logit_cap = (float)pick(1, 60);
        if (pick(0, 1)) sc.window = pick(1, 5000);
        if (pick(0, 1)) sc.slopes = slopes.data();
        if (nothing || pick(0, 1)) sc.doc_start = docs.data();
        if (pick(0, 1)) sc.prefix_len = nothing ? nullptr : prefix.data();
        switch (pick(0, 19)) {                     // now and then something that is refused
        case 0: sc.logit_cap = -1.f; break;
        case 1: sc.window = -3; break;
        case 2: if (sc.doc_start && n_rows) docs[(size_t)(n_rows - 1)] = -1; break;
        case 3: if (sc.prefix_len && n_req) prefix[0] = -1; break;
        case 4: slopes[0] = NAN; break;
        default: break;
        }
        pod::Plan plan;
        std::string err;
        const pod_status st = pod::build_plan(prm, meta.data(), 256, plan, err, &sc);
        if (st != POD_OK) { require(!err.empty(), "no message", seed); ++n_refused; continue; }
        ++n_ok;
        require(plan.ranges.size() == 2 * (size_t)n_rows && !plan.heavy_pays &&
                    (!plan.units_merge || plan.unit_splits.size() == plan.dunits.size()), "shape of the plan", seed);
        for (const pod::PrefillItem &it : plan.pitems) {
            require(it.kv_begin >= 0 && it.kv_begin <= it.kv_end && it.kv_end <= meta[4 * (size_t)it.req + 2], "keys of an item", seed);
            require(it.split == 0 || it.kv_begin % 16 == 0, "a split inside a step", seed);
        }
        for (const pod::DecodeUnit &u : plan.dunits) {
            const int32_t *range = plan.ranges.data() + 2 * (size_t)(at + u.q_start);
            require(u.t0 >= range[0] && u.t0 < u.t1 && u.t1 <= range[1], "keys of a unit", seed);
            require(u.t0 == range[0] || u.t0 % 16 == 0, "a unit begins inside a step", seed);
        }
        size_t empty = 0;
        for (int r = 0; r < prm.n_decode; ++r) empty += plan.ranges[2 * (size_t)(at + r)] >= plan.ranges[2 * (size_t)(at + r) + 1];
        require(plan.zero_rows.size() == empty, "decode rows that see nothing", seed);
        for (const pod::CombineRow &c : plan.merge_rows) {
            const uint64_t out_row = ((uint64_t)(c.out_row_hi & 0x7fffffffu) << 32 | c.out_row_lo) / (uint64_t)prm.n_q_heads;
            require(out_row < (uint64_t)n_rows && plan.ranges[2 * out_row] < plan.ranges[2 * out_row + 1], "a merged row that sees nothing", seed);
            require(c.n_splits >= 2 && c.prow >= 0 && c.prow < plan.n_partial_rows, "partials of a merged row", seed);
        }
    }
    std::printf("plans checked under the sanitizers: %d accepted, %d refused\n", n_ok, n_refused);
    return 0;
}
