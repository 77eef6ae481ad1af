// The shares of the prompts' attention, walked on the host as a CTA's roles walk them (test_operators_host.py).  Prints the calls, the tiles of tokens
// that were not walked exactly once, CTAs with more pieces than they have places for, and walks that left the call's requests.
#include "attend_prompts.cu"

#include <algorithm>
#include <cstdio>
#include <vector>

namespace {

uint32_t state = 7;
uint32_t next(uint32_t n) { return ((state = state * 1664525u + 1013904223u) >> 8) % n; }

struct Call {
    AttendParams P{};
    std::vector<int32_t> starts, lens;
    std::vector<uint32_t> prefix;

    // behind the arrays' ends lie requests with rows and tokens, which nobody may see
    Call(uint32_t B, uint32_t H, uint32_t G, bool cut) {
        starts.assign(1, int32_t(next(3)));
        for (uint32_t b = 0; b < B; ++b) {
            const uint32_t kind = next(8);
            starts.push_back(starts[b] + int32_t(kind == 0 ? 0 : kind == 1 ? next(300) : 1 + next(4)));
            lens.push_back(int32_t(kind == 2 ? 0 : cut ? next(900) : next(256)));
        }
        P.q.N = uint32_t(starts[B]) + next(5);
        for (uint32_t k = 0; k < 64; ++k) starts.push_back(k % 2 ? int32_t(P.q.N) : 0), lens.push_back(200);
        P.q.starts = starts.data(), P.q.seq_lens = lens.data();
        P.q.B = B, P.q.H = H, P.q.columns = cut ? 15 : 4, P.q.page = 64, P.q.shift = 6;
        P.G = G, P.Hq = G * H, P.causal = next(2), P.grid = 148;
        P.workspace = cut ? reinterpret_cast<float *>(16) : nullptr;          // (never read)
        prefix.assign(B + 1, 0);
        for (uint32_t b = 0; b < B; ++b) {
            const Extent r = extent_of(P.q, b);
            for (uint32_t j = 0; j < row_tiles_of(P, r); ++j) prefix[b + 1] += (tiles_of(P, r, j) + kStart) * H;
        }
        for (uint32_t b = 0; b < B; ++b) prefix[b + 1] += prefix[b];
    }
    // where CTA k of `ctas` begins
    Place start(uint32_t k, uint32_t ctas) const {
        const uint64_t all = prefix.back();
        const uint32_t from = uint32_t(all * k / ctas), to = uint32_t(all * (k + 1) / ctas);
        Place p{0, 0, 0, 0, from, to - from};
        p.b = uint32_t(std::upper_bound(prefix.begin(), prefix.end(), from) - prefix.begin()) - 1u;
        const Extent r = extent_of(P.q, p.b);
        uint32_t v = from - prefix[p.b];
        while (v >= (tiles_of(P, r, p.j) + kStart) * P.q.H) v -= (tiles_of(P, r, p.j++) + kStart) * P.q.H;
        const uint32_t per_head = tiles_of(P, r, p.j) + kStart;
        p.h = v / per_head, p.off = v % per_head;
        if (!P.workspace && p.off) {
            const uint32_t skip = per_head - p.off;
            p.left -= std::min(p.left, skip), p.at += skip, p.off = 0;
            if (++p.h == P.q.H) p.h = 0, ++p.j;
        }
        return p;
    }
};

}  // namespace

int main() {
    uint32_t calls = 0, wrong = 0, crowded = 0, outside = 0;
    for (const uint32_t B : {1u, 2u, 7u, 100u, 511u, 513u, 700u, 2000u})
        for (uint32_t round = 0; round < 12; ++round, ++calls) {
            const Call c(B, 1 + next(3), 1 + next(9), round % 2);
            const AttendParams &P = c.P;
            std::vector<std::vector<uint32_t>> seen(B);      // how often tile i of (row tile, head) was walked
            for (uint32_t b = 0; b < B; ++b) {
                const Extent r = extent_of(P.q, b);
                for (uint32_t j = 0; j < row_tiles_of(P, r); ++j) seen[b].resize(seen[b].size() + P.q.H * tiles_of(P, r, j));
            }
            const uint32_t ctas = std::min(P.grid, c.prefix.back());
            for (uint32_t k = 0; k < ctas; ++k) {
                uint32_t begun = 0, continued = 0;
                for (Cursor x(P, c.start(k, ctas)); x.more(); x.next()) {
                    if (x.p.b >= B || x.row0() >= x.r.rows * P.G) { ++outside; break; }
                    uint32_t at = 0;
                    for (uint32_t j = 0; j < x.p.j; ++j) at += P.q.H * tiles_of(P, x.r, j);
                    for (uint32_t i = 0; i < x.count; ++i) ++seen[x.p.b][at + x.p.h * x.total + x.first + i];
                    if (x.count && x.count != x.total) ++(x.first ? continued : begun);
                }
                crowded += begun > 1 || continued > 1;
            }
            for (const auto &s : seen) for (const uint32_t n : s) wrong += n != 1;
            // a share that has more places left than there are: it ends with the last request
            uint32_t steps = 0;
            for (Cursor x(P, Place{B - 1, 0, 0, 0, 0, 100000}); x.more(); x.next())
                if (x.p.b >= B || ++steps > 200000) { ++outside; break; }
        }
    std::printf("%u %u %u %u\n", calls, wrong, crowded, outside);
    return 0;
}
