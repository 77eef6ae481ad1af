// The list of the attention's requests as its kernels make it, on the host (test_operators_host.py): every thread's part of the sums, one
// after the other, over counts that the sums read from where they are written (the prompts' kernel) and over counts that are made again.
#include "kv_cache.hpp"

#include <algorithm>
#include <cstdio>
#include <vector>

struct Counts {
    const uint32_t *of;
    __host__ __device__ uint32_t operator()(uint32_t b) const { return of[b]; }
};

int main() {
    uint32_t wrong = 0, calls = 0, state = 1;
    auto next = [&] { return (state = state * 1664525u + 1013904223u) >> 8; };
    for (const uint32_t threads : {256u, 384u, 512u})
        for (uint32_t B = 1; B <= ep::kMaxRequests; B += B < 1200 ? 1 : 97) {
            std::vector<uint32_t> counts(B), own(B + 1), again(B + 1), want(B + 1);
            for (uint32_t b = 0; b < B; ++b) counts[b] = next() % 3 ? next() % 50 : 0, want[b + 1] = want[b] + counts[b];
            for (uint32_t b = 0; b < B; ++b) own[b] = counts[b];
            const uint32_t per = (B + threads - 1) / threads;
            std::vector<uint32_t> at(threads + 1);
            auto b0 = [&](uint32_t t) { return std::min(t * per, B); };
            auto b1 = [&](uint32_t t) { return std::min(b0(t) + per, B); };
            for (uint32_t t = 0; t < threads; ++t) at[t + 1] = at[t] + ep::sum_units(b0(t), b1(t), Counts{own.data()});
            for (uint32_t t = 0; t < threads; ++t) {
                ep::lay_prefix(b0(t), b1(t), at[t], Counts{own.data()}, own.data());
                ep::lay_prefix(b0(t), b1(t), at[t], Counts{counts.data()}, again.data());
            }
            own[B] = again[B] = at[threads];
            for (uint32_t b = 0; b <= B; ++b) wrong += (own[b] != want[b]) + (again[b] != want[b]);
            ++calls;
        }
    std::printf("%u %u\n", calls, wrong);
    return 0;
}
