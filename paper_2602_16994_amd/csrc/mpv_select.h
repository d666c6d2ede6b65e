// The largest of many keys that a workgroup holds in registers, and the order of those that are chosen.

#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace mpv {

// Thread t of BLOCK holds the keys t, t + BLOCK, ..: `held[i]` is key i * BLOCK + t, 0 where there is none (rounds: how many there are in all,
// the same for all threads).  LOW: lowest bits in which no two keys differ.
template <int BLOCK, int HELD, int LOW>
struct Select {
    static constexpr int kWaves = BLOCK / 64, kTurns = (32 - LOW) / 2, kEntries = HELD * kWaves;
    static_assert(BLOCK % 64 == 0 && (32 - LOW) % 2 == 0, "whole waves and turns");
    struct Shared {
        int counts[kTurns + 1][3];
        int2 before[kEntries];             // of a wave's keys of one round: larger ones and equal ones before them
    };

    // `limit`: the want-th largest key (its bits from LOW on; 0 if there are fewer), `above`: how many are larger.  As soon as exactly `want`
    // keys reach a number that is all there is to know: `limit` is the one below it then, and `above` is `want`.  Two bits a turn: the keys
    // that reach each of three numbers are counted by ballots, so that equal digits cost no more than different ones.
    static __device__ __forceinline__ void largest(const uint32_t (&held)[HELD], int rounds, int want, Shared& sh, uint32_t& limit, int& above) {
        __syncthreads();                                           // (a call before this one may still be read)
        for (int i = threadIdx.x; i < (kTurns + 1) * 3; i += BLOCK) sh.counts[i / 3][i % 3] = 0;
        __syncthreads();
        limit = 0;
#pragma unroll 1
        for (int turn = 0; turn < kTurns; ++turn) {
            const int shift = 30 - 2 * turn;
            int reach[3] = {};
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i < rounds) {
#pragma unroll
                    for (int d = 0; d < 3; ++d) reach[d] += __popcll(__ballot(held[i] >= (limit | static_cast<uint32_t>(d + 1) << shift)));
                }
            if ((threadIdx.x & 63) < 3) {
                const int d = threadIdx.x & 63;
                atomicAdd(&sh.counts[turn][d], d == 0 ? reach[0] : d == 1 ? reach[1] : reach[2]);
            }
            __syncthreads();
            uint32_t digit = 0;
            bool just = false;
#pragma unroll
            for (int d = 0; d < 3; ++d) {
                const int count = sh.counts[turn][d];
                digit += count >= want;
                just = just || count == want;
            }
            limit |= digit << shift;
            if (just) {
                limit -= 1u << LOW;
                above = want;
                return;
            }
        }
        int larger = 0;
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i < rounds) larger += __popcll(__ballot(held[i] >> LOW > limit >> LOW));
        if ((threadIdx.x & 63) == 0) atomicAdd(&sh.counts[kTurns][0], larger);
        __syncthreads();
        above = sh.counts[kTurns][0];
    }

    // The same where `want` is large, by counts of eleven bits at a time in a table: fewer instructions, and equal digits meet in a
    // word of LDS (1024 lists of up to 6000 scores, 512 threads each: 33 us, 50 with ballots).
    struct Table {
        int counts[2048];
        int part[kWaves];
        int digit, above, count;
    };
    static __device__ __forceinline__ void largest_by_table(const uint32_t (&held)[HELD], int rounds, int want, Table& sh, uint32_t& limit, int& above) {
        constexpr int kBins = 2048 / BLOCK;
        static_assert(2048 % BLOCK == 0, "bins");
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        limit = 0;
        above = 0;
#pragma unroll
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11;
#pragma unroll
            for (int j = 0; j < kBins; ++j) sh.counts[j * BLOCK + threadIdx.x] = 0;
            __syncthreads();
#pragma unroll
            for (int i = 0; i < HELD; ++i)
                if (i < rounds && (pass == 0 || held[i] >> (shift + bits) == limit >> (shift + bits)))
                    atomicAdd(&sh.counts[held[i] >> shift & ((1 << bits) - 1)], 1);
            __syncthreads();
            // the bins from the largest on, kBins a thread
            int mine[kBins], sum = 0;
#pragma unroll
            for (int j = 0; j < kBins; ++j) sum += mine[j] = sh.counts[2047 - (static_cast<int>(threadIdx.x) * kBins + j)];
            int upto = sum;
            for (int d = 1; d < 64; d <<= 1) {
                const int o = __shfl_up(upto, d);
                if (lane >= d) upto += o;
            }
            if (lane == 63) sh.part[wave] = upto;
            __syncthreads();
            int reached = above + upto - sum;
            for (int w = 0; w < wave; ++w) reached += sh.part[w];
#pragma unroll
            for (int j = 0; j < kBins; ++j) {
                if (reached < want && reached + mine[j] >= want) {
                    sh.digit = 2047 - (static_cast<int>(threadIdx.x) * kBins + j);
                    sh.above = reached;
                    sh.count = mine[j];
                }
                reached += mine[j];
            }
            __syncthreads();
            limit |= static_cast<uint32_t>(sh.digit) << shift;
            above = sh.above;
            if (above + sh.count == want && limit > 0) {           // all of this digit
                limit -= 1;
                above = want;
                return;
            }
        }
    }

    // take(i, place) for the chosen ones of this thread's keys: those above the limit, and the first `equal` of those that have it; `place` is
    // the key's among the chosen ones, in the order of the keys.  `size`: keys in all.
    template <class F>
    static __device__ __forceinline__ void chosen(const uint32_t (&held)[HELD], int rounds, int size, uint32_t limit, int equal, Shared& sh, const F& take) {
        const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
        auto is_equal = [&](int i) { return held[i] >> LOW == limit >> LOW && i * BLOCK + static_cast<int>(threadIdx.x) < size; };
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i < rounds) {
                const int l = __popcll(__ballot(held[i] >> LOW > limit >> LOW)), e = __popcll(__ballot(is_equal(i)));
                if (lane == 0) sh.before[i * kWaves + wave] = make_int2(l, e);
            }
        __syncthreads();
        if (wave == 0) {
            int2 sum = {0, 0};
            for (int first = 0; first < rounds * kWaves; first += 64) {
                const int at = first + lane;
                const int2 mine = at < rounds * kWaves ? sh.before[at] : make_int2(0, 0);
                int2 upto = mine;
                for (int d = 1; d < 64; d <<= 1) {
                    const int x = __shfl_up(upto.x, d), y = __shfl_up(upto.y, d);
                    if (lane >= d) { upto.x += x; upto.y += y; }
                }
                if (at < rounds * kWaves) sh.before[at] = make_int2(sum.x + upto.x - mine.x, sum.y + upto.y - mine.y);
                sum.x += __shfl(upto.x, 63);
                sum.y += __shfl(upto.y, 63);
            }
        }
        __syncthreads();
        const unsigned long long lower = (1ull << lane) - 1;
#pragma unroll
        for (int i = 0; i < HELD; ++i)
            if (i < rounds) {
                const unsigned long long l = __ballot(held[i] >> LOW > limit >> LOW), e = __ballot(is_equal(i));
                const int2 base = sh.before[i * kWaves + wave];
                const int larger = base.x + __popcll(l & lower), same = base.y + __popcll(e & lower);
                if ((l >> lane & 1) || ((e >> lane & 1) && same < equal)) take(i, larger + min(same, equal));
            }
    }
};

}  // namespace mpv
