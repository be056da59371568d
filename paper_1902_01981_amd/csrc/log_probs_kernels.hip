// Log probabilities of tokens, entropy and the most probable alternatives, and the gradient of the first two, for gfx950.
//
// With c the largest x_j of a row (or of a part):  S = sum_j exp(x_j - c),  E = sum_j exp(x_j - c) (x_j - c);  l_j = x_j - c - log S,  entropy = log S - E / S.  Sums about two
// references meet by S exp(c - c') and (E + S (c - c')) exp(c - c').
// The alternatives: at least `top` values are no smaller than the top-th largest of the largest values of disjoint sets, so what is no smaller than that is
// all that can be among them, and few other than them; their order is that of numbers with the value above and the index's complement below, of which no two are equal.
//
//   log_probs_narrow_kernel    four rows in a wavefront
//   log_probs_slices_kernel    a row, or a slice of it, in the registers of a wavefront or a workgroup, read once
//   log_probs_join_kernel      rows of several slices
//   log_probs_gradient_kernel, log_probs_narrow_gradient_kernel   the gradient
//
// Without alternatives reads bound it, and arithmetic about as much: 8 192 x 131 071 bf16 413 us, 5.2 TB/s; 4 099 x 50 008 bf16 73 us, 5.6 TB/s; 2 048 x 128 000
// fp32 158 us, 6.6 TB/s.  With them a slice's bound, list and ranks, each of which waits for the one before: 4 099 x 50 008 with 8 84 us, with 64 114, with 128 153;
// 8 192 x 131 071 with 8 431; rows of equal values 335 (64).  A bound of 16 bits tells few fp32 logits apart whose common offset is large beside their spread, and
// every slice is then searched bit by bit: 2 048 x 128 000 fp32 with 64, normal logits of deviation 3, 220 us, 263 around 300, 4.3 ms around 3 000; bf16, 4 099 x 50 008, 114, 125 and
// 334, where what is left of the logits are equal values.  A workgroup's lanes have eight chunks whether the slice fills them or not: 40 990 x 5 000 bf16 109 us, 3.8 TB/s,
// x 8 000 130, x 16 384 199, 6.8 TB/s, x 4 096 by wavefronts 55, 6.1 TB/s; with 20 177, 184, 253 and 86.  Teams of 512 threads took 122 with 64 and 464 (8 192 x 131 071 with 8), of 1 024 182 and 780.
// 100 000 x 100 bf16 with five 32 us, without 10.  Gradient: 8 192 x 131 071 bf16 812 us, 5.3 TB/s; 100 000 x 100 12 us.
#include "softmax_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr int kThreads = 256, kTeam = 256, kMostTop = 128;
constexpr float kLowest = -3.4028234663852886e38f;

struct Part {
    float c, S, E, unused;
};
// distances past which exp is 0, so that what it is multiplied with may be anything finite
__device__ __forceinline__ float bounded(float d) { return fmaxf(d, -128.f); }
// the same sums about a reference that is no smaller
__device__ __forceinline__ Part about(const Part &p, float c)
{
    const float d = p.c - usable(c), f = exp_fast(d);
    return {c, p.S * f, fmaf(p.S, bounded(d), p.E) * f, 0.f};
}
__device__ __forceinline__ Part joined(const Part &a, const Part &b)
{
    const float c = fmaxf(a.c, b.c);
    const Part u = about(a, c), v = about(b, c);
    return {c, u.S + v.S, u.E + v.E, 0.f};
}
template <int LANES> __device__ __forceinline__ void join_lanes(Part &p)
{
    p = about(p, lanes_most<LANES>(p.c));
    // rounded here: a product taken into the first of the additions would give every lane another sum
    hold(p.S);
    hold(p.E);
    p.S = lanes_total<LANES>(p.S);
    p.E = lanes_total<LANES>(p.E);
}

// numbers in the order of the values, both zeros the same
__device__ __forceinline__ uint32_t ordered(float x)
{
    const uint32_t u = __float_as_uint(x + 0.f);
    return u >> 31 ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o >> 31 ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t entry_of(float x, int index) { return uint64_t(ordered(x)) << 32 | (0xffffffffu - static_cast<uint32_t>(index)); }

// log S comes as log2 S, and every use of it is one multiply-add, spelled out: the same bits wherever it is.
__device__ __forceinline__ float log_prob(float x, const Part &p, float log2_S) { return fmaf(-kLn2, log2_S, x - p.c); }
struct Token {
    int64_t t;
    float x;
};
__device__ __forceinline__ Token read_token(const LogProbsArgs &a, int64_t row)
{
    if (!a.logp) return {-1, 0.f};
    const int64_t t = a.tokens[row], at = row * a.row_stride + (t >= 0 && t < a.classes ? t : 0);
    return {t, a.bf16 ? Element<true>::get(static_cast<const uint16_t *>(a.logits) + at) : static_cast<const float *>(a.logits)[at]};
}
// what is written of a row
__device__ __forceinline__ void write_row(const LogProbsArgs &a, int64_t row, const Token &token, const Part &p, float log2_S)
{
    if (a.logp) a.logp[row] = token.t < 0 ? 0.f : token.t >= a.classes ? __builtin_nanf("") : p.S == 0.f ? -infinity() : log_prob(token.x, p, log2_S);
    if (a.entropy) a.entropy[row] = p.S == 0.f ? 0.f : fmaf(kLn2, log2_S, -(p.E / p.S));
    if (a.largest) {
        // a NaN that the largest value does not show is in the sum
        a.largest[row] = p.S == p.S ? p.c : __builtin_nanf("");
        a.log_sum[row] = kLn2 * log2_S;
    }
}
__device__ __forceinline__ void write_entry(const LogProbsArgs &a, int64_t row, int place, uint64_t entry, const Part &p, float log2_S)
{
    const bool number = p.S == p.S;
    const int64_t to = row * a.top + place;
    a.top_index[to] = entry && number ? int64_t(0xffffffffu - static_cast<uint32_t>(entry)) : -1;
    a.top_logp[to] = !number ? __builtin_nanf("") : entry ? log_prob(unordered(static_cast<uint32_t>(entry >> 32)), p, log2_S) : -infinity();
}

// The team that has a row or slice: a wavefront, or a workgroup.
template <int SIZE> struct Team {
    static constexpr bool kWave = SIZE == 64;
    static constexpr int kWaves = SIZE / 64;
    static __device__ __forceinline__ void sync()
    {
        if constexpr (kWave) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }
    // f over the team's wavefronts, each of which has a value of its own; meet: a place for each
    template <typename F> static __device__ __forceinline__ float over_waves(float v, float *meet, F f)
    {
        if constexpr (!kWave) {
            if (threadIdx.x % 64 == 0) meet[threadIdx.x / 64] = v;
            __syncthreads();
            v = meet[0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v = f(v, meet[w]);
            __syncthreads();
        }
        return v;
    }
    // the sum over the team of small numbers
    static __device__ __forceinline__ int total(int mine, float *meet)
    {
        return static_cast<int>(over_waves(lanes_total<64>(static_cast<float>(mine)), meet, [](float a, float b) { return a + b; }));
    }
};

// The top-th largest of a wavefront's numbers of 16 bits, 0 if there are no so many above 0: bit by bit, from the first in which any differ.
template <int N> __device__ __forceinline__ uint32_t reached(const uint32_t (&keys)[N], int top)
{
    uint32_t all = keys[0], any = keys[0];
#pragma unroll
    for (int i = 1; i < N; ++i) {
        all &= keys[i];
        any |= keys[i];
    }
    // what the lanes have in common, as numbers of 16 bits beside each other
    uint32_t both = any << 16 | (~all & 0xffffu);
    both |= __builtin_amdgcn_update_dpp(0, both, 0xB1, 0xf, 0xf, false);
    both |= __builtin_amdgcn_update_dpp(0, both, 0x4E, 0xf, 0xf, false);
    both |= __builtin_amdgcn_update_dpp(0, both, 0x141, 0xf, 0xf, false);
    both |= __builtin_amdgcn_update_dpp(0, both, 0x140, 0xf, 0xf, false);
    const uint32_t joined = __builtin_amdgcn_readlane(both, 0) | __builtin_amdgcn_readlane(both, 16) | __builtin_amdgcn_readlane(both, 32) | __builtin_amdgcn_readlane(both, 48);
    const uint32_t differ = joined >> 16 & joined & 0xffffu;         // bits that some have and some have not
    const int first = 31 - __builtin_clz(differ | 1u);
    uint32_t least = (joined >> 16 & ~differ) >> (first + 1) << (first + 1);
    int reach = 0;
#pragma unroll 1
    for (int bit = first; bit >= 0; --bit) {
        const uint32_t more = least | 1u << bit;
        int count = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) count += __popcll(__ballot(keys[i] >= more));
        if (count >= top) {
            least = more;
            reach = count;
        }
    }
    // no bit was taken: whether the prefix itself is reached is not known yet
    if (reach == 0) {
#pragma unroll
        for (int i = 0; i < N; ++i) reach += __popcll(__ballot(keys[i] >= max(least, 1u)));
    }
    return reach >= top ? least : 0u;
}
__device__ __forceinline__ uint32_t short_key(float x) { return x > -infinity() ? ordered(x) >> 16 : 0u; }       // 0 of -infinity and NaN

constexpr int kWaveEntries = 512, kBlockEntries = 1024;  // that a team keeps of those that may be among the largest

// The `top` largest of chunks [begin, end) of a row, where too many are no smaller than `least`: the top-th largest value itself, which is the smallest of them if all the
// others are too few (two passes, where many are equal), and is found bit by bit if not (32 more); then as many of its places as are wanted, lowest first (two).  The chunks are
// read again each time: 32 KB at most, from the caches.
template <bool BF16, int VEC, int TEAM>
__device__ __noinline__ int select_exactly(const typename Chunk<BF16, VEC>::element *x, int begin, int end, int nq, int classes, int top, float least, uint64_t *list, int *count, float *meet)
{
    using C = Chunk<BF16, VEC>;
    using Group = Team<TEAM>;
    const int lane = threadIdx.x % TEAM, doubled = nq * VEC - classes;
    // f(number in order, index, value) for the elements of a step that are this thread's; places of a step lie behind those of the one before
    auto of_step = [&](int q0, auto &&f) {
        const int q = q0 + lane;
        if (q >= end) return;
        const int at = chunk_at<VEC>(q, nq, classes);
        float v[VEC];
        C::widen(C::load(x + at), v);
#pragma unroll
        for (int i = 0; i < VEC; ++i)
            if (v[i] > -infinity() && (q < nq - 1 || i >= doubled)) f(ordered(v[i]), at + i, v[i]);
    };
    auto number = [&](auto &&counts) {
        int mine = 0;
        for (int q0 = begin; q0 < end; q0 += TEAM) of_step(q0, [&](uint32_t o, int, float) { mine += counts(o); });
        return Group::total(mine, meet);
    };
    Group::sync();
    float smallest = infinity();
    for (int q0 = begin; q0 < end; q0 += TEAM) of_step(q0, [&](uint32_t, int, float v) { smallest = v >= least ? fminf(smallest, v) : smallest; });
    smallest = Group::over_waves(-lanes_most<64>(-smallest), meet, [](float a, float b) { return fminf(a, b); });
    uint32_t value = ordered(smallest);
    if (number([&](uint32_t o) { return o > value; }) >= top) {
        value = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t more = value | 1u << bit;
            if (number([&](uint32_t o) { return o >= more; }) >= top) value = more;
        }
    }
    if (lane == 0) *count = 0;
    Group::sync();
    for (int q0 = begin; q0 < end; q0 += TEAM)
        of_step(q0, [&](uint32_t o, int index, float v) {
            if (o > value) {
                const int to = atomicAdd(count, 1);
                if (to < kMostTop) list[to] = entry_of(v, index);
            }
        });
    Group::sync();
    int n = min(*count, top);                            // fewer than `top`; places of the value itself fill them up
    for (int q0 = begin; q0 < end && n < top; q0 += TEAM) {
        int mine = 0;
        of_step(q0, [&](uint32_t o, int, float) { mine += o == value; });
        int sum = mine;                                  // up to and with this lane
        for (int d = 1; d < 64; d *= 2) {
            const int other = __shfl_up(sum, d);
            if (static_cast<int>(threadIdx.x % 64) >= d) sum += other;
        }
        int total = __shfl(sum, 63), before = 0;
        if constexpr (!Group::kWave) {
            if (threadIdx.x % 64 == 63) meet[threadIdx.x / 64] = static_cast<float>(sum);
            __syncthreads();
            total = 0;
            for (int w = 0; w < Group::kWaves; ++w) {
                if (w < static_cast<int>(threadIdx.x / 64)) before += static_cast<int>(meet[w]);
                total += static_cast<int>(meet[w]);
            }
            __syncthreads();
        }
        int to = n + before + sum - mine;
        of_step(q0, [&](uint32_t o, int index, float v) {
            if (o == value) {
                if (to < top) list[to] = entry_of(v, index);
                ++to;
            }
        });
        n = min(n + total, top);
    }
    Group::sync();
    return n;
}

// K chunks of a lane; TOP: alternatives are wanted.  A team has one unit, a row or a slice of one: where it stayed and read the next unit's chunks as it was done with
// these, 4 099 x 50 008 bf16 took 102 us and 246 with 64 alternatives, since that took registers from the other teams, whose loads hide the waits as well.
// Arithmetic bounds it as much as reads do (an exponential is four operations), so a sweep over a lane's chunks has no operation too many: the largest first, then
// the sums, E without a bound on the distances: where a class cannot be it is NaN (0 times infinity), and those lanes add up once more.
constexpr int kWavesOf[2] = {6, 8};                      // of a SIMD: where a lane has eight chunks, and where it has fewer
template <bool BF16, int VEC, int K, int TEAM, bool TOP>
__global__ void __launch_bounds__(TEAM == 64 ? kThreads : TEAM) __attribute__((amdgpu_waves_per_eu(kWavesOf[K < 8])))
log_probs_slices_kernel(LogProbsArgs a, int slice, int slices, Part *parts, uint64_t *lists)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    using Group = Team<TEAM>;
    constexpr bool WAVE = Group::kWave;
    constexpr int kTeams = WAVE ? kThreads / 64 : 1, kEntries = !TOP ? 1 : WAVE ? kWaveEntries : kBlockEntries;
    __shared__ uint64_t entries[kTeams][kEntries];
    __shared__ int counts[kTeams];
    __shared__ float meet[3][Group::kWaves];
    __shared__ uint32_t maxima[WAVE || !TOP ? 1 : TEAM];
    __shared__ float bound;
    __shared__ int ranks[WAVE || !TOP ? 1 : 128];
    constexpr int kHits = WAVE || !TOP ? 1 : 512;
    __shared__ typename C::raw hit[kHits];
    __shared__ int hit_at[kHits], hits;
    const int wave = threadIdx.x / 64, team = WAVE ? wave : 0, lane = threadIdx.x % TEAM;
    const int unit = WAVE ? blockIdx.x * kTeams + team : blockIdx.x;               // fewer than 2^22 in a batch
    const int row = WAVE || slices == 1 ? unit : unit / slices;
    if (row >= a.rows) return;                           // whole teams; there is no barrier of the workgroup where a team is a wavefront
    const int nq = (a.classes + VEC - 1) / VEC, begin = WAVE ? 0 : (unit - row * slices) * slice, end = min(begin + slice, nq);
    const int doubled = nq * VEC - a.classes;            // of the last chunk, which is moved back to end with the row
    const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
    auto place = [&](int k) { return chunk_at<VEC>(min(begin + lane + k * TEAM, end - 1), nq, a.classes); };
    auto has = [&](int k) { return begin + lane + k * TEAM < end; };

    typename C::raw raw[K];
#pragma unroll
    for (int k = 0; k < K; ++k) raw[k] = C::load_once(x + place(k));
    const bool alone = WAVE || slices == 1;
    Token token = {};
    if (alone) token = read_token(a, row);
    float v[VEC], most[K], own = -infinity();            // own: the largest of this thread
#pragma unroll
    for (int k = 0; k < K; ++k) {
        // what the neighbour has is here a class that cannot be
        if (begin + lane + k * TEAM == nq - 1 && doubled > 0) {
            C::widen(raw[k], v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = i < doubled ? -infinity() : v[i];
            raw[k] = C::narrow(v);
        }
        C::widen(raw[k], v);
        float m = v[0];
#pragma unroll
        for (int i = 1; i < VEC; ++i) m = fmaxf(m, v[i]);
        most[k] = has(k) ? m : -infinity();
        own = fmaxf(own, most[k]);
        hold(raw[k]);                                    // widened again later, rather than kept wide
    }
    Part p = {own, 0.f, 0.f, 0.f};
    const float from = usable(own);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        if (has(k)) {
            C::widen(raw[k], v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = v[i] - from, e = exp_fast(d);
                p.S += e;
                p.E = fmaf(e, d, p.E);
            }
        }
        hold(raw[k]);
    }
    if (!(p.E == p.E)) {
        p.E = 0.f;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (!has(k)) continue;
            C::widen(raw[k], v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const float d = v[i] - from;
                p.E = fmaf(exp_fast(d), bounded(d), p.E);
            }
            if constexpr (TOP) hold(raw[k]);
        }
    }
    join_lanes<64>(p);
    if constexpr (!WAVE) {
        if (threadIdx.x % 64 == 0) {
            meet[0][wave] = p.c;
            meet[1][wave] = p.S;
            meet[2][wave] = p.E;
        }
        if constexpr (TOP) maxima[threadIdx.x] = short_key(own);
        __syncthreads();
        const int w = threadIdx.x % Group::kWaves;
        p = {meet[0][w], meet[1][w], meet[2][w], 0.f};
        join_lanes<Group::kWaves>(p);
    }
    const float log2_S = __builtin_amdgcn_logf(p.S);     // the hardware's logarithm is that to base 2
    if (lane == 0) {
        if (alone) write_row(a, row, token, p, log2_S);
        else parts[unit] = p;
    }
    if constexpr (TOP) {
        uint64_t *list = entries[team];
        int *count = &counts[team];
        float least;
        if constexpr (WAVE) {
            // sets of a lane's elements: the chunks; where they are too few for a bound that is one, eight sets of a lane if it has so many elements
            constexpr int kSets = K >= 8 ? 1 : VEC < 8 / K ? VEC : 8 / K, kOfSet = VEC / kSets;
            uint32_t key;
            if (kSets == 1 || 2 * a.top <= nq) {
                uint32_t keys[K];
#pragma unroll
                for (int k = 0; k < K; ++k) keys[k] = short_key(most[k]);
                key = reached(keys, a.top);
            } else {
                uint32_t keys[K * kSets];
#pragma unroll
                for (int k = 0; k < K; ++k) {
                    C::widen(raw[k], v);
#pragma unroll
                    for (int set = 0; set < kSets; ++set) {
                        float m = v[set * kOfSet];
#pragma unroll
                        for (int i = 1; i < kOfSet; ++i) m = fmaxf(m, v[set * kOfSet + i]);
                        keys[k * kSets + set] = has(k) ? short_key(m) : 0u;
                    }
                }
                key = reached(keys, a.top);
            }
            least = key ? unordered(key << 16) : kLowest;
        } else if (wave == 0) {
            uint32_t keys[Group::kWaves];
#pragma unroll
            for (int i = 0; i < Group::kWaves; ++i) keys[i] = maxima[threadIdx.x + 64 * i];
            const uint32_t key = reached(keys, a.top);
            if (threadIdx.x == 0) bound = key ? unordered(key << 16) : kLowest;
        }
        if (lane == 0) {
            *count = 0;
            if constexpr (!WAVE) hits = 0;
        }
        Group::sync();
        if constexpr (!WAVE) least = bound;
        bool all_kept = true;
        if constexpr (WAVE) {
            // the chunks with such elements, one of each lane at a time: few lanes have any, and fewer have several
            unsigned chunks = 0;
#pragma unroll
            for (int k = 0; k < K; ++k) chunks |= most[k] >= least ? 1u << k : 0u;
            while (chunks) {
                const int which = __builtin_ctz(chunks);
                chunks &= chunks - 1;
                typename C::raw one = raw[0];
#pragma unroll
                for (int k = 1; k < K; ++k) one = which == k ? raw[k] : one;
                C::widen(one, v);
                const int at = chunk_at<VEC>(begin + lane + which * TEAM, nq, a.classes);
                int hits = 0;
#pragma unroll
                for (int i = 0; i < VEC; ++i) hits += v[i] >= least;
                int to = atomicAdd(count, hits);
#pragma unroll
                for (int i = 0; i < VEC; ++i)
                    if (v[i] >= least) {
                        if (to < kEntries) list[to] = entry_of(v[i], at + i);
                        ++to;
                    }
            }
        } else {
            // the chunks with such elements to where all threads can look at them, an element each
#pragma unroll
            for (int k = 0; k < K; ++k)
                if (most[k] >= least) {
                    const int to = atomicAdd(&hits, 1);
                    if (to < kHits) {
                        hit[to] = raw[k];
                        hit_at[to] = lane + k * TEAM;
                    }
                }
            __syncthreads();
            const int found = hits;
            all_kept = found <= kHits;
            if (all_kept)
                for (int e = threadIdx.x; e < found * VEC; e += TEAM) {
                    const float one = Element<BF16>::get(reinterpret_cast<const T *>(hit) + e);
                    if (one >= least) {
                        const int to = atomicAdd(count, 1);
                        if (to < kEntries) list[to] = entry_of(one, chunk_at<VEC>(begin + hit_at[e / VEC], nq, a.classes) + e % VEC);
                    }
                }
        }
        Group::sync();
        int n = *count;
        if (n > kEntries || !all_kept) n = select_exactly<BF16, VEC, TEAM>(x, begin, end, nq, a.classes, a.top, least, list, count, meet[0]);
        auto leave = [&](int rank, uint64_t entry) {
            if (alone) write_entry(a, row, rank, entry, p, log2_S);
            else lists[int64_t(unit) * a.top + rank] = entry;
        };
        if (!WAVE && n <= 128) {
            // several threads an entry, each against a part of the others
            const int across = n <= 64 ? 64 : 128, each = (n * across + TEAM - 1) / TEAM, i = threadIdx.x % across, first = threadIdx.x / across * each;
            if (threadIdx.x < across) ranks[threadIdx.x] = 0;
            __syncthreads();
            uint64_t entry = 0;
            if (i < n) {
                entry = list[i];
                int rank = 0;
#pragma unroll 8
                for (int j = first; j < min(first + each, n); ++j) rank += list[j] > entry;
                atomicAdd(&ranks[i], rank);
            }
            __syncthreads();
            if (threadIdx.x < n && ranks[i] < a.top) leave(ranks[i], entry);
        } else {
            for (int i = lane; i < n; i += TEAM) {
                const uint64_t entry = list[i];
                int rank = 0;
#pragma unroll 8
                for (int j = 0; j < n; ++j) rank += list[j] > entry;
                if (rank < a.top) leave(rank, entry);
            }
        }
        for (int rank = n + lane; rank < a.top; rank += TEAM) leave(rank, 0);
    }
}

// Rows of up to 32 chunks: sixteen lanes each, four rows beside each other in a wavefront.  (A wavefront per row took 100 000 x 100 bf16 66 us with five
// alternatives: its instructions, whatever the row has.)  The bound is the top-th largest element's upper half here, found bit by bit by all four rows at once.
template <bool BF16, int VEC, int K, bool TOP> __global__ void __launch_bounds__(kThreads) log_probs_narrow_kernel(LogProbsArgs a)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    constexpr int kLanes = 16, kElements = kLanes * K * VEC;
    __shared__ uint64_t entries[TOP ? kThreads / kLanes : 1][TOP ? kElements + 1 : 1];             // teams begin in other banks
    const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
    const int64_t own_row = int64_t(blockIdx.x) * (kThreads / kLanes) + team, row = std::min(own_row, a.rows - 1);
    const bool here = own_row < a.rows;                  // the others go along
    const int nq = (a.classes + VEC - 1) / VEC, doubled = nq * VEC - a.classes;
    const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
    typename C::raw raw[K];
#pragma unroll
    for (int k = 0; k < K; ++k) raw[k] = C::load_once(x + chunk_at<VEC>(min(lane + k * kLanes, nq - 1), nq, a.classes));
    const Token token = read_token(a, row);
    float v[K][VEC], most = -infinity();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        C::widen(raw[k], v[k]);
        const int q = lane + k * kLanes, none = q >= nq ? VEC : q == nq - 1 ? doubled : 0;         // no elements of this place
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            v[k][i] = i < none ? -infinity() : v[k][i];
            most = fmaxf(most, v[k][i]);
        }
    }
    Part p = {most, 0.f, 0.f, 0.f};
    const float from = usable(most);
#pragma unroll
    for (int k = 0; k < K; ++k) {
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float d = v[k][i] - from, e = exp_fast(d);
            p.S += e;
            p.E = fmaf(e, bounded(d), p.E);
        }
    }
    join_lanes<kLanes>(p);
    const float log2_S = __builtin_amdgcn_logf(p.S);
    if (lane == 0 && here) write_row(a, row, token, p, log2_S);
    if constexpr (TOP) {
        auto number = [&](uint32_t bound) {              // of the row's elements that reach it
            int mine = 0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) mine += short_key(v[k][i]) >= bound;
            }
            return static_cast<int>(lanes_total<kLanes>(static_cast<float>(mine)));
        };
        uint32_t key = 0;
#pragma unroll 1
        for (int bit = 15; bit >= 0; --bit) {
            const uint32_t more = key | 1u << bit;
            if (number(more) >= a.top) key = more;
        }
        const float least = key ? unordered(key << 16) : kLowest;
        uint64_t *list = entries[team];
        int hits = 0;
#pragma unroll
        for (int k = 0; k < K; ++k) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) hits += v[k][i] >= least;
        }
        int to = hits;                                   // up to and with this lane, then before it
#pragma unroll
        for (int d = 1; d < kLanes; d *= 2) {
            const int other = __shfl_up(to, d, kLanes);
            if (lane >= d) to += other;
        }
        const int n = __shfl(to, kLanes - 1, kLanes);
        to -= hits;
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int at = chunk_at<VEC>(min(lane + k * kLanes, nq - 1), nq, a.classes);
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (v[k][i] >= least) list[to++] = entry_of(v[k][i], at + i);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        if (!here) return;
        for (int i = lane; i < n; i += kLanes) {
            const uint64_t entry = list[i];
            int rank = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) rank += list[j] > entry;
            if (rank < a.top) write_entry(a, row, rank, entry, p, log2_S);
        }
        for (int rank = n + lane; rank < a.top; rank += kLanes) write_entry(a, row, rank, 0, p, log2_S);
    }
}

// A row's slices: their sums, and the largest of their lists, a few lists at a time beside those found so far.  A number's place is the number of larger ones in
// every list, each of which is in order.
constexpr int kListsAtOnce = 8;
template <int THREADS> __global__ void __launch_bounds__(THREADS) log_probs_join_kernel(LogProbsArgs a, int slices, const Part *parts, const uint64_t *lists)
{
    extern __shared__ uint64_t some[];                   // [list][place], the ones found so far first; behind them those that are found
    __shared__ float meet[3][4];
    const int64_t row = blockIdx.x;
    const int top = a.top;
    const Token token = read_token(a, row);
    Part p = {-infinity(), 0.f, 0.f, 0.f};
    for (int i = threadIdx.x; i < slices; i += THREADS) p = joined(p, parts[row * slices + i]);
    uint64_t *best = some + (kListsAtOnce + 1) * top;
    for (int i = threadIdx.x; i < top; i += THREADS) best[i] = 0;
    for (int first = 0; first < slices && top > 0; first += kListsAtOnce) {
        const int now = min(kListsAtOnce, slices - first);
        __syncthreads();
        for (int i = threadIdx.x; i < now * top; i += THREADS) some[top + i] = lists[(row * slices + first) * top + i];
        for (int i = threadIdx.x; i < top; i += THREADS) {
            some[i] = best[i];
            best[i] = 0;
        }
        __syncthreads();
        // of `count` lists the first ones of each, `top` or more together, are no smaller than the smallest of the last of these
        const int empty = first == 0 ? 1 : 0, count = now + 1 - empty, share = (top + count - 1) / count;
        uint64_t bound = ~uint64_t(0);
        for (int list = empty; list <= now; ++list) bound = min(bound, some[list * top + share - 1]);
        for (int i = threadIdx.x; i < count * top; i += THREADS) {
            const int rank = i / count, mine = empty + i - rank * count;
            const uint64_t entry = some[mine * top + rank];
            if (!entry || entry < bound) continue;
            int before[kListsAtOnce + 1];                // larger ones of each list, all lists a step at a time
#pragma unroll
            for (int other = 0; other <= kListsAtOnce; ++other) before[other] = 0;
            for (int step = 1 << (31 - __builtin_clz(top)); step > 0; step /= 2) {
#pragma unroll
                for (int other = 0; other <= kListsAtOnce; ++other) {
                    const int to = before[other] + step;
                    if (other >= empty && other <= now && to <= top && some[other * top + to - 1] > entry) before[other] = to;
                }
            }
            int place = rank;
#pragma unroll
            for (int other = 0; other <= kListsAtOnce; ++other) place += other == mine ? 0 : before[other];
            if (place < top) best[place] = entry;
        }
    }
    join_lanes<64>(p);
    if constexpr (THREADS > 64) {
        if (threadIdx.x % 64 == 0) {
            meet[0][threadIdx.x / 64] = p.c;
            meet[1][threadIdx.x / 64] = p.S;
            meet[2][threadIdx.x / 64] = p.E;
        }
        __syncthreads();
        p = {meet[0][threadIdx.x % 4], meet[1][threadIdx.x % 4], meet[2][threadIdx.x % 4], 0.f};
        join_lanes<4>(p);
    }
    const float log2_S = __builtin_amdgcn_logf(p.S);
    if (threadIdx.x == 0) write_row(a, row, token, p, log2_S);
    __syncthreads();
    for (int i = threadIdx.x; i < top; i += THREADS) write_entry(a, row, i, best[i], p, log2_S);
}

// dx_j = a ([j = t] - p_j) - b p_j (l_j + entropy)
struct RowGradient {
    float c, L, by_logp, by_entropy, H, value;
    int64_t t;
    bool flat;                   // all of the row is `value`
    __device__ __forceinline__ RowGradient(const LogProbsGradArgs &a, int64_t row)
    {
        c = a.largest[row];
        L = a.log_sum[row];
        t = a.tokens ? a.tokens[row] : -1;
        by_logp = t >= 0 ? a.dlogp[row] : 0.f;
        by_entropy = a.entropy ? a.dentropy[row] : 0.f;
        H = a.entropy ? a.entropy[row] : 0.f;
        flat = t >= a.classes || c == -infinity();
        value = t >= a.classes ? __builtin_nanf("") : 0.f;
    }
    __device__ __forceinline__ float of(float x, int j) const
    {
        const float l = x - c - L, p = exp_fast(l);
        const float g = -p * (by_logp + by_entropy * (H + fmaxf(l, -256.f)));              // p is 0 there already
        return flat ? value : j == t ? g + by_logp : g;
    }
};
// A thread has K chunks of a row, and an element of those behind the whole chunks.
template <bool BF16, int VEC, int K> __global__ void __launch_bounds__(kThreads) log_probs_gradient_kernel(LogProbsGradArgs a, int tiles)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    const int whole = a.classes / VEC, left = a.classes % VEC;
    const int64_t units = a.rows * tiles;
    for (int64_t unit = blockIdx.x; unit < units; unit += gridDim.x) {
        const int64_t row = unit / tiles;
        const int tile = static_cast<int>(unit - row * tiles);
        const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
        T *dx = static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride;
        const RowGradient g(a, row);
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int q = (tile * K + k) * kThreads + threadIdx.x;
            if (q < whole) {
                float v[VEC];
                C::widen(C::load(x + q * VEC), v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = g.of(v[i], q * VEC + i);
                C::store(dx + q * VEC, C::narrow(v));
            }
        }
        if (tile == 0 && threadIdx.x < left) {
            const int j = whole * VEC + threadIdx.x;
            Element<BF16>::put(dx + j, g.of(Element<BF16>::get(x + j), j));
        }
    }
}
// Rows of fewer chunks than a workgroup has threads: their chunks, and the elements behind them, beside each other.  (100 000 x 100 bf16 78 us a workgroup per row.)
template <bool BF16, int VEC> __global__ void __launch_bounds__(kThreads) log_probs_narrow_gradient_kernel(LogProbsGradArgs a, Divisor items)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    const int whole = a.classes / VEC, per = items.d;
    const int64_t all = a.rows * per;
    for (int64_t first = int64_t(blockIdx.x) * kThreads; first < all; first += int64_t(gridDim.x) * kThreads) {
        const int64_t row0 = first / per;
        const uint32_t l = static_cast<uint32_t>(first - row0 * per) + threadIdx.x, r = items.of(l);
        const int64_t row = row0 + r;
        const int item = l - r * per;
        if (row >= a.rows) continue;
        const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
        T *dx = static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride;
        const RowGradient g(a, row);
        if (item < whole) {
            float v[VEC];
            C::widen(C::load(x + item * VEC), v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = g.of(v[i], item * VEC + i);
            C::store(dx + item * VEC, C::narrow(v));
        } else {
            const int j = whole * (VEC - 1) + item;      // whole * VEC + (item - whole)
            Element<BF16>::put(dx + j, g.of(Element<BF16>::get(x + j), j));
        }
    }
}

struct LogProbsPlan {
    int vec, chunks;             // of a chunk, of a row
    int k;                       // chunks per thread
    bool wave;                   // a wavefront per row
    int slice, slices;           // chunks of a slice, slices of a row
    int64_t batch;               // rows per pair of launches
};
LogProbsPlan plan_log_probs(int64_t rows, int64_t classes, bool bf16, int top)
{
    LogProbsPlan p = {};
    p.vec = classes < (bf16 ? 8 : 4) ? 1 : bf16 ? 8 : 4;
    p.chunks = static_cast<int>((classes + p.vec - 1) / p.vec);
    p.wave = p.chunks <= 64 * 8;
    const int threads = p.wave ? 64 : kTeam;
    p.slices = p.wave ? 1 : (p.chunks + threads * 8 - 1) / (threads * 8);
    p.slice = (p.chunks + p.slices - 1) / p.slices;
    p.slices = (p.chunks + p.slice - 1) / p.slice;
    for (p.k = 1; p.k * threads < p.slice;) p.k *= 2;
    const int64_t bytes = p.slices * (sizeof(Part) + 8 * int64_t(top));
    p.batch = std::max<int64_t>(1, std::min<int64_t>(rows, (int64_t(64) << 20) / (p.slices == 1 ? 16 : bytes)));       // and at most 2^22 workgroups
    return p;
}

template <bool BF16, int VEC, int K, int TEAM> void launch_slices(const LogProbsArgs &a, const LogProbsPlan &p, Part *parts, uint64_t *lists, hipStream_t stream)
{
    const unsigned groups = static_cast<unsigned>(TEAM == 64 ? (a.rows + 3) / 4 : a.rows * p.slices);
    (a.top ? log_probs_slices_kernel<BF16, VEC, K, TEAM, true> : log_probs_slices_kernel<BF16, VEC, K, TEAM, false>)<<<groups, TEAM == 64 ? kThreads : TEAM, 0, stream>>>(a, p.slice, p.slices, parts,
                                                                                                                                                   lists);
}

template <bool BF16, int VEC, int K> void launch_narrow(const LogProbsArgs &a, hipStream_t stream)
{
    const unsigned groups = static_cast<unsigned>((a.rows + 15) / 16);
    (a.top ? log_probs_narrow_kernel<BF16, VEC, K, true> : log_probs_narrow_kernel<BF16, VEC, K, false>)<<<groups, kThreads, 0, stream>>>(a);
}

template <bool BF16> hipError_t launch(const LogProbsArgs &a, const LogProbsPlan &p, void *workspace, hipStream_t stream)
{
    constexpr int VEC = BF16 ? 8 : 4;
    Part *parts = static_cast<Part *>(workspace);
    uint64_t *lists = reinterpret_cast<uint64_t *>(parts + p.batch * p.slices);
    for (int64_t row = 0; row < a.rows; row += p.batch) {
        LogProbsArgs b = a;
        b.rows = std::min(p.batch, a.rows - row);
        b.logits = static_cast<const char *>(a.logits) + row * a.row_stride * (BF16 ? 2 : 4);
        if (b.tokens) b.tokens += row;
        if (b.logp) b.logp += row;
        if (b.entropy) b.entropy += row;
        if (b.top_index) b.top_index += row * a.top;
        if (b.top_logp) b.top_logp += row * a.top;
        if (b.largest) b.largest += row;
        if (b.log_sum) b.log_sum += row;
        if (p.vec == 1) launch_narrow<BF16, 1, 1>(b, stream);
        else if (p.chunks <= 16) launch_narrow<BF16, VEC, 1>(b, stream);
        else if (p.chunks <= 32) launch_narrow<BF16, VEC, 2>(b, stream);
        else if (!p.wave) launch_slices<BF16, VEC, 8, kTeam>(b, p, parts, lists, stream);
        else if (p.k == 1) launch_slices<BF16, VEC, 1, 64>(b, p, parts, lists, stream);
        else if (p.k == 2) launch_slices<BF16, VEC, 2, 64>(b, p, parts, lists, stream);
        else if (p.k == 4) launch_slices<BF16, VEC, 4, 64>(b, p, parts, lists, stream);
        else launch_slices<BF16, VEC, 8, 64>(b, p, parts, lists, stream);
        if (p.slices > 1) {
            const unsigned groups = static_cast<unsigned>(b.rows);
            const size_t lds = (kListsAtOnce + 2) * size_t(a.top) * 8;
            // a wavefront where there is little to do: as many rows at once as there are wavefronts
            if (int64_t(std::min(p.slices, kListsAtOnce) + 1) * a.top <= 128 && p.slices <= 64) log_probs_join_kernel<64><<<groups, 64, lds, stream>>>(b, p.slices, parts, lists);
            else log_probs_join_kernel<256><<<groups, 256, lds, stream>>>(b, p.slices, parts, lists);
        }
    }
    return hipGetLastError();
}

}  // namespace

size_t log_probs_bytes(int64_t rows, int64_t classes, bool bf16, int top)
{
    if (rows == 0) return 0;
    const LogProbsPlan p = plan_log_probs(rows, classes, bf16, top);
    return p.slices > 1 ? static_cast<size_t>(p.batch) * p.slices * (sizeof(Part) + 8 * size_t(top)) : 0;
}

hipError_t launch_log_probs(const LogProbsArgs &a, void *workspace, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const LogProbsPlan p = plan_log_probs(a.rows, a.classes, a.bf16, a.top);
    return a.bf16 ? launch<true>(a, p, workspace, stream) : launch<false>(a, p, workspace, stream);
}

hipError_t launch_log_probs_backward(const LogProbsGradArgs &a, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const int vec = a.classes < (a.bf16 ? 8 : 4) ? 1 : a.bf16 ? 8 : 4, whole = a.classes / vec;
    if (whole < kThreads) {
        const int per = whole + a.classes % vec;
        const unsigned grid = static_cast<unsigned>(std::min<int64_t>((a.rows * per + kThreads - 1) / kThreads, 1 << 20));
        if (vec == 1) (a.bf16 ? log_probs_narrow_gradient_kernel<true, 1> : log_probs_narrow_gradient_kernel<false, 1>)<<<grid, kThreads, 0, stream>>>(a, Divisor(per));
        else if (a.bf16) log_probs_narrow_gradient_kernel<true, 8><<<grid, kThreads, 0, stream>>>(a, Divisor(per));
        else log_probs_narrow_gradient_kernel<false, 4><<<grid, kThreads, 0, stream>>>(a, Divisor(per));
        return hipGetLastError();
    }
    constexpr int K = 4;
    const int tiles = (whole + kThreads * K - 1) / (kThreads * K);
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(a.rows * tiles, 1 << 20));
    if (a.bf16) log_probs_gradient_kernel<true, 8, K><<<grid, kThreads, 0, stream>>>(a, tiles);
    else log_probs_gradient_kernel<false, 4, K><<<grid, kThreads, 0, stream>>>(a, tiles);
    return hipGetLastError();
}

}  // namespace cr
