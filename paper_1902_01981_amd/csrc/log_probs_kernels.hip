// Log probabilities of tokens, entropy and the most probable alternatives, and the gradient of the first two, for gfx950.
//
// With c the largest x_j of a row (or of a part):  S = sum_j exp(x_j - c),  E = sum_j exp(x_j - c) (x_j - c);  l_j = x_j - c - log S,  entropy = log S - E / S.  Sums about two
// references meet by S exp(c - c') and (E + S (c - c')) exp(c - c').
// The alternatives: at least `top` values are no smaller than the top-th largest of the largest values of disjoint sets, so what is no smaller than that is
// all that can be among them, and few other than them; their order is that of numbers with the value above and the index's complement below, of which no two are equal.
//
//   log_probs_slices_kernel    a row, or a slice of it, in the registers of a wavefront or a workgroup, read once
//   log_probs_join_kernel      rows of several slices
//   log_probs_gradient_kernel  the gradient
#include "softmax_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr int kThreads = 256, kMostTop = 128;
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
// what is written of a row
__device__ __forceinline__ void write_row(const LogProbsArgs &a, int64_t row, const Part &p, float log2_S)
{
    if (a.logp) {
        const int64_t t = a.tokens[row];
        float logp = 0.f;
        if (t >= a.classes) {
            logp = __builtin_nanf("");
        } else if (t >= 0) {
            const float x = a.bf16 ? Element<true>::get(static_cast<const uint16_t *>(a.logits) + row * a.row_stride + t)
                                   : static_cast<const float *>(a.logits)[row * a.row_stride + t];
            logp = p.S == 0.f ? -infinity() : log_prob(x, p, log2_S);
        }
        a.logp[row] = logp;
    }
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
template <bool WAVE> struct Team {
    static constexpr int kSize = WAVE ? 64 : kThreads;
    static __device__ __forceinline__ void sync()
    {
        if constexpr (WAVE) {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        } else {
            __syncthreads();
        }
    }
    // the sum over the team of small numbers
    static __device__ __forceinline__ int total(int mine, float *meet)
    {
        float sum = lanes_total<64>(static_cast<float>(mine));
        if constexpr (!WAVE) {
            if (threadIdx.x % 64 == 0) meet[threadIdx.x / 64] = sum;
            __syncthreads();
            sum = meet[0] + meet[1] + meet[2] + meet[3];
            __syncthreads();
        }
        return static_cast<int>(sum);
    }
};

// The largest number of 16 bits that at least `top` of a wavefront's numbers reach, 0 if there are no so many above 0.
template <int N> __device__ __forceinline__ uint32_t reached(const uint32_t (&keys)[N], int top)
{
    uint32_t least = 0;
#pragma unroll 1
    for (int bit = 15; bit >= 0; --bit) {
        const uint32_t more = least | 1u << bit;
        int count = 0;
#pragma unroll
        for (int i = 0; i < N; ++i) count += __popcll(__ballot(keys[i] >= more));
        if (count >= top) least = more;
    }
    return least;
}
__device__ __forceinline__ uint32_t short_key(float x) { return x > -infinity() ? ordered(x) >> 16 : 0u; }       // 0 of -infinity and NaN

constexpr int kWaveEntries = 512, kBlockEntries = 1024;  // that a team keeps of those that may be among the largest

template <bool BF16, int VEC, int K, bool WAVE>
__global__ void __launch_bounds__(kThreads) log_probs_slices_kernel(LogProbsArgs a, int slice, int slices, Part *parts, uint64_t *lists)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    using Group = Team<WAVE>;
    constexpr int kTeams = kThreads / Group::kSize, kEntries = WAVE ? kWaveEntries : kBlockEntries;
    __shared__ uint64_t entries[kTeams][kEntries];
    __shared__ int counts[kTeams];
    __shared__ float meet[3][4];
    __shared__ uint32_t maxima[WAVE ? 1 : kThreads];
    __shared__ float bound;
    const int wave = threadIdx.x / 64, team = WAVE ? wave : 0, lane = threadIdx.x % Group::kSize;
    const int64_t unit = WAVE ? int64_t(blockIdx.x) * kTeams + team : int64_t(blockIdx.x);
    const int64_t row = WAVE ? unit : unit / slices;
    if (row >= a.rows) return;                           // whole teams; there is no barrier of the workgroup where a team is a wavefront
    const int nq = (a.classes + VEC - 1) / VEC, begin = WAVE ? 0 : static_cast<int>(unit - row * slices) * slice, end = min(begin + slice, nq);
    const int doubled = nq * VEC - a.classes;            // of the last chunk, which is moved back to end with the row
    const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;

    typename C::raw raw[K];
#pragma unroll
    for (int k = 0; k < K; ++k) raw[k] = C::load(x + chunk_at<VEC>(min(begin + lane + k * Group::kSize, end - 1), nq, a.classes));
    float v[VEC], most[K], c = -infinity();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        // what is no element of this place is a class that cannot be
        const int q = begin + lane + k * Group::kSize, none = q >= end ? VEC : q == nq - 1 ? doubled : 0;
        if (none) {
            C::widen(raw[k], v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = i < none ? -infinity() : v[i];
            raw[k] = C::narrow(v);
        }
        C::widen(raw[k], v);
        most[k] = v[0];
#pragma unroll
        for (int i = 1; i < VEC; ++i) most[k] = fmaxf(most[k], v[i]);
        c = fmaxf(c, most[k]);
    }
    const float own = c;                                 // the largest of this thread
    Part p = {own, 0.f, 0.f, 0.f};
    const float from = usable(own);
#pragma unroll
    for (int k = 0; k < K; ++k) {
        C::widen(raw[k], v);
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float d = v[i] - from, e = exp_fast(d);
            p.S += e;
            p.E = fmaf(e, bounded(d), p.E);
        }
    }
    join_lanes<64>(p);
    if constexpr (!WAVE) {
        if (threadIdx.x % 64 == 0) {
            meet[0][wave] = p.c;
            meet[1][wave] = p.S;
            meet[2][wave] = p.E;
        }
        __syncthreads();
        p = {meet[0][threadIdx.x % 4], meet[1][threadIdx.x % 4], meet[2][threadIdx.x % 4], 0.f};
        join_lanes<4>(p);
    }
    const float log2_S = __builtin_amdgcn_logf(p.S);                 // the hardware's logarithm is that to base 2
    const bool alone = WAVE || slices == 1;
    if (lane == 0) {
        if (alone) write_row(a, row, p, log2_S);
        else parts[unit] = p;
    }
    if (a.top == 0) return;

    float least;
    if constexpr (WAVE) {
        uint32_t keys[K];
#pragma unroll
        for (int k = 0; k < K; ++k) keys[k] = short_key(most[k]);
        const uint32_t key = reached(keys, a.top);
        least = key ? unordered(key << 16) : kLowest;
    } else {
        maxima[threadIdx.x] = short_key(own);
        __syncthreads();
        if (wave == 0) {
            uint32_t keys[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) keys[i] = maxima[threadIdx.x + 64 * i];
            const uint32_t key = reached(keys, a.top);
            if (threadIdx.x == 0) bound = key ? unordered(key << 16) : kLowest;
        }
    }
    uint64_t *list = entries[team];
    int *count = &counts[team];
    if (lane == 0) *count = 0;
    Group::sync();
    if constexpr (!WAVE) least = bound;
    if (own >= least) {
#pragma unroll
        for (int k = 0; k < K; ++k) {
            if (most[k] < least) continue;
            C::widen(raw[k], v);
            const int at = chunk_at<VEC>(min(begin + lane + k * Group::kSize, end - 1), nq, a.classes);
#pragma unroll
            for (int i = 0; i < VEC; ++i)
                if (v[i] >= least) {
                    const int to = atomicAdd(count, 1);
                    if (to < kEntries) list[to] = entry_of(v[i], at + i);
                }
        }
    }
    Group::sync();
    int n = *count;
    if (n > kEntries) {
        // Too many, equal ones mostly: the top-th largest value itself, bit by bit, then as many of its places as are wanted, lowest first.
        auto number = [&](auto &&counts_if) {
            int mine = 0;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                C::widen(raw[k], v);
                const int at = chunk_at<VEC>(min(begin + lane + k * Group::kSize, end - 1), nq, a.classes);
#pragma unroll
                for (int i = 0; i < VEC; ++i) mine += v[i] > -infinity() && counts_if(ordered(v[i]), at + i);
            }
            return Group::total(mine, meet[0]);
        };
        Group::sync();
        uint32_t value = 0;
        for (int bit = 31; bit >= 0; --bit) {
            const uint32_t more = value | 1u << bit;
            if (number([&](uint32_t o, int) { return o >= more; }) >= a.top) value = more;
        }
        const int wanted = a.top - number([&](uint32_t o, int) { return o > value; });
        int behind = 0;                                  // the largest index before which there are fewer places than wanted
        for (int bit = 28; bit >= 0; --bit) {
            const int more = behind | 1 << bit;
            if (more <= a.classes && number([&](uint32_t o, int index) { return o == value && index < more; }) < wanted) behind = more;
        }
        if (lane == 0) *count = 0;
        Group::sync();
#pragma unroll
        for (int k = 0; k < K; ++k) {
            C::widen(raw[k], v);
            const int at = chunk_at<VEC>(min(begin + lane + k * Group::kSize, end - 1), nq, a.classes);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
                const uint32_t o = ordered(v[i]);
                if (v[i] > -infinity() && (o > value || (o == value && at + i <= behind))) {
                    const int to = atomicAdd(count, 1);
                    if (to < kEntries) list[to] = entry_of(v[i], at + i);
                }
            }
        }
        Group::sync();
        n = min(*count, kEntries);
    }
    auto leave = [&](int place, uint64_t entry) {
        if (alone) write_entry(a, row, place, entry, p, log2_S);
        else lists[unit * a.top + place] = entry;
    };
    for (int i = lane; i < n; i += Group::kSize) {
        const uint64_t entry = list[i];
        int place = 0;
        for (int j = 0; j < n; ++j) place += list[j] > entry;
        if (place < a.top) leave(place, entry);
    }
    for (int place = n + lane; place < a.top; place += Group::kSize) leave(place, 0);
}

// A row's slices: their sums, and the largest of their lists, a few lists at a time beside those found so far.  A number's place is the number of larger ones in
// every list, each of which is in order.
constexpr int kListsAtOnce = 8;
__global__ void __launch_bounds__(kThreads) log_probs_join_kernel(LogProbsArgs a, int slices, const Part *parts, const uint64_t *lists)
{
    __shared__ uint64_t some[kListsAtOnce + 1][kMostTop], best[kMostTop];
    __shared__ float meet[3][4];
    const int64_t row = blockIdx.x;
    Part p = {-infinity(), 0.f, 0.f, 0.f};
    for (int i = threadIdx.x; i < slices; i += kThreads) p = joined(p, parts[row * slices + i]);
    join_lanes<64>(p);
    if (threadIdx.x % 64 == 0) {
        meet[0][threadIdx.x / 64] = p.c;
        meet[1][threadIdx.x / 64] = p.S;
        meet[2][threadIdx.x / 64] = p.E;
    }
    __syncthreads();
    p = {meet[0][threadIdx.x % 4], meet[1][threadIdx.x % 4], meet[2][threadIdx.x % 4], 0.f};
    join_lanes<4>(p);
    const float log2_S = __builtin_amdgcn_logf(p.S);                 // the hardware's logarithm is that to base 2
    if (threadIdx.x == 0) write_row(a, row, p, log2_S);
    const int top = a.top;
    if (top == 0) return;
    if (threadIdx.x < top) best[threadIdx.x] = 0;
    for (int first = 0; first < slices; first += kListsAtOnce) {
        const int now = min(kListsAtOnce, slices - first);
        __syncthreads();
        for (int i = threadIdx.x; i < now * top; i += kThreads) some[1 + i / top][i % top] = lists[(row * slices + first) * top + i];
        if (threadIdx.x < top) {
            some[0][threadIdx.x] = best[threadIdx.x];
            best[threadIdx.x] = 0;
        }
        __syncthreads();
        for (int i = threadIdx.x; i < (now + 1) * top; i += kThreads) {
            const int mine = i / top;
            int place = i % top;
            const uint64_t entry = some[mine][place];
            if (!entry) continue;
            for (int other = 0; other <= now; ++other) {
                if (other == mine) continue;
                int lo = 0, hi = top;                    // entries before lo are larger, from hi on they are not
                while (lo < hi) {
                    const int mid = (lo + hi) / 2;
                    if (some[other][mid] > entry) lo = mid + 1;
                    else hi = mid;
                }
                place += lo;
            }
            if (place < top) best[place] = entry;
        }
    }
    __syncthreads();
    if (threadIdx.x < top) write_entry(a, row, threadIdx.x, best[threadIdx.x], p, log2_S);
}

// dx_j = a ([j = t] - p_j) - b p_j (l_j + entropy); a thread has K chunks of a row, and an element of those behind the whole chunks.
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
        const float c = a.largest[row], L = a.log_sum[row];
        const int64_t t = a.tokens ? a.tokens[row] : -1;
        const float by_logp = t >= 0 ? a.dlogp[row] : 0.f, by_entropy = a.entropy ? a.dentropy[row] : 0.f, H = a.entropy ? a.entropy[row] : 0.f;
        const bool flat = t >= a.classes || c == -infinity();
        const float value = t >= a.classes ? __builtin_nanf("") : 0.f;
        auto form = [&](float xi, int j) {
            const float l = xi - c - L, p = exp_fast(l);
            const float g = -p * (by_logp + by_entropy * (H + fmaxf(l, -256.f)));          // p is 0 there already
            return flat ? value : j == t ? g + by_logp : g;
        };
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int q = (tile * K + k) * kThreads + threadIdx.x;
            if (q < whole) {
                float v[VEC];
                C::widen(C::load(x + q * VEC), v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = form(v[i], q * VEC + i);
                C::store(dx + q * VEC, C::narrow(v));
            }
        }
        if (tile == 0 && threadIdx.x < left) {
            const int j = whole * VEC + threadIdx.x;
            Element<BF16>::put(dx + j, form(Element<BF16>::get(x + j), j));
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
    const int threads = p.wave ? 64 : kThreads;
    p.slices = p.wave ? 1 : (p.chunks + threads * 8 - 1) / (threads * 8);
    p.slice = (p.chunks + p.slices - 1) / p.slices;
    p.slices = (p.chunks + p.slice - 1) / p.slice;
    for (p.k = 1; p.k * threads < p.slice;) p.k *= 2;
    const int64_t bytes = p.slices * (sizeof(Part) + 8 * int64_t(top));
    p.batch = std::max<int64_t>(1, std::min<int64_t>(rows, (int64_t(64) << 20) / (p.slices == 1 ? 16 : bytes)));       // and at most 2^22 workgroups
    return p;
}

template <bool BF16, int VEC, int K, bool WAVE> void launch_slices(const LogProbsArgs &a, const LogProbsPlan &p, Part *parts, uint64_t *lists, hipStream_t stream)
{
    const int64_t groups = WAVE ? (a.rows + 3) / 4 : a.rows * p.slices;
    log_probs_slices_kernel<BF16, VEC, K, WAVE><<<static_cast<unsigned>(groups), kThreads, 0, stream>>>(a, p.slice, p.slices, parts, lists);
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
        if (p.vec == 1) launch_slices<BF16, 1, 1, true>(b, p, parts, lists, stream);
        else if (!p.wave) launch_slices<BF16, VEC, 8, false>(b, p, parts, lists, stream);
        else if (p.k == 1) launch_slices<BF16, VEC, 1, true>(b, p, parts, lists, stream);
        else if (p.k == 2) launch_slices<BF16, VEC, 2, true>(b, p, parts, lists, stream);
        else if (p.k == 4) launch_slices<BF16, VEC, 4, true>(b, p, parts, lists, stream);
        else launch_slices<BF16, VEC, 8, true>(b, p, parts, lists, stream);
        if (p.slices > 1) log_probs_join_kernel<<<static_cast<unsigned>(b.rows), kThreads, 0, stream>>>(b, p.slices, parts, lists);
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
    const int vec = a.classes < (a.bf16 ? 8 : 4) ? 1 : a.bf16 ? 8 : 4;
    constexpr int K = 4;
    const int tiles = std::max(1, (a.classes / vec + kThreads * K - 1) / (kThreads * K));
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(a.rows * tiles, 1 << 20));
    if (vec == 1) (a.bf16 ? log_probs_gradient_kernel<true, 1, K> : log_probs_gradient_kernel<false, 1, K>)<<<grid, kThreads, 0, stream>>>(a, tiles);
    else if (a.bf16) log_probs_gradient_kernel<true, 8, K><<<grid, kThreads, 0, stream>>>(a, tiles);
    else log_probs_gradient_kernel<false, 4, K><<<grid, kThreads, 0, stream>>>(a, tiles);
    return hipGetLastError();
}

}  // namespace cr
