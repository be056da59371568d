// The loss of a student's logits against a teacher's largest ones, and its gradient, for gfx950.
//
// With q the teacher's shares at temperature T, about their largest logit, and c, S as of the softmax loss with exp(x / T) in place of exp(x):
//     loss = w T sum_i q_i ((z_i - largest z) - (x_(j_i) - c) + T (log S - log S_q)),   dx_j = w T (exp((x_j - c) / T) / S - sum_(j_i = j) q_i).
//
//   distill_narrow_kernel  four rows in a wavefront
//   distill_wave_kernel    a row in the registers of a wavefront
//   distill_rows_kernel    a row in the registers of a workgroup, read once; a wavefront of its own reads the teacher's entries, forms the loss and puts the
//                          teacher's classes into the gradient
//   distill_slices_kernel, distill_join_kernel   rows wider than that: a row cut into slices, read twice with the gradient
//
// Reads and writes bound it: 8 192 x 131 071 bf16 with 20 entries 933 us, 4.6 TB/s (the loss of one target 908); 4 099 x 50 008 bf16 with five 167 us, with 64
// 179, 4.6 TB/s, fp32 351, 4.7 TB/s; without the gradient 74 and, 8 192 x 131 071, 436 us, 4.9 TB/s.  Slices: 2 048 x 128 000 fp32 188 us without the gradient, 5.6 TB/s, 705 with it, 4.5 TB/s
// of what moves; 8 192 x 152 064 bf16 1.65 ms.  100 000 x 100 bf16 with 20 33 us, 1.2 TB/s: the entries, all of which every lane goes through.
#include "softmax_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr int kMostTop = 128, kEntries = kMostTop / 64;  // entries of a lane

__device__ __forceinline__ float first_lane(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }
__device__ __forceinline__ float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

// What a wavefront knows of a row's teacher: entries lane and lane + 64.
struct Teacher {
    int index[kEntries];         // -1: not there
    float q[kEntries];           // shares
    float d[kEntries];           // distances from the largest logit
    float at[kEntries];          // the student's logits there
    bool any, unknown;           // entries at all; one of no class
    float sum;                   // of exp(d / T): NaN where there is no sense in it
    float w;
};
// A row's entries as they are given.
struct Entries {
    int64_t index[kEntries];
    float z[kEntries], w;
};
__device__ __forceinline__ void read_entries(Entries &n, const DistillArgs &a, int64_t row)
{
    n.w = a.weights ? a.weights[row] : 1.f;
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
        const int i = threadIdx.x % 64 + 64 * e;
        n.index[e] = -1;
        n.z[e] = -infinity();
        if (i < a.top) {
            n.index[e] = a.top_index[row * a.top_row_stride + i];
            n.z[e] = a.top_logits[row * a.top_row_stride + i];
        }
    }
}
// All of it but the student's logits; their places.
__device__ __forceinline__ void settle(Teacher &t, const Entries &n, const DistillArgs &a, float unit)
{
    float z[kEntries], most = -infinity();
    bool there = false, unknown = false;
    t.w = n.w;
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
        const bool is = n.index[e] >= 0 && n.z[e] != -infinity(), known = is && n.index[e] < a.classes;
        z[e] = is ? n.z[e] : -infinity();
        t.index[e] = known ? static_cast<int>(n.index[e]) : -1;
        there |= is;
        unknown |= is && !known;
        most = fmaxf(most, z[e]);
    }
    most = lanes_most<64>(most);
    t.any = __ballot(there) != 0;
    t.unknown = __ballot(unknown) != 0;
    const float from = usable(most);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
        t.d[e] = z[e] - from;
        t.q[e] = exp_fast(t.d[e], unit);
        sum += t.q[e];
    }
    t.sum = lanes_total<64>(sum);
    const float by = 1.f / t.sum;
#pragma unroll
    for (int e = 0; e < kEntries; ++e) t.q[e] *= by;
}
template <bool BF16> __device__ __forceinline__ void read_logits(float (&at)[kEntries], const Entries &n, const DistillArgs &a, int64_t row)
{
    const auto *x = static_cast<const typename Element<BF16>::type *>(a.logits) + row * a.row_stride;
#pragma unroll
    for (int e = 0; e < kEntries; ++e) at[e] = Element<BF16>::get(x + (n.index[e] >= 0 && n.index[e] < a.classes ? n.index[e] : 0));
}
// what a row's gradient is, but for the shares
enum Kind : int { kShares, kZero, kNan };
__device__ __forceinline__ Kind kind_of(const Teacher &t) { return !t.any ? kZero : t.unknown || !(t.sum == t.sum) ? kNan : kShares; }

// The loss, for every lane.
__device__ __forceinline__ float loss_of(const Teacher &t, const DistillArgs &a, const Softmax &s)
{
    // Not distances over T, and a fourth of each: they, and sums of them, could be infinite where the loss is not (masks of the type's lowest value).
    const float from = usable(s.c), both = 0.25f * a.temperature * kLn2 * (__builtin_amdgcn_logf(s.S) - __builtin_amdgcn_logf(t.sum));
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
        const float term = t.q[e] * (0.25f * t.d[e] - (0.25f * t.at[e] - 0.25f * from) + both);
        sum += t.index[e] >= 0 && t.q[e] != 0.f ? term : 0.f;
    }
    sum = lanes_total<64>(sum);
    return !t.any ? 0.f : 4.f * (t.w * a.temperature * (t.unknown ? __builtin_nanf("") : s.S == 0.f ? infinity() * t.sum : sum));
}
// The gradient at the teacher's classes: an index that comes several times has the same bits from each of its entries.  Which do is found by a table of the last
// entry in each of its places; going through all entries for each took the teacher's wavefront 2 us a row of 64 (4 099 x 50 008 bf16 184 us).
constexpr int kSlots = 4096;
__device__ __forceinline__ void at_entries(float (&value)[kEntries], const Teacher &t, const DistillArgs &a, const Softmax &s, float unit, float factor, uint8_t *slots)
{
    const int lane = threadIdx.x % 64;
    float q[kEntries];
    bool met[kEntries];
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
        q[e] = t.q[e];
        if (t.index[e] >= 0) slots[t.index[e] % kSlots] = static_cast<uint8_t>(lane + 64 * e);
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < kEntries; ++e) met[e] = t.index[e] >= 0 && slots[t.index[e] % kSlots] != lane + 64 * e;
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
        uint64_t left = __ballot(met[e]);
        while (left) {
            const int index = __builtin_amdgcn_readlane(t.index[e], __builtin_ctzll(left));
            float total = 0.f;                           // of all entries with this index, in their order
#pragma unroll
            for (int f = 0; f < kEntries; ++f)
                for (uint64_t same = __ballot(t.index[f] == index); same; same &= same - 1) total += lane_of(t.q[f], __builtin_ctzll(same));
#pragma unroll
            for (int f = 0; f < kEntries; ++f) q[f] = t.index[f] == index ? total : q[f];
            left &= ~__ballot(t.index[e] == index);
        }
    }
    const float from = usable(s.c);
#pragma unroll
    for (int e = 0; e < kEntries; ++e) value[e] = fmaf(exp_fast(t.at[e] - from, unit), factor, -(t.w * a.temperature * q[e]));
}

// ---- sixteen lanes' rows ---------------------------------------------------------------------------------------------------------
// Rows of up to 16 chunks, four beside each other in a wavefront.  (A wavefront per row took 100 000 x 100 bf16 with 20 entries 59 us: its instructions,
// whatever the row has.)  Every lane goes through all entries and adds up the shares of those that are in its own chunk, so that nothing follows the gradient.
template <bool BF16, int VEC, bool GRAD> __global__ void __launch_bounds__(256) distill_narrow_kernel(DistillArgs a)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    constexpr int kLanes = 16, kTeams = 256 / kLanes, kOwn = kMostTop / kLanes;
    __shared__ int indices[GRAD ? kTeams : 1][GRAD ? kMostTop + 1 : 1];            // teams begin in other banks
    __shared__ float shares[GRAD ? kTeams : 1][GRAD ? kMostTop + 1 : 1];
    const int lane = threadIdx.x % kLanes, team = threadIdx.x / kLanes;
    const int64_t own_row = int64_t(blockIdx.x) * kTeams + team, row = std::min(own_row, a.rows - 1);
    const bool here = own_row < a.rows;                  // the others go along
    const int nq = (a.classes + VEC - 1) / VEC, doubled = nq * VEC - a.classes, at = chunk_at<VEC>(min(lane, nq - 1), nq, a.classes);
    const float unit = kLog2e / a.temperature, nan = __builtin_nanf("");
    const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
    const typename C::raw raw = C::load(x + at);
    const float w = a.weights ? a.weights[row] : 1.f;
    int index[kOwn];
    float z[kOwn], logit[kOwn], most = -infinity();
    bool there = false, unknown = false;
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        index[e] = -1;
        z[e] = -infinity();
        logit[e] = 0.f;
        const int i = lane + kLanes * e;
        if (kLanes * e >= a.top) continue;
        if (i < a.top) {
            const int64_t given = a.top_index[row * a.top_row_stride + i];
            const float zi = a.top_logits[row * a.top_row_stride + i];
            const bool is = given >= 0 && zi != -infinity(), known = is && given < a.classes;
            there |= is;
            unknown |= is && !known;
            if (is) z[e] = zi;
            if (known) {
                index[e] = static_cast<int>(given);
                logit[e] = Element<BF16>::get(x + given);
            }
        }
        most = fmaxf(most, z[e]);
    }
    most = lanes_most<kLanes>(most);
    const uint32_t flags = static_cast<uint32_t>(__ballot(there) >> (threadIdx.x % 64 / kLanes * kLanes)) & 0xffffu;
    const uint32_t unknowns = static_cast<uint32_t>(__ballot(unknown) >> (threadIdx.x % 64 / kLanes * kLanes)) & 0xffffu;
    const float from_z = usable(most);
    float q[kOwn], sum_q = 0.f;
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        if (kLanes * e >= a.top) continue;
        q[e] = exp_fast(z[e] - from_z, unit);
        sum_q += q[e];
    }
    sum_q = lanes_total<kLanes>(sum_q);
    const float by = 1.f / sum_q;
    float v[VEC];
    C::widen(raw, v);
    Softmax s;
    float counted[VEC];
#pragma unroll
    for (int i = 0; i < VEC; ++i) counted[i] = lane >= nq || (lane == nq - 1 && i < doubled) ? -infinity() : v[i];
    take<VEC>(s, counted, true, unit);
    const float c = lanes_most<kLanes>(s.c), from = usable(c);
    float S = s.S * exp_fast(s.c - from, unit);
    hold(S);                                             // rounded here: taken into an addition it would give every lane another sum
    S = lanes_total<kLanes>(S);
    const float both = 0.25f * a.temperature * kLn2 * (__builtin_amdgcn_logf(S) - __builtin_amdgcn_logf(sum_q));
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < kOwn; ++e) {
        if (kLanes * e >= a.top) continue;
        q[e] *= by;
        const float term = q[e] * (0.25f * (z[e] - from_z) - (0.25f * logit[e] - 0.25f * from) + both);
        sum += index[e] >= 0 && q[e] != 0.f ? term : 0.f;
        if constexpr (GRAD) {
            indices[team][lane + kLanes * e] = index[e];
            shares[team][lane + kLanes * e] = q[e];
        }
    }
    sum = lanes_total<kLanes>(sum);
    if (lane == 0 && here) a.loss[row] = !flags ? 0.f : 4.f * (w * a.temperature * (unknowns ? nan : S == 0.f ? infinity() * sum_q : sum));
    if constexpr (GRAD) {
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const Kind kind = !flags ? kZero : unknowns || !(sum_q == sum_q) ? kNan : kShares;
        const bool flat = kind != kShares || S == 0.f;
        const float value = kind == kNan ? nan : 0.f, factor = w * a.temperature / S;
        float taken[VEC];                                // of the teacher's shares, by this chunk's classes
#pragma unroll
        for (int i = 0; i < VEC; ++i) taken[i] = 0.f;
        for (int e = 0; e < a.top; ++e) {
            const int place = indices[team][e] - at;
            const float share = shares[team][e];
#pragma unroll
            for (int i = 0; i < VEC; ++i) taken[i] += place == i ? share : 0.f;
        }
        if (!here || lane >= nq) return;
#pragma unroll
        for (int i = 0; i < VEC; ++i) {
            const float share = exp_fast(v[i] - from, unit);
            v[i] = flat ? value : taken[i] == 0.f ? share * factor : fmaf(share, factor, -(w * a.temperature * taken[i]));
        }
        C::store(static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride + at, C::narrow(v));
    }
}

// ---- a wavefront's rows ----------------------------------------------------------------------------------------------------------
// A lane has K chunks; the last chunk of a row is moved back to end with it, where it has elements twice: they count once and are stored twice, the same bits.
template <bool BF16, int VEC, int K, bool GRAD> __global__ void __launch_bounds__(256) distill_wave_kernel(DistillArgs a)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    __shared__ uint8_t slots[GRAD ? 4 : 1][GRAD ? kSlots : 1];
    const int lane = threadIdx.x % 64, nq = (a.classes + VEC - 1) / VEC, doubled = nq * VEC - a.classes;
    const float unit = kLog2e / a.temperature;
    for (int64_t row = int64_t(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x / 64); row < a.rows; row += int64_t(gridDim.x) * 4) {
        const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
        typename C::raw raw[K];
#pragma unroll
        for (int k = 0; k < K; ++k) raw[k] = C::load(x + chunk_at<VEC>(min(lane + 64 * k, nq - 1), nq, a.classes));
        Entries entries;
        Teacher teacher;
        read_entries(entries, a, row);
        read_logits<BF16>(teacher.at, entries, a, row);
        settle(teacher, entries, a, unit);
        Softmax s;
        float v[VEC];
#pragma unroll
        for (int k = 0; k < K; ++k) {
            const int q = lane + 64 * k;
            C::widen(raw[k], v);
            if (q == nq - 1) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = i < doubled ? -infinity() : v[i];
            }
            take<VEC>(s, v, q < nq, unit);
        }
        join_lanes<64>(s, unit);
        s.c = first_lane(s.c);                           // the lanes' sums may differ by a rounding
        s.S = first_lane(s.S);
        const float loss = loss_of(teacher, a, s);
        if (lane == 0) a.loss[row] = loss;
        if constexpr (GRAD) {
            T *dx = static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride;
            const Kind kind = kind_of(teacher);
            const bool flat = kind != kShares || s.S == 0.f;
            const float value = kind == kNan ? __builtin_nanf("") : 0.f, from = usable(s.c), factor = teacher.w * a.temperature / s.S;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                const int q = lane + 64 * k;
                if (q >= nq) break;
                hold(raw[k]);                            // widened again rather than kept wide since the sum
                C::widen(raw[k], v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = flat ? value : exp_fast(v[i] - from, unit) * factor;
                C::store(dx + chunk_at<VEC>(q, nq, a.classes), C::narrow(v));
            }
            if (!flat) {
                float put[kEntries];
                at_entries(put, teacher, a, s, unit, factor, slots[threadIdx.x / 64]);
                // behind the shares of the same places
                __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "workgroup");
                __builtin_amdgcn_wave_barrier();
#pragma unroll
                for (int e = 0; e < kEntries; ++e)
                    if (teacher.index[e] >= 0) Element<BF16>::put(dx + teacher.index[e], put[e]);
            }
        }
    }
}

// ---- a workgroup's rows ----------------------------------------------------------------------------------------------------------
// All wavefronts but the last have chunks of the row, K a lane, lanes = ceil(whole / K) of them: as they were read, added to the running sum as they arrive, and
// as soon as a chunk's gradient is stored its place takes the chunk of the workgroup's next row.  Whoever has no chunk at a place forms the last
// whole one again, with the same bits, and does not count it.  The last wavefront has the elements behind the whole chunks, and the teacher: its entries' loads
// depend on each other, and a wait for them would be a wait for all chunks in flight.  A row's barrier has the parts of its sums on one side and the
// shares on the other; the teacher's classes follow behind the next one, when all shares have been stored.
constexpr int kMostWaves = 16;
template <bool BF16, int K, bool GRAD> __global__ void __launch_bounds__(64 * kMostWaves) distill_rows_kernel(DistillArgs a, int lanes)
{
    constexpr int VEC = BF16 ? 8 : 4;
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    constexpr unsigned kBytes = VEC * sizeof(T);
    __shared__ float meet[2][2][kMostWaves];
    __shared__ int kinds[2];
    __shared__ float weights[2];
    __shared__ uint8_t slots[GRAD ? kSlots : 1];
    const int waves = blockDim.x / 64, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
    const int whole = a.classes / VEC, left = a.classes % VEC;
    const float unit = kLog2e / a.temperature;
    int turn = 0;                                        // two places in turn: one barrier a row
    auto meet_all = [&](Softmax &s) {
        join_lanes<64>(s, unit);
        if (threadIdx.x % 64 == 0) {
            meet[turn][0][wave] = s.c;
            meet[turn][1][wave] = s.S;
        }
        __syncthreads();
        s = Softmax();
        if (threadIdx.x % 16 < waves) {
            s.c = meet[turn][0][threadIdx.x % 16];
            s.S = meet[turn][1][threadIdx.x % 16];
        }
        join_lanes<16>(s, unit);
        s.c = first_lane(s.c);                           // scalars, and the same for all: the lanes' sums may differ by a rounding
        s.S = first_lane(s.S);
    };
    const int64_t stride = gridDim.x;
    int64_t row = blockIdx.x;
    if (row >= a.rows) return;                           // the whole workgroup

    if (wave == waves - 1) {
        const int lane = threadIdx.x % 64, edge_at = whole * VEC + min(lane, max(left - 1, 0));
        const bool has_edge = lane < left;
        int64_t last = -1;                               // the row before, whose classes are still to be put there
        int places[kEntries];
        float put[kEntries];
        auto follow = [&] {
            if (last < 0) return;
            T *dx = static_cast<T *>(a.dlogits) + last * a.dlogits_row_stride;
#pragma unroll
            for (int e = 0; e < kEntries; ++e)
                if (places[e] >= 0) Element<BF16>::put(dx + places[e], put[e]);
        };
        // entries are read a row ahead, and the logits that they point at before this row's own work
        Entries entries;
        Teacher teacher;
        float next_edge;
        auto read_next = [&](int64_t of) {
            read_logits<BF16>(teacher.at, entries, a, of);
            next_edge = Element<BF16>::get(static_cast<const T *>(a.logits) + of * a.row_stride + min(edge_at, a.classes - 1));
        };
        read_entries(entries, a, row);
        read_next(row);
        for (; row < a.rows; row += stride) {
            const int64_t next = std::min(row + stride, a.rows - 1);
            settle(teacher, entries, a, unit);
            const float edge = next_edge;
            const float edges[1] = {edge};
            read_entries(entries, a, next);
            Softmax s;
            take<1>(s, edges, has_edge, unit);
            const Kind kind = kind_of(teacher);
            if (lane == 0) {
                kinds[turn] = kind;
                weights[turn] = teacher.w;
            }
            meet_all(s);
            turn ^= 1;
            const Teacher now = teacher;
            if (row + stride < a.rows) read_next(next);
            const float loss = loss_of(now, a, s);
            if (lane == 0) a.loss[row] = loss;
            if constexpr (GRAD) {
                follow();
                const bool flat = kind != kShares || s.S == 0.f;
                const float factor = now.w * a.temperature / s.S;
                if (has_edge) {
                    const float value = kind == kNan ? __builtin_nanf("") : 0.f;
                    Element<BF16>::put(static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride + edge_at, flat ? value : exp_fast(edge - usable(s.c), unit) * factor);
                }
                last = flat ? -1 : row;
                if (!flat) at_entries(put, now, a, s, unit, factor, slots);
#pragma unroll
                for (int e = 0; e < kEntries; ++e) places[e] = now.index[e];
            }
        }
        if constexpr (GRAD) {
            __syncthreads();
            follow();
        }
        return;
    }

    const int tl = min(static_cast<int>(threadIdx.x), lanes - 1);
    auto row_at = [&](int64_t of) { return static_cast<const T *>(a.logits) + std::min(of, a.rows - 1) * a.row_stride; };
    typename C::raw raw[K];
    const unsigned lane_byte = tl * kBytes;
    const unsigned last_byte = min(tl + (K - 1) * lanes, whole - 1) * kBytes;
    auto chunk = [&](auto *x, int k) {                   // a scalar address and the lane's offset
        using P = std::remove_pointer_t<decltype(x)>;
        auto *bytes = reinterpret_cast<std::conditional_t<std::is_const_v<P>, const char, char> *>(x);
        if (k < K - 1) return reinterpret_cast<P *>(scalar(bytes + static_cast<unsigned>(k * lanes) * kBytes) + lane_byte);
        return reinterpret_cast<P *>(scalar(bytes) + last_byte);
    };
    auto fetch = [&](int k, const T *x) { raw[k] = GRAD ? C::load(chunk(x, k)) : C::load_once(chunk(x, k)); };
    Softmax s;
    auto add = [&](int k) {
        float x[VEC];
        C::widen(raw[k], x);
        take<VEC>(s, x, k < K - 1 || static_cast<int>(threadIdx.x) + k * lanes < whole, unit);
    };
    auto settle = [&] {
        if (static_cast<int>(threadIdx.x) >= lanes) s = Softmax();     // had the chunks of the last lane that has any
    };
    // the gradient of a row, each chunk making place for one of the row at x
    auto form = [&](int64_t of, Kind kind, float w, auto more, const T *x) {
        T *dx = static_cast<T *>(a.dlogits) + of * a.dlogits_row_stride;
        const float from = usable(s.c), factor = w * a.temperature / s.S;
        float v[VEC];
        if (kind != kShares || s.S == 0.f) {
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = kind == kNan ? __builtin_nanf("") : 0.f;
#pragma unroll
            for (int k = 0; k < K; ++k) {
                C::store(chunk(dx, k), C::narrow(v));
                if (more()) fetch(k, x);
            }
        } else {
#pragma unroll
            for (int k = 0; k < K; ++k) {
                hold(raw[k]);                            // widened again rather than kept wide since the sum
                C::widen(raw[k], v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = exp_fast(v[i] - from, unit) * factor;
                C::store(chunk(dx, k), C::narrow(v));
                if (more()) fetch(k, x);
            }
        }
    };

    const T *x = row_at(row);
#pragma unroll
    for (int k = 0; k < K; ++k) fetch(k, x);
    if constexpr (GRAD) {
        auto step = [&](auto more) {
#pragma unroll
            for (int k = 0; k < K; ++k) add(k);
            settle();
            meet_all(s);
            const Kind kind = static_cast<Kind>(__builtin_amdgcn_readfirstlane(kinds[turn]));
            const float w = first_lane(weights[turn]);
            turn ^= 1;
            form(row, kind, w, more, row_at(row + stride));
            s = Softmax();
        };
        for (; row + stride < a.rows; row += stride) step(std::true_type());
        step(std::false_type());
        __syncthreads();
    } else {
        for (; row < a.rows; row += stride) {
            x = row_at(row + stride);                    // past the last row: that row once more, from the caches
            s = Softmax();
#pragma unroll
            for (int k = 0; k < K; ++k) {
                add(k);
                fetch(k, x);
            }
            settle();
            meet_all(s);
            turn ^= 1;
        }
    }
}

// ---- a row in slices -------------------------------------------------------------------------------------------------------------
constexpr int kSliceThreads = 256, kSliceChunks = 8;     // chunks that a thread has in flight
__device__ __forceinline__ void join_block(Softmax &s, float (&lds)[2][kSliceThreads / 64], float unit)
{
    join_lanes<64>(s, unit);
    if (threadIdx.x % 64 == 0) {
        lds[0][threadIdx.x / 64] = s.c;
        lds[1][threadIdx.x / 64] = s.S;
    }
    __syncthreads();
    s.c = lds[0][threadIdx.x % (kSliceThreads / 64)];
    s.S = lds[1][threadIdx.x % (kSliceThreads / 64)];
    join_lanes<kSliceThreads / 64>(s, unit);
    s.c = first_lane(s.c);
    s.S = first_lane(s.S);
}

// parts[row of the batch][slice] = (c, S).  The logits at the teacher's classes go to at[row][entry]: in the next kernel the gradient may have replaced them.
template <bool BF16, int VEC> __global__ void __launch_bounds__(kSliceThreads) distill_slices_kernel(DistillArgs a, int slice, f2 *parts, float *at)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    __shared__ float lds[2][kSliceThreads / 64];
    const int nq = (a.classes + VEC - 1) / VEC, begin = blockIdx.x * slice, end = min(begin + slice, nq), doubled = nq * VEC - a.classes;
    const int64_t row = blockIdx.y;
    const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
    const float unit = kLog2e / a.temperature;
    if (blockIdx.x == 0 && static_cast<int>(threadIdx.x) < a.top) {
        const int64_t index = a.top_index[row * a.top_row_stride + threadIdx.x];
        at[row * a.top + threadIdx.x] = Element<BF16>::get(x + (index >= 0 && index < a.classes ? index : 0));
    }
    Softmax s;
    for (int q0 = begin + threadIdx.x; q0 < end; q0 += kSliceThreads * kSliceChunks) {
        typename C::raw raw[kSliceChunks];
#pragma unroll
        for (int k = 0; k < kSliceChunks; ++k) raw[k] = C::load(x + chunk_at<VEC>(min(q0 + k * kSliceThreads, end - 1), nq, a.classes));
#pragma unroll
        for (int k = 0; k < kSliceChunks; ++k) {
            const int q = q0 + k * kSliceThreads;
            float v[VEC];
            C::widen(raw[k], v);
            if (q == nq - 1) {
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = i < doubled ? -infinity() : v[i];
            }
            take<VEC>(s, v, q < end, unit);
        }
    }
    join_block(s, lds, unit);
    if (threadIdx.x == 0) parts[row * gridDim.x + blockIdx.x] = f2{s.c, s.S};
}
// Joins a row's slices, every workgroup for itself, and forms the gradient of its own slice.
template <bool BF16, int VEC, bool GRAD>
__global__ void __launch_bounds__(kSliceThreads) distill_join_kernel(DistillArgs a, int slice, int slices, const f2 *parts, const float *at)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    __shared__ float lds[2][kSliceThreads / 64];
    __shared__ uint8_t slots[GRAD ? kSlots : 1];
    const int64_t row = blockIdx.y;
    const int lane = threadIdx.x % 64;
    const float unit = kLog2e / a.temperature;
    Entries entries;
    Teacher teacher;
    read_entries(entries, a, row);
    settle(teacher, entries, a, unit);
#pragma unroll
    for (int e = 0; e < kEntries; ++e) teacher.at[e] = at[row * a.top + min(lane + 64 * e, a.top - 1)];
    Softmax s;
    for (int i = threadIdx.x; i < slices; i += kSliceThreads) {
        const f2 p = parts[row * slices + i];
        const float c = fmaxf(s.c, p.x), from = usable(c);
        s.S = s.S * exp_fast(s.c - from, unit) + p.y * exp_fast(p.x - from, unit);
        s.c = c;
    }
    join_block(s, lds, unit);
    if (blockIdx.x == 0 && threadIdx.x < 64) {
        const float loss = loss_of(teacher, a, s);
        if (lane == 0) a.loss[row] = loss;
    }
    if constexpr (GRAD) {
        const int nq = (a.classes + VEC - 1) / VEC, begin = blockIdx.x * slice, end = min(begin + slice, nq);
        const int doubled = nq * VEC - a.classes;
        const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
        T *dx = static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride;
        const Kind kind = kind_of(teacher);
        const bool flat = kind != kShares || s.S == 0.f;
        const float value = kind == kNan ? __builtin_nanf("") : 0.f, from = usable(s.c), factor = teacher.w * a.temperature / s.S;
        for (int q0 = begin + threadIdx.x; q0 < end; q0 += kSliceThreads * kSliceChunks) {
            typename C::raw raw[kSliceChunks];
#pragma unroll
            for (int k = 0; k < kSliceChunks; ++k) raw[k] = C::load(x + chunk_at<VEC>(min(q0 + k * kSliceThreads, end - 1), nq, a.classes));
#pragma unroll
            for (int k = 0; k < kSliceChunks; ++k) {
                const int q = q0 + k * kSliceThreads, to = chunk_at<VEC>(q, nq, a.classes);
                if (q >= end) break;
                float v[VEC];
                C::widen(raw[k], v);
#pragma unroll
                for (int i = 0; i < VEC; ++i) v[i] = flat ? value : exp_fast(v[i] - from, unit) * factor;
                if (q < nq - 1 || doubled == 0) {
                    C::store(dx + to, C::narrow(v));
                } else {                                 // what the neighbour has too may have been read after it was replaced: it is the neighbour's
#pragma unroll
                    for (int i = 0; i < VEC; ++i)
                        if (i >= doubled) Element<BF16>::put(dx + to + i, v[i]);
                }
            }
        }
        if (flat) return;                                // the whole workgroup
        __syncthreads();
        if (threadIdx.x < 64) {                          // the teacher's classes in this slice follow
            float put[kEntries];
            at_entries(put, teacher, a, s, unit, factor, slots);
#pragma unroll
            for (int e = 0; e < kEntries; ++e)
                if (teacher.index[e] >= begin * VEC && teacher.index[e] < min(end * VEC, a.classes)) Element<BF16>::put(dx + teacher.index[e], put[e]);
        }
    }
}

struct DistillPlan {
    int vec;
    bool narrow, wave, slices;
    int k, waves;                // chunks per lane, wavefronts of a workgroup with the teacher's
    int slice, per_row;          // chunks of a slice, slices of a row
    int64_t batch, with_gradient;        // rows per pair of launches: most; what the caches hold from its first to its second
};
// Chunks of a lane: 8 take 58 registers, so that two workgroups of 16 wavefronts fit a compute unit, and 18 are the least that hold 131 072 bf16 classes.  18 take 95
// registers, one workgroup a unit; 24, 184 320 bf16 classes, would take 122 and leave it at one, but are not built: rows from 138 248 bf16 and 69 124 fp32 classes on are cut into
// slices and read twice (8 192 x 138 240 bf16 878 us, x 152 064 1 660).
constexpr int kFew = 8, kMany = 18;

DistillPlan plan_distill(int64_t rows, int64_t classes, bool bf16)
{
    DistillPlan p = {};
    p.vec = classes < (bf16 ? 8 : 4) ? 1 : bf16 ? 8 : 4;
    const int64_t whole = classes / p.vec, chunks = (classes + p.vec - 1) / p.vec;
    p.narrow = chunks <= 16;
    if (chunks <= 64 * 8) {
        p.wave = true;
        p.k = static_cast<int>((chunks + 63) / 64);
        return p;
    }
    constexpr int kLanes = 64 * (kMostWaves - 1);
    if (whole <= kLanes * kMany) {
        p.k = whole <= kLanes * kFew ? kFew : kMany;
        p.waves = 1 + static_cast<int>((whole + p.k * 64 - 1) / (p.k * 64));
        return p;
    }
    constexpr int kStep = kSliceThreads * kSliceChunks;
    p.slices = true;
    int64_t slice = kStep;
    while (whole > slice * 512) slice *= 2;
    p.slice = static_cast<int>(slice);
    p.per_row = static_cast<int>((chunks + slice - 1) / slice);
    p.with_gradient = std::max<int64_t>(1, std::min<int64_t>(rows, (int64_t(64) << 20) / (classes * (bf16 ? 2 : 4))));
    p.batch = std::max(p.with_gradient, std::min<int64_t>({rows, (int64_t(1) << 21) / p.per_row, 65535}));
    return p;
}

constexpr int kUnits = 256;      // compute units, for the number of workgroups that stay

template <bool BF16, int VEC> void launch_narrow(const DistillArgs &a, hipStream_t stream)
{
    const unsigned groups = static_cast<unsigned>((a.rows + 15) / 16);
    (a.dlogits ? distill_narrow_kernel<BF16, VEC, true> : distill_narrow_kernel<BF16, VEC, false>)<<<groups, 256, 0, stream>>>(a);
}
template <bool BF16, int VEC, int K> void launch_wave(const DistillArgs &a, hipStream_t stream)
{
    const unsigned groups = static_cast<unsigned>(std::min<int64_t>((a.rows + 3) / 4, 1 << 20));
    (a.dlogits ? distill_wave_kernel<BF16, VEC, K, true> : distill_wave_kernel<BF16, VEC, K, false>)<<<groups, 256, 0, stream>>>(a);
}
template <bool BF16, int K> void launch_rows(const DistillArgs &a, int waves, hipStream_t stream)
{
    // as many workgroups as the registers of the compute units take at once
    constexpr int kWaves = K >= 16 ? 16 : 32;
    const int lanes = (a.classes / (BF16 ? 8 : 4) + K - 1) / K;
    const unsigned groups = static_cast<unsigned>(std::min<int64_t>(a.rows, kUnits * (kWaves / waves)));
    (a.dlogits ? distill_rows_kernel<BF16, K, true> : distill_rows_kernel<BF16, K, false>)<<<groups, waves * 64, 0, stream>>>(a, lanes);
}

template <bool BF16> hipError_t launch(const DistillArgs &a, const DistillPlan &p, void *workspace, hipStream_t stream)
{
    constexpr int VEC = BF16 ? 8 : 4;
    if (p.slices) {
        f2 *parts = static_cast<f2 *>(workspace);
        float *at = reinterpret_cast<float *>(parts + p.batch * p.per_row);
        constexpr int64_t e = BF16 ? 2 : 4;
        const int64_t batch = a.dlogits ? p.with_gradient : p.batch;
        for (int64_t row = 0; row < a.rows; row += batch) {
            DistillArgs b = a;
            b.rows = std::min(batch, a.rows - row);
            b.logits = static_cast<const char *>(a.logits) + row * a.row_stride * e;
            b.top_index += row * a.top_row_stride;
            b.top_logits += row * a.top_row_stride;
            if (b.weights) b.weights += row;
            b.loss += row;
            if (b.dlogits) b.dlogits = static_cast<char *>(a.dlogits) + row * a.dlogits_row_stride * e;
            const dim3 grid(p.per_row, static_cast<unsigned>(b.rows));
            distill_slices_kernel<BF16, VEC><<<grid, kSliceThreads, 0, stream>>>(b, p.slice, parts, at);
            if (b.dlogits) distill_join_kernel<BF16, VEC, true><<<grid, kSliceThreads, 0, stream>>>(b, p.slice, p.per_row, parts, at);
            else distill_join_kernel<BF16, VEC, false><<<dim3(1, grid.y), kSliceThreads, 0, stream>>>(b, p.slice, p.per_row, parts, at);
        }
        return hipGetLastError();
    }
    if (p.narrow) {
        // at most 2^24 workgroups' threads are numbered in a launch
        for (int64_t row = 0; row < a.rows; row += int64_t(1) << 26) {
            constexpr int64_t e = BF16 ? 2 : 4;
            DistillArgs b = a;
            b.rows = std::min<int64_t>(int64_t(1) << 26, a.rows - row);
            b.logits = static_cast<const char *>(a.logits) + row * a.row_stride * e;
            b.top_index += row * a.top_row_stride;
            b.top_logits += row * a.top_row_stride;
            if (b.weights) b.weights += row;
            b.loss += row;
            if (b.dlogits) b.dlogits = static_cast<char *>(a.dlogits) + row * a.dlogits_row_stride * e;
            if (p.vec == 1) launch_narrow<BF16, 1>(b, stream);
            else launch_narrow<BF16, VEC>(b, stream);
        }
    } else if (p.wave) {
        switch (p.k) {
        case 1: launch_wave<BF16, VEC, 1>(a, stream); break;
        case 2: launch_wave<BF16, VEC, 2>(a, stream); break;
        case 3: launch_wave<BF16, VEC, 3>(a, stream); break;
        case 4: launch_wave<BF16, VEC, 4>(a, stream); break;
        case 5: launch_wave<BF16, VEC, 5>(a, stream); break;
        case 6: launch_wave<BF16, VEC, 6>(a, stream); break;
        case 7: launch_wave<BF16, VEC, 7>(a, stream); break;
        default: launch_wave<BF16, VEC, 8>(a, stream);
        }
    } else if (p.k == kFew) {
        launch_rows<BF16, kFew>(a, p.waves, stream);
    } else {
        launch_rows<BF16, kMany>(a, p.waves, stream);
    }
    return hipGetLastError();
}

}  // namespace

size_t distill_bytes(int64_t rows, int64_t classes, bool bf16, int top)
{
    if (rows == 0) return 0;
    const DistillPlan p = plan_distill(rows, classes, bf16);
    return p.slices ? static_cast<size_t>(p.batch) * (p.per_row * sizeof(f2) + top * sizeof(float)) : 0;
}

hipError_t launch_distill(const DistillArgs &a, void *workspace, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const DistillPlan p = plan_distill(a.rows, a.classes, a.bf16);
    return a.bf16 ? launch<true>(a, p, workspace, stream) : launch<false>(a, p, workspace, stream);
}

}  // namespace cr
