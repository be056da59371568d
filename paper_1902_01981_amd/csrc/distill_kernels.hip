// The loss of a student's logits against a teacher's largest ones, and its gradient, for gfx950.
//
// With q the teacher's shares at temperature T, about their largest logit, and c, S as of the softmax loss with exp(x / T) in place of exp(x):
//     loss = w T sum_i q_i ((z_i - largest z) - (x_(j_i) - c) + T (log S - log S_q)),   dx_j = w T (exp((x_j - c) / T) / S - sum_(j_i = j) q_i).
#include "softmax_device.h"

#include <algorithm>

namespace cr {

namespace {

constexpr int kThreads = 256, kWaves = kThreads / 64, kMostTop = 128, kEntries = kMostTop / 64;     // entries of a lane

__device__ __forceinline__ float first_lane(float v) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(v))); }

// What a wavefront knows of a row's teacher: entries lane and lane + 64.
struct Teacher {
    int index[kEntries];         // -1: not there
    float q[kEntries];           // shares
    float d[kEntries];           // distances from the largest logit
    bool any, unknown;           // entries at all; one of no class
    float sum;                   // of exp(d / T): NaN where there is no sense in it
};
__device__ __forceinline__ void read_teacher(Teacher &t, const DistillArgs &a, int64_t row, float unit)
{
    const int lane = threadIdx.x % 64;
    float z[kEntries], most = -infinity();
    bool there = false, unknown = false;
#pragma unroll
    for (int e = 0; e < kEntries; ++e) {
        const int i = lane + 64 * e;
        int64_t index = -1;
        z[e] = -infinity();
        if (i < a.top) {
            index = a.top_index[row * a.top_row_stride + i];
            z[e] = a.top_logits[row * a.top_row_stride + i];
        }
        if (index < 0 || z[e] == -infinity()) {
            index = -1;
            z[e] = -infinity();
        }
        there |= index >= 0;
        unknown |= index >= a.classes;
        t.index[e] = index >= a.classes ? -1 : static_cast<int>(index);
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

template <bool BF16, int VEC> __global__ void __launch_bounds__(kThreads) distill_kernel(DistillArgs a)
{
    using C = Chunk<BF16, VEC>;
    using T = typename C::element;
    __shared__ float meet[2][kWaves], shares[kMostTop];
    __shared__ int places[kMostTop];
    const int lane = threadIdx.x % 64, wave = threadIdx.x / 64;
    const int whole = a.classes / VEC, left = a.classes % VEC;
    const float unit = kLog2e / a.temperature;
    for (int64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = static_cast<const T *>(a.logits) + row * a.row_stride;
        Teacher teacher;
        read_teacher(teacher, a, row, unit);
        float at[kEntries];
#pragma unroll
        for (int e = 0; e < kEntries; ++e) at[e] = Element<BF16>::get(x + max(teacher.index[e], 0));
        Softmax s;
        float v[VEC];
        for (int q = threadIdx.x; q < whole; q += kThreads) {
            C::widen(C::load(x + q * VEC), v);
            take<VEC>(s, v, true, unit);
        }
        if (threadIdx.x < left) {
            const float last[1] = {Element<BF16>::get(x + whole * VEC + threadIdx.x)};
            take<1>(s, last, true, unit);
        }
        join_lanes<64>(s, unit);
        __syncthreads();                                 // the last row's places are read
        if (lane == 0) {
            meet[0][wave] = s.c;
            meet[1][wave] = s.S;
        }
        if (wave == 0) {
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                places[lane + 64 * e] = teacher.index[e];
                shares[lane + 64 * e] = teacher.q[e];
            }
        }
        __syncthreads();
        s.c = meet[0][threadIdx.x % kWaves];
        s.S = meet[1][threadIdx.x % kWaves];
        join_lanes<kWaves>(s, unit);
        s.c = first_lane(s.c);                           // the lanes' sums may differ by a rounding
        s.S = first_lane(s.S);
        const float w = a.weights ? a.weights[row] : 1.f, from = usable(s.c), log2_S = __builtin_amdgcn_logf(s.S);
        const float nan = __builtin_nanf("");
        if (wave == 0) {
            // Not distances over T, and a fourth of each: they, and sums of them, could be infinite where the loss is not (masks of the type's lowest value).
            float sum = 0.f;
            const float both = 0.25f * a.temperature * kLn2 * (log2_S - __builtin_amdgcn_logf(teacher.sum));
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                const float term = teacher.q[e] * (0.25f * teacher.d[e] - (0.25f * at[e] - 0.25f * from) + both);
                sum += teacher.index[e] >= 0 && teacher.q[e] != 0.f ? term : 0.f;
            }
            sum = lanes_total<64>(sum);
            if (lane == 0)
                a.loss[row] = !teacher.any ? 0.f : 4.f * (w * a.temperature * (teacher.unknown ? nan : s.S == 0.f ? infinity() * teacher.sum : sum));
        }
        if (!a.dlogits) continue;
        T *dx = static_cast<T *>(a.dlogits) + row * a.dlogits_row_stride;
        const bool no_sense = teacher.unknown || !(teacher.sum == teacher.sum);
        const bool flat = !teacher.any || no_sense || s.S == 0.f;
        const float value = teacher.any && no_sense ? nan : 0.f;
        const float factor = w * a.temperature / s.S;
        auto form = [&](float xi) { return flat ? value : exp_fast(xi - from, unit) * factor; };
        for (int q = threadIdx.x; q < whole; q += kThreads) {
            C::widen(C::load(x + q * VEC), v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) v[i] = form(v[i]);
            C::store(dx + q * VEC, C::narrow(v));
        }
        if (threadIdx.x < left) {
            const int j = whole * VEC + threadIdx.x;
            Element<BF16>::put(dx + j, form(Element<BF16>::get(x + j)));
        }
        __syncthreads();
        // the teacher's classes follow; an index that comes several times has the same bits from each of its entries
        if (wave == 0 && !flat) {
#pragma unroll
            for (int e = 0; e < kEntries; ++e) {
                if (teacher.index[e] < 0) continue;
                float q = 0.f;
                for (int i = 0; i < a.top; ++i) q += places[i] == teacher.index[e] ? shares[i] : 0.f;
                Element<BF16>::put(dx + teacher.index[e], fmaf(exp_fast(at[e] - from, unit), factor, -(w * a.temperature * q)));
            }
        }
    }
}

}  // namespace

size_t distill_bytes(int64_t, int64_t, bool, int) { return 0; }

hipError_t launch_distill(const DistillArgs &a, void *, hipStream_t stream)
{
    if (a.rows == 0) return hipSuccess;
    const unsigned grid = static_cast<unsigned>(std::min<int64_t>(a.rows, 1 << 20));
    if (a.classes < (a.bf16 ? 8 : 4)) (a.bf16 ? distill_kernel<true, 1> : distill_kernel<false, 1>)<<<grid, kThreads, 0, stream>>>(a);
    else if (a.bf16) distill_kernel<true, 8><<<grid, kThreads, 0, stream>>>(a);
    else distill_kernel<false, 4><<<grid, kThreads, 0, stream>>>(a);
    return hipGetLastError();
}

}  // namespace cr
