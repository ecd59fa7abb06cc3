// Norm of every query and key head and its rotation by (time, height, width), from the projections' rows into the
// attention's query rows and the K/V slots.
//
//   y = x * rsqrt(mean x^2 + eps) * w        per head, d elements
//   (y_a, y_b) -> (y_a cos - y_b sin, y_a sin + y_b cos)     for every pair, angle = position on the pair's axis * frequency
//
// One pass: every element is read once, held as fp32 and rounded once.  HBM bound.
#include <type_traits>

#include "fc_common.hpp"

namespace {

constexpr int kThreads = 256;
constexpr int kWaves = kThreads / FC_WAVE;
constexpr int kAhead = 4;

// Sum over groups of G neighbouring lanes, in all of them.
template <int G>
__device__ __forceinline__ float group_sum(float v) {
    auto dpp = [](float x, auto ctrl) { return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), decltype(ctrl)::value, 0xF, 0xF, true)); };
    v += dpp(v, std::integral_constant<int, 0xB1>());                   // quad_perm 1 0 3 2
    v += dpp(v, std::integral_constant<int, 0x4E>());                   // quad_perm 2 3 0 1
    v += dpp(v, std::integral_constant<int, 0x141>());                  // the other quad of eight lanes (mirrored: its lanes agree)
    if (G >= 16) v += dpp(v, std::integral_constant<int, 0x140>());     // the other eight of sixteen lanes
    if (G >= 32) v += __shfl_xor(v, 16, FC_WAVE);
    return v;
}

// Heads whose mean square leaves a float's range, or its normal numbers: the elements times a power of two first (small ones), or the
// root's inverse and then the power (large ones; the other order would lose bits of small elements).  f becomes what the returned
// factor has yet to be multiplied with.  Rare: a group's lanes agree, so it is a branch that others skip.
template <int G, int V>
__device__ __forceinline__ float norm_far(float (&f)[V], bool small, float eps, float inv_d) {
    const float to = small ? 0x1p100f : 0x1p-68f;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < V; ++i) ss = fmaf(f[i] * to, f[i] * to, ss);
    const float inv = rsqrtf(group_sum<G>(ss) * inv_d + eps * to * to);
#pragma unroll
    for (int i = 0; i < V; ++i) f[i] = small ? f[i] * to : f[i] * inv * to;
    return small ? inv : 1.0f;
}

// A lane's 16 bytes of a head, as two halves of the pairs' elements: neighbours (HALVES: one from each side of the head).
template <typename T, int D, bool HALVES>
struct Part {
    static constexpr int V = Elem<T>::kVec, G = D / V, NP = V / 2;
    static __device__ __forceinline__ uint4 load(const T* head, int l) {
        if constexpr (HALVES) {
            const uint2 a = *reinterpret_cast<const uint2*>(head + l * NP), b = *reinterpret_cast<const uint2*>(head + D / 2 + l * NP);
            return make_uint4(a.x, a.y, b.x, b.y);
        } else {
            return *reinterpret_cast<const uint4*>(head + l * V);
        }
    }
    static __device__ __forceinline__ void store(T* head, int l, const uint4& u) {
        if constexpr (HALVES) {
            *reinterpret_cast<uint2*>(head + l * NP) = make_uint2(u.x, u.y);
            *reinterpret_cast<uint2*>(head + D / 2 + l * NP) = make_uint2(u.z, u.w);
        } else {
            *reinterpret_cast<uint4*>(head + l * V) = u;
        }
    }
    // pair i of the lane: elements first(i) and second(i) of the 16 bytes
    static constexpr __device__ int first(int i) { return HALVES ? i : 2 * i; }
    static constexpr __device__ int second(int i) { return HALVES ? NP + i : 2 * i + 1; }
    // ... and of the head
    static __device__ __forceinline__ int first_at(int l, int i) { return HALVES ? l * NP + i : 2 * (l * NP + i); }
    static __device__ __forceinline__ int second_at(int l, int i) { return HALVES ? D / 2 + l * NP + i : 2 * (l * NP + i) + 1; }
};
__device__ __forceinline__ uint4 pack16(const float (&f)[8], bf16_t) {
    // (f32_to_bf16() is for finite values: some NaN become zeros there)
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    auto two = [](float x, float y) { return __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)x, (__bf16)y}); };
    return make_uint4(two(f[0], f[1]), two(f[2], f[3]), two(f[4], f[5]), two(f[6], f[7]));
}
__device__ __forceinline__ uint4 pack16(const float (&f)[4], float) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}

// A group of G lanes takes one token and goes through its heads, one per pass: queries, then keys, then values (a launch of few
// tokens deals a token's passes to several groups).  A lane has the same place in every head, so it computes its sines and cosines
// once; the wavefront's 64 / G tokens are neighbours, and so are the rows of a cache that it writes.  kAhead passes are read
// before the first of them is worked on.
template <typename T, int D, bool HALVES>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(FcRopeArgs a, int slices) {
    typedef Part<T, D, HALVES> P;
    constexpr int G = P::G, PER = FC_WAVE / G, NP = P::NP;
    const int r = blockIdx.y;
    if (r >= *a.n_rec || r >= a.A) return;
    const int c = a.rec_idx[r];
    if ((unsigned)c >= (unsigned)a.A) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int item = blockIdx.x * kWaves + wave;
    const int n = item / slices * PER + lane / G, slice = item % slices, l = lane % G;
    if (n >= a.L_c) return;
    const int total = a.H_q + (a.v ? 2 : 1) * a.H_k;
    const int first = (int)((int64_t)total * slice / slices), last = (int)((int64_t)total * (slice + 1) / slices);
    const int64_t row = (int64_t)r * a.L_c + n;
    const int64_t slot = (int64_t)(a.active_off[c] + n) * a.tok_stride;
    const T *q = (const T*)a.q + row * a.q_stride, *k = (const T*)a.k + row * a.kv_stride, *v = (const T*)a.v + row * a.kv_stride;

    float cs[NP], sn[NP], wq[P::V], wk[P::V];
    if (first < a.H_q + a.H_k) {
        const int frame = n / (a.grid_h * a.grid_w), in = n - frame * (a.grid_h * a.grid_w);
        const double pt = (double)a.frame0[c] + frame, ph = in / a.grid_w, pw = in % a.grid_w;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int p = l * NP + i;
            // In revolutions, whole ones dropped before anything is rounded (turns and turns_rest: rope_turns.hpp), so far positions lose
            // nothing: with turns alone, frame 2^31 is off by 8 units of 2^-24.
            const double pos = p < a.pairs_t ? pt : p < a.pairs_th ? ph : pw, turns = a.turns[p];
            const double t = fma(pos, turns, -rint(pos * turns)) + pos * a.turns_rest[p];
            sincospif(2.0f * (float)t, &sn[i], &cs[i]);
            wq[P::first(i)] = a.q_weight ? a.q_weight[P::first_at(l, i)] : 1.0f;
            wq[P::second(i)] = a.q_weight ? a.q_weight[P::second_at(l, i)] : 1.0f;
            wk[P::first(i)] = a.k_weight ? a.k_weight[P::first_at(l, i)] : 1.0f;
            wk[P::second(i)] = a.k_weight ? a.k_weight[P::second_at(l, i)] : 1.0f;
        }
    }
    for (int pass0 = first; pass0 < last; pass0 += kAhead) {
        uint4 u[kAhead];
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int pass = pass0 + e < last ? pass0 + e : last - 1;        // (past the end: read again, not written)
            const bool is_q = pass < a.H_q, is_k = pass < a.H_q + a.H_k;
            const int h = pass - (is_q ? 0 : is_k ? a.H_q : a.H_q + a.H_k);
            u[e] = P::load((is_q ? q : is_k ? k : v) + h * D, l);
        }
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
            const int pass = pass0 + e;
            if (pass >= last) break;
            const bool is_q = pass < a.H_q, is_k = pass < a.H_q + a.H_k;
            const int h = pass - (is_q ? 0 : is_k ? a.H_q : a.H_q + a.H_k);
            if (is_k) {                                                      // a query or a key
                float f[P::V];
                unpack16(u[e], f, T());
                if (a.norm) {
                    float ss = 0.f;
#pragma unroll
                    for (int i = 0; i < P::V; ++i) ss = fmaf(f[i], f[i], ss);
                    const float ms = group_sum<G>(ss) * (1.0f / D) + a.eps;
                    float inv = rsqrtf(ms);
                    if (!(ms >= 0x1p-96f && ms <= 0x1p120f)) inv = norm_far<G>(f, ms < 0x1p-96f, a.eps, 1.0f / D);
#pragma unroll
                    for (int i = 0; i < P::V; ++i) f[i] = f[i] * inv * (is_q ? wq[i] : wk[i]);
                }
#pragma unroll
                for (int i = 0; i < NP; ++i) {
                    const float x = f[P::first(i)], y = f[P::second(i)];
                    f[P::first(i)] = x * cs[i] - y * sn[i];
                    f[P::second(i)] = x * sn[i] + y * cs[i];
                }
                u[e] = pack16(f, T());
            }
            P::store(is_q ? (T*)a.q_out + (row * a.H_q + h) * D : (is_k ? (T*)a.k_cache : (T*)a.v_cache) + h * a.head_stride + slot, l, u[e]);
        }
    }
}

template <typename T, int D>
int launch(const FcRopeArgs& a, hipStream_t s) {
    constexpr int per = FC_WAVE / (D / Elem<T>::kVec);        // tokens per wavefront
    const int total = a.H_q + (a.v ? 2 : 1) * a.H_k;
    const int64_t groups = (a.L_c + per - 1) / per;
    // eight wavefronts for every compute unit, if a chunk's passes are so many
    int64_t slices = (2048 + groups - 1) / groups;
    slices = slices < total ? slices : total;
    const int64_t blocks = (groups * slices + kWaves - 1) / kWaves;
    if (a.pairing)
        qk_norm_rope_kernel<T, D, true><<<dim3((unsigned)blocks, a.A), kThreads, 0, s>>>(a, (int)slices);
    else
        qk_norm_rope_kernel<T, D, false><<<dim3((unsigned)blocks, a.A), kThreads, 0, s>>>(a, (int)slices);
    FC_LAUNCH_CHECK();
    return FC_OK;
}

}  // namespace

int fc_launch_qk_norm_rope(const FcRopeArgs& a, hipStream_t s) {
    if (a.dtype == FC_BF16) return a.d == 128 ? launch<bf16_t, 128>(a, s) : launch<bf16_t, 64>(a, s);
    return a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}
