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

// A lane's V elements: pairs are neighbours (HALVES: one half from each side of the head).
template <typename T, int D, bool HALVES>
struct Part {
    static constexpr int V = Elem<T>::kVec, G = D / V;
    float a[V / 2], b[V / 2];
    __device__ __forceinline__ void load(const T* row, int l) {
        if constexpr (HALVES) {
            load_half(row + l * (V / 2), a);
            load_half(row + D / 2 + l * (V / 2), b);
        } else {
            float f[V];
            unpack16(*reinterpret_cast<const uint4*>(row + l * V), f, T());
#pragma unroll
            for (int i = 0; i < V / 2; ++i) { a[i] = f[2 * i]; b[i] = f[2 * i + 1]; }
        }
    }
    __device__ __forceinline__ void store(T* row, int l) const {
        if constexpr (HALVES) {
            store_half(row + l * (V / 2), a);
            store_half(row + D / 2 + l * (V / 2), b);
        } else if constexpr (V == 8) {
            uint4 u;
            u.x = pack2(a[0], b[0]); u.y = pack2(a[1], b[1]); u.z = pack2(a[2], b[2]); u.w = pack2(a[3], b[3]);
            *reinterpret_cast<uint4*>(row + l * V) = u;
        } else {
            *reinterpret_cast<float4*>(row + l * V) = make_float4(a[0], b[0], a[1], b[1]);
        }
    }
    static __device__ __forceinline__ uint32_t pack2(float x, float y) {
        return (uint32_t)f32_to_bf16(x) | ((uint32_t)f32_to_bf16(y) << 16);
    }
    static __device__ __forceinline__ void load_half(const bf16_t* p, float* f) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        f[0] = bf16lo_to_f32(u.x); f[1] = bf16hi_to_f32(u.x); f[2] = bf16lo_to_f32(u.y); f[3] = bf16hi_to_f32(u.y);
    }
    static __device__ __forceinline__ void load_half(const float* p, float* f) {
        const float2 u = *reinterpret_cast<const float2*>(p);
        f[0] = u.x; f[1] = u.y;
    }
    static __device__ __forceinline__ void store_half(bf16_t* p, const float* f) {
        *reinterpret_cast<uint2*>(p) = make_uint2(pack2(f[0], f[1]), pack2(f[2], f[3]));
    }
    static __device__ __forceinline__ void store_half(float* p, const float* f) { *reinterpret_cast<float2*>(p) = make_float2(f[0], f[1]); }
};

// One wavefront takes the heads of one token, 64 / G of them at a time (`passes` first .. last): queries, then keys, then
// values.  Its lanes have the same place in every head, so a token's sines and cosines are computed once for all of them.
template <typename T, int D, bool HALVES>
__global__ __launch_bounds__(kThreads) void qk_norm_rope_kernel(FcRopeArgs a, int slices) {
    typedef Part<T, D, HALVES> P;
    constexpr int G = P::G, PER = FC_WAVE / G, NP = P::V / 2;
    const int r = blockIdx.y;
    if (r >= *a.n_rec || r >= a.A) return;
    const int c = a.rec_idx[r];
    if ((unsigned)c >= (unsigned)a.A) return;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
    const int64_t item = (int64_t)blockIdx.x * kWaves + wave;
    const int n = (int)(item / slices), slice = (int)(item % slices);
    if (n >= a.L_c) return;
    const int l = lane % G, sub = lane / G;
    const int nq = (a.H_q + PER - 1) / PER, nk = (a.H_k + PER - 1) / PER, nv = a.v ? nk : 0;
    const int total = nq + nk + nv;
    const int first = (int)((int64_t)total * slice / slices), last = (int)((int64_t)total * (slice + 1) / slices);
    const int64_t row = (int64_t)r * a.L_c + n;
    const int64_t slot = (int64_t)(a.active_off[c] + n) * a.tok_stride;

    float cs[NP], sn[NP], w[P::V];
    if (first < nq + nk) {
        const int frame = n / (a.grid_h * a.grid_w), in = n - frame * (a.grid_h * a.grid_w);
        const double pt = (double)a.frame0[c] + frame, ph = in / a.grid_w, pw = in % a.grid_w;
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const int p = l * NP + i;
            // in revolutions: whole ones are dropped in 64 bits, so far positions lose nothing
            const double t = (p < a.pairs_t ? pt : p < a.pairs_th ? ph : pw) * a.turns[p];
            sincospif(2.0f * (float)(t - rint(t)), &sn[i], &cs[i]);
        }
    }
    for (int pass = first; pass < last; ++pass) {
        const bool is_q = pass < nq, is_k = !is_q && pass < nq + nk;
        const int h = (pass - (is_q ? 0 : is_k ? nq : nq + nk)) * PER + sub;
        if (h >= (is_q ? a.H_q : a.H_k)) continue;
        const T* src = is_q ? (const T*)a.q + row * a.q_stride : (is_k ? (const T*)a.k : (const T*)a.v) + row * a.kv_stride;
        T* dst = is_q ? (T*)a.q_out + (row * a.H_q + h) * D : (is_k ? (T*)a.k_cache : (T*)a.v_cache) + h * a.head_stride + slot;
        src += h * D;
        if (!is_q && !is_k) {
            *reinterpret_cast<uint4*>(dst + l * P::V) = *reinterpret_cast<const uint4*>(src + l * P::V);
            continue;
        }
        P x;
        x.load(src, l);
        if (a.norm) {
            const float* wp = is_q ? a.q_weight : a.k_weight;
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < NP; ++i) ss = fmaf(x.a[i], x.a[i], fmaf(x.b[i], x.b[i], ss));
            const float inv = rsqrtf(group_sum<G>(ss) * (1.0f / D) + a.eps);
#pragma unroll
            for (int i = 0; i < NP; ++i) {
                x.a[i] *= inv; x.b[i] *= inv;
                if (wp) {
                    x.a[i] *= wp[HALVES ? l * NP + i : 2 * (l * NP + i)];
                    x.b[i] *= wp[HALVES ? D / 2 + l * NP + i : 2 * (l * NP + i) + 1];
                }
            }
        }
#pragma unroll
        for (int i = 0; i < NP; ++i) {
            const float u = x.a[i] * cs[i] - x.b[i] * sn[i], v = x.a[i] * sn[i] + x.b[i] * cs[i];
            x.a[i] = u; x.b[i] = v;
        }
        x.store(dst, l);
    }
}

template <typename T, int D>
int launch(const FcRopeArgs& a, hipStream_t s) {
    const int per = FC_WAVE / (D / Elem<T>::kVec);
    const int passes = (a.H_q + per - 1) / per + (a.v ? 2 : 1) * ((a.H_k + per - 1) / per);
    int slices = 1;
    const int64_t blocks = ((int64_t)a.L_c * slices + kWaves - 1) / kWaves;
    (void)passes;
    if (a.pairing)
        qk_norm_rope_kernel<T, D, true><<<dim3((unsigned)blocks, a.A), kThreads, 0, s>>>(a, slices);
    else
        qk_norm_rope_kernel<T, D, false><<<dim3((unsigned)blocks, a.A), kThreads, 0, s>>>(a, slices);
    FC_LAUNCH_CHECK();
    return FC_OK;
}

}  // namespace

int fc_launch_qk_norm_rope(const FcRopeArgs& a, hipStream_t s) {
    if (a.dtype == FC_BF16) return a.d == 128 ? launch<bf16_t, 128>(a, s) : launch<bf16_t, 64>(a, s);
    return a.d == 128 ? launch<float, 128>(a, s) : launch<float, 64>(a, s);
}
