// Rows of a projection on their way to the caches, for gfx950: per-head norm of queries and keys, position rotation, and
// the turn from token-major rows [B][n][heads][d] to the head-major ones [B][heads][n][d] that prompt scoring and the caches
// hold, in one pass.
//
//   x' = x / sqrt(mean(x^2) + eps) * weight                                 (queries and keys, if asked for)
//   (a, b) -> (a cos t - b sin t, a sin t + b cos t),  t = position * inv_freq[i]
//
// with (a, b) = elements (2i, 2i+1) or (i, i + rot/2) of a row.  Everything is computed in 32 bits and rounded once, when the
// row is stored; the angle's turns are counted in 64 bits, so that a position of 100 000 costs no accuracy.
//
// What bounds it is bytes: each row is read and written once (8 x 4096 tokens x 96 heads x 128, padded: 1.0 GB in 222 to 246 us on
// four cards, 4.1 to 4.5 TB/s; a large copy runs at 4.7).  One token a sequence is bound by a chain: positions and frequencies, the
// angles, then the rows' own trip to memory, which waits for them although no address asks for it (64 sequences x 96 heads x 128
// 5.0 us).  A lane takes 16 bytes of a row, d * sizeof(T) / 16 adjacent lanes a row.  A workgroup takes `tt` neighbouring
// tokens of one sequence and `hc` heads: the cosines and sines of its tokens are formed once, in LDS, for all its heads.
#include "kf_device.h"
#include "kf_internal.h"

namespace kf {

constexpr int kRowsThreads = 256;

template <typename T>
__device__ __forceinline__ uint4 pack16(const float* f);
template <>
__device__ __forceinline__ uint4 pack16<float>(const float* f) {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
}
typedef __bf16 rows_bf2_t __attribute__((ext_vector_type(2)));
typedef _Float16 rows_h2_t __attribute__((ext_vector_type(2)));
template <>
__device__ __forceinline__ uint4 pack16<bf16_t>(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, rows_bf2_t{(__bf16)f[2 * i], (__bf16)f[2 * i + 1]});
    return make_uint4(w[0], w[1], w[2], w[3]);
}
template <>
__device__ __forceinline__ uint4 pack16<f16_t>(const float* f) {
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __builtin_bit_cast(uint32_t, rows_h2_t{(_Float16)f[2 * i], (_Float16)f[2 * i + 1]});
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <typename T, int D, int STYLE>
__global__ void __launch_bounds__(kRowsThreads) rows_kernel(const RowsArgs a) {
    constexpr int EPV = ElemTraits<T>::kPerVec, LPR = D / EPV, RPW = kWave / LPR, NW = kRowsThreads / kWave, RPB = RPW * NW;
    extern __shared__ float2 turn[];  // [tt][half] cosine and sine of the workgroup's tokens
    __shared__ __attribute__((aligned(16))) float part[STYLE == KF_ROTATE_HALVES ? NW * RPW * D : 1];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, sub = lane / LPR, cl = lane % LPR;
    const uint32_t chunk = blockIdx.x % (uint32_t)a.chunks, bt = blockIdx.x / (uint32_t)a.chunks;
    const int b = (int)(bt / (uint32_t)a.tiles), t0 = (int)(bt % (uint32_t)a.tiles) << a.tt_shift;
    int nb = a.n;
    if (a.seq_n) {
        nb = a.seq_n[b];
        if (nb < 1 || nb > a.n) nb = 0;  // no such length: the sequence is left out (and nb - t0 does not leave its range)
    }
    const int cnt = min(1 << a.tt_shift, nb - t0);
    if (cnt <= 0) return;
    if constexpr (STYLE != KF_ROTATE_NONE) {
        const int64_t first = (a.seq_pos ? (int64_t)a.seq_pos[b] : (int64_t)a.pos0) + t0;
        for (int i = tid; i < cnt * a.half; i += kRowsThreads) {
            const int t = i / a.half, f = i - t * a.half;
            double rev = (double)(first + t) * ((double)a.freq[f] * 0.15915494309189533577);  // in turns
            rev -= rint(rev);
            float s, c;
            sincospif((float)(2.0 * rev), &s, &c);
            turn[i] = make_float2(c, s);
        }
        __syncthreads();
    }
    float qw[EPV], kw[EPV];
#pragma unroll
    for (int e = 0; e < EPV; ++e) qw[e] = kw[e] = 1.0f;
    if (a.qw) unpack16<T>(((const uint4*)a.qw)[cl], qw);
    if (a.kw) unpack16<T>(((const uint4*)a.kw)[cl], kw);

    const int h0 = (int)chunk * a.hc, heads = min(a.hc, a.nq + a.nk + a.nv - h0);
    const int rows = heads << a.tt_shift;
    for (int r0 = wv * RPW; r0 < rows; r0 += RPB) {
        const int r = r0 + sub, t = r & ((1 << a.tt_shift) - 1), hd = h0 + (r >> a.tt_shift);
        const bool ok = r < rows && t < cnt;
        const int kind = hd < a.nq ? 0 : hd < a.nq + a.nk ? 1 : 2;  // query, key, value
        const int h = kind == 0 ? hd : kind == 1 ? hd - a.nq : hd - a.nq - a.nk;
        const int64_t tok = t0 + t;
        uint4 raw = make_uint4(0u, 0u, 0u, 0u);
        if (ok) {
            const T* src = kind == 0 ? (const T*)a.q + b * a.q_sb + tok * a.q_st : kind == 1 ? (const T*)a.k + b * a.k_sb + tok * a.k_st
                                                                                    : (const T*)a.v + b * a.v_sb + tok * a.v_st;
            raw = stream_load((const uint4*)(src + (int64_t)h * D) + cl);
        }
        float x[EPV];
        unpack16<T>(raw, x);
        if (a.qw || a.kw) {
            float ss = 0.0f;
#pragma unroll
            for (int e = 0; e < EPV; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
            for (int o = 1; o < LPR; o <<= 1) ss += __shfl_xor(ss, o, kWave);
            if (kind == 0 ? a.qw != nullptr : kind == 1 && a.kw) {
                const float inv = 1.0f / sqrtf(ss * (1.0f / D) + a.eps);
#pragma unroll
                for (int e = 0; e < EPV; ++e) x[e] = x[e] * inv * (kind == 0 ? qw[e] : kw[e]);
            }
        }
        if constexpr (STYLE == KF_ROTATE_PAIRS) {
            if (ok && kind < 2) {
#pragma unroll
                for (int e = 0; e < EPV; e += 2) {
                    const int i = (cl * EPV + e) / 2;
                    if (i < a.half) {
                        const float2 cs = turn[t * a.half + i];
                        const float u = x[e], v = x[e + 1];
                        x[e] = u * cs.x - v * cs.y;
                        x[e + 1] = u * cs.y + v * cs.x;
                    }
                }
            }
        }
        if constexpr (STYLE == KF_ROTATE_HALVES) {  // a row's other half lies with other lanes of the wave
            float* mine = part + (wv * RPW + sub) * D;
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int e = 0; e < EPV; ++e) mine[cl * EPV + e] = x[e];
            __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
            __builtin_amdgcn_wave_barrier();
            __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
            if (ok && kind < 2) {
#pragma unroll
                for (int e = 0; e < EPV; ++e) {
                    const int c = cl * EPV + e;
                    if (c < 2 * a.half) {
                        const bool low = c < a.half;
                        const int i = low ? c : c - a.half;
                        const float2 cs = turn[t * a.half + i];
                        const float other = mine[low ? c + a.half : i];
                        x[e] = low ? x[e] * cs.x - other * cs.y : other * cs.y + x[e] * cs.x;
                    }
                }
            }
        }
        if (ok) {
            T* dst = kind == 0 ? (T*)a.Q + (((int64_t)b * a.nq + h) * a.n + tok) * D
                               : (T*)(kind == 1 ? a.K : a.V) + (((int64_t)b * (kind == 1 ? a.nk : a.nv) + h) * a.kv_rows + tok) * D;
            stream_store((uint4*)dst + cl, kind == 2 ? raw : pack16<T>(x));
        }
    }
}

template <typename T, int D>
static hipError_t launch_rows_d(const RowsArgs& a, int64_t blocks, hipStream_t st) {
    const dim3 grid((unsigned)blocks), block(kRowsThreads);
    const size_t lds = (size_t)a.half << (a.tt_shift + 3);
    if (a.half == 0) hipLaunchKernelGGL((rows_kernel<T, D, KF_ROTATE_NONE>), grid, block, 0, st, a);
    else if (a.pairs) hipLaunchKernelGGL((rows_kernel<T, D, KF_ROTATE_PAIRS>), grid, block, lds, st, a);
    else hipLaunchKernelGGL((rows_kernel<T, D, KF_ROTATE_HALVES>), grid, block, lds, st, a);
    return hipGetLastError();
}

// Tokens and heads of a workgroup: 8 tokens share a trip through the heads where there are as many; fewer heads than all
// where the launch would else have under 1024 workgroups.
int64_t plan_rows(RowsArgs* a) {
    a->tt_shift = a->n >= 8 ? 3 : a->n >= 4 ? 2 : a->n >= 2 ? 1 : 0;
    a->tiles = (int32_t)(((int64_t)a->n + (1 << a->tt_shift) - 1) >> a->tt_shift);
    const int64_t bt = (int64_t)a->B * a->tiles;
    const int32_t heads = a->nq + a->nk + a->nv;
    int64_t want = (1024 + bt - 1) / bt;
    if (want > heads) want = heads;
    a->hc = (int32_t)((heads + want - 1) / want);
    a->chunks = (heads + a->hc - 1) / a->hc;
    return bt * a->chunks;
}

hipError_t launch_rows(const RowsArgs& a, int64_t blocks, int32_t d, int32_t dtype, hipStream_t stream) {
    if (dtype == KF_BF16) {
        if (d == 64) return launch_rows_d<bf16_t, 64>(a, blocks, stream);
        if (d == 128) return launch_rows_d<bf16_t, 128>(a, blocks, stream);
        if (d == 256) return launch_rows_d<bf16_t, 256>(a, blocks, stream);
    } else if (dtype == KF_F16) {
        if (d == 64) return launch_rows_d<f16_t, 64>(a, blocks, stream);
        if (d == 128) return launch_rows_d<f16_t, 128>(a, blocks, stream);
        if (d == 256) return launch_rows_d<f16_t, 256>(a, blocks, stream);
    } else if (dtype == KF_F32) {
        if (d == 64) return launch_rows_d<float, 64>(a, blocks, stream);
        if (d == 128) return launch_rows_d<float, 128>(a, blocks, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace kf
