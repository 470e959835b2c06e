// Caches of 4 bits for gfx950: the decode step's split kernel over them, and the eviction of 16-bit rows into them.
//
// A row of D elements is D/2 bytes of codes -- E2M1: sign, two exponent bits, one mantissa bit, i.e. 0 1/2 1 3/2 2 3 4 6 --
// and 16 scale bytes, one for every D/16 elements: a power of two, the smallest with which none of them is above 7 (what
// lies between 6 and 7 becomes 6, no further off than half the last step).  Powers of two keep a value of two significant bits
// exact in bf16, so the conversion instructions of the matrix formats (two codes and a scale in, two bf16 or fp32 out) do
// all of the decoding; and sixteen scales fill the 16 bytes that keep rows aligned.
//
// The step is that of kf_decode.hip, with the same arguments, workspace records and merge:
//   x_j = scale*<q, K_j> - slope*(q_pos - pos_j);  out = sum_j softmax(x)_j V_j;  f_j += softmax((x + zeta)/tau)_j
// A workgroup streams the rows [j0, j1) of one cached head; a lane takes EPL elements of a row (16 bytes of codes, or 8 where
// many query heads need the registers).  The new token's own key and value enter as they were given, in 16 bits.
#include "kf_device.h"
#include "kf_internal.h"
#include "kf_merge.h"

namespace kf {

constexpr int kQuantThreads = 256;
constexpr int kQuantWaves = kQuantThreads / kWave;
constexpr int kQuantUnroll = 4;                       // rows a lane has in flight
constexpr size_t kQuantLds = 81920 - 1024;            // two workgroups on a compute unit at least
constexpr int quant_epl(int G) { return G >= 8 ? 16 : 32; }

typedef __bf16 q_bf2_t __attribute__((ext_vector_type(2)));
typedef float q_f2_t __attribute__((ext_vector_type(2)));

// ---------------------------------------------------------------- encoding
// Scale byte of a group whose largest magnitude is `a`: 255 for one that holds an infinity or a NaN.
__device__ __forceinline__ uint32_t quant_scale(float a) {
    const uint32_t b = __float_as_uint(a), E = b >> 23;
    if (E == 255) return 255u;
    const int s = (int)E - 2 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)min(max(s, 1), 252);
}
// Nearest code, ties to the even one; `inv`: two to the power of minus the scale's exponent.
__device__ __forceinline__ uint32_t quant_code(float v, float inv) {
    const float y = fabsf(v) * inv;
    const uint32_t c = (y > 0.25f) + (y >= 0.75f) + (y > 1.25f) + (y >= 1.75f) + (y > 2.5f) + (y >= 3.5f) + (y > 5.0f);
    return c | ((__float_as_uint(v) >> 28) & 8u);
}
// One group of N = D/16 elements at `src` (16 bits each) -> its codes and scale byte in the row at `dst`.
template <typename T, int D>
__device__ __forceinline__ void quant_group(const char* src, char* dst, int g) {
    constexpr int N = D / 16;
    float v[N];
    if constexpr (N == 4) {
        const uint2 r = *(const uint2*)(src + g * 8);
        float t[8];
        unpack16<T>(make_uint4(r.x, r.y, 0u, 0u), t);
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] = t[i];
    } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) unpack16<T>(((const uint4*)(src + g * 2 * N))[i], v + 8 * i);
    }
    float a = 0.0f;
    uint32_t bad = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        a = fmaxf(a, fabsf(v[i]));
        bad |= ((__float_as_uint(v[i]) >> 23) & 255u) == 255u ? 1u : 0u;
    }
    const uint32_t s = bad ? 255u : quant_scale(a);
    const float inv = __uint_as_float((254u - min(s, 252u)) << 23);
    uint32_t w[(N + 7) / 8];
#pragma unroll
    for (int i = 0; i < (N + 7) / 8; ++i) w[i] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) w[i / 8] |= (bad ? 7u : quant_code(v[i], inv)) << (4 * (i % 8));
    if constexpr (N == 4) *(uint16_t*)(dst + g * 2) = (uint16_t)w[0];
    else if constexpr (N == 8) *(uint32_t*)(dst + g * 4) = w[0];
    else *(uint2*)(dst + g * 8) = make_uint2(w[0], w[N / 8 - 1]);
    ((uint8_t*)dst)[D / 2 + g] = (uint8_t)s;
}

// ---------------------------------------------------------------- decoding
// What a lane holds of a row: EPL codes and the scales of their groups.
template <int D, int EPL>
struct QuantPiece {
    static constexpr int W = EPL / 8, SB = EPL / (D / 16);  // words of codes, scale bytes (1, 2, 4 or 8)
    uint32_t w[W];
    uint32_t s[(SB + 3) / 4];
    __device__ __forceinline__ void load(const char* row, int cl) {
        if constexpr (W == 4) {
            const uint4 r = *(const uint4*)(row + cl * 16);
            w[0] = r.x, w[1] = r.y, w[2] = r.z, w[3] = r.w;
        } else {
            const uint2 r = *(const uint2*)(row + cl * 8);
            w[0] = r.x, w[1] = r.y;
        }
        const char* sp = row + D / 2 + cl * SB;
        if constexpr (SB == 8) {
            const uint2 r = *(const uint2*)sp;
            s[0] = r.x, s[1] = r.y;
        } else if constexpr (SB == 4) s[0] = *(const uint32_t*)sp;
        else if constexpr (SB == 2) s[0] = *(const uint16_t*)sp;
        else s[0] = *(const uint8_t*)sp;
    }
    __device__ __forceinline__ float scale(int g) const {  // of the lane's g-th group
        const uint32_t b = s[g / 4];
        return __uint_as_float(SB == 1 ? b << 23 : ((b >> (8 * (g % 4))) & 255u) << 23);
    }
};
template <int SEL>
__device__ __forceinline__ q_bf2_t quant_bf16(uint32_t w, float s) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL); }
template <int SEL>
__device__ __forceinline__ q_f2_t quant_f32(uint32_t w, float s) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, SEL); }

// <q, row piece>: the decoded pairs against a query kept as pairs of bf16; a half of 11 significant bits is the sum of two.
template <typename T, int EPL>
struct QuantQuery {
    static constexpr int TERMS = sizeof(T) == 2 && ElemTraits<T>::kPerVec == 8 && __is_same(T, f16_t) ? 2 : 1;
    uint32_t q[TERMS][EPL / 2];
    __device__ __forceinline__ void load(const T* p) {
#pragma unroll
        for (int i = 0; i < EPL / 8; ++i) {
            const uint4 r = ((const uint4*)p)[i];
            if constexpr (TERMS == 1) {
                q[0][4 * i] = r.x, q[0][4 * i + 1] = r.y, q[0][4 * i + 2] = r.z, q[0][4 * i + 3] = r.w;
            } else {
                float f[8];
                unpack16<T>(r, f);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint32_t a = __float_as_uint(f[2 * j]), b = __float_as_uint(f[2 * j + 1]);
                    q[0][4 * i + j] = (a >> 16) | (b & 0xFFFF0000u);  // upper 8 significant bits; the rest is exact too
                    const float ra = f[2 * j] - __uint_as_float(a & 0xFFFF0000u), rb = f[2 * j + 1] - __uint_as_float(b & 0xFFFF0000u);
                    q[TERMS - 1][4 * i + j] = (__float_as_uint(ra) >> 16) | (__float_as_uint(rb) & 0xFFFF0000u);
                }
            }
        }
    }
    __device__ __forceinline__ float dot(const q_bf2_t (&k)[EPL / 2]) const {
        float p = 0.0f;
#pragma unroll
        for (int t = 0; t < TERMS; ++t) {
#pragma unroll
            for (int i = 0; i < EPL / 2; ++i) p = __builtin_amdgcn_fdot2_f32_bf16(k[i], __builtin_bit_cast(q_bf2_t, q[t][i]), p, false);
        }
        return p;
    }
};
template <int D, int EPL>
__device__ __forceinline__ void quant_decode(const QuantPiece<D, EPL>& p, q_bf2_t (&v)[EPL / 2]) {
#pragma unroll
    for (int w = 0; w < EPL / 8; ++w) {
        v[4 * w + 0] = quant_bf16<0>(p.w[w], p.scale((8 * w + 0) / (D / 16)));
        v[4 * w + 1] = quant_bf16<1>(p.w[w], p.scale((8 * w + 2) / (D / 16)));
        v[4 * w + 2] = quant_bf16<2>(p.w[w], p.scale((8 * w + 4) / (D / 16)));
        v[4 * w + 3] = quant_bf16<3>(p.w[w], p.scale((8 * w + 6) / (D / 16)));
    }
}
template <int D, int EPL>
__device__ __forceinline__ void quant_decode(const QuantPiece<D, EPL>& p, q_f2_t (&v)[EPL / 2]) {
#pragma unroll
    for (int w = 0; w < EPL / 8; ++w) {
        v[4 * w + 0] = quant_f32<0>(p.w[w], p.scale((8 * w + 0) / (D / 16)));
        v[4 * w + 1] = quant_f32<1>(p.w[w], p.scale((8 * w + 2) / (D / 16)));
        v[4 * w + 2] = quant_f32<2>(p.w[w], p.scale((8 * w + 4) / (D / 16)));
        v[4 * w + 3] = quant_f32<3>(p.w[w], p.scale((8 * w + 6) / (D / 16)));
    }
}

// What a lane O lanes away holds.
template <int O>
__device__ __forceinline__ float from_lane_xor(float v) {
    if constexpr (O == 1) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0xB1, 0xF, 0xF, true));
    else if constexpr (O == 2) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, true));
    else if constexpr (O == 4) return __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x101F));
    else if constexpr (O == 8) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xF, 0xF, true));
    else if constexpr (O == 16) return __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401F));
    else return __shfl_xor(v, 32, kWave);
}
// Sum over the LPR lanes of a row, in every one of them.
template <int LPR>
__device__ __forceinline__ float row_sum(float p) {
    p += from_lane_xor<1>(p);
    if constexpr (LPR >= 4) p += from_lane_xor<2>(p);
    if constexpr (LPR >= 8)  // (the lanes of a quad hold the same by now: any lane of the other quad will do)
        p += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, p), 0x141, 0xF, 0xF, true));
    if constexpr (LPR >= 16) p += __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, p), 0x140, 0xF, 0xF, true));
    return p;
}
// N sums spread over the lanes that differ in bits O, O/2, .. LPR: each step sends half away and adds what comes, so a lane is left
// with N / (64 / LPR) of them, the ones from `off` on.
template <int N, int O, int LPR>
__device__ __forceinline__ void spread_sums(float* v, int lane, int& off) {
    if constexpr (O >= LPR) {
        const bool up = (lane & O) != 0;
#pragma unroll
        for (int i = 0; i < N / 2; ++i) {
            const float keep = up ? v[N / 2 + i] : v[i], send = up ? v[i] : v[N / 2 + i];
            v[i] = keep + from_lane_xor<O>(send);
        }
        off += up ? N / 2 : 0;
        spread_sums<N / 2, O / 2, LPR>(v, lane, off);
    }
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(kQuantThreads) quant_split_kernel(const DecodeArgs a) {
    constexpr int NT = kQuantThreads, NW = kQuantWaves, UNR = kQuantUnroll, EPL = quant_epl(G), LPR = D / EPL, RPW = kWave / LPR;
    constexpr int RPB = RPW * NW, TILE = RPB * UNR, PW = D + 4, RB = D / 2 + 16;
    extern __shared__ float smem[];
    __shared__ float red[2 * G * NW];
    const int CS = a.chunk + 1;
    float* xs = smem;               // [G][CS] logits, then attention weights
    float* ys = smem + G * CS;      // [G][CS] adjusted logits / tau, then their exponentials
    float* red_o = smem + 2 * G * CS;  // [NW][G*D]

    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, sub = lane / LPR, cl = lane % LPR;
    const int S = a.S;
    const uint32_t ui = blockIdx.x / (uint32_t)S, lb = ui / (uint32_t)a.H;
    const int64_t u = ui;
    const int s = (int)(blockIdx.x - ui * (uint32_t)S);
    const int h = (int)(ui - lb * (uint32_t)a.H), b = (int)(lb % (uint32_t)a.B), l = a.layer0 + (int)(lb / (uint32_t)a.B);
    const bool random = a.noise == kNoiseGumbel || a.noise == kNoiseGaussian;
    char* Ku = (char*)a.K + (size_t)u * a.cap * RB;
    char* Vu = (char*)a.V + (size_t)u * a.cap * RB;
    const T* qu = (const T*)a.q + (size_t)u * G * D;
    const T* knew = (const T*)a.k_new + (size_t)u * D;
    const T* vnew = (const T*)a.v_new + (size_t)u * D;
    int32_t* pu = a.pos + (size_t)u * a.cap;

    const uint64_t seed_b = random ? a.seeds[b] : 0;
    int q_pos = a.q_pos;
    float inv_tau = a.inv_tau;
    if (a.step) {  // as in the step over 16-bit caches
        const int t = max(*a.step, 1);
        q_pos = a.n0 + t - 1;
        inv_tau = 1.0f / schedule_tau(a.tau_init, a.dtau, min(t, a.T));
    }
    if (a.seq_q_pos) q_pos = a.seq_q_pos[b];
    if (a.seq_tau) inv_tau = 1.0f / a.seq_tau[b];
    const int len0 = a.len[u], m = len0 + 1;
    if (len0 < 0 || len0 >= a.cap || len0 > S * a.chunk) {  // no room for the new token: leave the unit alone, report it
        if (s == 0) {
            for (int c = tid; c < G * D; c += NT) a.out[u * G * D + c] = 0.0f;
            if (tid == 0) {
                atomicAdd(a.ws_err, 1);
                a.ws_m[u] = 0;
            }
        }
        return;
    }
    const int j0 = s * a.chunk, j1 = min(len0, j0 + a.chunk), cnt_c = max(j1 - j0, 0);
    const bool owner = s == S - 1;
    const int cnt = cnt_c + (owner ? 1 : 0);

    // ---- append (nobody reads the row back in this launch)
    if (owner) {
        if (tid < 32) {
            const int g = tid & 15;
            const size_t at = (size_t)len0 * RB;
            if (tid < 16) quant_group<T, D>((const char*)knew, Ku + at, g);
            else quant_group<T, D>((const char*)vnew, Vu + at, g);
        }
        if (tid == 2 * kWave) pu[len0] = q_pos;
    }

    // rows past the split re-read its last one; their logits are dropped, their weights are zero
    typedef QuantPiece<D, EPL> Piece;
    Piece cur[UNR], nxt[UNR];
    const int base0 = j0 + wv * RPW;
    auto load_tile = [&](const char* rows, int base, Piece(&p)[UNR]) {
#pragma unroll
        for (int i = 0; i < UNR; ++i) p[i].load(rows + (size_t)min(base + i * RPB + sub, j1 - 1) * RB, cl);
    };

    // ---- K: plain products into LDS
    {
        QuantQuery<T, EPL> q[G];
#pragma unroll
        for (int g = 0; g < G; ++g) q[g].load(qu + g * D + cl * EPL);
        if (base0 < j1) load_tile(Ku, base0, cur);
        for (int base = base0; base < j1; base += TILE) {
            if (base + TILE < j1) load_tile(Ku, base + TILE, nxt);
#pragma unroll
            for (int i = 0; i < UNR; ++i) {
                q_bf2_t kv[EPL / 2];
                quant_decode<D, EPL>(cur[i], kv);
                const int j = base + i * RPB + sub;
#pragma unroll
                for (int g = 0; g < G; ++g) {
                    const float p = row_sum<LPR>(q[g].dot(kv));
                    if (cl == g % LPR && j < j1) xs[g * CS + j - j0] = p;
                }
            }
#pragma unroll
            for (int i = 0; i < UNR; ++i) cur[i] = nxt[i];
        }
    }
    if (owner && wv == NW - 1) {  // the new token's
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float p = 0.0f;
            for (int c = lane; c < D; c += kWave) {
                float kq[2];
                if constexpr (__is_same(T, bf16_t)) kq[0] = bf16_lo(knew[c].bits), kq[1] = bf16_lo(qu[g * D + c].bits);
                else kq[0] = f16_lo(knew[c].bits), kq[1] = f16_lo(qu[g * D + c].bits);
                p = fmaf(kq[0], kq[1], p);
            }
            p = wave_sum(p);
            if (lane == 0) xs[g * CS + cnt_c] = p;
        }
    }
    if (base0 < j1) load_tile(Vu, base0, cur);  // in flight while the statistics are formed
    __syncthreads();

    // ---- position bias, logit adjustment, the two softmaxes' statistics (base 2)
    float mx[2 * G], sum[2 * G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        const int hq = h * G + g;
        const float slope = a.slopes ? a.slopes[hq] : 0.0f;
        const uint32_t rk = random ? row_key(unit_key(seed_b, (uint32_t)l, (uint32_t)hq), (uint32_t)q_pos) : 0u;
        float m0 = -INFINITY, m1 = -INFINITY;
        for (int t = tid; t < cnt; t += NT) {
            const int j = j0 + t, pj = t == cnt_c ? q_pos : pu[j];
            const int dist = t == cnt_c ? 0 : a.new_pos ? len0 - j : q_pos - pj;
            const float x = (xs[g * CS + t] * a.scale - slope * (float)dist) * kLog2e;
            const float y = (x + zeta_log2e(a.noise, rk, (uint32_t)pj)) * inv_tau;
            xs[g * CS + t] = x;
            ys[g * CS + t] = y;
            m0 = fmaxf(m0, x);
            m1 = fmaxf(m1, y);
        }
        mx[2 * g] = wave_max(m0);
        mx[2 * g + 1] = wave_max(m1);
        if (lane == 0) red[2 * G * wv + 2 * g] = mx[2 * g], red[2 * G * wv + 2 * g + 1] = mx[2 * g + 1];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2 * G; ++i) {
        mx[i] = red[i];
#pragma unroll
        for (int w = 1; w < NW; ++w) mx[i] = fmaxf(mx[i], red[2 * G * w + i]);
    }
    __syncthreads();
#pragma unroll
    for (int g = 0; g < G; ++g) {
        float s0 = 0.0f, s1 = 0.0f;
        for (int t = tid; t < cnt; t += NT) {
            const float p = hw_exp2(xs[g * CS + t] - mx[2 * g]), e = hw_exp2(ys[g * CS + t] - mx[2 * g + 1]);
            xs[g * CS + t] = p;
            ys[g * CS + t] = e;
            s0 += p;
            s1 += e;
        }
        s0 = wave_sum(s0);
        s1 = wave_sum(s1);
        if (lane == 0) red[2 * G * wv + 2 * g] = s0, red[2 * G * wv + 2 * g + 1] = s1;
    }
    __syncthreads();  // the weights too
#pragma unroll
    for (int i = 0; i < 2 * G; ++i) {
        sum[i] = red[i];
#pragma unroll
        for (int w = 1; w < NW; ++w) sum[i] += red[2 * G * w + i];
    }

    // ---- V
    float acc[G * EPL];
#pragma unroll
    for (int i = 0; i < G * EPL; ++i) acc[i] = 0.0f;
    for (int base = base0; base < j1; base += TILE) {
        if (base + TILE < j1) load_tile(Vu, base + TILE, nxt);
#pragma unroll
        for (int i = 0; i < UNR; ++i) {
            q_f2_t v[EPL / 2];
            quant_decode<D, EPL>(cur[i], v);
            const int j = base + i * RPB + sub;
#pragma unroll
            for (int g = 0; g < G; ++g) {
                const float p = j < j1 ? xs[g * CS + j - j0] : 0.0f;
#pragma unroll
                for (int e = 0; e < EPL / 2; ++e) {
                    acc[g * EPL + 2 * e] = fmaf(p, v[e].x, acc[g * EPL + 2 * e]);
                    acc[g * EPL + 2 * e + 1] = fmaf(p, v[e].y, acc[g * EPL + 2 * e + 1]);
                }
            }
        }
#pragma unroll
        for (int i = 0; i < UNR; ++i) cur[i] = nxt[i];
    }
    int off = 0;
    spread_sums<G * EPL, 32, LPR>(acc, lane, off);
    constexpr int LEFT = G * EPL / RPW;
#pragma unroll
    for (int i = 0; i < LEFT; ++i) {
        const int f = off + i;
        red_o[wv * G * D + (f / EPL) * D + cl * EPL + f % EPL] = acc[i];
    }
    __syncthreads();

    // ---- records for the merge
    float* we = a.ws_e + (size_t)u * G * a.cap;
    for (int t = tid; t < cnt; t += NT) {
        const int slot = t == cnt_c ? len0 : j0 + t;
#pragma unroll
        for (int g = 0; g < G; ++g) we[(size_t)g * a.cap + slot] = ys[g * CS + t];
    }
    float* part = a.ws_part + ((size_t)u * S + s) * G * PW;
    for (int c = tid; c < G * D; c += NT) {
        float o = red_o[c];
#pragma unroll
        for (int w = 1; w < NW; ++w) o += red_o[w * G * D + c];
        if (owner) {
            const uint32_t bits = vnew[c % D].bits;
            o = fmaf(xs[(c / D) * CS + cnt_c], __is_same(T, bf16_t) ? bf16_lo(bits) : f16_lo(bits), o);
        }
        part[(c / D) * PW + c % D] = o;
    }
    if (tid == 0) {
#pragma unroll
        for (int g = 0; g < G; ++g) *(float4*)(part + g * PW + D) = make_float4(mx[2 * g], sum[2 * g], mx[2 * g + 1], sum[2 * g + 1]);
        if (owner) a.ws_m[u] = m;
    }
}

// ---------------------------------------------------------------- eviction of 16-bit rows into 4-bit ones
constexpr int kQuantGatherRows = 64;
template <typename T, int D>
__global__ void __launch_bounds__(kQuantThreads) quant_gather_kernel(const GatherArgs g) {
    constexpr int RB = D / 2 + 16;
    const int64_t u = blockIdx.y + (int64_t)blockIdx.z * gridDim.y;
    if (u >= g.units) return;
    const int64_t ud = u + g.dst_unit0;
    const int tid = threadIdx.x, k = g.k, row0 = blockIdx.x * kQuantGatherRows;
    const int32_t* idx = g.idx + (size_t)u * k;
    for (int p = tid; p < 2 * kQuantGatherRows * 16; p += kQuantThreads) {
        const int t = p / (kQuantGatherRows * 16), q = p % (kQuantGatherRows * 16), i = row0 + q / 16;
        if (i >= k) continue;
        const int s = idx[i];
        if (s < 0 || s >= g.src_cap) continue;
        quant_group<T, D>((const char*)(t ? g.src_V : g.src_K) + ((size_t)u * g.src_cap + s) * D * 2, (char*)(t ? g.dst_V : g.dst_K) + ((size_t)ud * g.dst_cap + i) * RB,
                          q % 16);
    }
    if (tid < kQuantGatherRows && row0 + tid < k) {
        const int i = row0 + tid, s = idx[i];
        if (s >= 0 && s < g.src_cap) {
            g.dst_score[(size_t)ud * g.dst_cap + i] = g.src_score[(size_t)u * g.src_cap + s];
            g.dst_pos[(size_t)ud * g.dst_cap + i] = g.src_pos[(size_t)u * g.src_cap + s];
        }
    }
    if (blockIdx.x == 0 && tid == 0) g.dst_len[ud] = min(g.src_len[u], k);
}

template <typename T>
static hipError_t launch_quant_gather_t(const GatherArgs& g, int32_t d, const dim3& grid, hipStream_t stream) {
    if (d == 64) hipLaunchKernelGGL((quant_gather_kernel<T, 64>), grid, dim3(kQuantThreads), 0, stream, g);
    else if (d == 128) hipLaunchKernelGGL((quant_gather_kernel<T, 128>), grid, dim3(kQuantThreads), 0, stream, g);
    else if (d == 256) hipLaunchKernelGGL((quant_gather_kernel<T, 256>), grid, dim3(kQuantThreads), 0, stream, g);
    else return hipErrorInvalidValue;
    return hipGetLastError();
}
hipError_t launch_quant_gather(const GatherArgs& g, int32_t d, int32_t dtype, hipStream_t stream) {
    const unsigned gy = (unsigned)(g.units < 32768 ? g.units : 32768);
    const unsigned gz = (unsigned)((g.units + gy - 1) / gy);
    const dim3 grid((unsigned)((g.k + kQuantGatherRows - 1) / kQuantGatherRows), gy, gz);
    return dtype == KF_BF16 ? launch_quant_gather_t<bf16_t>(g, d, grid, stream) : launch_quant_gather_t<f16_t>(g, d, grid, stream);
}

// ---------------------------------------------------------------- host
static int quant_rpb(int32_t d, int32_t G) { return kWave / (d / quant_epl(G)) * kQuantWaves; }
static size_t quant_lds(int32_t G, int64_t chunk, int32_t d) { return (size_t)(2 * G * (chunk + 1) + kQuantWaves * G * d) * sizeof(float); }

// Most splits of a unit of up to m tokens (what the records are sized for): enough for 1024 workgroups in all, each of two
// rounds of rows at least, and as many as the logits in LDS ask for.
int32_t quant_max_splits(int64_t U, int32_t m, int32_t d, int32_t G) {
    const int64_t rows = m > 1 ? m - 1 : 1, rpb = quant_rpb(d, G);
    const int64_t fit = (int64_t)((kQuantLds / sizeof(float) - (size_t)kQuantWaves * G * d) / (2 * G) - 1) / rpb * rpb;
    const int64_t lo = (rows + fit - 1) / fit, hi = (rows + 2 * rpb - 1) / (2 * rpb);
    int64_t S = (1024 + U - 1) / U;
    if (S > hi) S = hi;
    if (S > kDecodeMaxSplits) S = kDecodeMaxSplits;
    if (S < lo) S = lo;
    return (int32_t)S;
}
DecodePlan plan_quant(int64_t U, int32_t m, int32_t d, int32_t G) {
    DecodePlan p;
    const int64_t rows = m > 1 ? m - 1 : 1, rpb = quant_rpb(d, G), S = quant_max_splits(U, m, d, G);
    p.chunk = (int32_t)(((rows + S - 1) / S + rpb - 1) / rpb * rpb);
    p.S = (int32_t)((rows + p.chunk - 1) / p.chunk);
    p.lds_bytes = quant_lds(G, p.chunk, d);
    return p;
}

template <typename T, int D>
static hipError_t launch_quant_split_d(const DecodeArgs& a, int64_t U, hipStream_t st) {
    const dim3 grid((unsigned)(U * a.S)), block(kQuantThreads);
    const size_t lds = quant_lds(a.G, a.chunk, D);
    if (lds > kQuantLds || a.S > kDecodeMaxSplits) return hipErrorInvalidValue;
    switch (a.G) {
        case 1: hipLaunchKernelGGL((quant_split_kernel<T, D, 1>), grid, block, lds, st, a); break;
        case 2: hipLaunchKernelGGL((quant_split_kernel<T, D, 2>), grid, block, lds, st, a); break;
        case 4: hipLaunchKernelGGL((quant_split_kernel<T, D, 4>), grid, block, lds, st, a); break;
        case 8: hipLaunchKernelGGL((quant_split_kernel<T, D, 8>), grid, block, lds, st, a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
hipError_t launch_quant_split(const DecodeArgs& a, int64_t U, int32_t d, int32_t dtype, hipStream_t stream) {
    if (dtype == KF_BF16_Q4) {
        if (d == 64) return launch_quant_split_d<bf16_t, 64>(a, U, stream);
        if (d == 128) return launch_quant_split_d<bf16_t, 128>(a, U, stream);
        if (d == 256) return launch_quant_split_d<bf16_t, 256>(a, U, stream);
    } else if (dtype == KF_F16_Q4) {
        if (d == 64) return launch_quant_split_d<f16_t, 64>(a, U, stream);
        if (d == 128) return launch_quant_split_d<f16_t, 128>(a, U, stream);
        if (d == 256) return launch_quant_split_d<f16_t, 256>(a, U, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace kf
