// Caches of 4 bits for gfx950: the decode step over them, and the eviction of 16-bit rows into them.
//
// A row of D elements is D/2 bytes of codes -- E2M1: sign, two exponent bits, one mantissa bit, i.e. 0 1/2 1 3/2 2 3 4 6 --
// and 16 scale bytes, one for every D/16 elements: a power of two, the smallest with which none of them is above 7 (what
// lies between 6 and 7 becomes 6, no further off than half the last step).  Powers of two keep a value of two significant bits
// exact in bf16, so the conversion instructions of the matrix formats (two codes and a scale in, two bf16 or fp32 out) do
// all of the decoding; and sixteen scales fill the 16 bytes that keep rows aligned.
//
// The step is that of kf_decode.hip, with the same arguments, workspace records and merge:
//   x_j = scale*<q, K_j> - slope*(q_pos - pos_j);  out = sum_j softmax(x)_j V_j;  f_j += softmax((x + zeta)/tau)_j
// A workgroup streams the rows [j0, j1) of one cached head: keys through the matrix cores, then values, of which a lane takes EPL
// elements of a row (16 bytes of codes, or 8 where several query heads need the registers).  The new token's own key and value
// enter as they were given, in 16 bits.  With a quarter to a third of the bytes of 16-bit rows the launch is close to being bound by
// its instructions as well as by bytes.  Steps in the slot layout, one launch: 2048 units x 1024 x 128 75 us (4.9 TB/s of rows, scores and
// positions), 2048 x 2048 x 128 139 us (5.2 TB/s); with 4 query heads 512 x 2048 x 128 71 us (2.6 TB/s).  Few units gain nothing by 4 bits:
// their chains of trips are as long, and 16-bit rows have a form for them that these have not (slot layout, 16 bits / 4 bits, replayed: 16 x
// 1024 x 256 14.9 / 13.9 us, 64 x 1024 x 128 16.3 / 17.8, 512 x 1024 x 128 48 / 30; ordered 13.3 / 18.6, 18.8 / 23.3, 78 / 43).  Non-temporal loads lose 20 %
// here: a cache line holds pieces of two rows' codes and scales, and is asked for more than once.
#include "kf_device.h"
#include "kf_internal.h"
#include "kf_merge.h"

namespace kf {

constexpr int kQuantThreads = 256;
constexpr int kQuantWaves = kQuantThreads / kWave;
constexpr int quant_unroll(int G) { return G == 2 ? 2 : 4; }  // rows a lane has in use, and as many on their way
constexpr size_t kQuantLds = 81920 - 1024;            // two workgroups on a compute unit at least
constexpr int quant_epl(int G) { return G >= 4 ? 16 : 32; }   // elements of a row that a lane takes
constexpr int quant_heads(int G) { return G >= 4 ? 4 : G; }   // query heads of a wave

typedef __bf16 q_bf2_t __attribute__((ext_vector_type(2)));
typedef _Float16 q_h2_t __attribute__((ext_vector_type(2)));
typedef unsigned short q_us2_t __attribute__((ext_vector_type(2)));
typedef float q_f2_t __attribute__((ext_vector_type(2)));
typedef __bf16 q_bf8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- encoding
// Scale byte of a group whose largest magnitude is `a`.
__device__ __forceinline__ uint32_t quant_scale(float a) {
    const uint32_t b = __float_as_uint(a), E = b >> 23;
    const int s = (int)E - 2 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return (uint32_t)min(max(s, 1), 252);
}
// Two elements -> two codes in byte SEL of `w`: the nearest, ties to the even one, at most 6 in magnitude.
template <typename T, int SEL>
__device__ __forceinline__ uint32_t quant_codes(uint32_t w, uint32_t pair, float scale) {
    if constexpr (__is_same(T, bf16_t)) return __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_bit_cast(q_bf2_t, pair), scale, SEL);
    else return __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, __builtin_bit_cast(q_h2_t, pair), scale, SEL);
}
// One group of N = D/16 elements at `src` (16 bits each) -> its codes and scale byte in the row at `dst`.  Magnitudes compare as
// 15-bit numbers, pair by pair; one conversion instruction makes two codes.  (Element by element in fp32, with the seven borders
// between codes, the eviction of 512 units of 1024 rows x 128 took 112 us, 87 so; a step of 16 heads x 1024 x 256 lost 3.2 of 10.7 us.)
template <typename T, int D>
__device__ __forceinline__ void quant_group(const char* src, char* dst, int g) {
    constexpr int N = D / 16, P = N / 2;
    uint32_t v[P];
    if constexpr (N == 4) {
        const uint2 r = *(const uint2*)(src + g * 8);
        v[0] = r.x, v[1] = r.y;
    } else {
#pragma unroll
        for (int i = 0; i < N / 8; ++i) {
            const uint4 r = ((const uint4*)(src + g * 2 * N))[i];
            v[4 * i] = r.x, v[4 * i + 1] = r.y, v[4 * i + 2] = r.z, v[4 * i + 3] = r.w;
        }
    }
    q_us2_t top = __builtin_bit_cast(q_us2_t, v[0] & 0x7FFF7FFFu);
#pragma unroll
    for (int i = 1; i < P; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(q_us2_t, v[i] & 0x7FFF7FFFu));
    const uint32_t most = max((uint32_t)top.x, (uint32_t)top.y);
    const bool bad = most >= (__is_same(T, bf16_t) ? 0x7F80u : 0x7C00u);  // an infinity or a NaN
    const float a = __is_same(T, bf16_t) ? __uint_as_float(most << 16) : f16_lo(most);
    const uint32_t s = bad ? 255u : quant_scale(a);
    const float scale = __uint_as_float(s << 23);
    uint32_t w[(N + 7) / 8];
#pragma unroll
    for (int i = 0; i < (N + 7) / 8; ++i) {
        w[i] = 0;
        w[i] = quant_codes<T, 0>(w[i], v[4 * i], scale);
        w[i] = quant_codes<T, 1>(w[i], v[4 * i + 1], scale);
        if constexpr (N > 4) {
            w[i] = quant_codes<T, 2>(w[i], v[4 * i + 2], scale);
            w[i] = quant_codes<T, 3>(w[i], v[4 * i + 3], scale);
        }
        if (bad) w[i] = 0x77777777u;
    }
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
    // codes at voff behind a base that the wave shares, scale bytes at soff
    __device__ __forceinline__ void load(const char* base, uint32_t voff, uint32_t soff) {
        if constexpr (W >= 4) {
#pragma unroll
            for (int i = 0; i < W / 4; ++i) {
                const uint4 r = *(const uint4*)(base + voff + 16 * i);
                w[4 * i] = r.x, w[4 * i + 1] = r.y, w[4 * i + 2] = r.z, w[4 * i + 3] = r.w;
            }
        } else {
            const uint2 r = *(const uint2*)(base + voff);
            w[0] = r.x, w[1] = r.y;
        }
        const char* sp = base + soff;
        if constexpr (SB == 8) {
            const uint2 r = *(const uint2*)sp;
            s[0] = r.x, s[1] = r.y;
        } else if constexpr (SB == 4) s[0] = *(const uint32_t*)sp;
        else if constexpr (SB == 2) s[0] = *(const uint16_t*)sp;
        else s[0] = *(const uint8_t*)sp;
    }
    // of the lane's g-th group; the conversions read the exponent bits of it alone, so that one shift will do
    __device__ __forceinline__ float scale(int g) const {
        const uint32_t b = s[g / 4];
        return __uint_as_float(g % 4 == 3 ? b >> 1 : b << (23 - 8 * (g % 4)));
    }
};
template <int SEL>
__device__ __forceinline__ q_bf2_t quant_bf16(uint32_t w, float s) { return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, s, SEL); }
template <int SEL>
__device__ __forceinline__ q_f2_t quant_f32(uint32_t w, float s) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, s, SEL); }

// Eight elements of a query as bf16, for the products with decoded pairs; a half's 11 significant bits are the sum of two.
template <typename T>
struct QuantQuery {
    static constexpr int TERMS = __is_same(T, f16_t) ? 2 : 1;
    uint4 q[TERMS];
    __device__ __forceinline__ void load(const T* p) {
        const uint4 r = *(const uint4*)p;
        if constexpr (TERMS == 1) {
            q[0] = r;
        } else {
            float f[8];
            unpack16<T>(r, f);
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint32_t a = __float_as_uint(f[2 * j]), b = __float_as_uint(f[2 * j + 1]);
                hi[j] = (a >> 16) | (b & 0xFFFF0000u);  // upper 8 significant bits; the rest is exact too
                const float ra = f[2 * j] - __uint_as_float(a & 0xFFFF0000u), rb = f[2 * j + 1] - __uint_as_float(b & 0xFFFF0000u);
                lo[j] = (__float_as_uint(ra) >> 16) | (__float_as_uint(rb) & 0xFFFF0000u);
            }
            q[0] = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            q[TERMS - 1] = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
    }
};
// The eight elements of word w of a piece, as pairs.
template <int D, int EPL>
__device__ __forceinline__ void quant_decode(const QuantPiece<D, EPL>& p, int w, q_bf2_t (&v)[4]) {
    v[0] = quant_bf16<0>(p.w[w], p.scale((8 * w + 0) / (D / 16)));
    v[1] = quant_bf16<1>(p.w[w], p.scale((8 * w + 2) / (D / 16)));
    v[2] = quant_bf16<2>(p.w[w], p.scale((8 * w + 4) / (D / 16)));
    v[3] = quant_bf16<3>(p.w[w], p.scale((8 * w + 6) / (D / 16)));
}
template <int D, int EPL>
__device__ __forceinline__ void quant_decode(const QuantPiece<D, EPL>& p, int w, q_f2_t (&v)[4]) {
    v[0] = quant_f32<0>(p.w[w], p.scale((8 * w + 0) / (D / 16)));
    v[1] = quant_f32<1>(p.w[w], p.scale((8 * w + 2) / (D / 16)));
    v[2] = quant_f32<2>(p.w[w], p.scale((8 * w + 4) / (D / 16)));
    v[3] = quant_f32<3>(p.w[w], p.scale((8 * w + 6) / (D / 16)));
}

// What a lane O lanes away holds.
template <int O>
__device__ __forceinline__ float from_lane_xor(float v) {
    if constexpr (O == 2) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x4E, 0xF, 0xF, true));
    else if constexpr (O == 4) return __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x101F));
    else if constexpr (O == 8) return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), 0x128, 0xF, 0xF, true));
    else if constexpr (O == 16) return __builtin_bit_cast(float, __builtin_amdgcn_ds_swizzle(__builtin_bit_cast(int, v), 0x401F));
    else return __shfl_xor(v, 32, kWave);
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

// The workgroup: NT / 64 waves over the rows [j0, j1), or, with 8 query heads, four over the rows for heads 0-3 and four for heads
// 4-7 (a row comes from the cache the second time; 8 heads in one wave would take 128 registers of sums).
template <typename T, int D, int G>
__device__ __forceinline__ void quant_block(const DecodeArgs& a) {
    constexpr int UNR = quant_unroll(G), EPL = quant_epl(G), HG = quant_heads(G), HS = G / HG, NT = kQuantThreads * HS;
    constexpr int NW = kQuantWaves, WA = NT / kWave, LPR = D / EPL, RPW = kWave / LPR, RPB = RPW * NW, TILE = RPB * UNR;
    constexpr int PW = D + 4, RB = D / 2 + 16;
    extern __shared__ float smem[];
    __shared__ float red[2 * WA], red_s[2 * WA];
    __shared__ float stat[4 * G];  // per query head: max x, sum p, max y, sum e
    __shared__ unsigned long long evict_min[WA];
    __shared__ int evict_slot;
    __shared__ float new_score;
    const int CS = a.chunk + 1;
    float* xs = smem;                  // [G][CS] logits, then attention weights
    float* ys = smem + G * CS;         // [G][CS] adjusted logits / tau, then their exponentials
    int32_t* ps = (int32_t*)(smem + 2 * G * CS);              // [CS] positions (several query heads)
    float* red_o = smem + (2 * G + (G > 1 ? 1 : 0)) * CS;     // [NW][G*D]

    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), sub = lane / LPR, cl = lane % LPR;
    const int wr = wv % NW, g0 = wv / NW * HG;  // the wave's share of the rows, its first head
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
    float* fu = a.score + (size_t)u * a.cap;
    int32_t* pu = a.pos + (size_t)u * a.cap;

    // The words of device memory that the launch depends on, asked for together; an absent one is read from where something else lies.
    uint64_t seed_b = uniform_load(random ? a.seeds + b : (const uint64_t*)a.q);
    int32_t step_now = uniform_load(a.step ? a.step : a.len);
    int32_t seq_pos = uniform_load(a.seq_q_pos ? a.seq_q_pos + b : a.len);
    float seq_tau = uniform_load(a.seq_tau ? a.seq_tau + b : (const float*)a.len);
    int len0 = uniform_load(a.len + u);
    asm volatile("" : "+s"(seed_b), "+s"(step_now), "+s"(seq_pos), "+s"(seq_tau), "+s"(len0));  // (read once)
    int q_pos = a.q_pos;
    float inv_tau = a.inv_tau;
    if (a.step) {  // as in the step over 16-bit caches
        const int t = max(step_now, 1);
        q_pos = a.n0 + t - 1;
        inv_tau = 1.0f / schedule_tau(a.tau_init, a.dtau, min(t, a.T));
    }
    if (a.seq_q_pos) q_pos = seq_pos;
    if (a.seq_tau) inv_tau = 1.0f / seq_tau;
    const int m = len0 + 1;
    if (len0 < 0 || len0 >= a.cap || len0 > S * a.chunk) {  // no room for the new token: leave the unit alone, report it
        if (s == 0) {
            for (int c = tid; c < G * D; c += NT) a.out[u * G * D + c] = 0.0f;
            if (tid == 0) {
                atomicAdd(a.ws_err, 1);
                a.ws_m[u] = 0;
                if (a.fuse_k > 0 && len0 > a.fuse_k + 1) atomicAdd(a.ws_err, 1);  // the selection would have refused it as well
            }
        }
        return;
    }
    const int j0 = s * a.chunk, j1 = min(len0, j0 + a.chunk), cnt_c = max(j1 - j0, 0);
    const bool owner = s == S - 1;
    const int cnt = cnt_c + (owner ? 1 : 0);
    // a step in one launch (one split, slot layout): a unit one token over its budget evicts here, and the new token goes
    // straight into the freed slot
    const bool over = a.fuse_k > 0 && m > a.fuse_k, evict_here = over && m == a.fuse_k + 1;
    auto store_new = [&](int slot) {  // called by all; nobody reads the row back in this launch
        if (tid < 32) {
            if (tid < 16) quant_group<T, D>((const char*)knew, Ku + (size_t)slot * RB, tid);
            else quant_group<T, D>((const char*)vnew, Vu + (size_t)slot * RB, tid - 16);
        }
        if (tid == 2 * kWave) pu[slot] = q_pos;
    };
    if (owner && !evict_here) store_new(len0);

    // Rows past the split re-read its last one; their logits are dropped, their weights are zero.  A tile that lies inside is
    // addressed by one scalar base and offsets that stay the same.
    typedef QuantPiece<D, EPL> Piece;
    Piece ping[UNR], pong[UNR];
    const int base0 = j0 + wr * RPW;
    const uint32_t voff = (uint32_t)(sub * RB + cl * (EPL / 2)), soff = (uint32_t)(sub * RB + D / 2 + cl * Piece::SB);
    auto load_tile = [&](const char* rows, int base, Piece(&p)[UNR]) {
        if (base + (UNR - 1) * RPB + RPW <= j1) {
            const char* at = rows + (size_t)base * RB;
#pragma unroll
            for (int i = 0; i < UNR; ++i) p[i].load(at + i * RPB * RB, voff, soff);
        } else {
#pragma unroll
            for (int i = 0; i < UNR; ++i) {
                const uint32_t at = (uint32_t)((min(base + i * RPB + sub, j1 - 1) - j0) * RB);  // (at least 0: offsets are unsigned)
                p[i].load(rows + (size_t)j0 * RB, at + cl * (EPL / 2), at + D / 2 + cl * Piece::SB);
            }
        }
    };
    // The V stream alternates between two sets of registers, one under way while the other is used.
    auto stream = [&](const char* rows, auto use) {  // the first tile is in `ping`, or on its way there
        int base = base0;
        while (base < j1) {
            if (base + TILE < j1) load_tile(rows, base + TILE, pong);
            use(base, ping);
            base += TILE;
            if (base >= j1) break;
            if (base + TILE < j1) load_tile(rows, base + TILE, ping);
            use(base, pong);
            base += TILE;
        }
    };

    // ---- K: plain products into LDS
    {
        // On the matrix cores, 16 rows by 16 heads (the others zero) a tile.  Lane (i, kb) holds the kb-th quarter of row i, D/4 codes and four scale bytes; the order of a contraction is free, so word w of the
        // quarters is one 16x16x32 product, with the queries laid out alike.  A lane gets the logits of head i, rows 4*kb .. +3.
        constexpr int QW = D / 32, TERMS = QuantQuery<T>::TERMS;
        typedef QuantPiece<D, D / 4> Quarter;
        const int i16 = lane & 15, kb = lane >> 4;
        uint4 bq[TERMS][QW];
#pragma unroll
        for (int w = 0; w < QW; ++w) {
            QuantQuery<T> one;
            one.load(qu + min(i16, G - 1) * D + kb * (D / 4) + 8 * w);
#pragma unroll
            for (int t = 0; t < TERMS; ++t)
                bq[t][w] = i16 < G ? one.q[t] : make_uint4(0u, 0u, 0u, 0u);
        }
        constexpr int KT = 16 * WA;
        const char* rows = Ku + (size_t)j0 * RB;
        auto load = [&](int base, Quarter& q) {
            const uint32_t at = (uint32_t)((min(base + i16, j1 - 1) - j0) * RB);
            q.load(rows, at + kb * (D / 8), at + D / 2 + 4 * kb);
        };
        auto logits = [&](int base, const Quarter& q) {
            f32x4_t acc = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
            for (int w = 0; w < QW; ++w) {
                q_bf2_t kv[4];
                quant_decode<D, D / 4>(q, w, kv);
                const q_bf8_t av = __builtin_bit_cast(q_bf8_t, make_uint4(__builtin_bit_cast(uint32_t, kv[0]), __builtin_bit_cast(uint32_t, kv[1]),
                                                                         __builtin_bit_cast(uint32_t, kv[2]), __builtin_bit_cast(uint32_t, kv[3])));
#pragma unroll
                for (int t = 0; t < TERMS; ++t) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(av, __builtin_bit_cast(q_bf8_t, bq[t][w]), acc, 0, 0, 0);
            }
            if (i16 < G) {
                float* xg = xs + i16 * CS + base - j0 + 4 * kb;
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (base + 4 * kb + r < j1) xg[r] = acc[r];
            }
        };
        constexpr int KU = D >= 256 ? 2 : 4;  // tiles a wave has in flight
        Quarter q[KU];
        const int kbase = j0 + wv * 16;
#pragma unroll
        for (int i = 0; i < KU; ++i)
            if (kbase + i * KT < j1) load(kbase + i * KT, q[i]);
        // Several heads: the positions, which the logits' adjustment asks for, on their way behind the first tiles.  (A wave
        // adjusts a head's tokens, stride after stride, and each waited for a trip to memory: 512 units x 2048 x 128 with 4 query
        // heads 89.6 us, 79.7 so; one head has four waves, a quarter of the strides, and gains nothing.)
        if constexpr (G > 1) {
            for (int t0 = tid; t0 < cnt_c; t0 += 4 * NT) {
                int32_t pj[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) pj[i] = pu[j0 + min(t0 + i * NT, cnt_c - 1)];
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (t0 + i * NT < cnt_c) ps[t0 + i * NT] = pj[i];
            }
            if (tid == 0) ps[cnt_c] = q_pos;
        }
        for (int base = kbase; base < j1; base += KU * KT) {
#pragma unroll
            for (int i = 0; i < KU; ++i) {
                if (base + i * KT >= j1) break;
                logits(base + i * KT, q[i]);
                if (base + (KU + i) * KT < j1) load(base + (KU + i) * KT, q[i]);
            }
        }
    }
    if (owner && wv == WA - 1) {  // the new token's
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float p = 0.0f;
#pragma unroll
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
    if (base0 < j1) load_tile(Vu, base0, ping);  // under way while the statistics are formed
    __syncthreads();

    // ---- position bias, logit adjustment, the two softmaxes' statistics (base 2)
    // A wave takes a head, or a share of one's tokens: WPH waves a head.
    constexpr int WPH = WA / G;
    static_assert(WPH >= 1, "a wave for each head");
    {
        const int g = wv / WPH, t0 = wv % WPH * kWave + lane, hq = h * G + g;
        float *xg = xs + g * CS, *yg = ys + g * CS;
        const float slope = a.slopes ? a.slopes[hq] : 0.0f;
        const uint32_t rk = random ? row_key(unit_key(seed_b, (uint32_t)l, (uint32_t)hq), (uint32_t)q_pos) : 0u;
        float m0 = -INFINITY, m1 = -INFINITY;
        for (int t = t0; t < cnt; t += kWave * WPH) {
            const int pj = G > 1 ? ps[t] : t == cnt_c ? q_pos : pu[j0 + t];
            const int dist = t == cnt_c ? 0 : a.new_pos ? len0 - j0 - t : q_pos - pj;
            const float x = (xg[t] * a.scale - slope * (float)dist) * kLog2e;
            const float y = (x + zeta_log2e(a.noise, rk, (uint32_t)pj)) * inv_tau;
            xg[t] = x;
            yg[t] = y;
            m0 = fmaxf(m0, x);
            m1 = fmaxf(m1, y);
        }
        m0 = wave_max(m0);
        m1 = wave_max(m1);
        if constexpr (WPH > 1) {
            if (lane == 0) red[2 * wv] = m0, red[2 * wv + 1] = m1;
            __syncthreads();
            m0 = red[2 * g * WPH], m1 = red[2 * g * WPH + 1];
#pragma unroll
            for (int w = 1; w < WPH; ++w) m0 = fmaxf(m0, red[2 * (g * WPH + w)]), m1 = fmaxf(m1, red[2 * (g * WPH + w) + 1]);
        }
        float s0 = 0.0f, s1 = 0.0f;
        for (int t = t0; t < cnt; t += kWave * WPH) {
            const float p = hw_exp2(xg[t] - m0), e = hw_exp2(yg[t] - m1);
            xg[t] = p;
            yg[t] = e;
            s0 += p;
            s1 += e;
        }
        s0 = wave_sum(s0);
        s1 = wave_sum(s1);
        if (lane == 0) {
            red_s[2 * wv] = s0, red_s[2 * wv + 1] = s1;
            if (wv % WPH == 0) stat[4 * g] = m0, stat[4 * g + 2] = m1;
        }
    }
    __syncthreads();  // the weights too
    if (tid < 2 * G) {  // (read behind the barrier that follows the V stream)
        float r = red_s[2 * (tid / 2) * WPH + (tid & 1)];
#pragma unroll
        for (int w = 1; w < WPH; ++w) r += red_s[2 * ((tid / 2) * WPH + w) + (tid & 1)];
        stat[4 * (tid / 2) + 1 + 2 * (tid & 1)] = r;
    }

    // ---- V
    float acc[HG * EPL];
#pragma unroll
    for (int i = 0; i < HG * EPL; ++i) acc[i] = 0.0f;
    stream(Vu, [&](int base, const Piece(&p)[UNR]) {
#pragma unroll
        for (int i = 0; i < UNR; ++i) {
            const int j = base + i * RPB + sub;
            float weight[HG];
#pragma unroll
            for (int g = 0; g < HG; ++g) {
                weight[g] = xs[(g0 + g) * CS + min(j, j1 - 1) - j0];  // (no branch for each)
                weight[g] = j < j1 ? weight[g] : 0.0f;
            }
#pragma unroll
            for (int w = 0; w < EPL / 8; ++w) {
                q_f2_t v[4];
                quant_decode<D, EPL>(p[i], w, v);
#pragma unroll
                for (int g = 0; g < HG; ++g) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        acc[g * EPL + 8 * w + 2 * e] = fmaf(weight[g], v[e].x, acc[g * EPL + 8 * w + 2 * e]);
                        acc[g * EPL + 8 * w + 2 * e + 1] = fmaf(weight[g], v[e].y, acc[g * EPL + 8 * w + 2 * e + 1]);
                    }
                }
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    });
    int off = 0;
    spread_sums<HG * EPL, 32, LPR>(acc, lane, off);
    constexpr int LEFT = HG * EPL / RPW;
#pragma unroll
    for (int i = 0; i < LEFT; ++i) {
        const int f = off + i;
        red_o[wr * G * D + (g0 + f / EPL) * D + cl * EPL + f % EPL] = acc[i];
    }
    __syncthreads();
    auto output = [&](int c) {  // element c of [G][D], un-normalised
        float o = red_o[c];
#pragma unroll
        for (int w = 1; w < NW; ++w) o += red_o[w * G * D + c];
        if (owner) {
            const uint32_t bits = vnew[c % D].bits;
            o = fmaf(xs[(c / D) * CS + cnt_c], __is_same(T, bf16_t) ? bf16_lo(bits) : f16_lo(bits), o);
        }
        return o;
    };
    float* we = a.ws_e + (size_t)u * G * a.cap;
    if (S > 1) {  // ---- records for the merge
        for (int t = tid; t < cnt; t += NT) {
            const int slot = t == cnt_c ? len0 : j0 + t;
#pragma unroll
            for (int g = 0; g < G; ++g) we[(size_t)g * a.cap + slot] = ys[g * CS + t];
        }
        float* part = a.ws_part + ((size_t)u * S + s) * G * PW;
        for (int c = tid; c < G * D; c += NT) part[(c / D) * PW + c % D] = output(c);
        if (tid < 4 * G) part[(tid >> 2) * PW + D + (tid & 3)] = stat[tid];
        if (tid == 0 && owner) a.ws_m[u] = m;
        return;
    }
    // ---- the whole unit is here: scores, outputs, and the eviction of a step in one launch
    float inv[G];
#pragma unroll
    for (int g = 0; g < G; ++g) inv[g] = 1.0f / stat[4 * g + 3];
    unsigned long long best = ~0ull;  // smallest candidate: lowest score, of equal ones the highest position
    int best_slot = -1;
    for (int t = tid; t < cnt; t += NT) {
        const int slot = t;  // (j0 is 0, the new token's place len0 is cnt_c)
        float df = 0.0f;
#pragma unroll
        for (int g = 0; g < G; ++g) df = fmaf(ys[g * CS + t], inv[g], df);
        if (evict_here) {
            float f_new = df;
            int pj = q_pos;
            if (t == cnt_c) {
                new_score = df;
            } else {
                f_new = fu[slot] + df;
                fu[slot] = f_new;
                pj = pu[slot];
            }
            if (pj <= q_pos - a.fuse_w) {
                const unsigned long long pack = ((unsigned long long)float_key(f_new) << 32) | (uint32_t)(~(uint32_t)pj);
                if (pack < best) {
                    best = pack;
                    best_slot = slot;
                }
            }
        } else if (a.shared) {
            we[slot] = df;  // summed over the layers by the launch that follows
        } else if (t == cnt_c) {
            fu[slot] = df;
        } else {
            unsafeAtomicAdd(&fu[slot], df);  // no round trip; one add per address
        }
    }
    for (int c = tid; c < G * D; c += NT) a.out[u * G * D + c] = output(c) / stat[4 * (c / D) + 1];
    if (!evict_here) {
        if (tid == 0) {
            a.len[u] = m;
            if (a.shared) a.ws_m[u] = m;
            if (over) atomicAdd(a.ws_err, 1);  // more than one token over budget: appended, not evicted, reported
        }
        if (a.fuse_idx && !over) {
            int32_t* idx = a.fuse_idx + (size_t)u * a.fuse_k;
            for (int i = tid; i < a.fuse_k; i += NT) idx[i] = i < m ? i : -1;
        }
        return;
    }
    const unsigned long long mine = best;
    best = wave_min(best);
    if (lane == 0) evict_min[wv] = best;
    if (tid == 0) evict_slot = -1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < WA; ++i) best = evict_min[i] < best ? evict_min[i] : best;
    if (best != ~0ull && mine == best) evict_slot = best_slot;  // positions are unique: one lane
    __syncthreads();
    const int e = evict_slot, k = a.fuse_k;
    if (e < 0) {  // nothing lies outside the window: append after all, leave the unit one over budget and report it
        store_new(len0);
        if (tid == 2 * kWave) {
            fu[len0] = new_score;
            a.len[u] = m;
            atomicAdd(a.ws_err, 1);
        }
        return;
    }
    if (e != len0) {  // e == len0: the new token itself leaves (only without a recent window)
        store_new(e);
        if (tid == 2 * kWave) fu[e] = new_score;
    }
    if (a.fuse_idx) {
        int32_t* idx = a.fuse_idx + (size_t)u * k;
        for (int i = tid; i < k; i += NT) idx[i] = i == e ? k : i;
    }
    if (tid == 0) a.len[u] = k;
}

template <typename T, int D, int G>
__global__ void __launch_bounds__(kQuantThreads* G / quant_heads(G), 4) quant_step_kernel(const DecodeArgs a) {
    quant_block<T, D, G>(a);
    if (a.step_inc && threadIdx.x == 0) {  // step number in device memory: the workgroup that is done last moves it on
        if (atomicAdd(a.ws_ticket, 1) == (int)gridDim.x - 1) {
            *a.ws_ticket = 0;
            *a.step_inc += 1;
        }
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
static size_t quant_lds(int32_t G, int64_t chunk, int32_t d) { return (size_t)((2 * G + (G > 1 ? 1 : 0)) * (chunk + 1) + kQuantWaves * G * d) * sizeof(float); }

// Fewest and most splits of a unit of so many rows (the records are sized for the most): as many as the logits in LDS ask for, and
// as many as keep two rounds of rows for each, up to 2048 workgroups in all and 63 more than the fewest.  That bound is for few long units: the
// model below knows no price of a split in the merge, and would take 100 to 256 there, which lose (slot layout, best split / with the bound / without):
// 1 unit x 32000 x 128, 8 heads 48 splits 45 us, 91 51, 250 87; 2 x 32768 x 256, 8 heads 48 67, 108 89, 256 166; 4 x 16384 x 128, 4 heads
// 47 30, 64 32, 256 58; 1 x 40000 x 128 90 25, 70 26, 209 29; 8 x 40000 x 128 63 34, 63 34, 125 37.
static void quant_split_range(int64_t U, int64_t rows, int32_t d, int32_t G, int64_t* lo, int64_t* hi) {
    const int64_t rpb = quant_rpb(d, G);
    const int64_t fit = (int64_t)((kQuantLds / sizeof(float) - (size_t)kQuantWaves * G * d) / (2 * G + 1) - 1) / rpb * rpb;
    *lo = (rows + fit - 1) / fit;
    *hi = (rows + 2 * rpb - 1) / (2 * rpb);
    const int64_t most = (2048 + U - 1) / U;
    if (*hi > most) *hi = most;
    if (*hi > kDecodeMaxSplits) *hi = kDecodeMaxSplits;
    if (*hi > *lo + 63) *hi = *lo + 63;
    if (*hi < *lo) *hi = *lo;
}
int32_t quant_max_splits(int64_t U, int32_t m, int32_t d, int32_t G) {
    int64_t lo, hi;
    quant_split_range(U, m > 1 ? m - 1 : 1, d, G, &lo, &hi);
    return (int32_t)hi;
}
DecodePlan plan_quant(int64_t U, int32_t m, int32_t d, int32_t G) {
    DecodePlan p;
    int64_t lo, hi;
    const int64_t rows = m > 1 ? m - 1 : 1, rpb = quant_rpb(d, G);
    quant_split_range(U, rows, d, G, &lo, &hi);
    // A launch runs in rounds of as many workgroups as fit (registers: 16 waves on a compute unit; LDS); one of r workgroups on a
    // compute unit takes its chain of trips to memory and a time by its rows that falls short of proportion for small
    // r; splits add the launch that merges them.  Slot layout, replayed graphs, microseconds (the one taken first): 256 units x 4096 x 128,
    // 2 heads 4 splits 57, 2 62, 8 60; 512 x 2048 x 128, 4 heads 4 72, 3 70, 2 76; 128 x 4000 x 128 8 32, 4 32, 2 41; 16 x 1024 x 256 16
    // 14.6, 8 14.3, 2 19.5; 448 x 1024 x 256 1 38, 2 42.  Where the model falls short: few short units, whose one workgroup it takes to
    // be cheaper than it is (32 x 1024 x 128 1 18.3, 6 14.0; 64 x 2048 x 64 1 25.5, 6 16.7), and few units with 4 or 8 heads (8 x 5000 x
    // 128, 4 heads 53 27.5, 23 24.1; 64 x 300 x 256, 8 heads 7 25.6, 4 21.4).
    const double fixed = 6.0, row = (G == 1 ? 3.4e-5 : G == 2 ? 4e-5 : G == 4 ? 5.6e-5 : 1.1e-4) * (d / 2 + 16);
    double best = 0.0;
    for (int64_t S = lo; S <= hi; ++S) {
        const int64_t chunk = ((rows + S - 1) / S + rpb - 1) / rpb * rpb, n = (rows + chunk - 1) / chunk;
        const size_t lds = quant_lds(G, chunk, d);
        if (lds > kQuantLds) continue;
        int64_t fit = (int64_t)(163840 / (lds + 1024));
        if (fit > (G == 8 ? 2 : 4)) fit = G == 8 ? 2 : 4;
        const int64_t each = 256 * fit, full = U * n / each, left = (U * n - full * each + 255) / 256;
        auto round = [&](int64_t r) { return fixed + row * (double)(chunk * (r + 1)); };
        const double cost = (double)full * round(fit) + (left ? round(left) : 0.0) + (n > 1 ? 5.0 + 0.01 * (double)U : 0.0);
        if (best == 0.0 || cost < best) {
            best = cost;
            p.S = (int32_t)n;
            p.chunk = (int32_t)chunk;
        }
    }
    p.lds_bytes = quant_lds(G, p.chunk, d);
    return p;
}

template <typename T, int D>
static hipError_t launch_quant_step_d(const DecodeArgs& a, int64_t U, hipStream_t st) {
    const dim3 grid((unsigned)(U * a.S)), block(kQuantThreads);
    const size_t lds = quant_lds(a.G, a.chunk, D);
    if (lds > kQuantLds || a.S > kDecodeMaxSplits) return hipErrorInvalidValue;
    switch (a.G) {
        case 1: hipLaunchKernelGGL((quant_step_kernel<T, D, 1>), grid, block, lds, st, a); break;
        case 2: hipLaunchKernelGGL((quant_step_kernel<T, D, 2>), grid, block, lds, st, a); break;
        case 4: hipLaunchKernelGGL((quant_step_kernel<T, D, 4>), grid, block, lds, st, a); break;
        case 8: hipLaunchKernelGGL((quant_step_kernel<T, D, 8>), grid, 2 * kQuantThreads, lds, st, a); break;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}
hipError_t launch_quant_step(const DecodeArgs& a, int64_t U, int32_t d, int32_t dtype, hipStream_t stream) {
    if (dtype == KF_BF16_Q4) {
        if (d == 64) return launch_quant_step_d<bf16_t, 64>(a, U, stream);
        if (d == 128) return launch_quant_step_d<bf16_t, 128>(a, U, stream);
        if (d == 256) return launch_quant_step_d<bf16_t, 256>(a, U, stream);
    } else if (dtype == KF_F16_Q4) {
        if (d == 64) return launch_quant_step_d<f16_t, 64>(a, U, stream);
        if (d == 128) return launch_quant_step_d<f16_t, 128>(a, U, stream);
        if (d == 256) return launch_quant_step_d<f16_t, 256>(a, U, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace kf
