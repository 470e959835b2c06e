// Attention over prompts for gfx950: causal, grouped heads, sequences of their own lengths.
//
//   x_ij = scale*<q_i, k_j> - slope*(p_i - j)    j <= p_i = i + nk - nq        (query i of nq, key j of nk)
//   out_i = sum_j exp(x_ij - m_i) v_j / sum_j exp(x_ij - m_i)
//
// One pass over the keys with a running reference m and sum (in 32 bits); rows of both are never stored.  A wave takes 32 rows --
// a row is a query of one of the G heads that share a cached head, head by head inside a position, so that a tile of keys serves
// all of them -- and forms S^T = K Q^T and O^T = V^T P^T in tiles of 32 x 32: a lane then owns one row in both, its maximum and sum
// need one exchange between the wave's halves, and the exponentials, rounded to the element type, are the second product's operand as
// they lie.  (The order of the keys inside a product is free; the values' operand is read transposed from LDS in the same order.)
// Tiles of K and V go from memory straight to LDS, two buffers, swizzled so that both ways of reading meet each bank once.
//
// What bounds it: many rows, the matrix cores beside the vector unit (128 elements a row: 512 operations of the one for each exponential,
// sum and rounding of the other), and the power they draw.  8 x 32 heads x 4096 x 128 bf16, causal: 1180 us, 930 TFLOP/s (a product of
// 8192^3: 1155 to 1394); with a position bias, far tiles left out, 887; 8 heads of 8 x 512 rows at the end of 8192 keys 511 us, 1045 TFLOP/s; 256
// elements 760 (one wave a SIMD: a third of its cycles wait for data or a barrier), 64 elements 765 (the vector unit is busy two thirds of the
// cycles, the matrix cores one), fp32 79 (a product of 8192^3: 154).  Counters: no bank conflicts in LDS; 128 elements: matrix cores and vector unit
// each busy 45 % of the cycles; inputs of zeros run 18 % faster, which is power.  Few rows: the chain of a walk, 8 us for 1000 keys, and the join; 16 x 2048 x 128 40 us.
//
// Steps of 8 x 32 x 4096 x 128: tiles by way of registers, which spilled, 3133 us; infinities and NaNs of edge tiles taken out in LDS instead
// of beside every product 1328; direct loads to LDS 1245; keys a step ahead of the values 1190.  Tried, no gain: tiles of 32 keys (3 to 5 % more),
// workgroups of 256 rows (5 % less for 16384 keys, more for causal ones of 4096), wave priorities, three or four buffers, orders of
// instructions laid down by hand, two accumulators a block of logits (8 % more).
#include "kf_device.h"
#include "kf_internal.h"
#include "kf_prefill.h"

namespace kf {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) char lds_char;

// 16 bytes a lane from memory to LDS, at `lds` (the wave's) + 16 * lane.  The compiler does not know of them: whoever reads them waits for
// vmcnt(0) and the workgroup first.  (Its own form of this waits for all of them ahead of any read of LDS.)
__device__ __forceinline__ void to_lds(uint32_t lds, const char* base, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(off), "s"(base) : "memory");
}
__device__ __forceinline__ void to_lds(uint32_t lds, const char* p) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(p) : "memory");
}

// What a workgroup does: WR waves of 32 rows, times WK waves that share each tile's keys; SB blocks of 32 keys are a step of a wave, NB are
// a tile.
template <int WR_, int WK_, int SB_, int NB_>
struct AttendShape {
    static constexpr int WR = WR_, WK = WK_, SB = SB_, NB = NB_;
};

template <typename T>
__device__ __forceinline__ uint32_t pack_pair(float a, float b);
template <>
__device__ __forceinline__ uint32_t pack_pair<bf16_t>(float a, float b) { return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b}); }
template <>
__device__ __forceinline__ uint32_t pack_pair<f16_t>(float a, float b) { return __builtin_bit_cast(uint32_t, f16x2{(_Float16)a, (_Float16)b}); }

// A 16-byte piece with zeros in the place of infinities and NaNs; whether there were any.
template <typename T>
__device__ __forceinline__ bool clean_piece(u32x4_t& v) {
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (sizeof(T) == 4) {
            const bool odd = (v[i] & 0x7F800000u) == 0x7F800000u;
            v[i] = odd ? 0u : v[i];
            bad |= odd;
        } else {
            constexpr uint32_t e = __is_same(T, bf16_t) ? 0x7F80u : 0x7C00u;
            const bool lo = (v[i] & e) == e, hi = (v[i] & (e << 16)) == e << 16;
            v[i] = (lo ? 0u : v[i] & 0xFFFFu) | (hi ? 0u : v[i] & 0xFFFF0000u);
            bad |= lo || hi;
        }
    }
    return bad;
}

// Magnitudes in the order of their bits: the largest or the least (of two 16-bit ones in a word, in either half), and the number.
template <typename T, bool LEAST>
__device__ __forceinline__ uint32_t piece_magnitude(const u32x4_t& v, uint32_t m) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t lo = sizeof(T) == 4 ? v[i] & 0x7FFFFFFFu : v[i] & 0x7FFFu, hi = sizeof(T) == 4 ? lo : v[i] >> 16 & 0x7FFFu;
        m = LEAST ? min(m, min(lo, hi)) : max(m, max(lo, hi));
    }
    return m;
}
template <typename T>
__device__ __forceinline__ float magnitude(uint32_t m) {
    if constexpr (sizeof(T) == 4) return __uint_as_float(m);
    else return __is_same(T, bf16_t) ? __uint_as_float(m << 16) : (float)__builtin_bit_cast(_Float16, (uint16_t)m);
}

// Largest of a lane's and its partner's in the wave's other half.
__device__ __forceinline__ float half_max(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
__device__ __forceinline__ float half_sum(float v) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(x[0]) + __uint_as_float(x[1]);
}

constexpr int kFarTile = 128;         // keys whose largest norm and value are kept
// Keys are left out where all of them together have less than 2^-25 of what a row's own key has of each element, and of its weight; or
// where each weighs less than 2^-150 of the row's own key, which is nothing in 32 bits.
constexpr float kAttendFar = 25.0f, kAttendNothing = 150.0f;
// A reference is raised once a row's largest exponent is this far above the place where raising puts it.
constexpr float kAttendSlack = 8.0f;
// Raising puts a row's reference this far below its largest exponent.  In half precision terms then reach from 2^15 down to 2^-24, so that
// those below 2^-31 of the largest are all that is lost; the other types have bits of exponent enough.
template <typename T>
constexpr float kAttendLift = __is_same(T, f16_t) ? 7.0f : 0.0f;

template <typename T, int D, typename SHAPE, bool BIAS>
__global__ void __launch_bounds__(SHAPE::WR * SHAPE::WK * kWave, (D * (int)sizeof(T) > 256 || (SHAPE::WR * SHAPE::WK == 4 && D * (int)sizeof(T) * SHAPE::NB > 640) ? 1 : 2)) attend_kernel(const AttendArgs a) {
    constexpr int WR = SHAPE::WR, WK = SHAPE::WK, SB = SHAPE::SB, NB = SHAPE::NB, W = WR * WK, US = NB / (WK * SB);
    constexpr int EB = sizeof(T), RB = D * EB, CH = RB / 16, NT = W * kWave, BK = NB * 32, AHEAD = WK * SB * 32;
    constexpr int PT = BK * CH / NT;             // 16-byte pieces of a tile that a thread brings
    constexpr int KS = RB / 32, DT = D / 32, ROWS = WR * 32;
    static_assert(BK * CH % NT == 0 && PT >= 1 && US * WK * SB == NB, "a tile is brought in whole rounds and used in whole steps");
    constexpr int JOIN = (WK - 1) * WR * (D * 32 * 4 + 512);  // what the waves that share rows leave at the end
    constexpr int LDS = 4 * BK * RB > JOIN ? 4 * BK * RB : JOIN;
    __shared__ __attribute__((aligned(16))) char lds[LDS];
    char(*const kbuf)[BK * RB] = (char(*)[BK * RB]) lds;
    char(*const vbuf)[BK * RB] = kbuf + 2;
    __shared__ float4 far_s[BIAS ? W : 1];
    __shared__ int bad_s;                        // a tile of which some rows do not see all holds a value that is infinite or no number
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), n0 = lane & 31, half = lane >> 5;
    const int wr = wv % WR, wk = wv / WR;

    // The workgroups of a cached head share an XCD and its L2.  Where the heads are a multiple of the XCDs each takes its share of every
    // sequence's, to and fro and another share for the next sequence, the last heads first: what a position bias leaves them to do grows
    // with their number.  Else a head's blocks of rows are dealt out to as many XCDs as it takes to give each the same number, and the
    // heads of an XCD lie apart, so that no XCD has the long sequences or the heads with much to do.
    const unsigned xcd = blockIdx.x % kXcds, place = blockIdx.x / kXcds, spread = (unsigned)a.spread;
    const unsigned blocks = ((unsigned)a.tiles + spread - 1) / spread, per = blocks * (unsigned)a.S, local = place / per, rest = place - local * per;
    unsigned block = rest / (unsigned)a.S;
    int split = (int)(rest - block * (unsigned)a.S);
    int b, h;
    if (a.H % kXcds == 0) {
        const unsigned back = local / (unsigned)a.B, r = (unsigned)a.H / kXcds - 1 - back;
        b = (int)(local - back * (unsigned)a.B);
        const unsigned x = (xcd + (unsigned)b) % kXcds;
        h = (int)(r * kXcds + (r & 1 ? kXcds - 1 - x : x));
    } else {
        const unsigned group = local * kXcds + xcd;
        unsigned u = group / spread;
        block = block * spread + group % spread;
        if (spread == 1) {                       // heads of few blocks: one after the other
            const unsigned at = blockIdx.x / (unsigned)a.S;
            u = at / (unsigned)a.tiles;
            block = at - u * (unsigned)a.tiles;
            split = (int)(blockIdx.x - at * (unsigned)a.S);
        } else if (block >= (unsigned)a.tiles) return;
        b = (int)(u / (unsigned)a.H);
        h = a.H - 1 - (int)(u - (unsigned)b * (unsigned)a.H);
    }
    const unsigned unit = (unsigned)b * (unsigned)a.H + (unsigned)h;
    const int qt = a.tiles - 1 - (int)block;     // long walks first

    int64_t q0 = 0, k0 = 0;
    int nq = a.n, nk = a.m;
    if (a.q_start) q0 = a.q_start[b], nq = (int)min((int64_t)a.q_start[b + 1] - q0, (int64_t)0x7fffffff);
    else if (a.seq_n) nq = a.seq_n[b];
    if (a.k_start) k0 = a.k_start[b], nk = (int)min((int64_t)a.k_start[b + 1] - k0, (int64_t)0x7fffffff);
    else if (a.seq_m) nk = a.seq_m[b];
    if (nq < 1 || nq > a.n || nk < 0 || nk > a.m || q0 < 0 || k0 < 0) return;  // no such sequence
    const int rows = nq * a.G, R0 = qt * ROWS;   // (n * G fits 31 bits: the host asks)
    if (R0 >= rows) return;
    const int off = nk - nq;
    const char* Kh = (const char*)a.K + ((a.k_start ? k0 * a.k_st : b * a.k_sb) + h * a.k_sh) * EB;
    const char* Vh = (const char*)a.V + ((a.k_start ? k0 * a.v_st : b * a.v_sb) + h * a.v_sh) * EB;
    const int64_t krow = a.k_st * EB, vrow = a.v_st * EB;

    // this lane's row
    const int R = min(R0 + wr * 32 + n0, rows - 1), qi = R / a.G, qh = h * a.G + (R - qi * a.G), pos = off + qi;
    const bool mine = R0 + wr * 32 + n0 < rows;
    u32x4_t q[KS];
    {
        const char* p = (const char*)a.Q + ((a.q_start ? q0 * a.q_st : b * a.q_sb) + qh * a.q_sh + qi * a.q_st) * EB + half * 16;
#pragma unroll
        for (int s = 0; s < KS; ++s) q[s] = (*(const u32x4_t*)(p + s * 32) & a.q_keep) ^ a.q_flip;
    }
    float slope = 0.0f;
    if constexpr (BIAS) slope = a.slopes[qh] * kLog2e / a.sc;

    // tiles: the workgroup's rows see keys [0, kend)
    const int kend = min(nk, off + min(R0 + ROWS - 1, rows - 1) / a.G + 1);
    int t0 = 0, t1 = kend > 0 ? (kend + BK - 1) / BK : 0;
    if constexpr (BIAS) {
        // Far keys that cannot matter.  The logit of one at distance D is at most sc |q| |k| - slope D: where that lies so far below the own
        // key's of every row, as the number of keys, the tile's largest value and the least element of the row's own value ask for, a tile of
        // keys is left out, with all before it.  (A tile that holds a value which is no number, or infinite, has an infinite norm; what is no
        // number makes no row's bound hold, nor does a bias that rises.)
        if (a.ws_kn && t1 > 0) {
            float qq = 0.0f, own = 0.0f;
            const int64_t mine = min(max(pos, 0), nk - 1);
            u32x4_t k[KS], v[KS];
            uint32_t least = ~0u;
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                k[s] = *(const u32x4_t*)(Kh + mine * krow + half * 16 + s * 32);
                v[s] = *(const u32x4_t*)(Vh + mine * vrow + half * 16 + s * 32);
            }
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                qq = dot_piece<T>(__builtin_bit_cast(uint4, q[s]), __builtin_bit_cast(uint4, q[s]), qq);
                own = dot_piece<T>(__builtin_bit_cast(uint4, q[s]), __builtin_bit_cast(uint4, k[s]), own);
                least = piece_magnitude<T, true>(v[s], least);
            }
            qq = half_sum(qq);
            own = half_sum(own);
            const bool odd = __any(!(qq < INFINITY) || !(fabsf(own) < INFINITY) || slope < 0.0f);
            own *= -a.sc;
            const float value = own - hw_log2(-half_max(-magnitude<T>(least)));
            qq = odd ? INFINITY : wave_max(qq);
            const float flat = -wave_max(-slope), most = wave_max(own), most_value = wave_max(value);
            if (lane == 0) far_s[wv] = make_float4(qq, flat, most, most_value);
            __syncthreads();
            float4 all = far_s[0];
#pragma unroll
            for (int w = 1; w < W; ++w) all.x = fmaxf(all.x, far_s[w].x), all.y = fminf(all.y, far_s[w].y), all.z = fmaxf(all.z, far_s[w].z), all.w = fmaxf(all.w, far_s[w].w);
            const int lowest = off + R0 / a.G, count = (a.m + kFarTile - 1) / kFarTile;
            const float2* kn = a.ws_kn + (int64_t)unit * count;
            const float qn = sqrtf(all.x), need = kAttendFar + hw_log2((float)max(lowest, 1));
            int from = lowest > 0 ? lowest / kFarTile : 0;  // tiles that end before the lowest row
            for (int i = 0; i < from; i += kWave) {
                const int tile = i + lane;
                const float2 t = kn[min(tile, from - 1)];
                const float below = fminf(need + fmaxf(all.w + hw_log2(t.y), all.z), kAttendNothing + all.z);
                const bool far = tile < from && a.sc * (qn * t.x - all.y * (float)(lowest - (tile * kFarTile + kFarTile - 1))) < -below;
                const uint64_t no = __ballot(!far);
                if (no) {
                    from = min(from, i + __builtin_ctzll(no));
                    break;
                }
            }
            t0 = from * kFarTile / BK;
        }
    }
    // a workgroup walks at most a.chunk keys; one that walks all of them finishes its rows, of others the records are joined
    int parts = 1;
    if (a.S > 1) {
        const int each = a.chunk / BK;
        parts = max((t1 - t0 + each - 1) / each, 1);
        if (split >= parts) return;
        t0 += split * each;
        t1 = min(t0 + each, t1);
        if (split == 0 && tid == 0) a.ws_parts[unit * (unsigned)a.tiles + (unsigned)qt] = parts;
    }
    t0 = __builtin_amdgcn_readfirstlane(t0);     // (what the loads' bases are formed from)
    t1 = __builtin_amdgcn_readfirstlane(t1);
    const int first = off + min(R0 + wr * 32, rows - 1) / a.G;  // of the wave
    const int last = R0 + wr * 32 < rows ? off + min(R0 + wr * 32 + 31, rows - 1) / a.G : -1;
    const int lowest = off + R0 / a.G;           // of the workgroup

    // Pieces of keys are read 16 rows a time at one place of the row, pieces of values 4 rows at 64 neighbouring bytes: in LDS a row's
    // pieces are exchanged by the row's number, so that either way falls on all banks.
    auto key_piece = [](int row, int c) { return CH >= 16 ? c ^ (row & 15) : c ^ (row >> 1 & 7); };
    auto value_piece = [](int row, int c) { return CH >= 16 ? c ^ (row & 3) << 2 : c ^ (row >> 1 & 1) << 2; };
    // Tiles go from memory straight to LDS: an instruction of a wave fills 1 KB, a lane 16 bytes of it, so what a lane asks for is the
    // piece that belongs where it writes.  A wave's instructions lie RPX rows apart: the rows' part of an address that the wave shares
    // is the scalar unit's.  (The host refuses rows so far apart that the rest needs more than 32 bits.)
    constexpr int RPX = NT / CH, NV = RPX % 16 == 0 ? 1 : 16 / RPX;
    uint32_t koff[NV], voff[NV];
#pragma unroll
    for (int x = 0; x < NV; ++x) {
        const int row = tid / CH, mine = lane / CH, c = tid % CH;
        koff[x] = (uint32_t)mine * (uint32_t)krow + key_piece(row + x * RPX, c) * 16;
        voff[x] = (uint32_t)mine * (uint32_t)vrow + value_piece(row + x * RPX, c) * 16;
    }
    const uint32_t klds = (uint32_t)(uintptr_t)(lds_char*)kbuf + wv * 1024, vlds = (uint32_t)(uintptr_t)(lds_char*)vbuf + wv * 1024;
    // rows [r0, r0 + BK) of K or V; what lies outside the sequence is its nearest row again
    auto bring_rows = [&](int r0, const char* base, int64_t pitch, uint32_t lds, const uint32_t (&off)[NV], auto piece) {
        if (r0 >= 0 && r0 + BK <= nk) {
            const char* p = base + (int64_t)(r0 + wv * (kWave / CH)) * pitch;
#pragma unroll
            for (int x = 0; x < PT; ++x) to_lds(lds + x * NT * 16, p + x * RPX * pitch, off[x % NV]);
        } else {
            int here = tid;                      // (formed here: held over the loop it would be spilled)
            asm volatile("" : "+v"(here));
#pragma unroll
            for (int x = 0; x < PT; ++x) {
                const int row = here / CH + x * RPX, c = here % CH;
                to_lds(lds + x * NT * 16, base + (int64_t)min(max(r0 + row, 0), nk - 1) * pitch + piece(row, c) * 16);
            }
        }
    };
    // Keys run a step ahead of the values: while the exponentials of one step keep the vector unit busy, the matrix cores form the logits
    // of the next.  A tile of keys therefore begins AHEAD rows behind the tile of values.
    auto bring_keys = [&](int t, int buf) { bring_rows(t * BK + AHEAD, Kh, krow, klds + buf * BK * RB, koff, key_piece); };
    auto bring_values = [&](int t, int buf) { bring_rows(t * BK, Vh, vrow, vlds + buf * BK * RB, voff, value_piece); };

    f32x16 o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = (f32x16)(0.0f);
    float m = -INFINITY, l = 0.0f;
    f32x16 s[SB];                                // logits of the step that is next to be summed

    // Logits of the blocks from key j on, divided by sc.  The bias is where the products begin (in fp32, which would feel the roundings of
    // sums around a far key's bias, it is added behind them).
    auto logits = [&](const char* kt, int j, f32x16(&x)[SB]) {
        const float base = slope * (float)(j + half * 4 - pos);
#pragma unroll
        for (int c = 0; c < SB; ++c) {
#pragma unroll
            for (int r = 0; r < 16; ++r) x[c][r] = BIAS && EB == 2 ? fmaf(slope, (float)(c * 32 + (r >> 2) * 8 + (r & 3)), base) : 0.0f;
#pragma unroll
            for (int g = 0; g < KS; ++g) {
                const uint4 k = *(const uint4*)(kt + (c * 32 + n0) * RB + key_piece(n0, 2 * g + half) * 16);
                x[c] = Mma<T>::group(k, __builtin_bit_cast(uint4, q[g]), x[c]);
            }
            if constexpr (BIAS && EB == 4) {
#pragma unroll
                for (int r = 0; r < 16; ++r) x[c][r] = fmaf(slope, (float)(c * 32 + (r >> 2) * 8 + (r & 3)), base) + x[c][r];
            }
        }
    };
    auto masked = [&](f32x16(&x)[SB], int j) {
#pragma unroll
        for (int c = 0; c < SB; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) x[c][r] = j + half * 4 + c * 32 + (r >> 2) * 8 + (r & 3) > pos ? -INFINITY : x[c][r];
    };
    const float sc = a.sc;
    auto largest = [&](const f32x16(&x)[SB]) {
        float top = x[0][0];
#pragma unroll
        for (int c = 0; c < SB; ++c)
#pragma unroll
            for (int r = 0; r < 16; ++r) top = fmaxf(top, x[c][r]);
        return fmaf(half_max(top), sc, -kAttendLift<T>);
    };
    // the reference, where the largest exponent (less the lift) asks for it
    auto raise = [&](float top) {
        if (__any(top > m + kAttendSlack || m == -INFINITY)) {
            const float to = fmaxf(m, top), by = to == -INFINITY ? 1.0f : hw_exp2(m - to);
            m = to;
            l *= by;
#pragma unroll
            for (int i = 0; i < DT; ++i) o[i] *= by;
        }
    };
    // Operand x of the values, rows i * 32 .. of it: of 16 lanes each four bring 16 neighbouring elements of a key, and a lane
    // receives its element of the four keys.  In fp32 four products take one key of either half each.
    auto values = [&](const char* vt, int x, int i) {
        if constexpr (EB == 2) {
            const int row = x * 16 + half * 4 + (lane >> 2 & 3), c = i * 4 + (lane >> 4 & 1) * 2 + (lane >> 1 & 1);
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vt + row * RB + value_piece(row, c) * 16 + (lane & 1) * 8));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(vt + (row + 8) * RB + value_piece(row + 8, c) * 16 + (lane & 1) * 8));
            const uint2 u = __builtin_bit_cast(uint2, lo), v = __builtin_bit_cast(uint2, hi);
            return make_uint4(u.x, u.y, v.x, v.y);
        } else {
            uint32_t w[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
                const int row = x * 8 + half * 4 + y, byte = (i * 32 + n0) * 4;
                w[y] = *(const uint32_t*)(vt + row * RB + value_piece(row, byte / 16) * 16 + byte % 16);
            }
            return make_uint4(w[0], w[1], w[2], w[3]);
        }
    };
    constexpr int XS = EB == 2 ? 2 : 4, PX = 16 / XS;  // operands of 32 keys, terms of each
    // One step: its exponentials beside the next one's logits, then its values beside the next one's largest.
    auto step = [&](const char* next, const char* vt, int j, bool edge) {
        f32x16 y[SB];
        logits(next, j + AHEAD, y);
        const float ref = m == -INFINITY ? 0.0f : m;
        uint4 p[SB][XS];
#pragma unroll
        for (int c = 0; c < SB; ++c) {
#pragma unroll
            for (int r = 0; r < 16; ++r) s[c][r] = hw_exp2(fmaf(s[c][r], sc, -ref));
#pragma unroll
            for (int r = 0; r < 16; ++r) l += s[c][r];
#pragma unroll
            for (int x = 0; x < XS; ++x) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if constexpr (EB == 2) w[e] = pack_pair<T>(s[c][x * PX + 2 * e], s[c][x * PX + 2 * e + 1]);
                    else w[e] = __float_as_uint(s[c][x * PX + e]);
                }
                asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));  // here, beside the products, and not behind the branch
                p[c][x] = make_uint4(w[0], w[1], w[2], w[3]);
            }
        }
        if (edge) {
            asm volatile("");                    // a branch: the comparisons would be a fifth of a block's vector work
            masked(y, j + AHEAD);
        }
#pragma unroll
        for (int c = 0; c < SB; ++c)
#pragma unroll
            for (int x = 0; x < XS; ++x)
#pragma unroll
                for (int i = 0; i < DT; ++i) o[i] = Mma<T>::group(values(vt, c * XS + x, i), p[c][x], o[i]);
        const float top = largest(y);
        raise(top);
#pragma unroll
        for (int c = 0; c < SB; ++c) s[c] = y[c];
    };

    if (t0 < t1) {
        if (tid == 0) bad_s = 0;
        bring_keys(t0 - 1, 1);
        bring_keys(t0, 0);
        bring_values(t0, 0);
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
        logits(kbuf[1] + (BK - AHEAD + wk * SB * 32) * RB, t0 * BK + wk * SB * 32, s);
        masked(s, t0 * BK + wk * SB * 32);
        raise(largest(s));
    }
    for (int t = t0; t < t1; ++t) {
        const int buf = (t - t0) & 1;
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // the tile is there, and nobody reads the other buffers any more
        __syncthreads();
        if (t + 1 < t1) {
            bring_keys(t + 1, buf ^ 1);
            bring_values(t + 1, buf ^ 1);
        }
        if (t * BK + BK - 1 > lowest) {          // some row does not see all of the tile: see the end
            bool bad = false;
#pragma unroll
            for (int x = 0; x < PT; ++x) {
                u32x4_t* at = (u32x4_t*)(vbuf[buf] + (tid + x * NT) * 16);
                u32x4_t v = *at;
                if (clean_piece<T>(v)) *at = v, bad = true;
            }
            if (bad) bad_s = 1;
            __syncthreads();
        }
        if (t * BK > last) continue;             // the wave's rows see nothing of it
        const bool edge = (t + 1) * BK + AHEAD - 1 > first;
#pragma unroll 1
        for (int u = 0; u < US; ++u) {
            const int row = (u * WK + wk) * SB * 32;
            step(kbuf[buf] + row * RB, vbuf[buf] + row * RB, t * BK + row, edge);
        }
    }
    __syncthreads();
    const bool bad = t0 < t1 && bad_s;
    if constexpr (WK > 1) {                      // the waves that share rows
        if (wk > 0) {
            float4* w = (float4*)(lds + ((wk - 1) * WR + wr) * (D * 32 * 4 + 512));
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int y = 0; y < 4; ++y) w[(i * 4 + y) * 64 + lane] = make_float4(o[i][4 * y], o[i][4 * y + 1], o[i][4 * y + 2], o[i][4 * y + 3]);
            ((float2*)(w + DT * 256))[lane] = make_float2(m, l);
        }
        __syncthreads();
        if (wk > 0) return;
#pragma unroll 1
        for (int c = 0; c < WK - 1; ++c) {
            const float4* w = (const float4*)(lds + (c * WR + wr) * (D * 32 * 4 + 512));
            const float2 ml = ((const float2*)(w + DT * 256))[lane];
            const float to = fmaxf(m, ml.x), ref = to == -INFINITY ? 0.0f : to, mine_by = hw_exp2(m - ref), by = hw_exp2(ml.x - ref);
            m = to;
            l = fmaf(by, ml.y, l * mine_by);
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int y = 0; y < 4; ++y) {
                    const float4 v = w[(i * 4 + y) * 64 + lane];
                    o[i][4 * y] = fmaf(by, v.x, o[i][4 * y] * mine_by);
                    o[i][4 * y + 1] = fmaf(by, v.y, o[i][4 * y + 1] * mine_by);
                    o[i][4 * y + 2] = fmaf(by, v.z, o[i][4 * y + 2] * mine_by);
                    o[i][4 * y + 3] = fmaf(by, v.w, o[i][4 * y + 3] * mine_by);
                }
        }
    }
    l = half_sum(l);
    if (!mine) return;
    if (bad) {
        // 0 times an infinity would reach the rows that do not see it: such values were left out of the products with tiles of which
        // some rows do not see all, and go to the rows that do here
#pragma unroll 1
        for (int j = max(t0, (lowest + 1) / BK) * BK; j <= min(pos, t1 * BK - 1); ++j) {
            const char* row = Vh + j * vrow + half * 4 * EB;
#pragma unroll
            for (int i = 0; i < DT; ++i)
#pragma unroll
                for (int y = 0; y < 16; ++y) {
                    const char* p = row + (i * 32 + acc_row(y, 0)) * EB;
                    float v;
                    if constexpr (EB == 4) v = *(const float*)p;
                    else v = __is_same(T, bf16_t) ? __uint_as_float((uint32_t)*(const uint16_t*)p << 16) : (float)*(const _Float16*)p;
                    o[i][y] += (__float_as_uint(v) & 0x7F800000u) == 0x7F800000u ? v : 0.0f;
                }
        }
    }
    if (parts > 1) {
        const int64_t row = ((int64_t)unit * a.tiles * ROWS + R) * a.S + split;
        if (half == 0) a.ws_ml[row] = make_float2(m, l);
        float* w = a.ws_o + row * D;
#pragma unroll
        for (int i = 0; i < DT; ++i)
#pragma unroll
            for (int y = 0; y < 4; ++y)
                *(float4*)(w + i * 32 + y * 8 + half * 4) = make_float4(o[i][4 * y], o[i][4 * y + 1], o[i][4 * y + 2], o[i][4 * y + 3]);
        return;
    }
    if (l == 0.0f) {                             // nothing but logits at minus infinity, whatever their values hold
#pragma unroll
        for (int i = 0; i < DT; ++i) o[i] = (f32x16)(0.0f);
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    char* w = (char*)a.out + ((a.q_start ? q0 * a.o_st : b * a.o_sb) + qh * a.o_sh + qi * a.o_st) * EB;
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
            const float v0 = o[i][4 * y] * inv, v1 = o[i][4 * y + 1] * inv, v2 = o[i][4 * y + 2] * inv, v3 = o[i][4 * y + 3] * inv;
            char* p = w + (i * 32 + y * 8 + half * 4) * EB;
            if constexpr (EB == 4) *(float4*)p = make_float4(v0, v1, v2, v3);
            else *(uint2*)p = make_uint2(pack_pair<T>(v0, v1), pack_pair<T>(v2, v3));
        }
}

// Largest norm of kFarTile keys, or infinity where a key or a value among them is infinite or no number, and largest value: blockIdx = (tile, unit).
template <typename T, int D>
__global__ void __launch_bounds__(256) attend_norms_kernel(const AttendArgs a) {
    constexpr int CH = D * (int)sizeof(T) / 16, RPX = 256 / CH;
    __shared__ float red[4];
    const int b = blockIdx.y / a.H, h = blockIdx.y - b * a.H, tid = threadIdx.x;
    int64_t k0 = 0;
    int nk = a.m;
    if (a.k_start) k0 = a.k_start[b], nk = (int)min((int64_t)a.k_start[b + 1] - k0, (int64_t)0x7fffffff);
    else if (a.seq_m) nk = a.seq_m[b];
    if (nk < 0 || nk > a.m || k0 < 0) return;    // no such sequence
    const T* Kh = (const T*)a.K + (a.k_start ? k0 * a.k_st : b * a.k_sb) + h * a.k_sh + tid % CH * (16 / (int)sizeof(T));
    const T* Vh = (const T*)a.V + (a.k_start ? k0 * a.v_st : b * a.v_sb) + h * a.v_sh + tid % CH * (16 / (int)sizeof(T));
    uint4 k[kFarTile / RPX], v[kFarTile / RPX];
#pragma unroll
    for (int x = 0; x < kFarTile / RPX; ++x) {
        const int row = blockIdx.x * kFarTile + tid / CH + x * RPX;
        k[x] = v[x] = make_uint4(0u, 0u, 0u, 0u);
        if (row < nk) {
            k[x] = *(const uint4*)(Kh + row * a.k_st);
            v[x] = *(const uint4*)(Vh + row * a.v_st);
        }
    }
    float most = 0.0f;
    uint32_t value = 0;
#pragma unroll
    for (int x = 0; x < kFarTile / RPX; ++x) {
        float d = dot_piece<T>(k[x], k[x], 0.0f);
#pragma unroll
        for (int o = 1; o < CH; o <<= 1) d += __shfl_xor(d, o, kWave);
        u32x4_t w = {v[x].x, v[x].y, v[x].z, v[x].w};
        most = fmaxf(most, clean_piece<T>(w) || !(d < INFINITY) ? INFINITY : d);
        value = piece_magnitude<T, false>(w, value);
    }
    most = block_max<256>(most, red);
    const float large = block_max<256>(magnitude<T>(value), red);
    if (tid == 0) a.ws_kn[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = make_float2(sqrtf(most), large);
}

// Joins the parts of a row: one wave a row, a lane takes D / 64 elements.
template <typename T, int D>
__global__ void __launch_bounds__(256) attend_join_kernel(const AttendArgs a, int rows_pad) {
    constexpr int E = D / 64;
    const int lane = threadIdx.x & 63;
    const int64_t at = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6), unit = at / rows_pad;
    const int R = (int)(at - unit * rows_pad), b = (int)(unit / a.H), h = (int)(unit % a.H);
    if (b >= a.B) return;
    int64_t q0 = 0, k0 = 0;
    int nq = a.n, nk = a.m;
    if (a.q_start) q0 = a.q_start[b], nq = (int)min((int64_t)a.q_start[b + 1] - q0, (int64_t)0x7fffffff);
    else if (a.seq_n) nq = a.seq_n[b];
    if (a.k_start) k0 = a.k_start[b], nk = (int)min((int64_t)a.k_start[b + 1] - k0, (int64_t)0x7fffffff);
    else if (a.seq_m) nk = a.seq_m[b];
    if (nq < 1 || nq > a.n || nk < 0 || nk > a.m || q0 < 0 || k0 < 0 || R >= nq * a.G) return;
    const int qi = R / a.G, qh = h * a.G + (R - qi * a.G);
    const int parts = a.ws_parts[unit * a.tiles + R / a.block_rows];
    if (parts == 1) return;
    const int64_t row = at * a.S;
    // at most 64 parts: a lane a part's reference and sum, and the rows of sums come in one trip (eight at a time)
    float2 ml = make_float2(-INFINITY, 0.0f);
    if (lane < parts) ml = a.ws_ml[row + lane];
    const float m = wave_max(ml.x), by = hw_exp2(ml.x - (m == -INFINITY ? 0.0f : m));
    const float l = wave_sum(lane < parts ? by * ml.y : 0.0f);
    float x[E];
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = 0.0f;
    for (int s = 0; s < parts; s += 8) {
        float v[8][E];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int e = 0; e < E; ++e) v[i][e] = a.ws_o[(row + min(s + i, parts - 1)) * D + lane * E + e];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float w = s + i < parts ? __shfl(by, s + i, kWave) : 0.0f;
#pragma unroll
            for (int e = 0; e < E; ++e) x[e] = fmaf(w, s + i < parts ? v[i][e] : 0.0f, x[e]);
        }
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
#pragma unroll
    for (int e = 0; e < E; ++e) x[e] = l == 0.0f ? 0.0f : x[e];
    T* w = (T*)a.out + (a.q_start ? q0 * a.o_st : b * a.o_sb) + qh * a.o_sh + qi * a.o_st + lane * E;
#pragma unroll
    for (int e = 0; e < E; ++e) {
        if constexpr (sizeof(T) == 4) w[e] = x[e] * inv;
        else w[e].bits = (uint16_t)pack_pair<T>(x[e] * inv, 0.0f);
    }
}

// Shapes of a workgroup, by the bytes of a row: for many rows; for fewer; for about a workgroup of 64 rows a compute unit, whose waves are twice
// as many; for rows of a single wave.  Rows of 512 bytes fill registers and LDS with less.
template <int RB>
struct AttendShapes {
    using Many = AttendShape<4, 1, RB == 256 ? 2 : 1, 2>;
    using Fewer = AttendShape<2, 2, 1, 2>;
    using One = AttendShape<2, 4, 1, 4>;
    using Few = AttendShape<1, 4, 1, 4>;
};
template <>
struct AttendShapes<512> {
    using Many = AttendShape<4, 1, 1, 1>;
    using Fewer = AttendShape<2, 2, 1, 2>;
};
enum { kAttendMany, kAttendFewer, kAttendOne, kAttendFew };

void plan_attend(AttendArgs* a, int32_t d, int32_t dtype) {
    const int64_t units = (int64_t)a->B * a->H, rows = (int64_t)a->n * a->G, b64 = units * ((rows + 63) / 64);
    const bool wide = d * (dtype == KF_F32 ? 4 : 2) > 256;
    // 128 rows a workgroup where there are four rounds of them (two of wide rows): 32 heads x 4096 x 128 167 us, with 64 rows 174, 32 x 2048 63 and 59,
    // 16 x 4096 x 256 180 and 220, 16 x 2048 x 256 83 and 70.  64 rows and eight waves where these are a round at most and walks are long: 16 x
    // 2048 x 128 37 us, with four waves 40, 8 x 2048 26.5 and 30, but 32 x 1024 32 and 25; 16 x 16 sequences of 64 11 and 8.  A wave of rows: 2
    // heads x 1 x 8000 14.7 us, with two waves of them 15.2, 4 x (20 rows of 2 heads) x 5000 x 64 13.0 and 13.8.
    a->shape = kAttendFewer;
    if (units * ((rows + 127) / 128) >= (wide ? 512 : 1024)) a->shape = kAttendMany;
    else if (!wide && a->m > 512 && rows <= 32 && units <= 64) a->shape = kAttendFew;
    else if (!wide && a->m > 512 && b64 > 64 && b64 <= 256) a->shape = kAttendOne;
    a->block_rows = a->shape == kAttendMany ? 128 : a->shape == kAttendFew ? 32 : 64;
    a->threads = a->shape == kAttendOne ? 512 : 256;
    a->tiles = (int32_t)((rows + a->block_rows - 1) / a->block_rows);
    a->S = 1;
    const int64_t blocks = units * a->tiles;
    // Few workgroups share out the keys: a part costs the join as much as ten keys of a walk, and a row's record as much as a sixteenth of one.
    // (8 x 1 row x 1000 keys, 128 bf16: one part 15.6 us, parts of 128 keys 11.6; 2 x 1 x 8000: 66.6, 62 parts 15.9, 27 14; 8 x 1024 x 1024:
    // one part 17.9, two 21.1; 8 x 512 x 2048: 28.7, four 20.5.)
    int64_t least = (int64_t)sqrt(10.0 * a->m) + units * rows / 16, S = 256 / blocks;
    if (least < kFarTile) least = kFarTile;
    if (S > a->m / least) S = a->m / least;
    if (S > 64) S = 64;
    if (S > 1) {
        a->chunk = (int32_t)(((a->m + S - 1) / S + 127) / 128 * 128);
        a->S = (a->m + a->chunk - 1) / a->chunk;
    }
    // (20 heads x 2048 x 128: 47 us, a head after the other 62; 3 x 12 x 2900 120 and 125.)
    a->spread = 1;
    while (units * a->spread % kXcds) a->spread *= 2;
    if (a->H % kXcds == 0 || a->tiles < 4 * a->spread) a->spread = 1;
    a->blocks = units * a->spread * ((a->tiles + a->spread - 1) / a->spread) * a->S;  // of the launch
    // A row of far tiles is looked for where a key is read often enough: the search is a launch that reads K and V once more, 95 of 887 us of
    // 8 x 32 x 4096 x 128, which take 1350 without.  4 x 32 x 4096 450 and 665 us, 32 x 2048 62 and 67, 8 x 4096 73 and 70, 8 x 2048 40 and 32 (few
    // workgroups, which wait for the head of the gentlest slope); 8 x 32 x 1024 137 with it and 132.
    a->far_tiles = a->slopes && (int64_t)a->n * a->G >= 2048 && units <= 65535 ? (a->m + kFarTile - 1) / kFarTile : 0;
    a->ws_rows = a->S > 1 ? blocks * a->block_rows : 0;
}

template <typename T, int D, typename SHAPE>
static hipError_t launch_attend_s(const AttendArgs& a, hipStream_t st) {
    // tiles, records and the grid were sized for these
    if (a.block_rows != SHAPE::WR * 32 || a.threads != SHAPE::WR * SHAPE::WK * kWave) return hipErrorInvalidValue;
    const dim3 grid((unsigned)a.blocks), block((unsigned)a.threads);
    if (a.far_tiles)
        hipLaunchKernelGGL((attend_norms_kernel<T, D>), dim3((unsigned)a.far_tiles, (unsigned)(a.B * a.H)), dim3(256), 0, st, a);
    if (a.slopes) hipLaunchKernelGGL((attend_kernel<T, D, SHAPE, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((attend_kernel<T, D, SHAPE, false>), grid, block, 0, st, a);
    if (a.S > 1) hipLaunchKernelGGL((attend_join_kernel<T, D>), dim3((unsigned)(a.ws_rows / 4)), dim3(256), 0, st, a, a.tiles * a.block_rows);
    return hipGetLastError();
}
template <typename T, int D>
static hipError_t launch_attend_d(const AttendArgs& a, hipStream_t st) {
    using S = AttendShapes<D * (int)sizeof(T)>;
    if (a.shape == kAttendMany) return launch_attend_s<T, D, typename S::Many>(a, st);
    if (a.shape == kAttendFewer) return launch_attend_s<T, D, typename S::Fewer>(a, st);
    if constexpr (D * sizeof(T) <= 256) {
        if (a.shape == kAttendOne) return launch_attend_s<T, D, typename S::One>(a, st);
        if (a.shape == kAttendFew) return launch_attend_s<T, D, typename S::Few>(a, st);
    }
    return hipErrorInvalidValue;                 // wide rows have no such shape
}

hipError_t launch_attend(const AttendArgs& a, int32_t d, int32_t dtype, hipStream_t stream) {
    if (dtype == KF_BF16) {
        if (d == 64) return launch_attend_d<bf16_t, 64>(a, stream);
        if (d == 128) return launch_attend_d<bf16_t, 128>(a, stream);
        if (d == 256) return launch_attend_d<bf16_t, 256>(a, stream);
    } else if (dtype == KF_F16) {
        if (d == 64) return launch_attend_d<f16_t, 64>(a, stream);
        if (d == 128) return launch_attend_d<f16_t, 128>(a, stream);
        if (d == 256) return launch_attend_d<f16_t, 256>(a, stream);
    } else if (dtype == KF_F32) {
        if (d == 64) return launch_attend_d<float, 64>(a, stream);
        if (d == 128) return launch_attend_d<float, 128>(a, stream);
    }
    return hipErrorInvalidValue;
}

}  // namespace kf
