// Selection of a beam search for gfx950: the best W continuations of each request's W beams, over the whole vocabulary.
//
//   total(i, v) = score[i] + x[i][v] - lse(x[i]),   lse = log sum exp          (log-probability of beam i followed by word v)
//
// Larger totals first; of equal ones the lower beam, then the larger logit, then the lower word.  Two launches:
//   slices   a workgroup takes a slice of a row into registers, once, and leaves its largest logit, the sum of its
//            exponentials and its best W logits in order.  A wave finds the W-th largest of its lanes' maxima by a search
//            over the bits of the ordered key: at least W logits are as large, and only the lanes above it, fewer than W, hold
//            larger ones; so a short list holds what can be among the best, whatever the logits are.  The largest of the waves'
//            keys cuts all four lists.
//   request  a workgroup takes a request: each row's slices are joined (statistics in 64 bits, lists by taking their
//            smallest heads), then the rows' lists, totals in 64 bits; then the rows are numbered.
// The first launch (64 x 4 rows x 50304 in fp32 16 us, 3.2 TB/s; 16 x 16 x 128000 in halves, a fifth of the rows ended, 28 us) is
// bound by no one thing: its instructions, 700 to 900 a wave for 2048 words, are 6 to 10 of the 16 us, a trip to memory, the search's and the
// reductions' chains and the waves' starts the rest.  It grows by 1 us for 220 workgroups, also where the next round of them begins, and a
// row's last slice costs as much with one word as with 8192 (256 rows x 49152 18.8 us for both launches, x 49153 21.1).  What
// bounds the second is a chain of short steps, W picks a row, then W picks (4 beams 5.5 us, 16 beams 13.6).
#include "kf_device.h"
#include "kf_internal.h"

namespace kf {

constexpr int kBeamThreads = 256;
constexpr unsigned long long kBeamNone = ~0ull;  // behind every entry and total: (inverted key of the logit, word), the best is the smallest

__device__ __forceinline__ unsigned long long beam_entry(float x, int v) {
    return ((unsigned long long)(~float_key(x)) << 32) | (uint32_t)v;
}
__device__ __forceinline__ float beam_logit(unsigned long long c) {
    const uint32_t key = ~(uint32_t)(c >> 32);
    return __uint_as_float((key & 0x80000000u) ? key & 0x7FFFFFFFu : ~key);
}
// For the order a NaN counts as minus infinity, and minus zero as zero.
__device__ __forceinline__ float beam_ordered(float x) { return x != x ? -INFINITY : x + 0.0f; }

template <typename T>
__device__ __forceinline__ float beam_load(const T* p);
template <>
__device__ __forceinline__ float beam_load<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float beam_load<bf16_t>(const bf16_t* p) { return __uint_as_float((uint32_t)p->bits << 16); }
template <>
__device__ __forceinline__ float beam_load<f16_t>(const f16_t* p) { return (float)__builtin_bit_cast(_Float16, p->bits); }

// 16 bytes of a row, which may begin at any element.  (Slices begin at words, not at addresses: equal rows get equal sums
// wherever they lie.)
template <typename T>
__device__ __forceinline__ uint4 beam_load16(const T* p) {
    typedef unsigned int any4_t __attribute__((ext_vector_type(4), aligned(2)));
    const any4_t v = __builtin_nontemporal_load((const any4_t*)p);
    return make_uint4(v.x, v.y, v.z, v.w);
}

// Most entries that a wave adds to the list: the lanes above the W-th largest maximum hold all of theirs, the equal ones W.
constexpr int beam_list_cap(int W, int per_lane) { return (W - 1) * per_lane + W; }

// (six waves on a SIMD: 32 words a lane take 28 us at 16 x 16 x 128000, five waves 30, eight, with spills, 33)
template <typename T, int NL>
__global__ void __launch_bounds__(kBeamThreads, 6) beam_slice_kernel(const BeamArgs a) {
    constexpr int EPV = ElemTraits<T>::kPerVec, NW = kBeamThreads / kWave;
    extern __shared__ __attribute__((aligned(16))) unsigned long long list[];  // what can be among the best, and eight more
    __shared__ float w_max[NW];
    __shared__ double w_sum[NW];
    __shared__ uint32_t w_key[NW];
    __shared__ int w_cnt[NW], s_cnt;
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, W = a.W, V = a.V;
    const int64_t row = blockIdx.x / (uint32_t)a.S;
    const int s = (int)(blockIdx.x % (uint32_t)a.S);
    if (a.done && a.done[row]) return;  // the request launch does not look at its slices
    const T* base = (const T*)a.logits + row * a.row_stride;

    float x[NL][EPV];
    int first[NL];  // word of each vector's first element
    bool whole[NL];
    uint4 raw[NL];
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        const int vi = (s * NL + i) * kBeamThreads + tid;
        first[i] = vi * EPV;
        whole[i] = first[i] + EPV <= V;
        raw[i] = make_uint4(0u, 0u, 0u, 0u);
        if (whole[i]) raw[i] = beam_load16(base + first[i]);
    }
    bool any = false;  // whether the lane holds a word
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        unpack16<T>(raw[i], x[i]);
        any = any || first[i] < V;
        if (!whole[i]) {
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                x[i][e] = first[i] + e < V ? beam_load<T>(base + first[i] + e) : -INFINITY;
            }
        }
    }

    // ---- statistics
    float vmax[NL], lmax = -INFINITY;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        vmax[i] = x[i][0];
#pragma unroll
        for (int e = 1; e < EPV; ++e) vmax[i] = fmaxf(vmax[i], x[i][e]);  // (passes over NaN)
        lmax = fmaxf(lmax, vmax[i]);
    }
    // the W-th largest of the lanes' maxima, as a key; 0: fewer lanes hold words
    const uint32_t lkey = any ? float_key(beam_ordered(lmax)) : 0u;
    uint32_t T32 = 0;
    for (int bit = 31; bit >= 0; --bit) {
        const uint32_t t = T32 | (1u << bit);
        if ((int)__popcll(__ballot(lkey >= t)) >= W) T32 = t;
    }
    const float wmax = wave_max(lmax), ref = wmax == -INFINITY ? 0.0f : wmax;
    double sum = 0.0;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
        float part = 0.0f;
#pragma unroll
        for (int e = 0; e < EPV; ++e) {  // (a multiple of log2 e, its rounding put right by the second product)
            const float t = x[i][e] - ref, hi = t * kLog2e;
            const float lo = hi > -150.0f ? fmaf(t, kLog2e, -hi) + t * 1.92596299e-8f : 0.0f;
            part += hw_exp2(hi) * fmaf(lo, kLn2, 1.0f);
        }
        sum += (double)part;
    }
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o, kWave);
    if (lane == 0) {
        w_max[wv] = wmax;
        w_sum[wv] = sum;
        w_key[wv] = T32;
    }
    if (tid == 0) s_cnt = 0;
    __syncthreads();
    // ---- What can be among the slice's best W: the words above the largest of the waves' keys, and, of each wave, the first W (by
    // word) that equal it.  A wave has fewer than W lanes with words above its own key, so its list is bounded.
#pragma unroll
    for (int w = 0; w < NW; ++w) T32 = max(T32, w_key[w]);
    const float cut = __uint_as_float((T32 & 0x80000000u) ? T32 & 0x7FFFFFFFu : ~T32);
    const bool plain = T32 > 0x007FFFFFu;  // else minus infinity, as which a NaN counts, or less: every word is looked at
    // Usually those are few: every word that reaches the key, in any order (a branch that most of a wave's words skip; bits of each
    // word, and a list from them, took half of the kernel's instructions).  Many that equal it, or minus infinity as the
    // key: the lists with their bounds.
    const int room = NW * beam_list_cap(W, NL * EPV);
    int total = room + 1;
    if (plain) {
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            if (vmax[i] < cut) continue;
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                if (x[i][e] >= cut) {
                    const int at = atomicAdd(&s_cnt, 1);
                    if (at < room) list[at] = beam_entry(beam_ordered(x[i][e]), first[i] + e);
                }
            }
        }
        __syncthreads();
        total = s_cnt;
    }
    if (total > room) {
        uint32_t gt[NL], eq[NL];
        uint32_t n_lane = 0, n_eq = 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            gt[i] = eq[i] = 0;
#pragma unroll
            for (int e = 0; e < EPV; ++e) {
                if (!whole[i] && first[i] + e >= V) continue;
                const uint32_t key = float_key(beam_ordered(x[i][e]));
                gt[i] |= (key > T32 ? 1u : 0u) << e;
                eq[i] |= (key == T32 ? 1u : 0u) << e;
            }
            // equal ones in the order of words, vector by vector: the bits of the first W stay
            if (__ballot(eq[i] != 0) != 0) {
                const uint32_t c = (uint32_t)__popc(eq[i]), upto = wave_scan(c);
                uint32_t before = n_eq + upto - c;
                n_eq += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
                for (uint32_t left = eq[i]; left != 0; left &= left - 1, ++before)
                    if (before >= (uint32_t)W) eq[i] &= ~(left & (0u - left));
            }
            gt[i] |= eq[i];
            n_lane += (uint32_t)__popc(gt[i]);
        }
        const uint32_t upto = wave_scan(n_lane);
        if (lane == 63) w_cnt[wv] = (int)upto;
        __syncthreads();
        int at = (int)(upto - n_lane);
        total = 0;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            at += w < wv ? w_cnt[w] : 0;
            total += w_cnt[w];
        }
#pragma unroll
        for (int i = 0; i < NL; ++i) {
            if (gt[i] == 0) continue;
#pragma unroll
            for (int e = 0; e < EPV; ++e)
                if ((gt[i] >> e) & 1u) list[at++] = beam_entry(beam_ordered(x[i][e]), first[i] + e);
        }
    }
    if (tid < 8) list[total + tid] = kBeamNone;
    __syncthreads();
    // ---- in order: an entry's place is the number of entries before it, eight a step
    unsigned long long* out = a.ws_list + ((size_t)row * a.S + s) * W;
    for (int c = tid; c < total; c += kBeamThreads) {
        const unsigned long long v = list[c];
        int place = 0;
        for (int i = 0; i < total; i += 8) {
            ulonglong2 r[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = *(const ulonglong2*)&list[i + 2 * j];
#pragma unroll
            for (int j = 0; j < 4; ++j) place += (r[j].x < v ? 1 : 0) + (r[j].y < v ? 1 : 0);
        }
        if (place < W) out[place] = v;
    }
    for (int i = total + tid; i < W; i += kBeamThreads) out[i] = kBeamNone;
    if (tid == 0) {
        float m = w_max[0];
#pragma unroll
        for (int w = 1; w < NW; ++w) m = fmaxf(m, w_max[w]);
        double t = 0.0;
#pragma unroll
        for (int w = 0; w < NW; ++w) t += w_max[w] == -INFINITY && m != -INFINITY ? w_sum[w] * 0.0 : w_sum[w] * exp((double)(w_max[w] == m ? 0.0f : w_max[w] - m));
        a.ws_stat[(size_t)row * a.S + s] = make_double2((double)m, t);
    }
}

// Totals as keys of which the smallest is the best; NaN counts as minus infinity.
__device__ __forceinline__ unsigned long long total_key(double t) {
    if (t != t) t = -INFINITY;
    t += 0.0;
    const unsigned long long b = (unsigned long long)__double_as_longlong(t);
    return ~((b >> 63) ? ~b : (b | 0x8000000000000000ull));
}
__device__ __forceinline__ double key_total(unsigned long long k) {
    const unsigned long long o = ~k;
    return __longlong_as_double((long long)((o >> 63) ? (o & 0x7FFFFFFFFFFFFFFFull) : ~o));
}

// Smallest of the lanes' values, 32 bits.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t min32_step(uint32_t v) { return min(v, dpp_or<CTRL, ROWS>(~0u, v)); }
__device__ __forceinline__ uint32_t wave_min32(uint32_t v) {
    v = min32_step<0x111, 0xF>(v);
    v = min32_step<0x112, 0xF>(v);
    v = min32_step<0x114, 0xF>(v);
    v = min32_step<0x118, 0xF>(v);
    v = min32_step<0x142, 0xA>(v);
    v = min32_step<0x143, 0xC>(v);
    return (uint32_t)__builtin_amdgcn_readlane((int)v, 63);
}
// ... of 64-bit values, by halves: a chain of 32-bit minima is a third of one of 64-bit ones.
__device__ __forceinline__ unsigned long long wave_min_halves(unsigned long long v) {
    const uint32_t hi = wave_min32((uint32_t)(v >> 32));
    const uint32_t lo = wave_min32((uint32_t)(v >> 32) == hi ? (uint32_t)v : ~0u);
    return ((unsigned long long)hi << 32) | lo;
}
__device__ __forceinline__ void wave_sync_lds() {
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

__global__ void __launch_bounds__(1024) beam_request_kernel(const BeamArgs a) {
    extern __shared__ unsigned long long lists[];  // [waves][S][W]
    __shared__ unsigned long long best[kBeamMaxW][kBeamMaxW];      // a row's best W
    __shared__ unsigned long long totals[kBeamMaxW][kBeamMaxW];    // ... and their totals' keys
    __shared__ int p_s[kBeamMaxW], tok_s[kBeamMaxW];
    __shared__ double tot_s[kBeamMaxW];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6, waves = blockDim.x >> 6, W = a.W, S = a.S;
    const int64_t row0 = (int64_t)blockIdx.x * W;
    for (int i = wv; i < W; i += waves) {
        const int64_t row = row0 + i;
        const double sc = (double)a.score[row];
        if (a.done && a.done[row]) {  // one continuation, at its own score
            if (lane < W) {
                best[i][lane] = (unsigned long long)(uint32_t)a.eos;
                totals[i][lane] = lane == 0 ? total_key(sc) : kBeamNone;
            }
            continue;
        }
        unsigned long long* mine = lists + (size_t)wv * S * W;
        for (int j = lane; j < S * W; j += kWave) mine[j] = a.ws_list[(size_t)row * S * W + j];
        // statistics: a lane a slice (S <= 64)
        double m = -INFINITY, sum = 0.0;
        if (lane < S) {
            const double2 st = a.ws_stat[(size_t)row * S + lane];
            m = st.x;
            sum = st.y;
        }
        const double M = (double)wave_max((float)m);
        sum = (m == -INFINITY && M != -INFINITY) ? sum * 0.0 : sum * exp(m == M ? 0.0 : m - M);
#pragma unroll
        for (int o = 1; o < kWave; o <<= 1) sum += __shfl_xor(sum, o, kWave);
        const double lse = M + log(sum);
        // the slices' lists: a lane a list, the smallest head leaves
        wave_sync_lds();
        int at = 0;
        unsigned long long head = lane < S ? mine[lane * W] : kBeamNone;
        for (int j = 0; j < W; ++j) {
            const unsigned long long c = wave_min_halves(head);
            if (lane == 0) best[i][j] = c;
            if (c != kBeamNone && head == c) {  // (words are unique: one lane)
                ++at;
                head = at < W ? mine[lane * W + at] : kBeamNone;
            }
        }
        wave_sync_lds();
        if (lane < W) {
            const unsigned long long c = best[i][lane];
            totals[i][lane] = c == kBeamNone ? kBeamNone : total_key(sc + ((double)beam_logit(c) - lse));
        }
    }
    __syncthreads();
    if (wv != 0) return;
    // ---- the request's best W: a lane a beam
    int at = 0;
    unsigned long long head = lane < W ? totals[lane][0] : kBeamNone;
    for (int j = 0; j < W; ++j) {
        const unsigned long long c = wave_min_halves(head);
        const int owner = __ffsll((long long)__ballot(head == c)) - 1;  // the lowest beam of equals
        if (lane == owner) {
            p_s[j] = lane | (at << 8);
            tot_s[j] = key_total(c);
            ++at;
            head = lane < W && at < W ? totals[lane][at] : kBeamNone;
        }
    }
    wave_sync_lds();
    if (lane < W) {
        const int p = p_s[lane];
        tok_s[lane] = (int)(uint32_t)(best[p & 255][p >> 8] & 0xFFFFFFFFull);
        p_s[lane] = p & 255;
    }
    wave_sync_lds();
    // ---- numbering: a beam's best continuation keeps its row, the others take the rows that died, in order
    const int p = lane < W ? p_s[lane] : -1;
    bool first = lane < W, used = false;
    for (int j = 0; j < W; ++j) {
        const int o = p_s[j];
        if (j < lane && o == p) first = false;
        if (o == lane) used = true;
    }
    const unsigned long long later = __ballot(lane < W && !first), below = (1ull << lane) - 1ull;
    unsigned long long left = __ballot(lane < W && !used);
    if (lane < W) {
        int r = p;
        if (!first) {
            for (int i = __popcll(later & below); i > 0; --i) left &= left - 1;  // as many rows to die as continuations to place
            r = __ffsll((long long)left) - 1;
        }
        const bool was = a.done && a.done[row0 + p];
        a.parent[row0 + r] = (int32_t)(row0 + p);
        a.token[row0 + r] = tok_s[lane];
        if (a.rank) a.rank[row0 + r] = lane;
        a.new_score[row0 + r] = (float)tot_s[lane];
        if (a.new_done) p_s[lane] = was || tok_s[lane] == a.eos, tok_s[lane] = r;  // stored below: `done` may be the same array
    }
    if (a.new_done) {
        wave_sync_lds();
        if (lane < W) a.new_done[row0 + tok_s[lane]] = p_s[lane];
    }
}

// 16-byte loads per lane of a slice: as few as keep the slices of a row within the lanes of a wave and the launch within 2048
// workgroups (a lane's 32 words at most).
BeamPlan plan_beam(int64_t rows, int32_t W, int32_t V, int32_t dtype) {
    const int epv = dtype == KF_F32 ? 4 : 8;
    const int64_t vecs = ((int64_t)V + epv - 1) / epv;
    BeamPlan p;
    for (p.NL = 1; p.NL < 32 / epv; p.NL *= 2) {
        const int64_t S = (vecs + p.NL * kBeamThreads - 1) / (p.NL * kBeamThreads);
        if (S <= kWave && rows * S <= 2048) break;
    }
    p.S = (int32_t)((vecs + p.NL * kBeamThreads - 1) / (p.NL * kBeamThreads));
    p.lds_slice = ((size_t)(kBeamThreads / kWave) * beam_list_cap(W, p.NL * epv) + 8) * 8;
    const size_t per_row = (size_t)p.S * W * 8;
    p.waves = W < 16 ? W : 16;
    while (p.waves > 1 && p.waves * per_row > kBeamListLds) --p.waves;
    p.lds_request = p.waves * per_row;
    return p;
}

template <typename T>
static hipError_t launch_beam_slices(const BeamArgs& a, int64_t rows, const BeamPlan& p, hipStream_t st) {
    const dim3 grid((unsigned)(rows * a.S)), block(kBeamThreads);
    switch (p.NL) {
        case 1: hipLaunchKernelGGL((beam_slice_kernel<T, 1>), grid, block, p.lds_slice, st, a); break;
        case 2: hipLaunchKernelGGL((beam_slice_kernel<T, 2>), grid, block, p.lds_slice, st, a); break;
        case 4: hipLaunchKernelGGL((beam_slice_kernel<T, 4>), grid, block, p.lds_slice, st, a); break;
        case 8:
            if constexpr (ElemTraits<T>::kPerVec == 4) {
                hipLaunchKernelGGL((beam_slice_kernel<T, 8>), grid, block, p.lds_slice, st, a);
                break;
            }
            return hipErrorInvalidValue;
        default: return hipErrorInvalidValue;
    }
    return hipGetLastError();
}

hipError_t launch_beam(const BeamArgs& a, int32_t R, int32_t dtype, const BeamPlan& p, hipStream_t stream) {
    const int64_t rows = (int64_t)R * a.W;
    hipError_t e = dtype == KF_F32    ? launch_beam_slices<float>(a, rows, p, stream)
                   : dtype == KF_BF16 ? launch_beam_slices<bf16_t>(a, rows, p, stream)
                                      : launch_beam_slices<f16_t>(a, rows, p, stream);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(beam_request_kernel, dim3((unsigned)R), dim3(64 * p.waves), p.lds_request, stream, a);
    return hipGetLastError();
}

}  // namespace kf
