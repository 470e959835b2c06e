// Pages of an 8-bit cache for gfx950: rows in, the attention of a token over them, and who holds which page.
//
// A page is 64 tokens of every layer and cached head: key codes [64][D], value codes [D][64], and a power of two for each tensor, by
// which all codes of that page and head are multiplied.  Codes are E4M3 (sign, 4 bits of exponent, 3 of mantissa, up to 448, 0x7F no
// number): exact in bf16 and in half precision, so the conversion instructions decode two at a time and the matrix cores take them as
// they come.  The power is the smallest with which no finite element is above 448; a power of two, because a page's codes are then
// rounded again without a second error of their own (but for those that become subnormal) when a later row asks for a larger one.
//
// The step:  x_j = scale*<q, K_j> - slope*(n-1-j),  out = sum_j softmax(x)_j V_j  over the n tokens of a sequence, the last of which
// comes with the call and enters as it was given.  Pages need no exchange between lanes beyond a maximum and a sum: a wave takes a
// page whole,  S^T = K q^T  in tiles of 16 tokens x 16 columns and  O^T = V^T p^T  in tiles of 16 elements x 16 columns; a column is a
// query head, twice: once for the upper 11 bits of its probabilities and once for the rest, so that out keeps 22 bits of them.  Which
// token is which row of a tile is free: a lane's four tiles hold 16 neighbouring tokens, and 16 bytes of a row of V are the operand of
// two products.
//
// What bounds them: the bytes.  The step reads a page at 6.5 TB/s (2048 units x 4096 x 128: 331 us; a layer of 64 x 32 of 512 to 2048 tokens
// 131 us, 4.5; 32 units x 32768 49 us, 5.5; 8 units x 1501, 4 heads each: 10.4, two launches).  Steps of the first: pages
// looked up by the vector unit 382 us, by the scalar unit and the first ahead of the token 368, a wave a unit instead of four 331.  Tried: three workgroups a compute unit (registers spill),
// 2048 or 4096 workgroups (slower), workgroups of two waves (7 % more).  Rows in: 5.8 TB/s read and written (32 heads x 32768 x 128: 138 us).  Forks and
// reservations are launches of one workgroup, a chain of trips; kept rows are gathered a byte of V at a time (1024 units of 2048 tokens, 1024 kept: 177 us,
// 3.0 TB/s).
#include "kf_device.h"
#include "kf_internal.h"

namespace kf {

constexpr int kPageWaves = kPageThreads / kWave;
constexpr int kStepWaves = 4;        // of a workgroup of the step, or one
constexpr int kTableThreads = 1024;

typedef __bf16 p_bf2_t __attribute__((ext_vector_type(2)));
typedef __bf16 p_bf8_t __attribute__((ext_vector_type(8)));
typedef _Float16 p_h2_t __attribute__((ext_vector_type(2)));
typedef _Float16 p_h8_t __attribute__((ext_vector_type(8)));
typedef float p_f4_t __attribute__((ext_vector_type(4)));

// ---------------------------------------------------------------- codes
// Exponent of the scale for a largest finite magnitude `a`: a = f * 2^x with f in [1, 2); 448 = 1.75 * 2^8.
__device__ __forceinline__ int page_exponent(float a) {
    const uint32_t b = __float_as_uint(a);
    const int e = (int)(b >> 23) - 127 - 8 + ((b & 0x7FFFFFu) > 0x600000u ? 1 : 0);
    return min(max(e, -117), 119);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((uint32_t)(e + 127) << 23); }
__device__ __forceinline__ int exponent_of(float s) { return (int)(__float_as_uint(s) >> 23 & 255u) - 127; }
__device__ __forceinline__ bool finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }
// An element times 2^-e, ready to be rounded: at most 448 (a bf16 above 448 * 2^119 asks for more than the largest scale), and what is no
// number, or infinite, beyond all codes, which becomes 0x7F.
__device__ __forceinline__ float codable(float x, float inv) {
    const float y = __builtin_amdgcn_fmed3f(x * inv, -448.0f, 448.0f);
    return finite(x) ? y : INFINITY;
}
// Four elements, times 2^-e, rounded to the nearest code, ties to the even one.
__device__ __forceinline__ uint32_t encode4(float a, float b, float c, float d, float inv) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(codable(a, inv), codable(b, inv), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(codable(c, inv), codable(d, inv), w, true);
}
__device__ __forceinline__ uint8_t encode1(float a, float inv) { return (uint8_t)(__builtin_amdgcn_cvt_pk_fp8_f32(codable(a, inv), 0.0f, 0, false) & 255); }
typedef float p_f2_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ void decode4(uint32_t w, float* f) {
    const p_f2_t lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    f[0] = lo.x, f[1] = lo.y, f[2] = hi.x, f[3] = hi.y;
}
// Four codes whose scale grows by 1 / ratio.
__device__ __forceinline__ uint32_t again4(uint32_t w, float ratio) {
    float f[4];
    decode4(w, f);
    return encode4(f[0], f[1], f[2], f[3], ratio);
}

// ---------------------------------------------------------------- who holds which page (one workgroup)
__device__ __forceinline__ int pages_of(int n) { return (n >> 6) + ((n & 63) != 0); }
__device__ __forceinline__ int load_fresh(const int32_t* p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ __forceinline__ void count_error(const PageArgs& a) { atomicAdd(a.ws_err, 1); }

// Sum over the threads before this one, and over all.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t* red, uint32_t* all) {
    const uint32_t in = wave_scan(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 63) red[threadIdx.x >> 6] = in;
    __syncthreads();
    uint32_t before = 0, sum = 0;
    for (int i = 0; i < kTableThreads / 64; ++i) {
        if (i < (int)(threadIdx.x >> 6)) before += red[i];
        sum += red[i];
    }
    *all = sum;
    return before + in - v;
}

// need[b] in LDS: pages that sequence b asks for (0: none).  Free pages go out lowest number first, sequences in order; one that asks
// for more than are left gets none and its need becomes -1.  On return need[b] >= 0 is the place in ws_list of its first page, where
// asked[b] > 0.
__device__ __forceinline__ void take_pages(const PageArgs& a, int* need, uint32_t* red) {
    const int tid = threadIdx.x, per = (a.B + kTableThreads - 1) / kTableThreads, b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
    uint32_t mine = 0, total;
    for (int b = b0; b < b1; ++b) mine += (uint32_t)need[b];
    uint32_t at = block_scan(mine, red, &total);
    if (total == 0) {
        __syncthreads();
        return;
    }
    uint32_t found = 0;
    for (int base = 0; base < a.pages && found < total; base += kTableThreads * 4) {
        int r[4];
        uint32_t k = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int p = base + tid * 4 + i;
            r[i] = p < a.pages ? load_fresh(a.refs + p) : 1;
            k += r[i] == 0;
        }
        uint32_t here, place = found + block_scan(k, red, &here);
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r[i] == 0) {
                if (place < (uint32_t)a.pages) a.ws_list[place] = base + tid * 4 + i;
                ++place;
            }
        found += here;
    }
    if (found >= total) {
        for (int b = b0; b < b1; ++b) {
            const uint32_t k = (uint32_t)need[b];
            need[b] = (int)at;
            at += k;
        }
    } else if (tid == 0) {
        uint32_t place = 0;
        for (int b = 0; b < a.B; ++b) {
            const uint32_t k = (uint32_t)need[b];
            if (place + k > found) need[b] = -1;
            else need[b] = (int)place, place += k;
        }
    }
    __syncthreads();
}

// The rows of the table are shared out to teams of threads, as many as a row has pages, at most a wave: a launch of one workgroup is a
// chain of trips to memory, and what few rows ask for goes in one trip.
struct Team {
    int shift, first, step, lane;  // log2 of its threads; its first row, rows between two of its own; this thread's place
    __device__ __forceinline__ Team(int max_pages) {
        shift = 0;
        while ((1 << shift) < max_pages && shift < 6) ++shift;
        first = threadIdx.x >> shift;
        step = kTableThreads >> shift;
        lane = threadIdx.x & ((1 << shift) - 1);
    }
    __device__ __forceinline__ int size() const { return 1 << shift; }
};

// Gives up every page that a row of the table names (`size` threads).
__device__ __forceinline__ void release_row(const PageArgs& a, const int32_t* row, int lane, int size) {
    for (int j = lane; j < a.max_pages; j += size) {
        const int p = row[j];
        if ((unsigned)p < (unsigned)a.pages) atomicSub(a.refs + p, 1);
        else if (p != -1) count_error(a);
    }
}

__global__ void __launch_bounds__(kTableThreads) page_reserve_kernel(const PageArgs a) {
    extern __shared__ int need[];  // [B]
    __shared__ uint32_t red[kTableThreads / 64];
    const int tid = threadIdx.x;
    const int64_t room = (int64_t)a.max_pages * 64;
    auto asks = [&](int b, int* len, int* add) {
        *len = a.len[b];
        *add = a.seq_n ? a.seq_n[b] : a.n;
        if (*add < 1 || *add > a.n) *add = 0;
        return *add == 0 ? 0 : *len < 0 || *len + (int64_t)*add > room ? -1 : pages_of(*len + *add) - pages_of(*len);
    };
    for (int b = tid; b < a.B; b += kTableThreads) {
        int len, add;
        const int k = asks(b, &len, &add);
        if (k < 0) count_error(a);
        need[b] = max(k, 0);
    }
    __syncthreads();
    take_pages(a, need, red);
    const Team team(a.max_pages);
    const int lane = team.lane;
    for (int b = team.first; b < a.B; b += team.step) {
        int len, add;
        const int k = asks(b, &len, &add);
        __builtin_amdgcn_wave_barrier();         // (the length is read by all of the team before it is written)
        if (k < 0 || add == 0) continue;
        if (k > 0 && need[b] < 0) {
            if (lane == 0) count_error(a);
            continue;
        }
        const int have = pages_of(len);
        for (int j = lane; j < k; j += team.size()) {
            const int p = a.ws_list[need[b] + j];
            a.table[(int64_t)b * a.max_pages + have + j] = p;
            a.refs[p] = 1;
        }
        if (lane == 0) a.len[b] = len + add;
    }
}

__global__ void __launch_bounds__(kPageThreads) page_free_kernel(const PageArgs a) {
    const int b = blockIdx.x * kPageWaves + (threadIdx.x >> 6), lane = threadIdx.x & 63;
    if (b >= a.B || (a.which && a.which[b] == 0)) return;
    int32_t* row = a.table + (int64_t)b * a.max_pages;
    release_row(a, row, lane, kWave);
    for (int j = lane; j < a.max_pages; j += kWave) row[j] = -1;
    if (lane == 0) a.len[b] = 0;
}

// Rows that go on as another row's do: their pages are released, the parent's full ones shared, and a page taken for its last where that
// is not full; what is to be copied goes to ws_copy.
__global__ void __launch_bounds__(kTableThreads) page_fork_kernel(const PageArgs a) {
    extern __shared__ int need[];  // [B]; first the parent, -1: the row stays as it is, -2: it comes out empty
    __shared__ uint32_t red[kTableThreads / 64];
    const int tid = threadIdx.x;
    const int64_t room = (int64_t)a.max_pages * 64;
    const Team team(a.max_pages);
    const int lane = team.lane;
    for (int b = tid; b < a.B; b += kTableThreads) {
        const int p = a.which[b];
        int from = -1;
        if (p != b) {
            if ((unsigned)p < (unsigned)a.B) {
                const int further = a.which[p], n = a.len[p];
                if (further == p && n >= 0 && n <= room) from = p;
            }
            if (from < 0) count_error(a);
        }
        need[b] = from;
    }
    __syncthreads();
    for (int b = team.first; b < a.B; b += team.step) {
        const int p = need[b];
        if (p < 0) continue;
        const int32_t* theirs = a.table + (int64_t)p * a.max_pages;
        const int many = pages_of(a.len[p]);
        for (int j = lane; j < many; j += team.size())
            if ((unsigned)theirs[j] >= (unsigned)a.pages) need[b] = -2;  // the parent's row names a page that there is not
    }
    __syncthreads();
    for (int b = team.first; b < a.B; b += team.step) {
        const int p = need[b];
        if (p == -1) {
            if (lane == 0) a.ws_copy[b] = make_int2(-1, -1);
            continue;
        }
        int32_t* row = a.table + (int64_t)b * a.max_pages;
        const int32_t* theirs = a.table + (int64_t)max(p, 0) * a.max_pages;
        const int n = p < 0 ? 0 : a.len[p], full = n >> 6;
        for (int j = lane; j < a.max_pages; j += team.size()) {
            const int old = row[j], share = j < full ? theirs[j] : -1;
            if ((unsigned)old < (unsigned)a.pages) atomicSub(a.refs + old, 1);
            else if (old != -1) count_error(a);
            if (share >= 0) atomicAdd(a.refs + share, 1);
            row[j] = share;
        }
        if (lane == 0) {
            if (p < 0) count_error(a);
            // the page to copy; -3: no page more, -2: comes out empty
            a.ws_copy[b] = make_int2(p < 0 ? -2 : (n & 63) ? theirs[full] : -3, p);
        }
    }
    __threadfence();
    __syncthreads();
    for (int b = tid; b < a.B; b += kTableThreads) need[b] = a.ws_copy[b].x >= 0;
    __syncthreads();
    take_pages(a, need, red);
    for (int b = tid; b < a.B; b += kTableThreads) {
        const int2 c = a.ws_copy[b];
        if (c.x == -1) continue;
        const int n = c.x == -2 ? 0 : a.len[c.y];
        int2 copy = make_int2(-1, -1);
        if (c.x >= 0) {
            if (need[b] < 0) {                   // no page left: it comes out empty
                count_error(a);
                int32_t* row = a.table + (int64_t)b * a.max_pages;
                for (int j = 0; j < (n >> 6); ++j) {
                    atomicSub(a.refs + row[j], 1);
                    row[j] = -1;
                }
                a.len[b] = 0;
                a.ws_copy[b] = copy;
                continue;
            }
            const int to = a.ws_list[need[b]];
            a.table[(int64_t)b * a.max_pages + (n >> 6)] = to;
            a.refs[to] = 1;
            copy = make_int2(c.x, to);
        }
        a.len[b] = n;
        a.ws_copy[b] = copy;
    }
}

// Whole pages, a layer of one row's a workgroup group: blockIdx = (piece, row, layer).
__global__ void __launch_bounds__(kPageThreads) page_copy_kernel(const PageArgs a, int64_t bytes) {
    const int2 c = a.ws_copy[blockIdx.y];
    if (c.x < 0) return;
    const int64_t src = (int64_t)blockIdx.z * a.pages + c.x, dst = (int64_t)blockIdx.z * a.pages + c.y;
    const uint4* from[2] = {(const uint4*)(a.K + src * bytes), (const uint4*)(a.V + src * bytes)};
    uint4* to[2] = {(uint4*)(a.K + dst * bytes), (uint4*)(a.V + dst * bytes)};
    const int64_t pieces = bytes / 16;
    for (int64_t i = (int64_t)blockIdx.x * 2 * kPageThreads + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * 2 * kPageThreads) {
        const bool two = i + kPageThreads < pieces;
        uint4 v[4];
        v[0] = stream_load(from[0] + i);
        v[1] = stream_load(from[1] + i);
        if (two) v[2] = stream_load(from[0] + i + kPageThreads), v[3] = stream_load(from[1] + i + kPageThreads);
        to[0][i] = v[0];
        to[1][i] = v[1];
        if (two) to[0][i + kPageThreads] = v[2], to[1][i + kPageThreads] = v[3];
    }
    if (blockIdx.x == 0)
        for (int h = threadIdx.x; h < a.H; h += kPageThreads) {
            a.k_scale[dst * a.H + h] = a.k_scale[src * a.H + h];
            a.v_scale[dst * a.H + h] = a.v_scale[src * a.H + h];
        }
}

// New pages for the rows that keep k of their tokens; the old row of the table goes to ws_old (its length to ws_copy), and its pages are
// given up after the new ones were taken: they are read until the launch behind this one is done.
__global__ void __launch_bounds__(kTableThreads) page_shrink_kernel(const PageArgs a) {
    extern __shared__ int need[];  // [B]
    __shared__ uint32_t red[kTableThreads / 64];
    const int tid = threadIdx.x;
    const int64_t room = (int64_t)a.max_pages * 64;
    const Team team(a.max_pages);
    const int lane = team.lane, want = pages_of(a.kept);
    for (int b = tid; b < a.B; b += kTableThreads) {
        const int n = a.len[b], on = a.which ? a.which[b] : 1;
        const bool go = on != 0 && n > a.kept;
        need[b] = go ? n > room ? -1 : want : 0;
        a.ws_copy[b] = make_int2(go ? n : 0, 0);
    }
    __syncthreads();
    for (int b = team.first; b < a.B; b += team.step) {
        if (need[b] <= 0) continue;
        const int32_t* row = a.table + (int64_t)b * a.max_pages;
        const int many = pages_of(a.len[b]);
        for (int j = lane; j < many; j += team.size())
            if ((unsigned)row[j] >= (unsigned)a.pages) need[b] = -1;
    }
    __syncthreads();
    for (int b = tid; b < a.B; b += kTableThreads)
        if (need[b] < 0) {
            count_error(a);
            need[b] = 0;
            a.ws_copy[b] = make_int2(0, 0);
        }
    __syncthreads();
    take_pages(a, need, red);
    for (int b = tid; b < a.B; b += kTableThreads)
        if (a.ws_copy[b].x != 0) {
            if (need[b] < 0) {
                count_error(a);
                a.ws_copy[b] = make_int2(0, 0);
            } else a.len[b] = a.kept;
        }
    __threadfence_block();
    __syncthreads();
    for (int b = team.first; b < a.B; b += team.step) {
        if (a.ws_copy[b].x == 0) continue;
        int32_t* row = a.table + (int64_t)b * a.max_pages;
        int32_t* old = a.ws_old + (int64_t)b * a.max_pages;
        for (int j = lane; j < a.max_pages; j += team.size()) {
            const int had = row[j];
            int p = -1;
            if (j < want) {
                p = a.ws_list[need[b] + j];
                a.refs[p] = 1;
            }
            if ((unsigned)had < (unsigned)a.pages) atomicSub(a.refs + had, 1);
            else if (had != -1) count_error(a);
            old[j] = had;
            row[j] = p;
        }
    }
}

// ---------------------------------------------------------------- kept rows into new pages
__device__ __forceinline__ float block_most(float v, float* red) { return block_max<kPageThreads>(v, red); }

// A workgroup a new page of a head.  Keys: 16-byte pieces of rows.  Values: a wave's lanes are the page's tokens, a load a
// byte of each; a sequence's tokens are in order, so that a load falls on few lines.  Bound by these loads: a pass of 177 us where the bytes take 112.
// Tried: old rows of V whole in LDS (373 us: half of what a page holds is not kept), heads of a page on one XCD (296); whole words of the
// rows of up to four pages, whose bytes are exchanged between lanes (168, and 3 to 6 % more where less is kept).
template <int D>
__global__ void __launch_bounds__(kPageThreads) page_keep_kernel(const PageArgs a) {
    __shared__ int page_s[64], slot_s[64];
    __shared__ float ks_s[64], vs_s[64];
    __shared__ float red[kPageWaves];
    __shared__ __attribute__((aligned(16))) uint8_t turn_s[kPageWaves][D / kPageWaves * 64];
    const int tid = threadIdx.x, lane = tid & 63, wv = tid >> 6;
    // neighbouring workgroups take neighbouring heads, whose tiles lie side by side in a page
    const unsigned pages = (unsigned)(a.kept + 63) / 64, rest = blockIdx.x / (unsigned)a.H;
    const int h = (int)(blockIdx.x - rest * (unsigned)a.H), lb = (int)(rest / pages), j = (int)(rest - (unsigned)lb * pages);
    const int l = lb / a.B, b = lb - l * a.B, j0 = j * 64;
    // trips to memory in a row: the sequence, the kept tokens and the new page; the tokens' pages; their codes beside their scales
    const int live = min(64, a.kept - j0);
    const int s = a.keep[((int64_t)lb * a.H + h) * a.kept + j0 + min(lane, live - 1)];
    const int n = uniform_load(&a.ws_copy[b].x), fresh = uniform_load(a.table + (int64_t)b * a.max_pages + j);
    if (n == 0) return;
    float ks = 0.0f, vs = 0.0f;
    if (tid < 64) {
        int page = -1, slot = 0;
        if (tid < live) {
            if ((unsigned)s < (unsigned)n) {
                page = a.ws_old[(int64_t)b * a.max_pages + (s >> 6)];
                slot = s & 63;
            } else count_error(a);  // no such token: zeros
        }
        page_s[tid] = page;
        slot_s[tid] = slot;
        if (page >= 0) {
            ks = a.k_scale[((int64_t)l * a.pages + page) * a.H + h];
            vs = a.v_scale[((int64_t)l * a.pages + page) * a.H + h];
        }
    }
    __syncthreads();
    const int64_t tile = 64 * D, to = ((int64_t)l * a.pages + fresh) * a.H + h;
    const int64_t layer = (int64_t)l * a.pages;
    constexpr int CH = D / 16, PT = 64 * CH / kPageThreads, ROWS = D / kPageWaves;  // rows of values of a wave
    uint8_t vc[ROWS];
    const int vpage = page_s[lane];
    {
        const uint8_t* from = a.V + ((layer + max(vpage, 0)) * a.H + h) * tile + (int64_t)wv * ROWS * 64 + slot_s[lane];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) vc[r] = from[r * 64];
    }
    {
        uint4 c[PT];
        float most = 0.0f;
#pragma unroll
        for (int x = 0; x < PT; ++x) {
            const int p = tid + x * kPageThreads, t = p / CH;
            c[x] = make_uint4(0u, 0u, 0u, 0u);
            if (page_s[t] >= 0) c[x] = *(const uint4*)(a.K + ((layer + page_s[t]) * a.H + h) * tile + slot_s[t] * D + p % CH * 16);
        }
        if (tid < 64) ks_s[tid] = ks, vs_s[tid] = vs;
        __syncthreads();
#pragma unroll
        for (int x = 0; x < PT; ++x) {
            const float s = ks_s[(tid + x * kPageThreads) / CH];
            const uint32_t w[4] = {c[x].x, c[x].y, c[x].z, c[x].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float f[4];
                decode4(w[i], f);
#pragma unroll
                for (int e = 0; e < 4; ++e) most = fmaxf(most, finite(f[e]) ? fabsf(f[e] * s) : 0.0f);
            }
        }
        const int e = page_exponent(block_most(most, red));
        const float inv = power_of_two(-e);
#pragma unroll
        for (int x = 0; x < PT; ++x) {
            const int p = tid + x * kPageThreads, t = p / CH;
            const float s = ks_s[t];
            uint32_t w[4] = {c[x].x, c[x].y, c[x].z, c[x].w};
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float f[4];
                decode4(w[i], f);
                w[i] = encode4(f[0] * s, f[1] * s, f[2] * s, f[3] * s, inv);
            }
            if (t < live) *(uint4*)(a.K + to * tile + p * 16) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        if (tid == 0) a.k_scale[to] = power_of_two(e);
    }
    {
        uint8_t c[ROWS];
        const float s = vs_s[lane];
#pragma unroll
        for (int r = 0; r < ROWS; ++r) c[r] = vpage < 0 ? 0 : vc[r];
        float most = 0.0f;
#pragma unroll
        for (int r = 0; r < ROWS; r += 4) {
            float f[4];
            decode4(c[r] | c[r + 1] << 8 | c[r + 2] << 16 | (uint32_t)c[r + 3] << 24, f);
#pragma unroll
            for (int e = 0; e < 4; ++e) most = fmaxf(most, finite(f[e]) ? fabsf(f[e] * s) : 0.0f);
        }
        const int e = page_exponent(block_most(most, red));
        const float inv = power_of_two(-e);
        // by way of the wave's own LDS: 16 tokens of a row a store
        uint8_t* turn = turn_s[wv];
#pragma unroll
        for (int r = 0; r < ROWS; r += 4) {
            float f[4];
            decode4(c[r] | c[r + 1] << 8 | c[r + 2] << 16 | (uint32_t)c[r + 3] << 24, f);
            const uint32_t v = encode4(f[0] * s, f[1] * s, f[2] * s, f[3] * s, inv);
#pragma unroll
            for (int i = 0; i < 4; ++i) turn[(r + i) * 64 + lane] = (uint8_t)(v >> (8 * i));
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        uint8_t* w = a.V + to * tile + (int64_t)wv * ROWS * 64;
#pragma unroll
        for (int x = 0; x < ROWS / 16; ++x) {
            const int p = x * kWave + lane, t = p % 4 * 16;
            if (t + 16 <= live) *(uint4*)(w + p * 16) = *(const uint4*)(turn + p * 16);
            else
                for (int i = t; i < live; ++i) w[p * 16 + i - t] = turn[p * 16 + i - t];
        }
        if (tid == 0) a.v_scale[to] = power_of_two(e);
    }
}

// ---------------------------------------------------------------- rows into pages
// blockIdx.x = (layer * B + row, page behind the first that the call touches, head), the head fastest.  A thread holds 16-byte pieces of the page's new rows;
// values are turned in LDS.
template <typename T, int D>
__global__ void __launch_bounds__(kPageThreads) page_write_kernel(const PageArgs a) {
    constexpr int CH = D / 8, PT = 64 * CH / kPageThreads, Y = PT < 4 ? PT : 4, PITCH = 64 + 4;
    __shared__ __attribute__((aligned(16))) uint8_t turn[D * PITCH];
    // piece x of a thread: Y neighbouring tokens, then the next group of them
    auto token_of = [](int x) { return ((int)threadIdx.x / CH + x / Y * (kPageThreads / CH)) * Y + x % Y; };
    const int column = (int)threadIdx.x % CH;
    __shared__ float red[kPageWaves];
    const int tid = threadIdx.x;
    const unsigned pages = ((unsigned)a.n + 62u) / 64 + 1, rest = blockIdx.x / (unsigned)a.H;
    const int h = (int)(blockIdx.x - rest * (unsigned)a.H), lb = (int)(rest / pages), jx = (int)(rest - (unsigned)lb * pages);
    const int l = lb / a.B, b = lb - l * a.B;
    const int add = a.seq_n ? a.seq_n[b] : a.n, len = a.len[b];
    if (add < 1 || add > a.n) return;
    const bool none = len < add || len > (int64_t)a.max_pages * 64;
    const int first = len - add, j = (first >> 6) + jx;
    if (none || (int64_t)j * 64 >= len) {
        if (none && jx == 0 && tid == 0) count_error(a);  // no room was reserved for these rows
        return;
    }
    const int page = a.table[(int64_t)b * a.max_pages + j];
    if ((unsigned)page >= (unsigned)a.pages) {
        if (tid == 0) count_error(a);
        return;
    }
    const int s0 = max(first - j * 64, 0), s1 = min(len - j * 64, 64);  // slots of the new rows
    const int64_t at = ((int64_t)l * a.pages + page) * a.H + h;
    uint4 rows[2][PT];
    // what the page holds already, where not all of it is new: in the same trip
    constexpr int OT = 64 * D / 16 / kPageThreads;
    const bool beside = s0 > 0 || s1 < 64;
    const int holders = uniform_load(a.refs + page);
    uint4 held[2][OT];
    int was[2];
#pragma unroll
    for (int tensor = 0; tensor < 2; ++tensor) {
        const uint4* dst = (const uint4*)((tensor ? a.V : a.K) + at * 64 * D);
        was[tensor] = exponent_of(uniform_load((tensor ? a.v_scale : a.k_scale) + at));
#pragma unroll
        for (int x = 0; x < OT; ++x) {
            held[tensor][x] = make_uint4(0u, 0u, 0u, 0u);
            if (beside) held[tensor][x] = dst[tid + x * kPageThreads];
        }
        const T* src = (const T*)(tensor ? a.v : a.k) + (((int64_t)lb * a.H + h) * a.rows + (j * 64 - first)) * D;  // row of slot 0
#pragma unroll
        for (int x = 0; x < PT; ++x) {
            const int t = token_of(x);
            rows[tensor][x] = make_uint4(0u, 0u, 0u, 0u);
            if (t >= s0 && t < s1) rows[tensor][x] = stream_load((const uint4*)(src + t * D) + column);
        }
    }
    if (holders > 1) {                           // others hold the page: no room was reserved
        if (tid == 0) count_error(a);
        return;
    }
#pragma unroll
    for (int tensor = 0; tensor < 2; ++tensor) {
        uint8_t* dst = (tensor ? a.V : a.K) + at * 64 * D;
        float* scale = (tensor ? a.v_scale : a.k_scale) + at;
        const uint4(&r)[PT] = rows[tensor];
        float most = 0.0f;
#pragma unroll
        for (int x = 0; x < PT; ++x) {
            float f[8];
            unpack16<T>(r[x], f);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, finite(f[i]) ? fabsf(f[i]) : 0.0f);
        }
        int e = page_exponent(block_most(most, red));
        float ratio = 1.0f;                      // of the older rows' scale to the new one
        if (s0 > 0) {
            e = max(e, was[tensor]);
            ratio = power_of_two(max(was[tensor] - e, -126));
        }
        const float inv = power_of_two(-e);
        if (tensor == 0) {
#pragma unroll
            for (int x = 0; x < PT; ++x) {
                const int t = token_of(x);
                float f[8];
                unpack16<T>(r[x], f);
                if (t >= s0 && t < s1) *(uint2*)(dst + t * D + column * 8) = make_uint2(encode4(f[0], f[1], f[2], f[3], inv), encode4(f[4], f[5], f[6], f[7], inv));
            }
            if (ratio != 1.0f) {
#pragma unroll
                for (int x = 0; x < OT; ++x) {
                    const int p = tid + x * kPageThreads;
                    const uint4 o = held[0][x];
                    if (p < s0 * (D / 16)) ((uint4*)dst)[p] = make_uint4(again4(o.x, ratio), again4(o.y, ratio), again4(o.z, ratio), again4(o.w, ratio));
                }
            }
        } else {
            // an element of Y tokens is one write to LDS (a byte at a time, 16 lanes on a bank, 512-byte rows took twice as long)
#pragma unroll
            for (int x = 0; x < PT; x += Y) {
                uint32_t w[Y][2];
#pragma unroll
                for (int y = 0; y < Y; ++y) {
                    float f[8];
                    unpack16<T>(r[x + y], f);
                    w[y][0] = encode4(f[0], f[1], f[2], f[3], inv), w[y][1] = encode4(f[4], f[5], f[6], f[7], inv);
                }
                uint8_t* to = turn + column * 8 * PITCH + token_of(x);
#pragma unroll
                for (int q = 0; q < 2; ++q) {
                    if constexpr (Y == 4) {
                        const uint32_t a01 = __builtin_amdgcn_perm(w[1][q], w[0][q], 0x05010400u), b01 = __builtin_amdgcn_perm(w[1][q], w[0][q], 0x07030602u);
                        const uint32_t a23 = __builtin_amdgcn_perm(w[3][q], w[2][q], 0x05010400u), b23 = __builtin_amdgcn_perm(w[3][q], w[2][q], 0x07030602u);
                        *(uint32_t*)(to + (4 * q) * PITCH) = __builtin_amdgcn_perm(a23, a01, 0x05040100u);
                        *(uint32_t*)(to + (4 * q + 1) * PITCH) = __builtin_amdgcn_perm(a23, a01, 0x07060302u);
                        *(uint32_t*)(to + (4 * q + 2) * PITCH) = __builtin_amdgcn_perm(b23, b01, 0x05040100u);
                        *(uint32_t*)(to + (4 * q + 3) * PITCH) = __builtin_amdgcn_perm(b23, b01, 0x07060302u);
                    } else {
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            *(uint16_t*)(to + (4 * q + i) * PITCH) = (uint16_t)((w[0][q] >> (8 * i) & 255u) | (w[Y - 1][q] >> (8 * i) & 255u) << 8);
                    }
                }
            }
            __syncthreads();
#pragma unroll
            for (int x = 0; x < OT; ++x) {
                const int p = tid + x * kPageThreads, d = p >> 2, t = (p & 3) * 16;
                if (t + 16 <= s0 && ratio == 1.0f) continue;
                if (t >= s1) continue;
                const uint32_t* from = (const uint32_t*)(turn + d * PITCH + t);
                uint4 v = make_uint4(from[0], from[1], from[2], from[3]);
                if (t < s0 || t + 16 > s1) {     // older rows or none beside them
                    const uint4 o = held[1][x];
                    uint32_t w[4] = {v.x, v.y, v.z, v.w};
                    const uint32_t had[4] = {o.x, o.y, o.z, o.w};
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const uint32_t older = ratio == 1.0f ? had[i] : again4(had[i], ratio);
                        uint32_t out = 0;
#pragma unroll
                        for (int y = 0; y < 4; ++y) {
                            const int s = t + 4 * i + y;
                            out |= (s < s0 ? older : s < s1 ? w[i] : had[i]) & 0xFFu << (8 * y);
                        }
                        w[i] = out;
                    }
                    v = make_uint4(w[0], w[1], w[2], w[3]);
                }
                *(uint4*)(dst + d * 64 + t) = v;
            }
        }
        if (tid == 0) *scale = power_of_two(e);  // (read by the whole workgroup ahead of a barrier)
    }
}

// ---------------------------------------------------------------- the token's step
// Eight codes -> eight elements of a product's operand.
__device__ __forceinline__ p_h8_t halves8(uint32_t a, uint32_t b) {
    const p_h2_t x = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false), y = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
    const p_h2_t z = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false), w = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
    return p_h8_t{x.x, x.y, y.x, y.y, z.x, z.y, w.x, w.y};
}
__device__ __forceinline__ p_bf8_t brains8(uint32_t a, uint32_t b) {
    const p_bf2_t x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(a, 1.0f, true);
    const p_bf2_t z = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, false), w = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(b, 1.0f, true);
    return p_bf8_t{x.x, x.y, y.x, y.y, z.x, z.y, w.x, w.y};
}
template <typename T>
__device__ __forceinline__ p_f4_t key_product(const uint4& k, const uint4& q, p_f4_t c) {  // 16-bit elements on both sides
    if constexpr (__is_same(T, bf16_t)) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(p_bf8_t, k), __builtin_bit_cast(p_bf8_t, q), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(p_h8_t, k), __builtin_bit_cast(p_h8_t, q), c, 0, 0, 0);
}
template <typename T>
__device__ __forceinline__ p_f4_t code_product(uint32_t k0, uint32_t k1, const uint4& q, p_f4_t c) {
    if constexpr (__is_same(T, bf16_t)) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(brains8(k0, k1), __builtin_bit_cast(p_bf8_t, q), c, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(halves8(k0, k1), __builtin_bit_cast(p_h8_t, q), c, 0, 0, 0);
}
__device__ __forceinline__ p_h2_t truncated(float a, float b) { return __builtin_bit_cast(p_h2_t, __builtin_amdgcn_cvt_pkrtz(a, b)); }

__device__ __forceinline__ float across_max(float v) {  // over the four groups of 16 lanes
    v = fmaxf(v, __shfl_xor(v, 16, kWave));
    return fmaxf(v, __shfl_xor(v, 32, kWave));
}
__device__ __forceinline__ float across_sum(float v) {
    v += __shfl_xor(v, 16, kWave);
    return v + __shfl_xor(v, 32, kWave);
}

constexpr float kPageLift = 10.0f;   // probabilities are held 2^10 times as large, so that their lower half stays a normal number
constexpr float kPageSlack = 4.0f;   // a reference is raised once a row's largest exponent is this far above it: at most 2^14

// One element row into its page (a wave): values or keys, slot s.  A page that several sequences hold is not written: false.
template <typename T, int D>
__device__ __forceinline__ bool page_append(const T* row, uint8_t* dst, float* scale, const int32_t* refs, int s, bool values, int lane) {
    constexpr int E = D / 64;
    const int holders = *refs;
    float f[E], most = 0.0f;
#pragma unroll
    for (int i = 0; i < E; ++i) {
        const uint16_t w = ((const uint16_t*)row)[lane + 64 * i];
        f[i] = __is_same(T, bf16_t) ? __uint_as_float((uint32_t)w << 16) : f16_lo(w);
        most = fmaxf(most, finite(f[i]) ? fabsf(f[i]) : 0.0f);
    }
    int e = page_exponent(wave_max(most));
    if (holders > 1) return false;
    if (s > 0) {
        const int old = exponent_of(*scale);
        if (e > old) {  // the older rows are rounded again
            const float ratio = power_of_two(max(old - e, -126));
            if (values) {
#pragma unroll
                for (int i = 0; i < E; ++i) {
                    uint32_t* w = (uint32_t*)(dst + (lane + 64 * i) * 64);
                    for (int x = 0; x * 4 < s; ++x) {
                        const uint32_t had = w[x], mask = s - x * 4 >= 4 ? ~0u : (1u << 8 * (s - x * 4)) - 1u;
                        w[x] = (again4(had, ratio) & mask) | (had & ~mask);
                    }
                }
            } else {
                for (int p = lane; p < s * (D / 4); p += kWave) ((uint32_t*)dst)[p] = again4(((uint32_t*)dst)[p], ratio);
            }
        }
        e = max(e, old);
    }
    const float inv = power_of_two(-e);
#pragma unroll
    for (int i = 0; i < E; ++i) dst[values ? (lane + 64 * i) * 64 + s : s * D + lane + 64 * i] = encode1(f[i], inv);
    if (lane == 0) *scale = power_of_two(e);
    return true;
}

// blockIdx.x = unit * S + split, unit = (layer * B + row) * H + head.  A split is a.chunk pages, shared out to the waves.
template <typename T, int D, bool BIAS, int NW>
__global__ void __launch_bounds__(NW * kWave, 2) page_step_kernel(const PageArgs a) {
    constexpr int C = D / 64, NQ = D / 32, DT = D / 16;
    constexpr int PARTS = D > 128 ? 2 : 1, CP = C / PARTS, DP = DT / PARTS;  // a page of wide rows is held by halves: two waves on a SIMD
    __shared__ float o_s[NW][8][D];
    __shared__ float m_s[NW][8], l_s[NW][8];
    const int tid = threadIdx.x, lane = tid & 63, wv = __builtin_amdgcn_readfirstlane(tid >> 6), n0 = lane & 15, g = lane >> 4;
    const unsigned u = blockIdx.x / (unsigned)a.S;
    const int split = (int)(blockIdx.x - u * (unsigned)a.S);
    const unsigned lb = u / (unsigned)a.H;
    const int h = (int)(u - lb * (unsigned)a.H), l = (int)(lb / (unsigned)a.B), b = (int)(lb - (unsigned)l * (unsigned)a.B);
    // a wave's first page is looked up beside the length that says whether it is one
    const int32_t* table = a.table + (int64_t)b * a.max_pages;
    const int p0 = split * a.chunk;
    const int n = uniform_load(a.len + b), ask = a.seq_n ? uniform_load(a.seq_n + b) : 1;
    int ahead = uniform_load(table + min(p0 + wv, a.max_pages - 1));
    const bool asked = ask == 1, there = n >= 1 && n <= (int64_t)a.max_pages * 64;
    float* out = a.out + (int64_t)u * a.G * D;
    if (!asked || !there) {
        if (split == 0) {
            for (int i = tid; i < a.G * D; i += NW * kWave) out[i] = 0.0f;
            if (asked && tid == 0) count_error(a);
        }
        return;
    }
    const int old = n - 1, tail = old >> 6, owner = min(tail / a.chunk, a.S - 1);
    if (split > owner) return;
    const int p1 = split == owner ? tail + ((old & 63) != 0) : p0 + a.chunk;

    // A page's keys (or the half of them) are asked for when those before are used up, its values likewise: a wave always has some under way.
    uint4 k[4][CP], v[DP];
    float ks = 0.0f, vs = 0.0f;
    int page = -1;
    int64_t at = 0;
    const uint32_t klane = ((n0 >> 2) * 16 + (n0 & 3)) * D + g * 16, vlane = n0 * 64 + g * 16;
    auto find = [&](int j) {                     // a number that is no page's leaves the page's tokens out, and page 0 is read
        page = ahead;
        if (j < p1 && (unsigned)page >= (unsigned)a.pages) {
            if (lane == 0) count_error(a);
            page = -1;
        }
        ahead = uniform_load(table + min(j + NW, a.max_pages - 1));
        return ((int64_t)l * a.pages + max(page, 0)) * a.H + h;
    };
    auto bring_keys = [&](int64_t tile, int part) {
        const uint8_t* kp = a.K + tile * 64 * D + part * CP * 64 + klane;
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int c = 0; c < CP; ++c) k[t][c] = stream_load((const uint4*)(kp + t * 4 * D + c * 64));
        if (part == 0) ks = uniform_load(a.k_scale + tile) * a.sc;
    };
    auto bring_values = [&](int64_t tile, int part) {
        const uint8_t* vp = a.V + tile * 64 * D + part * DP * 16 * 64 + vlane;
#pragma unroll
        for (int i = 0; i < DP; ++i) v[i] = stream_load((const uint4*)(vp + i * 16 * 64));
        if (part == 0) vs = uniform_load(a.v_scale + tile);
    };
    if (p0 + wv < p1) {
        at = find(p0 + wv);
        bring_keys(at, 0);
        bring_values(at, 0);
    }

    const int head = n0 & 7, part = n0 >> 3;     // of this lane's column
    uint4 q[NQ];
    {
        const T* p = (const T*)a.q + ((int64_t)u * a.G + min(head, a.G - 1)) * D + g * 16;
#pragma unroll
        for (int c = 0; c < NQ; ++c) q[c] = *(const uint4*)(p + (c >> 1) * 64 + (c & 1) * 8);
    }
    float slope = 0.0f;
    if constexpr (BIAS) slope = a.slopes[h * a.G + min(head, a.G - 1)] * kLog2e;

    p_f4_t o[DT];
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] = p_f4_t{0.0f, 0.0f, 0.0f, 0.0f};
    float m = -INFINITY, sum = 0.0f;
    const T* kn = (const T*)a.k + (int64_t)u * D;
    const T* vn = (const T*)a.v + (int64_t)u * D;
    if (split == owner && wv == 0) {             // the token itself: row 0 of a tile
        p_f4_t x = p_f4_t{0.0f, 0.0f, 0.0f, 0.0f};
        uint4 row[NQ];
#pragma unroll
        for (int c = 0; c < NQ; ++c) row[c] = *(const uint4*)(kn + g * 16 + (c >> 1) * 64 + (c & 1) * 8);
#pragma unroll
        for (int c = 0; c < NQ; ++c) x = key_product<T>(n0 == 0 ? row[c] : make_uint4(0u, 0u, 0u, 0u), q[c], x);
        m = __shfl(x[0], n0, kWave) * a.sc;
        const float p = hw_exp2(m - (m == -INFINITY ? 0.0f : m) + kPageLift);
        sum = g == 0 ? p : 0.0f;
#pragma unroll
        for (int i = 0; i < DT; ++i) {
            const uint2 v = *(const uint2*)(vn + i * 16 + g * 4);
            float f[8];
            unpack16<T>(make_uint4(v.x, v.y, 0u, 0u), f);
#pragma unroll
            for (int r = 0; r < 4; ++r) o[i][r] = part == 0 ? p * f[r] : 0.0f;
        }
    }

    for (int j = p0 + wv; j < p1; j += NW) {
        const int live = page < 0 ? 0 : old;     // tokens that are there
        const float kby = ks, vby = page < 0 ? 0.0f : vs;
        const bool more = j + NW < p1;
        int64_t next = at;
        p_f4_t x[4];
#pragma unroll
        for (int t = 0; t < 4; ++t) x[t] = p_f4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int c = 0; c < CP; ++c) {
                    x[t] = code_product<T>(k[t][c].x, k[t][c].y, q[2 * (part * CP + c)], x[t]);
                    x[t] = code_product<T>(k[t][c].z, k[t][c].w, q[2 * (part * CP + c) + 1], x[t]);
                }
            if (part + 1 < PARTS) bring_keys(at, part + 1);
            else if (more) {
                next = find(j + NW);
                bring_keys(next, 0);
            }
        }
        const int j0 = j * 64 + g * 16;          // token of x[t][r]: j0 + 4 t + r
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (BIAS) x[t][r] = fmaf(x[t][r], kby, slope * (float)(j0 + 4 * t + r - old));
                else x[t][r] *= kby;
            }
        uint4 tail_mask = make_uint4(~0u, ~0u, ~0u, ~0u);
        if (j * 64 + 64 > live) {                // the last page: slots that hold no token of this sequence, or the new one's
#pragma unroll
            for (int t = 0; t < 4; ++t)
#pragma unroll
                for (int r = 0; r < 4; ++r) x[t][r] = j0 + 4 * t + r < live ? x[t][r] : -INFINITY;
            const int have = max(min(live - j0, 16), 0);
            uint32_t mask[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) mask[i] = have - 4 * i >= 4 ? ~0u : have - 4 * i <= 0 ? 0u : (1u << 8 * (have - 4 * i)) - 1u;
            tail_mask = make_uint4(mask[0], mask[1], mask[2], mask[3]);
        }
        float top = x[0][0];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, x[t][r]);
        top = across_max(top);
        if (__any(top > m + kPageSlack || m == -INFINITY)) {
            const float to = fmaxf(m, top), by = to == -INFINITY ? 1.0f : hw_exp2(m - to);
            m = to;
            sum *= by;
#pragma unroll
            for (int i = 0; i < DT; ++i) o[i] *= by;
        }
        const float ref = (m == -INFINITY ? 0.0f : m) - kPageLift;
        p_h8_t p[2];
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                const float e0 = hw_exp2(x[t][r] - ref), e1 = hw_exp2(x[t][r + 1] - ref);
                sum += e0 + e1;
                const p_h2_t hi = truncated(e0, e1), lo = truncated(e0 - (float)hi.x, e1 - (float)hi.y);
                const p_h2_t w = part == 0 ? hi : lo;
                p[t >> 1][(t & 1) * 4 + r] = w.x;
                p[t >> 1][(t & 1) * 4 + r + 1] = w.y;
            }
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            if (j * 64 + 64 > live) {
#pragma unroll
                for (int i = 0; i < DP; ++i) v[i].x &= tail_mask.x, v[i].y &= tail_mask.y, v[i].z &= tail_mask.z, v[i].w &= tail_mask.w;
            }
#pragma unroll
            for (int i = 0; i < DP; ++i) {
                p_f4_t y = p_f4_t{0.0f, 0.0f, 0.0f, 0.0f};
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves8(v[i].x, v[i].y), p[0], y, 0, 0, 0);
                y = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves8(v[i].z, v[i].w), p[1], y, 0, 0, 0);
#pragma unroll
                for (int r = 0; r < 4; ++r) o[part * DP + i][r] = fmaf(y[r], vby, o[part * DP + i][r]);
            }
            if (part + 1 < PARTS) bring_values(at, part + 1);
            else if (more) bring_values(next, 0);
        }
        at = next;
    }

    sum = across_sum(sum);
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            o[i][r] += __uint_as_float((uint32_t)__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(o[i][r]), 0x128, 0xF, 0xF, false));  // column +- 8
            if (n0 < 8) o_s[wv][n0][i * 16 + g * 4 + r] = o[i][r];
        }
    if (lane < 8) m_s[wv][lane] = m, l_s[wv][lane] = sum;
    __syncthreads();
    for (int i = tid; i < a.G * D; i += NW * kWave) {
        const int y = i / D, d = i - y * D;
        float top = m_s[0][y];
#pragma unroll
        for (int w = 1; w < NW; ++w) top = fmaxf(top, m_s[w][y]);
        const float ref = top == -INFINITY ? 0.0f : top;
        float s = 0.0f, v = 0.0f;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            const float by = hw_exp2(m_s[w][y] - ref);
            s = fmaf(by, l_s[w][y], s);
            v = fmaf(by, o_s[w][y][d], v);
        }
        if (a.S == 1) out[i] = s == 0.0f ? 0.0f : v / s;
        else {
            const int64_t at = ((int64_t)u * a.S + split) * a.G + y;
            a.ws_o[at * D + d] = v;
            if (d == 0) a.ws_ml[at] = make_float2(top, s);
        }
    }
    if (split == owner && wv < 2) {              // every wave is done with the page
        const int last = uniform_load(table + tail);
        if ((unsigned)last < (unsigned)a.pages) {
            const int64_t to = ((int64_t)l * a.pages + last) * a.H + h;
            for (int tensor = wv; tensor < 2; tensor += NW)
                if (!page_append<T, D>(tensor ? vn : kn, (tensor ? a.V : a.K) + to * 64 * D, (tensor ? a.v_scale : a.k_scale) + to, a.refs + last, old & 63,
                                       tensor != 0, lane) && tensor == 0 && lane == 0)
                    count_error(a);
        } else if (tid == 0 && (old & 63) == 0) count_error(a);
    }
}

// Joins the splits of a unit's head: D / 4 threads take a row of sums, the groups of them every so many-th split.
constexpr int kPageMaxSplits = 256;
template <int D>
__global__ void __launch_bounds__(kPageThreads) page_join_kernel(const PageArgs a) {
    constexpr int LANES = D / 4, GROUPS = kPageThreads / LANES;
    __shared__ float by_s[kPageMaxSplits];
    __shared__ float red[kPageWaves];
    __shared__ float4 part[GROUPS][LANES];
    const unsigned u = blockIdx.x / (unsigned)a.G;
    const int y = (int)(blockIdx.x - u * (unsigned)a.G), tid = threadIdx.x, grp = tid / LANES, e = tid % LANES;
    const int b = (int)(u / (unsigned)a.H % (unsigned)a.B), n = a.len[b];
    if ((a.seq_n && a.seq_n[b] != 1) || n < 1 || n > (int64_t)a.max_pages * 64) return;
    const int parts = min(((n - 1) >> 6) / a.chunk, a.S - 1) + 1;
    const int64_t at = (int64_t)u * a.S * a.G + y;
    float2 ml = make_float2(-INFINITY, 0.0f);
    if (tid < parts) ml = a.ws_ml[at + (int64_t)tid * a.G];
    const float top = block_max<kPageThreads>(ml.x, red), by = hw_exp2(ml.x - (top == -INFINITY ? 0.0f : top));
    if (tid < parts) by_s[tid] = by;
    const float sum = block_sum<kPageThreads>(tid < parts ? by * ml.y : 0.0f, red);
    float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int s = grp; s < parts; s += GROUPS) {
        const float4 x = ((const float4*)(a.ws_o + (at + (int64_t)s * a.G) * D))[e];
        const float w = by_s[s];
        v.x = fmaf(w, x.x, v.x), v.y = fmaf(w, x.y, v.y), v.z = fmaf(w, x.z, v.z), v.w = fmaf(w, x.w, v.w);
    }
    part[grp][e] = v;
    __syncthreads();
    if (grp > 0) return;
#pragma unroll
    for (int s = 1; s < GROUPS; ++s) {
        const float4 x = part[s][e];
        v.x += x.x, v.y += x.y, v.z += x.z, v.w += x.w;
    }
    const float inv = sum == 0.0f ? 0.0f : 1.0f / sum;
    float* out = a.out + ((int64_t)u * a.G + y) * D + 4 * e;  // (of any alignment)
    out[0] = v.x * inv, out[1] = v.y * inv, out[2] = v.z * inv, out[3] = v.w * inv;
}

// ---------------------------------------------------------------- launches
// Workgroups of four waves, or of one, and the splits of a unit's pages.  A wave keeps a page under way, so that one or two waves a SIMD, 1024
// to 2048 of them (twice as many with rows half as long), are what the memory asks for.
// As many units take one wave each (2048 units x 1000 x 128: 95 us, with four waves each 110; x 60: 18 and 29), of long ones up to four splits, lest
// a long unit among short ones is one chain; from half as many on two waves each where pages pay for the join (640 units x 1300: 44 us, with
// four waves each 51).  Fewer units take four waves and as many splits as make up to 512 workgroups, which all run at once (512 units x 1024 x 128: 29 us,
// two splits 35, two of one wave 34), a page a wave at least; long units, whose splits cost little, as many as hold 24 pages each, up to 1024
// workgroups (48 units of up to 31833 tokens: 58 us with 22 splits each, 90 with 6), where the 256 compute units get as many each (32 units x 32768: 16
// splits each 48 us, 19 splits 65, 32 splits 49; 288 x 6484: one split 114, four 90).
static int32_t page_splits(int64_t U, int32_t d, int32_t pages, int32_t* waves, bool bound) {
    const int64_t full = d == 64 ? kPageMostCut : kPageMostCut / 2, round = full / 2;
    *waves = U >= full || (U > round && (d > 64 || pages >= 8 || pages <= 2)) ? 1 : kStepWaves;
    int64_t S;
    if (*waves == 1) {
        S = (pages + 63) / 64 < 4 ? (pages + 63) / 64 : 4;
        if (U < full && pages >= 8 && S < 2) S = 2;
        return (int32_t)S;
    }
    const int64_t parts = pages / 24, fill = (full + U - 1) / U, most = (pages + kStepWaves - 1) / kStepWaves;
    const int64_t low = round / U < 1 ? 1 : round / U, high = parts < fill ? parts : fill;
    S = high > low ? high : low;
    if (!bound) {                                // the most splits that keep the compute units nearly as busy as can be
        auto busy = [&](int64_t x) { return U * x < 256 ? 1.0 : (double)(U * x) / (double)((U * x + 255) / 256 * 256); };
        double best = 0.0;
        for (int64_t x = low; x <= S; ++x) best = busy(x) > best ? busy(x) : best;
        while (S > low && busy(S) < 0.9 * best) --S;
    }
    if (S > most) S = most;
    return (int32_t)(S > kPageMaxSplits ? kPageMaxSplits : S);
}
// Bounds the splits of plan_page_step for any hint.
int32_t page_most_splits(int64_t U, int32_t d, int32_t max_pages) {
    int32_t waves;
    const int32_t S = page_splits(U, d, max_pages, &waves, true);
    return waves == 1 ? S : (5 * S + 3) / 4 < kPageMaxSplits ? (5 * S + 3) / 4 : kPageMaxSplits;
}
void plan_page_step(PageArgs* a, int64_t U, int32_t d, int32_t m_hint) {
    const int32_t pages = (m_hint + 63) / 64, S = page_splits(U, d, pages, &a->waves, false);
    a->chunk = (pages + S - 1) / S;
    // a fifth page would be a second round of one wave (58 units x 2518 x 256, 8 heads: 30 us, with four pages 25)
    if (a->waves == kStepWaves && a->chunk == kStepWaves + 1 && S > 1 && S * 5 / 4 < kPageMaxSplits) a->chunk = kStepWaves;
    a->S = (pages + a->chunk - 1) / a->chunk;
}

template <typename T, int D>
static void launch_step_d(const PageArgs& a, int64_t U, hipStream_t st) {
    const dim3 grid((unsigned)(U * a.S));
    if (a.waves == 1) {
        if (a.slopes) hipLaunchKernelGGL((page_step_kernel<T, D, true, 1>), grid, dim3(kWave), 0, st, a);
        else hipLaunchKernelGGL((page_step_kernel<T, D, false, 1>), grid, dim3(kWave), 0, st, a);
    } else {
        if (a.slopes) hipLaunchKernelGGL((page_step_kernel<T, D, true, kStepWaves>), grid, dim3(kStepWaves * kWave), 0, st, a);
        else hipLaunchKernelGGL((page_step_kernel<T, D, false, kStepWaves>), grid, dim3(kStepWaves * kWave), 0, st, a);
    }
    if (a.S > 1) hipLaunchKernelGGL((page_join_kernel<D>), dim3((unsigned)(U * a.G)), dim3(kPageThreads), 0, st, a);
}
template <typename T, int D>
static void launch_write_d(const PageArgs& a, hipStream_t st) {
    const int64_t blocks = ((int64_t)(a.n + 62) / 64 + 1) * a.H * a.L * a.B;
    const dim3 grid((unsigned)blocks), block(kPageThreads);
    hipLaunchKernelGGL((page_write_kernel<T, D>), grid, block, 0, st, a);
}

hipError_t launch_page_step(const PageArgs& a, int64_t U, int32_t d, int32_t dtype, hipStream_t st) {
    if (dtype == KF_BF16) {
        if (d == 64) launch_step_d<bf16_t, 64>(a, U, st);
        else if (d == 128) launch_step_d<bf16_t, 128>(a, U, st);
        else launch_step_d<bf16_t, 256>(a, U, st);
    } else {
        if (d == 64) launch_step_d<f16_t, 64>(a, U, st);
        else if (d == 128) launch_step_d<f16_t, 128>(a, U, st);
        else launch_step_d<f16_t, 256>(a, U, st);
    }
    return hipGetLastError();
}

hipError_t launch_page_write(const PageArgs& a, int32_t d, int32_t dtype, hipStream_t st) {
    if (dtype == KF_BF16) {
        if (d == 64) launch_write_d<bf16_t, 64>(a, st);
        else if (d == 128) launch_write_d<bf16_t, 128>(a, st);
        else launch_write_d<bf16_t, 256>(a, st);
    } else {
        if (d == 64) launch_write_d<f16_t, 64>(a, st);
        else if (d == 128) launch_write_d<f16_t, 128>(a, st);
        else launch_write_d<f16_t, 256>(a, st);
    }
    return hipGetLastError();
}

hipError_t launch_page_reserve(const PageArgs& a, hipStream_t st) {
    hipLaunchKernelGGL(page_reserve_kernel, dim3(1), dim3(kTableThreads), (size_t)a.B * 4, st, a);
    return hipGetLastError();
}
hipError_t launch_page_free(const PageArgs& a, hipStream_t st) {
    hipLaunchKernelGGL(page_free_kernel, dim3((unsigned)((a.B + kPageWaves - 1) / kPageWaves)), dim3(kPageThreads), 0, st, a);
    return hipGetLastError();
}
hipError_t launch_page_fork(const PageArgs& a, int32_t d, hipStream_t st) {
    hipLaunchKernelGGL(page_fork_kernel, dim3(1), dim3(kTableThreads), (size_t)a.B * 4, st, a);
    const int64_t bytes = (int64_t)a.H * 64 * d;
    int64_t pieces = bytes / 16 / (2 * kPageThreads);
    pieces = pieces < 1 ? 1 : pieces > 16 ? 16 : pieces;
    hipLaunchKernelGGL(page_copy_kernel, dim3((unsigned)pieces, (unsigned)a.B, (unsigned)a.L), dim3(kPageThreads), 0, st, a, bytes);
    return hipGetLastError();
}
hipError_t launch_page_compact(const PageArgs& a, int32_t d, hipStream_t st) {
    hipLaunchKernelGGL(page_shrink_kernel, dim3(1), dim3(kTableThreads), (size_t)a.B * 4, st, a);
    const int64_t blocks = (int64_t)((a.kept + 63) / 64) * a.H * a.L * a.B;
    const dim3 grid((unsigned)blocks), block(kPageThreads);
    if (d == 64) hipLaunchKernelGGL((page_keep_kernel<64>), grid, block, 0, st, a);
    else if (d == 128) hipLaunchKernelGGL((page_keep_kernel<128>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((page_keep_kernel<256>), grid, block, 0, st, a);
    return hipGetLastError();
}

}  // namespace kf
