// Device helpers of the operators: 16-bit types and their matrix
// instructions, the split of a ragged batch into jobs (gfx950, waves of 64).
//
// Lane layouts of the matrix instructions, with c = lane / 16 and h = lane / 32:
//   16x16x32: A lane holds row lane % 16, columns 8c .. 8c+7; B lane holds column
//             lane % 16, rows 8c .. 8c+7; C lane holds column lane % 16, rows 4c .. 4c+3
//   32x32x16: A row lane % 32, columns 8h .. 8h+7; B column lane % 32, rows 8h ..
//             8h+7; C column lane % 32, rows 8 (i / 4) + 4h + i % 4 for i = 0 .. 15
//   ds_read_tr16_b64: the 16 lanes of a group give the addresses of 4 rows x 4
//             pieces of 4 elements; lane i gets column i of the 4 rows
#pragma once

#include <hip/hip_runtime.h>

#include "mts_ops_internal.h"
#include "mts_wave.h"

namespace mts {
namespace ops {

typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));

struct Bf16 {
    using e = __bf16;
    using v4 = bf16x4;
    using v8 = bf16x8;
    static constexpr unsigned kExp = 0x7f80u;  // exponent bits: all set for infinities and NaN
    static __device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(s16x8 a, s16x8 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};

struct F16 {
    using e = _Float16;
    using v4 = f16x4;
    using v8 = f16x8;
    static constexpr unsigned kExp = 0x7c00u;
    static __device__ __forceinline__ f32x4 mfma16(s16x8 a, s16x8 b, f32x4 c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
    static __device__ __forceinline__ f32x16 mfma32(s16x8 a, s16x8 b, f32x16 c)
    {
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(v8, a), __builtin_bit_cast(v8, b), c, 0, 0, 0);
    }
};

// Eight floats rounded to the nearest even 16-bit values.
template <class T>
__device__ __forceinline__ s16x8 pack8(f32x8 x) { return __builtin_bit_cast(s16x8, __builtin_convertvector(x, typename T::v8)); }
template <class T>
__device__ __forceinline__ s16x4 pack4(f32x4 x) { return __builtin_bit_cast(s16x4, __builtin_convertvector(x, typename T::v4)); }
template <class T>
__device__ __forceinline__ float widen(short x) { return float(__builtin_bit_cast(typename T::e, x)); }

__device__ __forceinline__ s16x4 read_tr16(const void* lds)
{
    return __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(lds));
}

__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kLn2 = 0.69314718055994530942f;

// Orders a wave's own LDS writes before its reads of other lanes' values: LDS
// serves a wave's instructions in order, so only the compiler is held back.
__device__ __forceinline__ void lds_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

__device__ __forceinline__ int request_len(const Pool& p, const Batch& b, int r)
{
    const int most = b.width << p.lb;
    const int L = b.lens[r];
    return L < 0 ? 0 : L > most ? most : L;
}

__device__ __forceinline__ void request_tokens(const Batch& b, int r, int& first, int& T)
{
    int a = b.q_start[r], z = b.q_start[r + 1];
    a = a < 0 ? 0 : a > b.n_tokens ? b.n_tokens : a;
    z = z < a ? a : z > b.n_tokens ? b.n_tokens : z;
    first = a;
    T = z - a < b.max_q ? z - a : b.max_q;
}

// One job: part `split` of `nsplit` of request r's keys [k0, k1), for KV head
// hk and one group of its query rows.  `lead` is the id of the split 0 job.
struct Job {
    int id, lead;
    int r, hk, grp, split, nsplit;
    int L, T, first;
    int k0, k1;
};

struct SplitRule {
    int unit;         // keys that a workgroup passes over in one round
    int rows;         // query rows (token x head of the group) of a job; 0: all
    int G;            // query heads a KV head
    int target;       // jobs to aim for
    bool xcd;         // neighbouring jobs (which share keys) to one of the 8 dies
};

template <int NW>
__device__ __forceinline__ int64_t block_sum(int64_t v, int64_t* scratch)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    int64_t s = 0;
#pragma unroll
    for (int i = 0; i < NW; ++i) s += scratch[i];
    __syncthreads();
    return s;
}

// What one request adds: groups of query rows, rounds over its keys.
struct Share {
    int L, T, first, groups, rounds;
};

__device__ __forceinline__ Share share_of(const Pool& p, const Batch& b, const SplitRule& s, int r)
{
    Share q{0, 0, 0, 0, 1};
    if (r < b.n) {
        q.L = request_len(p, b, r);
        request_tokens(b, r, q.first, q.T);
        q.groups = s.rows ? int((int64_t(q.T) * s.G + s.rows - 1) / s.rows) : (q.T ? 1 : 0);
        q.rounds = q.L ? (q.L + s.unit - 1) / s.unit : 1;
    }
    return q;
}

// The jobs of a ragged batch, numbered head by head, in it request by request,
// group by group, split by split.  Lengths live on the device, so every
// workgroup (NW waves) finds its own job: it sums the requests' rounds, takes
// as many rounds a job as leave about `target` jobs, and finds its number
// among the requests' job counts.  One request a thread; more are passed over
// in turns.  Returns false for numbers past the last job; the results are
// uniform.  scratch: NW + 4 words of LDS.
template <int NW>
__device__ __forceinline__ bool find_job(const Pool& p, const Batch& b, const SplitRule& s, Job& j, int64_t* scratch)
{
    constexpr int NT = 64 * NW;
    const int t = threadIdx.x;
    Share q{};
    int64_t rounds = 0;
    for (int r0 = 0; r0 < b.n; r0 += NT) {
        q = share_of(p, b, s, r0 + t);
        rounds += int64_t(q.rounds) * q.groups;
    }
    const int64_t total = block_sum<NW>(rounds, scratch) * p.kv_heads;
    const int per = total > s.target ? int((total + s.target - 1) / s.target) : 1;
    int64_t mine = 0;
    for (int r0 = 0; r0 < b.n; r0 += NT) {
        if (b.n > NT) q = share_of(p, b, s, r0 + t);
        mine += int64_t((q.rounds + per - 1) / per) * q.groups;
    }
    const int64_t head = block_sum<NW>(mine, scratch), jobs = head * p.kv_heads;
    int64_t id = blockIdx.x;
    if (s.xcd) {
        const int64_t chunk = (jobs + 7) / 8;
        if ((id >> 3) >= chunk) return false;
        id = (id & 7) * chunk + (id >> 3);
    }
    if (id >= jobs) return false;
    const int hk = int(id / head), in = int(id % head);
    int* found = reinterpret_cast<int*>(scratch + NW);
    int64_t before = 0;
    for (int r0 = 0; r0 < b.n; r0 += NT) {
        if (b.n > NT) q = share_of(p, b, s, r0 + t);
        const int ns = (q.rounds + per - 1) / per;
        const int64_t n = int64_t(ns) * q.groups;
        int64_t incl = n;
        for (int o = 1; o < 64; o <<= 1) {
            const int64_t v = __shfl_up(incl, o);
            if ((t & 63) >= o) incl += v;
        }
        if ((t & 63) == 63) scratch[t >> 6] = incl;
        if (t == 0) found[0] = -1;
        __syncthreads();
        int64_t base = before;
#pragma unroll
        for (int w = 0; w < NW; ++w) {
            if (w < (t >> 6)) base += scratch[w];
            before += scratch[w];
        }
        const int64_t at = in - (base + incl - n);
        if (at >= 0 && at < n) {
            found[0] = r0 + t;
            found[1] = int(at);
            found[2] = ns;
            found[3] = q.L;
            found[4] = q.T;
            found[5] = q.first;
        }
        __syncthreads();
        if (found[0] >= 0) break;
    }
    const int at = __builtin_amdgcn_readfirstlane(found[1]);
    j.id = int(id);
    j.hk = hk;
    j.r = __builtin_amdgcn_readfirstlane(found[0]);
    j.nsplit = __builtin_amdgcn_readfirstlane(found[2]);
    j.L = __builtin_amdgcn_readfirstlane(found[3]);
    j.T = __builtin_amdgcn_readfirstlane(found[4]);
    j.first = __builtin_amdgcn_readfirstlane(found[5]);
    j.split = at % j.nsplit;
    j.grp = at / j.nsplit;
    j.lead = j.id - j.split;
    const int64_t k0 = int64_t(j.split) * per * s.unit, k1 = k0 + int64_t(per) * s.unit;
    j.k0 = int(k0);
    j.k1 = int(k1 < j.L ? k1 : j.L);
    return true;
}

// Most jobs that find_job can number for a call of these sizes.
inline uint64_t max_jobs(uint32_t n, uint64_t n_tokens, uint32_t kv_heads, uint32_t G, uint32_t rows, uint32_t target)
{
    const uint64_t groups = rows ? n + n_tokens * G / rows : n;
    return ((target + groups * kv_heads) + 7) / 8 * 8;
}

}  // namespace ops
}  // namespace mts
