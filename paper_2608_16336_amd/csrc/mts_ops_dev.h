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
    int r, hk, grp, split, nsplit, lead;
    int L, T, first;
    int k0, k1;
};

struct SplitRule {
    int unit;         // keys that a workgroup passes over in one round
    int rows;         // query rows (token x head of the group) of a job; 0: all
    int G;            // query heads a KV head
    int target;       // jobs to aim for
};

// The jobs of a ragged batch, numbered request by request.  Lengths live on
// the device, so every workgroup finds its own: it sums the requests' rounds,
// takes as many rounds a job as leave about `target` jobs, and walks the
// requests' job counts up to its id.  n / 256 loads a thread.  Returns false
// for ids past the last job; wave-uniform results.  scratch: 256 threads, 24
// words of LDS; two barriers a 256 requests and pass.
__device__ __forceinline__ long long block_sum(long long v, long long* scratch)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    const long long s = scratch[0] + scratch[1] + scratch[2] + scratch[3];
    __syncthreads();
    return s;
}

__device__ __forceinline__ bool find_job(const Pool& p, const Batch& b, const SplitRule& s, int id, Job& j, long long* scratch)
{
    const int t = threadIdx.x;
    long long rounds = 0;
    int L = 0, first = 0, T = 0, groups = 0, R = 0;
    for (int r0 = 0; r0 < b.n; r0 += 256) {
        const int r = r0 + t;
        if (r < b.n) {
            L = request_len(p, b, r);
            request_tokens(b, r, first, T);
            groups = s.rows ? int((int64_t(T) * s.G + s.rows - 1) / s.rows) : (T ? 1 : 0);
            R = L ? (L + s.unit - 1) / s.unit : 1;
            rounds += (long long)(R)*groups * p.kv_heads;
        }
    }
    const long long total = block_sum(rounds, scratch);
    const int per = total > s.target ? int((total + s.target - 1) / s.target) : 1;
    long long before = 0;
    int* found = reinterpret_cast<int*>(scratch + 8);
    for (int r0 = 0; r0 < b.n; r0 += 256) {
        const int r = r0 + t;
        if (b.n > 256) {
            groups = 0;
            R = 1;
            if (r < b.n) {
                L = request_len(p, b, r);
                request_tokens(b, r, first, T);
                groups = s.rows ? int((int64_t(T) * s.G + s.rows - 1) / s.rows) : (T ? 1 : 0);
                R = L ? (L + s.unit - 1) / s.unit : 1;
            }
        } else if (r >= b.n) {
            groups = 0;
            R = 1;
        }
        const int ns = (R + per - 1) / per;
        const long long jobs = (long long)(ns)*groups * p.kv_heads;
        long long incl = jobs;
        for (int o = 1; o < 64; o <<= 1) {
            const long long v = __shfl_up(incl, o);
            if ((t & 63) >= o) incl += v;
        }
        if ((t & 63) == 63) scratch[t >> 6] = incl;
        if (t == 0) found[0] = -1;
        __syncthreads();
        long long base = before;
        for (int w = 0; w < (t >> 6); ++w) base += scratch[w];
        const long long at = id - (base + incl - jobs);
        if (at >= 0 && at < jobs) {
            const int in = int(at);
            found[0] = r;
            found[1] = in;
            found[2] = ns;
            found[3] = groups;
            found[4] = L;
            found[5] = T;
            found[6] = first;
        }
        before += scratch[0] + scratch[1] + scratch[2] + scratch[3];
        __syncthreads();
        if (found[0] >= 0) break;
    }
    j.r = __builtin_amdgcn_readfirstlane(found[0]);
    if (j.r < 0) return false;
    const int in = __builtin_amdgcn_readfirstlane(found[1]);
    j.nsplit = __builtin_amdgcn_readfirstlane(found[2]);
    const int grp = __builtin_amdgcn_readfirstlane(found[3]);
    j.L = __builtin_amdgcn_readfirstlane(found[4]);
    j.T = __builtin_amdgcn_readfirstlane(found[5]);
    j.first = __builtin_amdgcn_readfirstlane(found[6]);
    j.split = in % j.nsplit;
    j.lead = id - j.split;
    const int rest = in / j.nsplit;
    j.grp = rest % grp;
    j.hk = rest / grp;
    const long long k0 = (long long)(j.split) * per * s.unit;
    const long long k1 = k0 + (long long)(per)*s.unit;
    j.k0 = int(k0);
    j.k1 = int(k1 < j.L ? k1 : j.L);
    return true;
}

// Most jobs that find_job can number for a call of these sizes.
inline uint64_t max_jobs(uint32_t n, uint64_t n_tokens, uint32_t kv_heads, uint32_t G, uint32_t rows, uint32_t target)
{
    const uint64_t groups = rows ? n + n_tokens * G / rows : n;
    return target + groups * kv_heads;
}

}  // namespace ops
}  // namespace mts
