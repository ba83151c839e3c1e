// The next token of a row of logits (mts_sample).
#include "mts_ops_dev.h"

namespace mts {
namespace ops {

struct SampleP {
    const char* logits;
    int64_t row_bytes;
    const float *u, *temperature, *top_p, *min_p;
    const int32_t* top_k;
    int32_t* token;
    float* logprob;
    int vocab, frac;  // frac: bits below the point of a summed weight
};

constexpr int kThreads = 1024, kWaves = 16;
typedef unsigned long long u64;

// A row as 16-byte vectors from the aligned address at or below its start;
// elements outside the row read as -inf with a key below all others'.
template <class E>
struct Row {
    static constexpr int N = 16 / int(sizeof(E));
    const char* start;  // of vector 0
    int skip;           // elements of vector 0 before the row
    int vocab, nvec;
    struct alignas(16) V {
        E e[N];
    };
    __device__ __forceinline__ Row(const char* row, int v) : vocab(v)
    {
        const uintptr_t a = reinterpret_cast<uintptr_t>(row);
        start = reinterpret_cast<const char*>(a & ~uintptr_t(15));
        skip = int((a & 15) / sizeof(E));
        nvec = (skip + v + N - 1) / N;
    }
    // index of element 0 of vector i
    __device__ __forceinline__ int first(int i) const { return i * N - skip; }
    __device__ __forceinline__ void load(int i, float x[N]) const
    {
        const int f = first(i);
        if (f >= 0 && f + N <= vocab) {
            const V v = *reinterpret_cast<const V*>(start + 16 * size_t(i));
#pragma unroll
            for (int e = 0; e < N; ++e) x[e] = float(v.e[e]);
        } else {
#pragma unroll
            for (int e = 0; e < N; ++e)
                x[e] = f + e >= 0 && f + e < vocab ? float(*reinterpret_cast<const E*>(start + 16 * size_t(i) + e * sizeof(E))) : -__builtin_inff();
        }
#pragma unroll
        for (int e = 0; e < N; ++e) x[e] = x[e] != x[e] ? -__builtin_inff() : x[e] + 0.f;
    }
};

__device__ __forceinline__ unsigned logit_key(float x)
{
    const unsigned u = __float_as_uint(x);
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

// Weights are summed as whole numbers of 2^-frac, to the nearest: the sums do
// not depend on any order, and are off by less than 2^-frac a token.  Adding
// 1.5 * 2^(52 - frac) leaves the rounded number in the low bits of the double.
struct Weigher {
    float top, inv_t, min_w;
    double magic;
    u64 magic_bits;
    __device__ __forceinline__ float weight(float x) const
    {
        return x == top ? 1.f : x == -__builtin_inff() ? 0.f : expf((x - top) * inv_t);
    }
    __device__ __forceinline__ u64 fixed(float w) const { return u64(__double_as_longlong(double(w) + magic)) - magic_bits; }
};

template <class F>
__device__ __forceinline__ u64 block_sum64(u64 v, F* scratch)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    u64 s = 0;
    for (int i = 0; i < kWaves; ++i) s += scratch[i];
    return s;
}

__device__ __forceinline__ u64 wave_incl(u64 v)
{
    const int lane = threadIdx.x & 63;
    for (int o = 1; o < 64; o <<= 1) {
        const u64 u = __shfl_up(v, o);
        if (lane >= o) v += u;
    }
    return v;
}

// One workgroup a row.  The kept set is a threshold key with a count of the
// lowest-numbered tokens of that key, found by radix selection over 11, 11 and
// 10 bits of the key: by counts for top-k, by summed weights for top-p.
template <class E>
__global__ __launch_bounds__(kThreads) void k_sample(const SampleP p)
{
    constexpr int N = Row<E>::N;
    __shared__ u64 hist[2048];
    __shared__ u64 scratch[kWaves];
    __shared__ u64 cut_sum;
    __shared__ int cut_bin;
    __shared__ unsigned wave_top[kWaves];
    __shared__ int wave_n[kWaves];
    const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const Row<E> row(p.logits + b * p.row_bytes, p.vocab);

    // the largest key and its lowest index
    unsigned best = 0;
    int at = 0x7fffffff;
    for (int i = tid; i < row.nvec; i += kThreads) {
        float x[N];
        row.load(i, x);
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const unsigned k = logit_key(x[e]);
            if (k > best) best = k, at = row.first(i) + e;
        }
    }
    for (int o = 32; o; o >>= 1) {
        const unsigned k = __shfl_xor(best, o);
        const int a = __shfl_xor(at, o);
        if (k > best || (k == best && a < at)) best = k, at = a;
    }
    if (lane == 0) wave_top[w] = best, wave_n[w] = at;
    __syncthreads();
    for (int i = 0; i < kWaves; ++i)
        if (wave_top[i] > best || (wave_top[i] == best && wave_n[i] < at)) best = wave_top[i], at = wave_n[i];
    const float t = p.temperature[b];
    if (best <= logit_key(-__builtin_inff()) || !(t > 0.f)) {
        const bool dead = best <= logit_key(-__builtin_inff());
        if (tid == 0) {
            p.token[b] = dead ? -1 : at;
            if (p.logprob) p.logprob[b] = dead ? -__builtin_inff() : 0.f;
        }
        return;
    }
    Weigher wt;
    wt.top = __uint_as_float(best ^ (best >> 31 ? 0x80000000u : 0xffffffffu));
    wt.inv_t = 1.f / t;
    wt.min_w = fminf(fmaxf(p.min_p[b], 0.f), 1.f);  // the first rank always stays
    wt.magic = ldexp(1.5, 52 - p.frac);
    wt.magic_bits = u64(__double_as_longlong(wt.magic));

    // kept: keys above thr, and the `need` lowest-numbered of those equal to it
    unsigned thr = 0;
    u64 need = ~0ull;
    const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
    const int k_top = p.top_k[b];
    const float top_p = p.top_p[b];
    const bool by_k = k_top > 0 && k_top < p.vocab, by_p = top_p < 1.f;
    for (int rule = 0; rule < 2; ++rule) {
        if (!(rule ? by_p : by_k)) continue;
        // rule 0: the first k_top ranks; rule 1: ranks while the weight before them is below the limit
        const unsigned old_thr = thr;
        const u64 old_need = need;
        double limit = 0.0;
        if (rule) {
            u64 z = 0, eq = 0;
            for (int i = tid; i < row.nvec; i += kThreads) {
                float x[N];
                row.load(i, x);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const unsigned k = logit_key(x[e]);
                    if (k > old_thr || (k == old_thr && old_need == ~0ull)) z += wt.fixed(wt.weight(x[e]));
                }
            }
            z = block_sum64(z, scratch);
            if (old_need != ~0ull) {
                const float x = __uint_as_float(old_thr ^ (old_thr >> 31 ? 0x80000000u : 0xffffffffu));
                eq = old_need * wt.fixed(wt.weight(x));
            }
            limit = double(top_p) * double(z + eq);
        }
        unsigned found = 0, mask = 0;
        u64 above = 0;  // counts or weights of the keys above the found prefix
        for (int d = 0; d < 3; ++d) {
            const int n = 1 << bits[d];
            __syncthreads();
            hist[tid] = 0;
            hist[tid + 1024] = 0;
            if (tid == 0) cut_bin = -1;
            __syncthreads();
            for (int i = tid; i < row.nvec; i += kThreads) {
                float x[N];
                row.load(i, x);
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    const unsigned k = logit_key(x[e]);
                    const int f = row.first(i) + e;
                    if (f < 0 || f >= p.vocab || (k & mask) != found || k < old_thr) continue;
                    atomicAdd(&hist[(k >> shifts[d]) & (n - 1)], rule ? wt.fixed(wt.weight(x[e])) : 1ull);
                }
            }
            __syncthreads();
            const int hi = n - 1 - 2 * tid, lo = hi - 1;
            const u64 a = hi >= 0 ? hist[hi] : 0, c = lo >= 0 ? hist[lo] : 0;
            const u64 incl = wave_incl(a + c);
            if (lane == 63) scratch[w] = incl;
            __syncthreads();
            u64 before = above;
            for (int i = 0; i < w; ++i) before += scratch[i];
            before += incl - a - c;
            // the last bin with anything in it whose ranks begin below the limit
            const auto below = [&](u64 s) { return rule ? s == 0 || double(s) < limit : s < u64(k_top); };
            if (a && below(before)) atomicMax(&cut_bin, 2047 - hi);
            if (c && below(before + a)) atomicMax(&cut_bin, 2047 - lo);
            __syncthreads();
            const int bin = 2047 - cut_bin;
            if (bin == hi && a) cut_sum = before;
            if (bin == lo && c) cut_sum = before + a;
            __syncthreads();
            above = cut_sum;
            found |= unsigned(bin) << shifts[d];
            mask |= unsigned(n - 1) << shifts[d];
        }
        thr = found;
        if (!rule) {
            need = u64(k_top) - above;
        } else {
            const float x = __uint_as_float(thr ^ (thr >> 31 ? 0x80000000u : 0xffffffffu));
            const u64 one = wt.fixed(wt.weight(x));
            // how many of the equal ones begin below the limit
            double more = one ? ceil((limit - double(above)) / double(one)) : 1.0;
            more = more < 1.0 ? 1.0 : more;
            need = more < 16777216.0 ? u64(more) : 16777216ull;
            if (thr == old_thr && old_need < need) need = old_need;
        }
    }

    // waves own consecutive stretches of the row
    const int seg = ((row.nvec + kWaves * 64 - 1) / (kWaves * 64)) * 64;
    const int v0 = min(w * seg, row.nvec), v1 = min(v0 + seg, row.nvec);
    u64 eq_before = 0;
    if (need != ~0ull) {
        u64 eq = 0;
        for (int i = v0 + lane; i < v1; i += 64) {
            float x[N];
            row.load(i, x);
#pragma unroll
            for (int e = 0; e < N; ++e) eq += logit_key(x[e]) == thr;
        }
        for (int o = 32; o; o >>= 1) eq += __shfl_xor(eq, o);
        __syncthreads();
        if (lane == 0) scratch[w] = eq;
        __syncthreads();
        for (int i = 0; i < w; ++i) eq_before += scratch[i];
        __syncthreads();
    }
    // a vector's kept weights, whole numbers; e0: equal keys before it in the row
    const auto kept = [&](int i, u64 e0, u64 out[N], float ws[N]) {
        float x[N];
        row.load(i, x);
        u64 sum = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) {
            const unsigned k = logit_key(x[e]);
            const int f = row.first(i) + e;
            bool in = f >= 0 && f < p.vocab && k >= thr;
            if (k == thr) in = in && e0++ < need;
            ws[e] = in ? wt.weight(x[e]) : 0.f;
            if (!(ws[e] >= wt.min_w)) ws[e] = 0.f;
            out[e] = wt.fixed(ws[e]);
            sum += out[e];
        }
        return sum;
    };
    const auto equals = [&](int i) {
        float x[N];
        row.load(i, x);
        u64 n = 0;
#pragma unroll
        for (int e = 0; e < N; ++e) n += logit_key(x[e]) == thr;
        return n;
    };
    u64 total = 0, e_run = eq_before;
    for (int i = v0; i < v1; i += 64) {
        const int v = i + lane;
        u64 e0 = 0;
        if (need != ~0ull) {
            const u64 n = v < v1 ? equals(v) : 0, incl = wave_incl(n);
            e0 = e_run + incl - n;
            e_run += __shfl(incl, 63);
        }
        u64 out[N];
        float ws[N];
        if (v < v1) total += kept(v, e0, out, ws);
    }
    for (int o = 32; o; o >>= 1) total += __shfl_xor(total, o);
    __syncthreads();
    if (lane == 0) scratch[w] = total;
    __syncthreads();
    u64 W = 0, lower = 0;
    for (int i = 0; i < kWaves; ++i) {
        if (i < w) lower += scratch[i];
        W += scratch[i];
    }
    const double target = double(fmaxf(p.u[b], 0.f)) * double(W);
    // the stretch that the target falls in finds the token; u of 1 and more ends at the last kept one
    const bool here = total && !(double(lower) > target) && (double(lower + total) > target || lower + total == W);
    if (!here) return;
    u64 run = lower;
    e_run = eq_before;
    int token = -1;
    float weight = 0.f;
    for (int i = v0; i < v1; i += 64) {
        const int v = i + lane;
        u64 e0 = 0;
        if (need != ~0ull) {
            const u64 n = v < v1 ? equals(v) : 0, incl = wave_incl(n);
            e0 = e_run + incl - n;
            e_run += __shfl(incl, 63);
        }
        u64 out[N];
        float ws[N];
        const u64 mine = v < v1 ? kept(v, e0, out, ws) : 0;
        const u64 incl = wave_incl(mine), all = __shfl(incl, 63);
        const u64 m = run + incl - mine;
        const bool hit = mine && double(m + mine) > target;
        const u64 who = __ballot(hit);
        if (who || run + all == W) {
            // past the last sum that exceeds the target, only u >= 1 gets here: the last lane with any weight
            const u64 any = __ballot(mine != 0);
            const int l = who ? __ffsll((long long)(who)) - 1 : 63 - __clzll((long long)(any));
            if (lane == l) {
                u64 s = m;
#pragma unroll
                for (int e = 0; e < N; ++e) {
                    if (!out[e]) continue;
                    if (token >= 0 && double(s) > target) continue;
                    s += out[e];
                    token = row.first(v) + e;
                    weight = ws[e];
                }
                p.token[b] = token;
                if (p.logprob) p.logprob[b] = float(log(ldexp(double(weight), p.frac) / double(W)));
            }
            break;
        }
        run += all;
    }
}

template <class E>
static void launch_sample(const SampleP& p, uint32_t rows, hipStream_t stream)
{
    hipLaunchKernelGGL(k_sample<E>, dim3(rows), dim3(kThreads), 0, stream, p);
}

}  // namespace ops
}  // namespace mts

using namespace mts::ops;

extern "C" int mts_sample(const mts_sample_args* a, hipStream_t stream)
{
    if (!a || a->reserved || a->type > MTS_F32 || a->vocab < 1 || a->vocab > (1u << 24) || a->rows > 0x7fffffffu) return MTS_EINVAL;
    if (a->rows == 0) return MTS_OK;
    const size_t e = a->type == MTS_F32 ? 4 : 2;
    if (!aligned(a->logits, e) || a->row_stride < 0 || (a->rows > 1 && uint64_t(a->row_stride) < a->vocab)) return MTS_EINVAL;
    if (!aligned(a->u, 4) || !aligned(a->temperature, 4) || !aligned(a->top_k, 4) || !aligned(a->top_p, 4) || !aligned(a->min_p, 4) ||
        !aligned(a->token, 4) || (a->logprob && !aligned(a->logprob, 4)))
        return MTS_EINVAL;
    SampleP p;
    p.logits = static_cast<const char*>(a->logits);
    p.row_bytes = int64_t(e) * a->row_stride;
    p.u = a->u;
    p.temperature = a->temperature;
    p.top_k = a->top_k;
    p.top_p = a->top_p;
    p.min_p = a->min_p;
    p.token = a->token;
    p.logprob = a->logprob;
    p.vocab = int(a->vocab);
    // the sum of all weights, each at most 1, stays below 2^62; one stays below 2^51
    int lv = 0;
    while ((1u << lv) < a->vocab) ++lv;
    p.frac = 62 - lv < 50 ? 62 - lv : 50;
    switch (a->type) {
    case MTS_BF16: launch_sample<__bf16>(p, a->rows, stream); break;
    case MTS_F16: launch_sample<_Float16>(p, a->rows, stream); break;
    default: launch_sample<float>(p, a->rows, stream); break;
    }
    return launched();
}
