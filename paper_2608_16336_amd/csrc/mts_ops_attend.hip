// Attention of new tokens over a paged cache (mts_attend).
#include "mts_ops_dev.h"

namespace mts {
namespace ops {

struct AttendP {
    Pool pool;
    Batch batch;
    const char* q;
    char* out;
    float* lse;
    int64_t q_token, q_head, out_token, out_head;  // bytes
    int G, q_heads;
    float scale2;  // scale * log2 e: the softmax runs in powers of two
    unsigned* count;
    float* part_ml;  // [job][rows][2] running maximum and sum
    float* part_o;   // [job][rows][D]
    int target;
};

constexpr int kRound = 128;  // keys of one round of a workgroup: 4 waves x 32

// Where slot j of request r lies: block id, or -1 for one outside the pool.
__device__ __forceinline__ int block_of(const Pool& p, const Batch& b, int r, int j)
{
    const int id = b.table[size_t(r) * b.width + (j >> p.lb)];
    return unsigned(id) < p.n_blocks ? id : -1;
}

// 16-byte pieces of a staged row are swapped by row so that the transposed
// reads of 16 rows fall on different banks.
template <int D>
__device__ __forceinline__ int swz(int row)
{
    constexpr int CH = D / 8;
    return CH % 16 == 0 ? (row & 15) : CH % 8 == 0 ? ((row >> 1) & 7) : ((row >> 2) & 3);
}

// Whether new token t of a request may see slot j at offset rel = j - (L - T) among the new ones.
__device__ __forceinline__ bool sees(const Batch& b, int tok, int t, int rel)
{
    if (rel < 0) return true;
    if (!b.tree) return rel <= t;
    return rel < 64 * b.words && ((b.tree[size_t(tok) * b.words + (rel >> 6)] >> (rel & 63)) & 1);
}

// Joins the parts of a job's rows, in the order of the splits, once the last
// of its workgroups has written its own: partial sums o, maxima m (in powers
// of two) and sums l of the waves or the splits.
//
// The softmax of a row over parts: o = sum_i 2^(m_i - M) o_i, l likewise.
template <class T, int D>
__device__ __forceinline__ void store_row(const AttendP& p, const Job& j, int row, int d, f32x4 o, float M, float l)
{
    const int t = row / p.G, h = j.hk * p.G + row % p.G;
    const size_t tok = size_t(j.first) + t;
    const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);  // a NaN sum stays one
    *reinterpret_cast<s16x4*>(p.out + tok * p.out_token + int64_t(h) * p.out_head + 2 * d) = pack4<T>(o * inv);
    if (d == 0 && p.lse) p.lse[tok * p.q_heads + h] = l == 0.f ? -__builtin_inff() : M * kLn2 + __logf(l);
}

// Few query rows (16 MT: tokens x heads of a group): a stream over K and V.
//
// Four waves take the keys of a round in turn, 32 each, and nothing is shared
// until the end.  Scores are formed transposed, S^T = K Q^T, so that a lane
// holds 8 keys of one query: that is the layout in which the product
// O^T += V^T P^T takes P^T, and the running maximum and sum are the lane's own.
// K goes from memory straight into the matrix instruction's layout; V is
// staged through LDS, whose transposed reads give V^T.
template <class T, int D, int MT>
__global__ __launch_bounds__(256, D == 256 ? 1 : 2) void k_attend_rows(const AttendP p)
{
    constexpr int KS = D / 32, DT = D / 16, RG = 16 * MT;
    __shared__ __attribute__((aligned(16))) char vst[4][32 * D * 2];
    __shared__ float wm[4][16], wl[4][16];
    __shared__ float pst[4][32 * 17];
    __shared__ long long scratch[16];
    __shared__ int last;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, lq = lane & 15, c = lane >> 4;
    Job j;
    const SplitRule rule{kRound, RG, p.G, p.target};
    if (!find_job(p.pool, p.batch, rule, blockIdx.x, j, scratch)) return;
    const int rows = min(RG, j.T * p.G - j.grp * RG), row0 = j.grp * RG;
    const int base = j.L - j.T;

    s16x8 qf[MT][KS];
    int tq[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        const int row = 16 * m + lq;
        const bool ok = row < rows;
        const int rr = row0 + (ok ? row : 0);
        tq[m] = rr / p.G;
        const char* qp = p.q + (size_t(j.first) + tq[m]) * p.q_token + int64_t(j.hk * p.G + rr % p.G) * p.q_head;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
            const s16x8 x = *reinterpret_cast<const s16x8*>(qp + (32 * s + 8 * c) * 2);
            qf[m][s] = ok ? x : s16x8{};
        }
    }

    f32x4 o[MT][DT];
    float m_run[MT], l_run[MT];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        m_run[m] = -__builtin_inff();
        l_run[m] = 0.f;
#pragma unroll
        for (int t = 0; t < DT; ++t) o[m][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    const char* kh = p.pool.k + int64_t(j.hk) * p.pool.k_head;
    const char* vh = p.pool.v + int64_t(j.hk) * p.pool.v_head;
    const int omask = (1 << p.pool.lb) - 1;

    for (int k0 = j.k0 + 32 * w; k0 < j.k1; k0 += kRound) {
        bool live[2];
        s16x8 kf[2][KS], vf[2][KS];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int key = k0 + 16 * u + lq;
            const int id = key < j.k1 ? block_of(p.pool, p.batch, j.r, key) : -1;
            live[u] = id >= 0;
            const int64_t blk = live[u] ? id : 0, off = live[u] ? key & omask : 0;
            const char* kp = kh + blk * p.pool.k_block + off * p.pool.k_token;
            const char* vp = vh + blk * p.pool.v_block + off * p.pool.v_token;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[u][s] = *reinterpret_cast<const s16x8*>(kp + (32 * s + 8 * c) * 2);
#pragma unroll
            for (int s = 0; s < KS; ++s) vf[u][s] = *reinterpret_cast<const s16x8*>(vp + (32 * s + 8 * c) * 2);
        }
        // unseen slots weigh nothing whatever they hold: their values must not reach the product as NaN
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < KS; ++s)
                if (!live[u]) vf[u][s] = s16x8{};
        const unsigned long long alive[2] = {__ballot(live[0]) & 0xffff, __ballot(live[1]) & 0xffff};
        const bool fresh = k0 + 32 > base;  // some of these slots are new tokens': rows differ in what they see
        bool odd = false;
        if (fresh) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int s = 0; s < KS; ++s)
#pragma unroll
                    for (int i = 0; i < 8; ++i) odd |= (unsigned(vf[u][s][i]) & T::kExp) == T::kExp;
            odd = __any(odd);
        }
        lds_order();
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const int row = 16 * u + lq;
                *reinterpret_cast<s16x8*>(&vst[w][row * D * 2 + (((4 * s + c) ^ swz<D>(row)) * 16)]) = vf[u][s];
            }
        lds_order();
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            f32x4 sc[2] = {};
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int s = 0; s < KS; ++s) sc[u] = T::mfma16(kf[u][s], qf[m][s], sc[u]);
            float x[8];
            float mx = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int in = 4 * c + (i & 3);
                bool see = (alive[i >> 2] >> in) & 1;
                if (fresh) see = see && sees(p.batch, j.first + tq[m], tq[m], k0 + 16 * (i >> 2) + in - base);
                x[i] = see ? sc[i >> 2][i & 3] * p.scale2 : -__builtin_inff();
                mx = fmaxf(mx, x[i]);
            }
            mx = fmaxf(mx, __shfl_xor(mx, 16));
            mx = fmaxf(mx, __shfl_xor(mx, 32));
            const float mn = fmaxf(m_run[m], mx);
            const float ref = mn == -__builtin_inff() ? 0.f : mn;
            const float alpha = exp2_fast(m_run[m] - ref);
            m_run[m] = mn;
            f32x8 pr;
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                pr[i] = exp2_fast(x[i] - ref);
                sum += pr[i];
            }
            l_run[m] = l_run[m] * alpha + sum;
#pragma unroll
            for (int t = 0; t < DT; ++t) o[m][t] *= alpha;
            if (!odd) {
                const s16x8 pf = pack8<T>(pr);
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    s16x8 a;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int row = 16 * u + 4 * c + (lq >> 2), piece = 2 * t + ((lq & 3) >> 1);
                        const s16x4 x4 = read_tr16(&vst[w][row * D * 2 + ((piece ^ swz<D>(row)) * 16) + (lq & 1) * 8]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) a[4 * u + i] = x4[i];
                    }
                    o[m][t] = T::mfma16(a, pf, o[m][t]);
                }
            } else {
                // infinities or NaN among the new tokens' values: only the rows that see a slot take its value
                lds_order();
#pragma unroll
                for (int i = 0; i < 8; ++i) pst[w][(16 * (i >> 2) + 4 * c + (i & 3)) * 17 + lq] = x[i] == -__builtin_inff() ? -1.f : pr[i];
                lds_order();
                for (int key = 0; key < 32; ++key) {
                    const float pk = pst[w][key * 17 + lq];
                    if (pk < 0.f) continue;
#pragma unroll
                    for (int t = 0; t < DT; ++t) {
                        const int d = 16 * t + 4 * c;
                        const s16x4 v4 = *reinterpret_cast<const s16x4*>(&vst[w][key * D * 2 + (((d >> 3) ^ swz<D>(key)) * 16) + (d & 4) * 2]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) o[m][t][i] += pk * widen<T>(v4[i]);
                    }
                }
                lds_order();
            }
        }
    }

    // the four waves' rows joined, 16 at a time
    const int slot = blockIdx.x;
    const bool whole = j.nsplit == 1;
#pragma unroll
    for (int m = 0; m < MT; ++m) {
        float l = l_run[m];
        l += __shfl_xor(l, 16);
        l += __shfl_xor(l, 32);
        __syncthreads();
        if (c == 0) {
            wm[w][lq] = m_run[m];
            wl[w][lq] = l;
        }
        float* mine = reinterpret_cast<float*>(vst[w]);
#pragma unroll
        for (int t = 0; t < DT; ++t) *reinterpret_cast<f32x4*>(&mine[lq * D + 16 * t + 4 * c]) = o[m][t];
        __syncthreads();
        for (int e = threadIdx.x; e < 16 * (D / 4); e += 256) {
            const int row = e / (D / 4), d = 4 * (e % (D / 4));
            if (16 * m + row >= rows) break;
            float M = fmaxf(fmaxf(wm[0][row], wm[1][row]), fmaxf(wm[2][row], wm[3][row]));
            const float ref = M == -__builtin_inff() ? 0.f : M;
            f32x4 s = {0.f, 0.f, 0.f, 0.f};
            float ls = 0.f;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float f = exp2_fast(wm[i][row] - ref);
                s += f * *reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(vst[i]) + row * D + d);
                ls += f * wl[i][row];
            }
            if (whole) {
                store_row<T, D>(p, j, row0 + 16 * m + row, d, s, M, ls);
            } else {
                const size_t at = size_t(slot) * RG + 16 * m + row;
                *reinterpret_cast<f32x4*>(&p.part_o[at * D + d]) = s;
                if (d == 0) {
                    p.part_ml[2 * at] = M;
                    p.part_ml[2 * at + 1] = ls;
                }
            }
        }
    }
    if (whole) return;

    // the last of the splits' workgroups joins them, in their order
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        const unsigned before = __hip_atomic_fetch_add(&p.count[j.lead], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        last = before + 1 == unsigned(j.nsplit);
        if (last) {
            p.count[j.lead] = 0;
            __threadfence();
        }
    }
    __syncthreads();
    if (!last) return;
    for (int e = threadIdx.x; e < rows * (D / 4); e += 256) {
        const int row = e / (D / 4), d = 4 * (e % (D / 4));
        float M = -__builtin_inff();
        for (int i = 0; i < j.nsplit; ++i) M = fmaxf(M, p.part_ml[2 * (size_t(j.lead + i) * RG + row)]);
        const float ref = M == -__builtin_inff() ? 0.f : M;
        f32x4 s = {0.f, 0.f, 0.f, 0.f};
        float ls = 0.f;
        for (int i = 0; i < j.nsplit; ++i) {
            const size_t at = size_t(j.lead + i) * RG + row;
            const float f = exp2_fast(p.part_ml[2 * at] - ref);
            s += f * *reinterpret_cast<const f32x4*>(&p.part_o[at * D + d]);
            ls += f * p.part_ml[2 * at + 1];
        }
        store_row<T, D>(p, j, row0 + row, d, s, M, ls);
    }
}

constexpr uint32_t kTarget = 512;

struct Sizes {
    uint32_t rows;  // query rows of a job
    uint64_t jobs;
    size_t ml, o;   // bytes of the two partial arrays
    size_t total;
};

// The counters of the splits take the first 64th of the workspace, whatever a
// call's sizes, so that no call's partial rows lie where a later one counts.
// A job's rows are at least 16 (8 + 256) bytes: its 4-byte counter always fits.
constexpr size_t kCountShare = 64;
static size_t count_bytes(size_t workspace) { return workspace / kCountShare & ~size_t(255); }

static Sizes sizes(uint32_t n, uint32_t n_tokens, uint32_t max_q, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim)
{
    const uint32_t G = q_heads / kv_heads;
    Sizes s;
    s.rows = uint64_t(max_q) * G <= 16 ? 16 : 32;
    s.jobs = max_jobs(n, n_tokens, kv_heads, G, s.rows, kTarget);
    s.ml = align256(8 * s.jobs * s.rows);
    s.o = align256(4 * s.jobs * s.rows * head_dim);
    s.total = align256((s.ml + s.o) / (kCountShare - 1) * kCountShare + 2 * 256 * kCountShare);
    return s;
}

template <class T, int D>
static void launch_d(const AttendP& p, const Sizes& s, hipStream_t stream)
{
    if (s.rows == 16)
        hipLaunchKernelGGL((k_attend_rows<T, D, 1>), dim3(uint32_t(s.jobs)), dim3(256), 0, stream, p);
    else
        hipLaunchKernelGGL((k_attend_rows<T, D, 2>), dim3(uint32_t(s.jobs)), dim3(256), 0, stream, p);
}

template <class T>
static void launch_t(const AttendP& p, uint32_t D, const Sizes& s, hipStream_t stream)
{
    switch (D) {
    case 64: launch_d<T, 64>(p, s, stream); break;
    case 96: launch_d<T, 96>(p, s, stream); break;
    case 128: launch_d<T, 128>(p, s, stream); break;
    default: launch_d<T, 256>(p, s, stream); break;
    }
}

}  // namespace ops
}  // namespace mts

using namespace mts::ops;

extern "C" {

int mts_attend_workspace(uint32_t n, uint32_t n_tokens, uint32_t max_q, uint32_t q_heads, uint32_t kv_heads, uint32_t head_dim,
                         size_t* bytes)
{
    if (!bytes || max_q < 1 || kv_heads < 1 || q_heads < kv_heads || q_heads % kv_heads || !head_dim_ok(head_dim))
        return MTS_EINVAL;
    const Sizes s = sizes(n, n_tokens, max_q, q_heads, kv_heads, head_dim);
    if (s.jobs > 0x7fffffffull) return MTS_ERANGE;
    *bytes = s.total;
    return MTS_OK;
}

int mts_attend(const mts_attend_args* a, hipStream_t stream)
{
    if (!a || !pool_ok(a->pool, true, true) || !head_dim_ok(a->pool.head_dim)) return MTS_EINVAL;
    if (!batch_ok(a->batch, a->pool.block_tokens, true)) return MTS_EINVAL;
    if (a->q_heads < a->pool.kv_heads || a->q_heads % a->pool.kv_heads || a->q_heads > kMaxHeads) return MTS_EINVAL;
    if (!(a->scale == a->scale)) return MTS_EINVAL;
    if (a->batch.n == 0 || a->batch.n_tokens == 0) return MTS_OK;
    if (!aligned(a->q, 16) || !aligned(a->out, 16) || !stride8(a->q_token) || !stride8(a->q_head) || !stride8(a->out_token) ||
        !stride8(a->out_head) || !aligned(a->workspace, 256))
        return MTS_EINVAL;
    const Sizes s = sizes(a->batch.n, a->batch.n_tokens, a->batch.max_q, a->q_heads, a->pool.kv_heads, a->pool.head_dim);
    if (s.jobs > 0x7fffffffull) return MTS_ERANGE;
    if (a->workspace_bytes < s.total) return MTS_ENOMEM;
    char* ws = static_cast<char*>(a->workspace);
    AttendP p;
    p.pool = device_pool(a->pool);
    p.batch = device_batch(a->batch);
    p.q = static_cast<const char*>(a->q);
    p.out = static_cast<char*>(a->out);
    p.lse = a->lse;
    p.q_token = 2 * a->q_token;
    p.q_head = 2 * a->q_head;
    p.out_token = 2 * a->out_token;
    p.out_head = 2 * a->out_head;
    p.q_heads = int(a->q_heads);
    p.G = int(a->q_heads / a->pool.kv_heads);
    p.scale2 = a->scale * kLog2e;
    p.count = reinterpret_cast<unsigned*>(ws);
    ws += count_bytes(a->workspace_bytes);
    p.part_ml = reinterpret_cast<float*>(ws);
    p.part_o = reinterpret_cast<float*>(ws + s.ml);
    p.target = int(kTarget);
    if (a->pool.type == MTS_BF16)
        launch_t<Bf16>(p, a->pool.head_dim, s, stream);
    else
        launch_t<F16>(p, a->pool.head_dim, s, stream);
    return launched();
}

}  // extern "C"
