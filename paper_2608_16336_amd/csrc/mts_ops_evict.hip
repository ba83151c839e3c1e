// Accumulated attention weights (mts_weigh) and the eviction by them (mts_evict).
#include "mts_ops_dev.h"

namespace mts {
namespace ops {

struct WeighP {
    Pool pool;
    Batch batch;
    const char* q;
    const float* lse;
    float* score;
    int64_t q_token, q_head;  // bytes
    int G, q_heads;
    float scale2, decay;
    int target;
};

constexpr int kWeighRound = 128;  // keys of one round of a workgroup: 4 waves x 32

// Every key's weight is one job's alone, so nothing is joined: a wave holds 32
// keys in the matrix instruction's layout and passes over the query rows, 16
// at a time; a lane's scores S^T = K Q^T are 8 keys of one query, so weights
// add up in the lane and over the 16 lanes of a group at the end.
template <class T, int D>
__global__ __launch_bounds__(256, 2) void k_weigh(const WeighP p)
{
    constexpr int KS = D / 32;
    __shared__ int64_t scratch[8];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, lq = lane & 15, c = lane >> 4;
    Job j;
    const SplitRule rule{kWeighRound, 0, p.G, p.target, false};
    if (!find_job<4>(p.pool, p.batch, rule, j, scratch)) return;
    const int rows = j.T * p.G, base = j.L - j.T;
    const char* kh = p.pool.k + int64_t(j.hk) * p.pool.k_head;
    const int omask = (1 << p.pool.lb) - 1;
    // the next tile's keys are on their way during the present one's rows, their block ids a tile earlier still
    int ids[2], held[2];
    s16x8 kn[2][KS];
    const auto load_ids = [&](int k0) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int key = k0 + 16 * u + lq;
            ids[u] = key < j.k1 ? p.batch.table[size_t(j.r) * p.batch.width + (key >> p.pool.lb)] : -1;
        }
    };
    const auto load_tile = [&](int k0) {
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const bool ok = unsigned(ids[u]) < p.pool.n_blocks;
            held[u] = ok ? ids[u] : -1;
            const char* kp = kh + int64_t(ok ? ids[u] : 0) * p.pool.k_block + int64_t(ok ? (k0 + 16 * u + lq) & omask : 0) * p.pool.k_token;
#pragma unroll
            for (int s = 0; s < KS; ++s) kn[u][s] = *reinterpret_cast<const s16x8*>(kp + (32 * s + 8 * c) * 2);
        }
    };
    int k0 = j.k0 + 32 * w;
    if (k0 < j.k1) {
        load_ids(k0);
        load_tile(k0);
        load_ids(k0 + kWeighRound);
    }
    for (; k0 < j.k1; k0 += kWeighRound) {
        s16x8 kf[2][KS];
        int id[2];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            id[u] = held[u];
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[u][s] = kn[u][s];
        }
        if (k0 + kWeighRound < j.k1) {
            load_tile(k0 + kWeighRound);
            load_ids(k0 + 2 * kWeighRound);
        }
        float acc[8] = {};
        const bool fresh = k0 + 32 > base;
        for (int row0 = 0; row0 < rows; row0 += 16) {
            const int row = row0 + lq;
            const bool ok = row < rows;
            const int t = (ok ? row : 0) / p.G, h = j.hk * p.G + (ok ? row : 0) % p.G;
            const size_t tok = size_t(j.first) + t;
            const char* qp = p.q + tok * p.q_token + int64_t(h) * p.q_head;
            // rows past the end and rows that saw nothing weigh 2^-inf
            float ref = p.lse[tok * p.q_heads + h] * kLog2e;
            if (!ok || ref == -__builtin_inff()) ref = __builtin_inff();
            f32x4 sc[2] = {};
#pragma unroll
            for (int s = 0; s < KS; ++s) {
                const s16x8 qf = *reinterpret_cast<const s16x8*>(qp + (32 * s + 8 * c) * 2);
                sc[0] = T::mfma16(kf[0][s], qf, sc[0]);
                sc[1] = T::mfma16(kf[1][s], qf, sc[1]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                float x = sc[i >> 2][i & 3] * p.scale2 - ref;
                bool see = ref != __builtin_inff();
                if (fresh) {
                    const int rel = k0 + 16 * (i >> 2) + 4 * c + (i & 3) - base;
                    if (rel >= 0)
                        see = see && (p.batch.tree ? rel < 64 * p.batch.words && ((p.batch.tree[tok * p.batch.words + (rel >> 6)] >> (rel & 63)) & 1)
                                                   : rel <= t);
                }
                acc[i] += see ? exp2_fast(x) : 0.f;
            }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int o = 1; o < 16; o <<= 1) acc[i] += __shfl_xor(acc[i], o);
        // lane lq < 8 of a group writes its 4c + lq % 4 of half lq / 4
        float mine = acc[0];
#pragma unroll
        for (int i = 1; i < 8; ++i) mine = lq == i ? acc[i] : mine;
        const int in = 16 * (lq >> 2) + 4 * c + (lq & 3), key = k0 + in;
        // the block of that key is known to the lane that loaded it
        const int b0 = __shfl(id[0], in & 15), b1 = __shfl(id[1], in & 15);
        const int b = in < 16 ? b0 : b1;
        if (lq < 8 && b >= 0) {
            float* at = p.score + ((size_t(b) * p.pool.kv_heads + j.hk) << p.pool.lb) + (key & omask);
            *at = p.decay == 0.f || key >= base ? mine : p.decay * *at + mine;
        }
    }
}

struct EvictP {
    Pool pool;
    Batch batch;
    const float* score;
    const int32_t* pos;
    const int32_t* next_pos;
    float* score_out;
    int32_t *pos_out, *lens_out;
    int budget, recent, sink;
    int cap;        // most moves of a request and head
    int* n_moves;   // [n][kv_heads]
    int* src;       // [n][kv_heads][cap] slots
    int* dst;
};

constexpr int kSelectThreads = 1024, kSelectWaves = 16;

// Larger score, larger key; below all of them 0 (a slot outside the pool),
// above all of them the slots that are kept first.
__device__ __forceinline__ unsigned score_key(float s)
{
    const unsigned u = __float_as_uint(s != s ? -__builtin_inff() : s + 0.f);  // -0 -> 0
    return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}

struct SlotView {
    const EvictP& p;
    int r, hk;
    long long from;  // next_pos - recent
    __device__ __forceinline__ size_t index(int slot, int& id) const
    {
        id = p.batch.table[size_t(r) * p.batch.width + (slot >> p.pool.lb)];
        return ((size_t(id) * p.pool.kv_heads + hk) << p.pool.lb) + (slot & ((1 << p.pool.lb) - 1));
    }
    __device__ __forceinline__ unsigned key(int slot) const
    {
        int id;
        const size_t at = index(slot, id);
        if (unsigned(id) >= p.pool.n_blocks) return 0u;
        const int ps = p.pos[at];
        if ((long long)(ps) < p.sink || ps >= from) return 0xffffffffu;
        return score_key(p.score[at]);
    }
};

// Sum over the lower threads, and the total, of a workgroup of 16 waves.
__device__ __forceinline__ int scan16(int v, int& total, int* scratch)
{
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    int incl = v;
    for (int o = 1; o < 64; o <<= 1) {
        const int u = __shfl_up(incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 63) scratch[w] = incl;
    __syncthreads();
    int base = 0;
    total = 0;
    for (int i = 0; i < kSelectWaves; ++i) {
        if (i < w) base += scratch[i];
        total += scratch[i];
    }
    __syncthreads();
    return base + incl - v;
}

// One workgroup finds which slots of a request and head stay, by a radix
// selection of the budget-th largest key in digits of 11, 11 and 10 bits, and
// lists the moves in slot order: waves own consecutive stretches of slots and
// count before they write, so that no order is left to chance.
__global__ __launch_bounds__(kSelectThreads) void k_evict_select(const EvictP p)
{
    __shared__ int hist[2048];
    __shared__ int scratch[kSelectWaves];
    __shared__ int cut[2];
    __shared__ int wave_a[kSelectWaves], wave_b[kSelectWaves];
    const int hk = blockIdx.x, r = blockIdx.y, tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
    const int L = request_len(p.pool, p.batch, r), B = p.budget;
    const SlotView v{p, r, hk, (long long)(p.next_pos[r]) - p.recent};
    if (hk == 0 && tid == 0) p.lens_out[r] = L < B ? L : B;
    const bool copy = p.score_out != p.score || p.pos_out != p.pos;
    if (L <= B) {
        if (tid == 0) p.n_moves[size_t(r) * p.pool.kv_heads + hk] = 0;
        if (copy)
            for (int s = tid; s < L; s += kSelectThreads) {
                int id;
                const size_t at = v.index(s, id);
                if (unsigned(id) >= p.pool.n_blocks) continue;
                p.score_out[at] = p.score[at];
                p.pos_out[at] = p.pos[at];
            }
        return;
    }
    // thr: the key of rank B; need: how many slots of that key stay, the lowest ones
    unsigned thr = 0, mask = 0;
    int need = B;
    const int shifts[3] = {21, 10, 0}, bits[3] = {11, 11, 10};
    for (int d = 0; d < 3; ++d) {
        const int n = 1 << bits[d];
        hist[tid] = 0;
        hist[tid + 1024] = 0;
        __syncthreads();
        for (int s = tid; s < L; s += kSelectThreads) {
            const unsigned k = v.key(s);
            if ((k & mask) == thr) atomicAdd(&hist[(k >> shifts[d]) & (n - 1)], 1);
        }
        __syncthreads();
        // from the largest digit down: thread t takes bins n-1-2t and n-2-2t
        const int hi = n - 1 - 2 * tid, lo = hi - 1;
        const int a = hi >= 0 ? hist[hi] : 0, b = lo >= 0 ? hist[lo] : 0;
        int total;
        const int above = scan16(a + b, total, scratch);
        if (above < need && need <= above + a) cut[0] = hi, cut[1] = need - above;
        if (above + a < need && need <= above + a + b) cut[0] = lo, cut[1] = need - above - a;
        __syncthreads();
        thr |= unsigned(cut[0]) << shifts[d];
        mask |= unsigned(n - 1) << shifts[d];
        need = cut[1];
        __syncthreads();
    }
    // consecutive stretches of slots for the waves
    const int seg = ((L + kSelectWaves * 64 - 1) / (kSelectWaves * 64)) * 64;
    const int s0 = w * seg < L ? w * seg : L, s1 = s0 + seg < L ? s0 + seg : L;
    int eq = 0;
    for (int s = s0 + lane; s - lane < s1; s += 64) {
        const bool e = s < s1 && v.key(s) == thr;
        eq += __popcll(__ballot(e));
    }
    if (lane == 0) wave_a[w] = eq;
    __syncthreads();
    int eq0 = 0;
    for (int i = 0; i < w; ++i) eq0 += wave_a[i];
    __syncthreads();
    int holes = 0, comers = 0;
    const unsigned long long lt = (1ull << lane) - 1;
    for (int pass = 0; pass < 2; ++pass) {
        int e0 = eq0;
        int* src = p.src + (size_t(r) * p.pool.kv_heads + hk) * p.cap;
        int* dst = p.dst + (size_t(r) * p.pool.kv_heads + hk) * p.cap;
        for (int s = s0 + lane; s - lane < s1; s += 64) {
            const bool in = s < s1;
            const unsigned k = in ? v.key(s) : 0u;
            const bool e = in && k == thr;
            const unsigned long long em = __ballot(e);
            const bool keep = in && (k > thr || (e && e0 + __popcll(em & lt) < need));
            e0 += __popcll(em);
            const unsigned long long hm = __ballot(in && s < B && !keep), cm = __ballot(in && s >= B && keep);
            if (pass) {
                if (in && s < B && !keep) dst[holes + __popcll(hm & lt)] = s;
                if (in && s >= B && keep) src[comers + __popcll(cm & lt)] = s;
                if (copy && s < B && keep) {
                    int id;
                    const size_t at = v.index(s, id);
                    if (unsigned(id) < p.pool.n_blocks) {
                        p.score_out[at] = p.score[at];
                        p.pos_out[at] = p.pos[at];
                    }
                }
            }
            holes += __popcll(hm);
            comers += __popcll(cm);
        }
        if (pass) break;
        if (lane == 0) wave_a[w] = holes, wave_b[w] = comers;
        __syncthreads();
        int total = 0;
        holes = comers = 0;
        for (int i = 0; i < kSelectWaves; ++i) {
            if (i < w) holes += wave_a[i], comers += wave_b[i];
            total += wave_b[i];
        }
        if (tid == 0) p.n_moves[size_t(r) * p.pool.kv_heads + hk] = total;
    }
}

constexpr int kMoveRows = 64;  // moves of a workgroup

// Kept rows above the budget into the holes below it: sources and holes are
// disjoint slots, so rows move in any order.
__global__ __launch_bounds__(256) void k_evict_move(const EvictP p, const int pieces)
{
    const int hk = blockIdx.y % p.pool.kv_heads, r = blockIdx.y / p.pool.kv_heads;
    const size_t at = size_t(r) * p.pool.kv_heads + hk;
    const int n = p.n_moves[at], m0 = blockIdx.x * kMoveRows;
    if (m0 >= n) return;
    const int rows = min(kMoveRows, n - m0);
    const int* src = p.src + at * p.cap + m0;
    const int* dst = p.dst + at * p.cap + m0;
    const int omask = (1 << p.pool.lb) - 1;
    const int32_t* table = p.batch.table + size_t(r) * p.batch.width;
    for (int u = threadIdx.x; u < rows * pieces; u += 256) {
        const int m = u / pieces, d = u % pieces * 16;
        const int a = src[m], b = dst[m];
        const int ia = table[a >> p.pool.lb], ib = table[b >> p.pool.lb];
        if (unsigned(ia) >= p.pool.n_blocks || unsigned(ib) >= p.pool.n_blocks) continue;
        const int64_t oa = a & omask, ob = b & omask;
        const int64_t ka = ia * p.pool.k_block + hk * p.pool.k_head + oa * p.pool.k_token + d;
        const int64_t kb = ib * p.pool.k_block + hk * p.pool.k_head + ob * p.pool.k_token + d;
        const int64_t va = ia * p.pool.v_block + hk * p.pool.v_head + oa * p.pool.v_token + d;
        const int64_t vb = ib * p.pool.v_block + hk * p.pool.v_head + ob * p.pool.v_token + d;
        *reinterpret_cast<u32x4*>(const_cast<char*>(p.pool.k) + kb) = *reinterpret_cast<const u32x4*>(p.pool.k + ka);
        *reinterpret_cast<u32x4*>(const_cast<char*>(p.pool.v) + vb) = *reinterpret_cast<const u32x4*>(p.pool.v + va);
        if (d == 0) {
            const size_t sa = ((size_t(ia) * p.pool.kv_heads + hk) << p.pool.lb) + oa, sb = ((size_t(ib) * p.pool.kv_heads + hk) << p.pool.lb) + ob;
            p.score_out[sb] = p.score[sa];
            p.pos_out[sb] = p.pos[sa];
        }
    }
}

constexpr uint32_t kWeighTarget = 2048;

struct EvictSizes {
    uint64_t cap;
    size_t src, dst, total;
};

static EvictSizes evict_sizes(uint32_t n, uint32_t kv_heads, uint32_t width, uint32_t bt, uint32_t budget)
{
    const uint64_t most = uint64_t(width) * bt, over = most > budget ? most - budget : 0;
    EvictSizes s;
    s.cap = over < budget ? over : budget;
    s.src = align256(4ull * n * kv_heads);
    s.dst = s.src + align256(4ull * n * kv_heads * s.cap);
    s.total = s.dst + align256(4ull * n * kv_heads * s.cap);
    return s;
}

template <class T>
static void launch_weigh(const WeighP& p, uint32_t D, uint32_t jobs, hipStream_t stream)
{
    switch (D) {
    case 64: hipLaunchKernelGGL((k_weigh<T, 64>), dim3(jobs), dim3(256), 0, stream, p); break;
    case 96: hipLaunchKernelGGL((k_weigh<T, 96>), dim3(jobs), dim3(256), 0, stream, p); break;
    case 128: hipLaunchKernelGGL((k_weigh<T, 128>), dim3(jobs), dim3(256), 0, stream, p); break;
    default: hipLaunchKernelGGL((k_weigh<T, 256>), dim3(jobs), dim3(256), 0, stream, p); break;
    }
}

}  // namespace ops
}  // namespace mts

using namespace mts::ops;

extern "C" {

int mts_weigh(const mts_weigh_args* a, hipStream_t stream)
{
    if (!a || !pool_ok(a->pool, true, false) || !head_dim_ok(a->pool.head_dim)) return MTS_EINVAL;
    if (!batch_ok(a->batch, a->pool.block_tokens, true)) return MTS_EINVAL;
    if (a->q_heads < a->pool.kv_heads || a->q_heads % a->pool.kv_heads || a->q_heads > kMaxHeads) return MTS_EINVAL;
    if (!(a->scale == a->scale) || !(a->decay >= 0.f && a->decay <= 1.f)) return MTS_EINVAL;
    if (a->batch.n == 0 || a->batch.n_tokens == 0) return MTS_OK;
    if (!aligned(a->q, 16) || !stride8(a->q_token) || !stride8(a->q_head) || !aligned(a->lse, 4) || !aligned(a->score, 4)) return MTS_EINVAL;
    const uint32_t G = a->q_heads / a->pool.kv_heads;
    if (uint64_t(a->batch.max_q) * G > 0x7fffffffull) return MTS_ERANGE;
    const uint64_t jobs = max_jobs(a->batch.n, a->batch.n_tokens, a->pool.kv_heads, G, 0, kWeighTarget);
    if (jobs > 0x7fffffffull) return MTS_ERANGE;
    WeighP p;
    p.pool = device_pool(a->pool);
    p.batch = device_batch(a->batch);
    p.q = static_cast<const char*>(a->q);
    p.lse = a->lse;
    p.score = a->score;
    p.q_token = 2 * a->q_token;
    p.q_head = 2 * a->q_head;
    p.G = int(G);
    p.q_heads = int(a->q_heads);
    p.scale2 = a->scale * kLog2e;
    p.decay = a->decay;
    p.target = int(kWeighTarget);
    if (a->pool.type == MTS_BF16)
        launch_weigh<Bf16>(p, a->pool.head_dim, uint32_t(jobs), stream);
    else
        launch_weigh<F16>(p, a->pool.head_dim, uint32_t(jobs), stream);
    return launched();
}

int mts_evict_workspace(uint32_t n, uint32_t kv_heads, uint32_t table_width, uint32_t block_tokens, uint32_t budget, size_t* bytes)
{
    if (!bytes || kv_heads < 1 || kv_heads > kMaxHeads || table_width < 1 || budget < 1 || block_tokens < 1 ||
        uint64_t(table_width) * block_tokens > kMaxSlots)
        return MTS_EINVAL;
    *bytes = evict_sizes(n, kv_heads, table_width, block_tokens, budget).total;
    return MTS_OK;
}

int mts_evict(const mts_evict_args* a, hipStream_t stream)
{
    if (!a || !pool_ok(a->pool, true, true) || a->pool.head_dim < 8 || a->pool.head_dim > 512 || a->pool.head_dim % 8) return MTS_EINVAL;
    if (!batch_ok(a->batch, a->pool.block_tokens, false) || a->reserved) return MTS_EINVAL;
    if (a->budget < 1 || a->budget > kMaxSlots || a->recent > kMaxSlots || a->sink > kMaxSlots) return MTS_EINVAL;
    if (a->batch.n == 0) return MTS_OK;
    if (!aligned(a->score, 4) || !aligned(a->pos, 4) || !aligned(a->next_pos, 4) || !aligned(a->score_out, 4) || !aligned(a->pos_out, 4) ||
        !aligned(a->lens_out, 4) || a->lens_out == a->batch.lens || !aligned(a->workspace, 256))
        return MTS_EINVAL;
    const uint64_t rows = uint64_t(a->batch.n) * a->pool.kv_heads;
    if (rows > 65535ull) return MTS_ERANGE;
    const EvictSizes s = evict_sizes(a->batch.n, a->pool.kv_heads, a->batch.table_width, a->pool.block_tokens, a->budget);
    if (a->workspace_bytes < s.total) return MTS_ENOMEM;
    char* ws = static_cast<char*>(a->workspace);
    EvictP p;
    p.pool = device_pool(a->pool);
    p.batch = device_batch(a->batch);
    p.score = a->score;
    p.pos = a->pos;
    p.next_pos = a->next_pos;
    p.score_out = a->score_out;
    p.pos_out = a->pos_out;
    p.lens_out = a->lens_out;
    p.budget = int(a->budget);
    p.recent = int(a->recent);
    p.sink = int(a->sink);
    p.cap = int(s.cap);
    p.n_moves = reinterpret_cast<int*>(ws);
    p.src = reinterpret_cast<int*>(ws + s.src);
    p.dst = reinterpret_cast<int*>(ws + s.dst);
    hipLaunchKernelGGL(k_evict_select, dim3(a->pool.kv_heads, a->batch.n), dim3(kSelectThreads), 0, stream, p);
    if (s.cap)
        hipLaunchKernelGGL(k_evict_move, dim3(uint32_t(ceil_div(s.cap, kMoveRows)), uint32_t(rows)), dim3(256), 0, stream, p,
                           int(a->pool.head_dim / 8));
    return launched();
}

}  // extern "C"
