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

// Called by every thread of a job of several splits after it has written its
// part: the last of the splits' workgroups joins them, in their order.  The
// counter's fences make the others' parts visible to it across the dies.
template <class T, int D, int NT>
__device__ __forceinline__ void join_splits(const AttendP& p, const Job& j, int row0, int rows, int RG, int* last)
{
    __syncthreads();
    if (threadIdx.x == 0) {
        __threadfence();
        const unsigned before = __hip_atomic_fetch_add(&p.count[j.lead], 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        *last = before + 1 == unsigned(j.nsplit);
        if (*last) {
            p.count[j.lead] = 0;
            __threadfence();
        }
    }
    __syncthreads();
    if (!*last) return;
    for (int e = threadIdx.x; e < rows * (D / 4); e += NT) {
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
    __shared__ int64_t scratch[8];
    __shared__ int last;
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, lq = lane & 15, c = lane >> 4;
    Job j;
    const SplitRule rule{kRound, RG, p.G, p.target, false};
    if (!find_job<4>(p.pool, p.batch, rule, j, scratch)) return;
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

    // the next tile's keys and values are asked for once the present ones have left their registers, the block ids a
    // tile earlier still
    int ids[2];
    bool live[2];
    s16x8 kf[2][KS], vf[2][KS];
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
            const int key = k0 + 16 * u + lq;
            live[u] = unsigned(ids[u]) < p.pool.n_blocks;
            const int64_t blk = live[u] ? ids[u] : 0, off = live[u] ? key & omask : 0;
            const char* kp = kh + blk * p.pool.k_block + off * p.pool.k_token;
            const char* vp = vh + blk * p.pool.v_block + off * p.pool.v_token;
#pragma unroll
            for (int s = 0; s < KS; ++s) kf[u][s] = *reinterpret_cast<const s16x8*>(kp + (32 * s + 8 * c) * 2);
#pragma unroll
            for (int s = 0; s < KS; ++s) vf[u][s] = *reinterpret_cast<const s16x8*>(vp + (32 * s + 8 * c) * 2);
        }
    };
    int k0 = j.k0 + 32 * w;
    if (k0 < j.k1) {
        load_ids(k0);
        load_tile(k0);
        load_ids(k0 + kRound);
    }
    for (; k0 < j.k1; k0 += kRound) {
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
        f32x4 sc[MT][2];
#pragma unroll
        for (int m = 0; m < MT; ++m)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                sc[m][u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int s = 0; s < KS; ++s) sc[m][u] = T::mfma16(kf[u][s], qf[m][s], sc[m][u]);
            }
        if (k0 + kRound < j.k1) {
            load_tile(k0 + kRound);
            load_ids(k0 + 2 * kRound);
        }
#pragma unroll
        for (int m = 0; m < MT; ++m) {
            float x[8];
            float mx = -__builtin_inff();
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int in = 4 * c + (i & 3);
                bool see = (alive[i >> 2] >> in) & 1;
                if (fresh) see = see && sees(p.batch, j.first + tq[m], tq[m], k0 + 16 * (i >> 2) + in - base);
                x[i] = see ? sc[m][i >> 2][i & 3] * p.scale2 : -__builtin_inff();
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
                const size_t at = size_t(j.id) * RG + 16 * m + row;
                *reinterpret_cast<f32x4*>(&p.part_o[at * D + d]) = s;
                if (d == 0) {
                    p.part_ml[2 * at] = M;
                    p.part_ml[2 * at + 1] = ls;
                }
            }
        }
    }
    if (whole) return;

    join_splits<T, D, 256>(p, j, row0, rows, RG, &last);
}

// Many query rows: tiles of 64 or 32 keys shared by the waves, 32 rows a wave.
//
// The tile after next's block ids and the next tile's keys and values are on
// their way to registers while the waves compute the present one from LDS;
// two tiles take turns there.  As in the other kernel scores are S^T = K Q^T,
// here 32 x 32, and a lane holds 32 scores of one query: their layout is that
// of P^T in O^T += V^T P^T, with V^T from transposed reads.  The running
// maximum is only followed when it grew by more than 2^kSlack since the sums
// were last scaled (weights up to 2^kSlack lose nothing in 32 bits nor in the
// rounding to 16).
//
// Values of new tokens that are not finite cannot go through the product,
// where rows that do not see them would take 0 x inf: they are staged as zero
// and added to the rows that see them, which is what weighting them gives.
constexpr float kSlack = 8.f;
// keys of a tile: half as many where a row is twice as long
constexpr int tile_keys(int D) { return D == 256 ? 32 : 64; }

template <class T, int D, int NW>
__global__ __launch_bounds__(64 * NW, D == 256 ? 1 : 2) void k_attend_tiles(const AttendP p)
{
    constexpr int NT = 64 * NW, RG = 32 * NW, CH = D / 8, KS = D / 16, DT = D / 32, kTile = tile_keys(D), UT = kTile / 32;
    constexpr int PIECES = (kTile * CH + NT - 1) / NT;  // 16-byte pieces a thread stages of each of K and V, at most
    constexpr bool EVEN = kTile * CH % NT == 0;
    __shared__ __attribute__((aligned(16))) char ks[2][kTile * D * 2];
    __shared__ __attribute__((aligned(16))) char vs[2][kTile * D * 2];
    __shared__ int64_t scratch[NW + 4];
    __shared__ int last;
    const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6, lq = lane & 31, h = lane >> 5;
    Job j;
    const SplitRule rule{64, RG, p.G, p.target, true};
    if (!find_job<NW>(p.pool, p.batch, rule, j, scratch)) return;
    const int row0 = j.grp * RG, rows = min(RG, j.T * p.G - row0), base = j.L - j.T;
    // a chain's later slots are seen by none of the group's rows
    if (!p.batch.tree) j.k1 = min(j.k1, base + (row0 + rows - 1) / p.G + 1);

    const int my = 32 * w + lq, rr = row0 + min(my, rows - 1), tq = rr / p.G;
    const size_t tok = size_t(j.first) + tq;
    s16x8 qf[KS];
    {
        const char* qp = p.q + tok * p.q_token + int64_t(j.hk * p.G + rr % p.G) * p.q_head;
#pragma unroll
        for (int s = 0; s < KS; ++s) qf[s] = *reinterpret_cast<const s16x8*>(qp + (16 * s + 8 * h) * 2);
        if (p.scale2 < 0.f) {
            // the running maximum is one of q.k: the sign of the scale goes to the queries
#pragma unroll
            for (int s = 0; s < KS; ++s) qf[s] ^= short(0x8000);
        }
    }
    const float scale2 = fabsf(p.scale2);
    const bool idle = 32 * w >= rows;  // this wave only stages

    f32x16 o[DT];
#pragma unroll
    for (int t = 0; t < DT; ++t)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[t][i] = 0.f;
    float m_ref = -__builtin_inff(), l_run = 0.f;

    const char* kh = p.pool.k + int64_t(j.hk) * p.pool.k_head;
    const char* vh = p.pool.v + int64_t(j.hk) * p.pool.v_head;
    const int32_t* table = p.batch.table + size_t(j.r) * p.batch.width;
    const int omask = (1 << p.pool.lb) - 1;

    int ids[PIECES], my_id;  // block ids of the staged rows, and of slot k0 + lane
    const auto load_ids = [&](int k0) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int key = k0 + (tid + NT * i) / CH;
            ids[i] = key < j.k1 && (EVEN || tid + NT * i < kTile * CH) ? table[key >> p.pool.lb] : -1;
        }
        my_id = lane < kTile && k0 + lane < j.k1 ? table[(k0 + lane) >> p.pool.lb] : -1;
    };
    s16x8 kr[PIECES], vr[PIECES];
    uint64_t alive_next = 0;
    const auto load_tile = [&](int k0) {
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int key = k0 + (tid + NT * i) / CH, piece = (tid + NT * i) % CH;
            const bool ok = unsigned(ids[i]) < p.pool.n_blocks;
            const int64_t blk = ok ? ids[i] : 0, off = ok ? key & omask : 0;
            kr[i] = *reinterpret_cast<const s16x8*>(kh + blk * p.pool.k_block + off * p.pool.k_token + piece * 16);
            const s16x8 x = *reinterpret_cast<const s16x8*>(vh + blk * p.pool.v_block + off * p.pool.v_token + piece * 16);
            vr[i] = ok ? x : s16x8{};
        }
        alive_next = __ballot(unsigned(my_id) < p.pool.n_blocks);
    };
    // Stores the staged tile; whether values of new tokens were not finite.
    const auto store_tile = [&](int buf, int k0) {
        bool odd = false;
        if (k0 + kTile > base) {
#pragma unroll
            for (int i = 0; i < PIECES; ++i)
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool bad = (unsigned(vr[i][e]) & T::kExp) == T::kExp;
                    odd |= bad;
                    vr[i][e] = bad ? short(0) : vr[i][e];
                }
        }
#pragma unroll
        for (int i = 0; i < PIECES; ++i) {
            const int row = (tid + NT * i) / CH, piece = (tid + NT * i) % CH;
            const int at = row * D * 2 + ((piece ^ swz<D>(row)) * 16);
            if (!EVEN && row >= kTile) continue;
            *reinterpret_cast<s16x8*>(&ks[buf][at]) = kr[i];
            *reinterpret_cast<s16x8*>(&vs[buf][at]) = vr[i];
        }
        return odd;
    };

    int k0 = j.k0, buf = 0;
    bool odd = false;
    uint64_t alive = 0;
    if (k0 < j.k1) {
        load_ids(k0);
        load_tile(k0);
        load_ids(k0 + kTile);
        alive = alive_next;
        odd = store_tile(0, k0);
    }
    for (; k0 < j.k1; k0 += kTile, buf ^= 1) {
        const bool fresh = k0 + kTile > base;
        if (fresh)
            odd = __syncthreads_or(odd);
        else
            __syncthreads();
        const bool more = k0 + kTile < j.k1;
        if (more) {
            load_tile(k0 + kTile);
            load_ids(k0 + 2 * kTile);
        }
        if (!idle) {
            f32x16 sc[UT];
#pragma unroll
            for (int u = 0; u < UT; ++u) {
#pragma unroll
                for (int i = 0; i < 16; ++i) sc[u][i] = 0.f;
                const int row = 32 * u + lq;
#pragma unroll
                for (int s = 0; s < KS; ++s) {
                    const s16x8 kf = *reinterpret_cast<const s16x8*>(&ks[buf][row * D * 2 + (((2 * s + h) ^ swz<D>(row)) * 16)]);
                    sc[u] = T::mfma32(kf, qf[s], sc[u]);
                }
            }
            uint64_t see = alive;
            if (fresh) {
                // the slots of the tile that this lane's row sees
                const int rel = k0 - base;
                if (!p.batch.tree) {
                    const int most = tq - rel;
                    see &= most >= 63 ? ~0ull : most < 0 ? 0ull : (2ull << most) - 1;
                } else {
                    const uint64_t* bits = p.batch.tree + tok * p.batch.words;
                    const auto word = [&](int i) { return i >= 0 && i < p.batch.words ? bits[i] : 0ull; };
                    if (rel >= 0) {
                        const int i = rel >> 6, s = rel & 63;
                        see &= (word(i) >> s) | (s ? word(i + 1) << (64 - s) : 0ull);
                    } else if (rel > -64) {
                        see &= (word(0) << -rel) | ((1ull << -rel) - 1);
                    }
                }
            }
            if (fresh || alive != (kTile == 64 ? ~0ull : 0xffffffffull)) {
                const uint64_t s = see >> (4 * h);
#pragma unroll
                for (int u = 0; u < UT; ++u) {
                    const unsigned bits = unsigned(s >> (32 * u));
#pragma unroll
                    for (int i = 0; i < 16; ++i) sc[u][i] = (bits >> (8 * (i / 4) + i % 4)) & 1 ? sc[u][i] : -__builtin_inff();
                }
            }
            float mx = sc[0][0];
#pragma unroll
            for (int i = 0; i < 16 * UT; ++i) mx = fmaxf(mx, sc[i >> 4][i & 15]);
            mx = fmaxf(mx, __shfl_xor(mx, 32)) * scale2;
            if (__any(mx > m_ref + kSlack)) {
                const float mn = fmaxf(m_ref, mx);
                const float alpha = mn == -__builtin_inff() ? 1.f : exp2_fast(m_ref - mn);
                m_ref = mn;
                l_run *= alpha;
#pragma unroll
                for (int t = 0; t < DT; ++t) o[t] *= alpha;
            }
            const float ref = m_ref == -__builtin_inff() ? 0.f : m_ref;
            float sum = 0.f;
#pragma unroll
            for (int u = 0; u < UT; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    sc[u][i] = exp2_fast(__builtin_fmaf(sc[u][i], scale2, -ref));
                    sum += sc[u][i];
                }
            l_run += sum;
#pragma unroll
            for (int kk = 0; kk < kTile / 16; ++kk) {
                f32x8 x;
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = sc[kk >> 1][8 * (kk & 1) + i];
                const s16x8 pf = pack8<T>(x);
#pragma unroll
                for (int t = 0; t < DT; ++t) {
                    s16x8 a;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const int row = 16 * kk + 8 * u + 4 * h + ((lane & 15) >> 2), piece = 4 * t + 2 * ((lane >> 4) & 1) + ((lane & 3) >> 1);
                        const s16x4 x4 = read_tr16(&vs[buf][row * D * 2 + ((piece ^ swz<D>(row)) * 16) + (lane & 1) * 8]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) a[4 * u + i] = x4[i];
                    }
                    o[t] = T::mfma32(a, pf, o[t]);
                }
            }
            if (fresh && odd) {
                for (int key = 0; key < kTile; ++key) {
                    if (!((alive >> key) & 1)) continue;
                    const char* vp = vh + int64_t(table[(k0 + key) >> p.pool.lb]) * p.pool.v_block + int64_t((k0 + key) & omask) * p.pool.v_token;
                    const bool mine = (see >> key) & 1;
#pragma unroll
                    for (int t = 0; t < DT; ++t)
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            const short x = reinterpret_cast<const short*>(vp)[32 * t + 8 * (i / 4) + 4 * h + i % 4];
                            if (mine && (unsigned(x) & T::kExp) == T::kExp) o[t][i] += widen<T>(x);
                        }
                }
            }
        }
        if (more) {
            odd = store_tile(buf ^ 1, k0 + kTile);
            alive = alive_next;
        }
    }

    l_run += __shfl_xor(l_run, 32);
    const float M = m_ref;
    if (my < rows) {
        if (j.nsplit == 1) {
            const float inv = l_run > 0.f ? 1.f / l_run : (l_run == 0.f ? 0.f : l_run);
            char* op = p.out + tok * p.out_token + int64_t(j.hk * p.G + rr % p.G) * p.out_head;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 x = {o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
                    *reinterpret_cast<s16x4*>(op + 2 * (32 * t + 8 * i + 4 * h)) = pack4<T>(x * inv);
                }
            if (h == 0 && p.lse) p.lse[tok * p.q_heads + j.hk * p.G + rr % p.G] = l_run == 0.f ? -__builtin_inff() : M * kLn2 + __logf(l_run);
        } else {
            const size_t at = size_t(j.id) * RG + my;
#pragma unroll
            for (int t = 0; t < DT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    *reinterpret_cast<f32x4*>(&p.part_o[at * D + 32 * t + 8 * i + 4 * h]) = f32x4{o[t][4 * i], o[t][4 * i + 1], o[t][4 * i + 2], o[t][4 * i + 3]};
            if (h == 0) {
                p.part_ml[2 * at] = M;
                p.part_ml[2 * at + 1] = l_run;
            }
        }
    }
    if (j.nsplit > 1) join_splits<T, D, NT>(p, j, row0, rows, RG, &last);
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
    const uint64_t most = uint64_t(max_q) * G;
    s.rows = most <= 16 ? 16 : most <= 128 || head_dim == 256 ? 128 : 256;
    s.jobs = max_jobs(n, n_tokens, kv_heads, G, s.rows, kTarget);
    s.ml = align256(8 * s.jobs * s.rows);
    s.o = align256(4 * s.jobs * s.rows * head_dim);
    s.total = align256((s.ml + s.o) / (kCountShare - 1) * kCountShare + 2 * 256 * kCountShare);
    return s;
}

template <class T, int D>
static void launch_d(const AttendP& p, const Sizes& s, hipStream_t stream)
{
    const dim3 grid(uint32_t(s.jobs));
    if (s.rows == 16)
        hipLaunchKernelGGL((k_attend_rows<T, D, 1>), grid, dim3(256), 0, stream, p);
    else if (s.rows == 128)
        hipLaunchKernelGGL((k_attend_tiles<T, D, 4>), grid, dim3(256), 0, stream, p);
    else if constexpr (D < 256)
        hipLaunchKernelGGL((k_attend_tiles<T, D, 8>), grid, dim3(512), 0, stream, p);
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
