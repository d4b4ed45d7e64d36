// Attention over packed prompts (prompt.h): o = sum_j p_j v_j, p = softmax(c q.k_j), and the log-sum-exp, in one pass over the keys
// with a running reference and sum per row.
//
// A workgroup takes 256 rows of one sequence and KV head -- with G query heads to a KV head the rows of 256 / G tokens, so that G heads share
// each key tile and all rows of a block reach about equally far -- and walks the keys in tiles of 64.  K and V go from the caller's
// tensors straight into LDS, three stages each, rows as they are: S^T = K.Q^T reads a tile's rows, O^T += V^T.P^T reads it transposed
// (ds_read_b64_tr_b16), and no packed copy is made first.  The eight wavefronts work in two sets in counter-phase, as the masked walk's
// do (attn_walk.hip): a SIMD's two wavefronts take turns at the matrix pipes, one's softmax under the other's products.
// A wavefront stops at the last tile that its own 32 rows reach.
//
// Score products are exact (bf16 x bf16 accumulated in fp32); the softmax scale is applied in fp32 with the reference, one
// instruction.  Weights are rounded to bf16 for P.V only: the sum is of the fp32 weights, so the log-sum-exp carries no bf16 rounding.
//
// Where the blocks are too few to fill the chip (a short turn on a long history), each block's keys are shared out to several
// workgroups, which leave fp32 partial results in the workspace, and prompt_join_kernel puts these together.
#include <algorithm>

#include "prompt.h"

namespace adaspark {

template <int D, int WAVES>
struct Prompt {
    static constexpr int THREADS = 64 * WAVES;
    static constexpr int NS = 2;
    static constexpr int ROWS = 16 * NS * WAVES;
    static constexpr int NST = WAVES == 8 ? 3 : 2;  // LDS stages of K and of V
    static constexpr int PF = 4;   // operand loads in flight ahead of the MFMAs
    static constexpr int TILE = KEY_TILE * D * 2;
    static constexpr int CPR = D / 8;              // 16-byte chunks of a row
    static constexpr int RPI = 64 / CPR;           // rows of one direct-to-LDS instruction
    static constexpr int DMA = TILE / 1024 / WAVES;
    static constexpr int OFF_V = NST * TILE;
    static constexpr int BYTES = 2 * NST * TILE;
    static_assert(BYTES <= 160 * 1024, "LDS of one CU");
};
constexpr float LN2 = 0.69314718055994530942f;

// A part's result: O unnormalised, fp32 [rows][D], then (m, l) of each row (m in base 2).
__host__ __device__ inline size_t prompt_part_floats(int rows, int D) { return (size_t)rows * (D + 2); }

template <int KEEP>
__device__ __forceinline__ void stage_barrier()
{
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(KEEP) : "memory");
}

template <int D, int WAVES, bool SPLIT>
__global__ __launch_bounds__(64 * WAVES, 2) void prompt_attn_kernel(PromptGeom g, int per_head, int parts, const uint16_t *__restrict__ Q,
                                                          const uint16_t *__restrict__ K, const uint16_t *__restrict__ V,
                                                          uint16_t *__restrict__ O, float *__restrict__ lse,
                                                          float *__restrict__ partial)
{
    using C = Prompt<D, WAVES>;
    constexpr int NS = C::NS, KSTEPS = D / 32, DT = D / 16, PF = C::PF;
    extern __shared__ __attribute__((aligned(256))) unsigned char smem[];

    const int lane = threadIdx.x & 63, n16 = lane & 15, q4 = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const bool set_y = WAVES == 8 && wave >= 4;

    int kv, slot;
    if (!head_slot(blockIdx.x, g.Hkv, per_head, kv, slot)) return;
    const int part = SPLIT ? slot % parts : 0;
    const PromptBlock b = longest_first(g, SPLIT ? slot / parts : slot, (g.Tk + KEY_TILE - 1) / KEY_TILE,
                                        [&](int n, int m, int t) { return row_blocks<C::ROWS>(n, m, g.G, g.causal, t); });
    if (b.seq < 0) return;
    const PromptSeq p = b.p;
    const int rows = p.n * g.G, i = (rows - 1) / C::ROWS - b.block, row0 = i * C::ROWS;
    auto reach_of = [&](int row) { return g.causal ? p.m - p.n + token_of_row(g, row) : p.m - 1; };  // the last key that a row attends
    auto tiles_to = [&](int row) { return max(0, reach_of(min(row, rows - 1)) / KEY_TILE + (reach_of(min(row, rows - 1)) >= 0 ? 1 : 0)); };

    // the tiles of the block's walk, and of the wavefront's: first .. first + count
    int first = 0, ntiles = __builtin_amdgcn_readfirstlane(tiles_to(row0 + C::ROWS - 1));
    int mine = row0 + 32 * wave < rows ? __builtin_amdgcn_readfirstlane(tiles_to(row0 + 32 * wave + 31)) : 0;
    if (SPLIT) {
        const int per = (ntiles + parts - 1) / parts;
        first = min(part * per, ntiles);
        ntiles = min(per, ntiles - first);
        mine = min(max(mine - first, 0), ntiles);
    }

    // the wavefront's rows (past the last one it is repeated)
    int reach[NS];
    bool valid[NS];
    size_t rid[NS];
    bf16x8 qf[NS][KSTEPS];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const int row = row0 + 32 * wave + 16 * s + n16, r = min(row, rows - 1), tok = token_of_row(g, r);
        valid[s] = row < rows;
        reach[s] = reach_of(r);
        const int head = kv * g.G + (r - tok * g.G);
        rid[s] = (size_t)(p.q0 + tok) * g.Hq + head;
        const uint16_t *q = Q + (size_t)(p.q0 + tok) * g.qs + (size_t)head * D + 8 * q4;
#pragma unroll
        for (int c = 0; c < KSTEPS; ++c) qf[s][c] = *reinterpret_cast<const bf16x8 *>(q + 32 * c);
    }
    const int reach_lo = __builtin_amdgcn_readfirstlane(reach[0]);  // of the wavefront's first row: no other reaches less far

    // Loads: piece u of this wavefront is RPI rows of a tile, a 16-byte slot to a lane, which fetches the chunk that belongs there.
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)smem);
    const uint32_t piece0 = __builtin_amdgcn_readfirstlane(lds0 + (uint32_t)(wave * C::DMA * 1024));
    uint32_t kofs[C::DMA], vofs[C::DMA];
    int prow[C::DMA], pchunk[C::DMA];
#pragma unroll
    for (int u = 0; u < C::DMA; ++u) {
        prow[u] = (wave * C::DMA + u) * C::RPI + lane / C::CPR;
        pchunk[u] = (((lane & 15) ^ row_swizzle<D>(prow[u])) & (C::CPR - 1)) * 8;
        kofs[u] = (uint32_t)(prow[u] * (int)g.ks + pchunk[u]) * 2u;
        vofs[u] = (uint32_t)(prow[u] * (int)g.vs + pchunk[u]) * 2u;
    }
    const uint16_t *khead = K + (size_t)p.k0 * g.ks + (size_t)kv * D, *vhead = V + (size_t)p.k0 * g.vs + (size_t)kv * D;
    // (keys past the sequence's last are that one again: its weights there are zero, its value finite where a row's are)
    auto issue = [&](const uint16_t *head, long long stride, const uint32_t (&ofs)[C::DMA], int t, int off) __attribute__((always_inline)) {
        const int key = (first + t) * KEY_TILE;
        const void *tile = uniform_ptr(head + (size_t)key * stride);
        if (key + KEY_TILE <= p.m) {
#pragma unroll
            for (int u = 0; u < C::DMA; ++u) dma_1k_s(piece0 + (uint32_t)(off + u * 1024), tile, ofs[u]);
        } else {
#pragma unroll
            for (int u = 0; u < C::DMA; ++u) {
                const int r = (wave * C::DMA + u) * C::RPI + lane / C::CPR;
                const int chunk = (((lane & 15) ^ row_swizzle<D>(r)) & (C::CPR - 1)) * 8;
                dma_1k_s(piece0 + (uint32_t)(off + u * 1024), tile, (uint32_t)(min(r, p.m - 1 - key) * (int)stride + chunk) * 2u);
            }
        }
    };
    auto issue_k = [&](int t, int st) __attribute__((always_inline)) { issue(khead, g.ks, kofs, t, st * C::TILE); };
    auto issue_v = [&](int t, int st) __attribute__((always_inline)) { issue(vhead, g.vs, vofs, t, C::OFF_V + st * C::TILE); };

    const float c2 = 1.44269504088896340736f / sqrtf((float)D);  // softmax scale in base 2
    float m_run[NS], l_run[NS];  // reference point of the exponentials; sum of the lane's keys' weights
    bool fresh[NS], settled = false;
    f32x4 oacc[NS][DT], sacc[NS][4];
    bf16x8 pf[NS][2];
#pragma unroll
    for (int s = 0; s < NS; ++s) {
        m_run[s] = l_run[s] = 0.f;
        fresh[s] = true;
#pragma unroll
        for (int e = 0; e < DT; ++e) oacc[s][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // Slot t works on K(t) and V(t-1).  Three stages: K(t+1) and V(t) may be in flight when it opens, K(t+2) and V(t+1) are started into
    // the stages that fell free (as in attn_walk.hip).  Two: K(t+1) and V(t) are started when it opens, and waited for at the next.
    int kst = 0;  // stage of K(t); V(t-1) sits in the one before
    auto before = [](int st) { return st == 0 ? C::NST - 1 : st - 1; };
    auto after = [](int st) { return st == C::NST - 1 ? 0 : st + 1; };
    auto open_slot = [&](int t) __attribute__((always_inline)) {
        if (C::NST == 3) {
            if (t > 0 && t + 1 < ntiles) stage_barrier<2 * C::DMA>();
            else stage_barrier<0>();
            if (t + 1 < ntiles) issue_v(t + 1, after(kst));
            if (t + 2 < ntiles) issue_k(t + 2, before(kst));
        } else {
            stage_barrier<0>();
            if (t > 0 && t < ntiles) issue_v(t, kst);
            if (t + 1 < ntiles) issue_k(t + 1, after(kst));
        }
    };
    auto next_slot = [&](int t) __attribute__((always_inline)) {
        kst = after(kst);
        open_slot(t);
    };

    // Operand reads (the lane's place in a tile, without the 16-row block and the chunk's high bits, which are flipped per read)
    const uint32_t nat0 = lds0 + (uint32_t)row_tile_off<D>(n16, q4);
    const uint32_t tr0 = lds0 + (uint32_t)(C::OFF_V + row_tile_off<D>(4 * q4 + (n16 >> 2), (n16 & 3) >> 1) + 8 * (n16 & 1));
    constexpr int BLK = 16 * D * 2;  // bytes of 16 tile rows
    auto k_operand = [&](uint32_t at, int c, int kg) __attribute__((always_inline)) {
        return lds_read<bf16x8>((at ^ (uint32_t)(c << 6)) + (uint32_t)(kg * BLK));
    };
    auto v_operand = [&](uint32_t at, int sl, int e) __attribute__((always_inline)) {
        return lds_read_tr2((at ^ (uint32_t)(e << 5)) + (uint32_t)(2 * sl * BLK), BLK);
    };
    // The products of a slot, P.V of tile t-1 and S of tile t, as one stream of operand reads and MFMAs: the reads run PF ahead
    // through a ring of registers, the order written is the order executed.
    auto products = [&](auto pv, auto qk) __attribute__((always_inline)) {
        constexpr bool PV = decltype(pv)::value, QK = decltype(qk)::value;
        constexpr int RV = PV ? 2 * DT : 0, R = RV + (QK ? 4 * KSTEPS : 0);
        const uint32_t kt = nat0 + (uint32_t)(kst * C::TILE), vt = tr0 + (uint32_t)(before(kst) * C::TILE);
        bf16x8 ring[PF];
        auto operand = [&](int r) __attribute__((always_inline)) {
            return r < RV ? v_operand(vt, r / DT, r % DT) : k_operand(kt, (r - RV) / 4, (r - RV) % 4);
        };
#pragma unroll
        for (int r = 0; r < PF && r < R; ++r) ring[r] = operand(r);
        __builtin_amdgcn_s_setprio(1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const bf16x8 a = ring[r % PF];
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                if (r < RV) oacc[s][r % DT] = mfma16(a, pf[s][r / DT], oacc[s][r % DT]);
                else sacc[s][(r - RV) % 4] = mfma16(a, qf[s][(r - RV) / 4], (r - RV) / 4 == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : sacc[s][(r - RV) % 4]);
            }
            if (r + PF < R) ring[r % PF] = operand(r + PF);
            __builtin_amdgcn_sched_barrier(0);
        }
        __builtin_amdgcn_s_setprio(0);
    };

    // Weights of tile t.  sacc[s][kg][v]: key 16 kg + 4 q4 + v, which is element 4 (kg % 2) + v of operand kg / 2.
    auto weights = [&](float (&sum)[NS]) __attribute__((always_inline)) {
#pragma unroll
        for (int s = 0; s < NS; ++s) sum[s] = 0.f;
#pragma unroll
        for (int kg = 0; kg < 4; ++kg)
#pragma unroll
            for (int v = 0; v < 4; ++v)
#pragma unroll
                for (int s = 0; s < NS; ++s) {
                    const float w = __builtin_amdgcn_exp2f(fmaf(sacc[s][kg][v], c2, -m_run[s]));
                    sum[s] += w;
                    pf[s][kg >> 1][4 * (kg & 1) + v] = (__bf16)w;
                }
    };
    auto softmax = [&](int t) __attribute__((always_inline)) {
        const int key0 = (first + t) * KEY_TILE;
        const bool edge = key0 + KEY_TILE - 1 > reach_lo;
        float sum[NS];
        bool done = false;
        if (settled && !edge) {
            // The weights straight away; a weight of 2 or more has the top exponent bit of its bf16 pattern set, and says that some row's
            // reference has to be moved first (attn_tile.h).
            weights(sum);
            uint32_t big = 0u;
#pragma unroll
            for (int s = 0; s < NS; ++s)
#pragma unroll
                for (int sl = 0; sl < 2; ++sl) {
                    const u32x4 w = __builtin_bit_cast(u32x4, pf[s][sl]);
                    big |= (w[0] | w[1]) | (w[2] | w[3]);
                }
            done = __ballot((big & 0x40004000u) != 0u) == 0ull;
        }
        if (!done) {
            if (edge) {
                int kb = key0 + 4 * q4;
                asm volatile("" : "+v"(kb));
#pragma unroll
                for (int s = 0; s < NS; ++s)
#pragma unroll
                    for (int kg = 0; kg < 4; ++kg)
#pragma unroll
                        for (int v = 0; v < 4; ++v)
                            if (kb + 16 * kg + v > reach[s]) sacc[s][kg][v] = -INFINITY;
            }
            bool open = false;
#pragma unroll
            for (int s = 0; s < NS; ++s) {
                float mx = vmax3(sacc[s][0][0], sacc[s][0][1], sacc[s][0][2]);
                mx = vmax3(mx, sacc[s][0][3], sacc[s][1][0]);
                mx = vmax3(mx, sacc[s][1][1], sacc[s][1][2]);
                mx = vmax3(mx, sacc[s][1][3], sacc[s][2][0]);
                mx = vmax3(mx, sacc[s][2][1], sacc[s][2][2]);
                mx = vmax3(mx, sacc[s][2][3], sacc[s][3][0]);
                mx = vmax3(mx, sacc[s][3][1], sacc[s][3][2]);
                mx = quad_max(vmax(mx, sacc[s][3][3])) * c2;
                const bool grow = fresh[s] ? mx > -INFINITY : mx >= m_run[s] + SOFTMAX_LAZY;
                if (__ballot(grow) != 0ull) {
                    const float to = grow ? mx + SOFTMAX_HEADROOM : m_run[s];
                    const float alpha = grow && !fresh[s] ? __builtin_amdgcn_exp2f(m_run[s] - to) : 1.f;  // (a fresh row has O = l = 0)
                    m_run[s] = to;
                    fresh[s] = fresh[s] && !grow;
#pragma unroll
                    for (int e = 0; e < DT; ++e) oacc[s][e] *= alpha;
                    l_run[s] *= alpha;
                }
                open = open || fresh[s];
            }
            settled = __ballot(open) == 0ull;
            weights(sum);
        }
#pragma unroll
        for (int s = 0; s < NS; ++s) l_run[s] += sum[s];
    };

    // prologue: K(0), V(0), K(1)
    if (ntiles > 0) {
        issue_k(0, 0);
        issue_v(0, 0);
        if (C::NST == 3 && ntiles > 1) issue_k(1, 1);
    }
    const std::true_type yes;
    const std::false_type no;
    open_slot(0);
    if (mine > 0) {
        products(no, yes);
        int t = 1;
        if (!set_y) {
            softmax(0);
            for (; t < mine; ++t) {
                next_slot(t);
                products(yes, yes);
                softmax(t);
            }
            next_slot(t);
        } else {
            for (; t < mine; ++t) {
                next_slot(t);
                softmax(t - 1);
                products(yes, yes);
            }
            next_slot(t);
            softmax(t - 1);
        }
        products(yes, no);
    }
    for (int t = mine > 0 ? mine + 1 : 1; t <= ntiles; ++t) next_slot(t);  // (its loads are others' keys)
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");  // no direct-to-LDS load may outlive the workgroup's LDS

#pragma unroll
    for (int s = 0; s < NS; ++s) {
        const float l = quad_sum(l_run[s]);
        if (!valid[s]) continue;
        if (SPLIT) {
            float *out = partial + (((size_t)kv * per_head / parts + row_block_id(g, C::ROWS, b.seq, p.q0, i)) * parts + part) * prompt_part_floats(C::ROWS, D);
            const int r = 32 * wave + 16 * s + n16;
#pragma unroll
            for (int e = 0; e < DT; ++e) *reinterpret_cast<f32x4 *>(out + r * D + 16 * e + 4 * q4) = oacc[s][e];
            if (q4 == 0) *reinterpret_cast<float2 *>(out + C::ROWS * D + 2 * r) = make_float2(fresh[s] ? -INFINITY : m_run[s], l);
        } else {
            const float inv = fresh[s] ? 0.f : 1.0f / l;  // (a row without keys: zero)
            uint16_t *o = O + rid[s] * D + 4 * q4;
#pragma unroll
            for (int e = 0; e < DT; ++e) *reinterpret_cast<uint2 *>(o + 16 * e) = pack_bf16(oacc[s][e] * inv);
            if (lse != nullptr && q4 == 0) lse[rid[s]] = fresh[s] ? -INFINITY : (m_run[s] + log2f(l)) * LN2;
        }
    }
}

// The parts of a row put together, a wavefront for each (token, query head): lane l has D / 64 columns.
template <int D, int ROWS>
__global__ __launch_bounds__(256) void prompt_join_kernel(PromptGeom g, int per_kv, int parts, const float *__restrict__ partial,
                                                          uint16_t *__restrict__ O, float *__restrict__ lse)
{
    constexpr int N = D / 64;
    const int lane = threadIdx.x & 63;
    const long long row = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (row >= (long long)g.Tq * g.Hq) return;
    const int tok = (int)(row / g.Hq), a = (int)(row - (long long)tok * g.Hq), kv = a / g.G;
    int lo = 0, hi = g.B;  // the last sequence with a start at or before the token
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (g.q_start[mid] <= tok) lo = mid;
        else hi = mid;
    }
    const PromptSeq p = prompt_seq(g, lo);
    if (tok < p.q0 || tok >= p.q0 + p.n) return;
    const int r = (tok - p.q0) * g.G + (a - kv * g.G), i = r / ROWS, at = r - i * ROWS;
    const float *from = partial + ((size_t)kv * per_kv + row_block_id(g, ROWS, lo, p.q0, i)) * parts * prompt_part_floats(ROWS, D);
    const float2 ml = lane < parts ? *reinterpret_cast<const float2 *>(from + lane * prompt_part_floats(ROWS, D) + ROWS * D + 2 * at)
                                   : make_float2(-INFINITY, 0.f);
    float M = ml.x;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) M = fmaxf(M, __shfl_xor(M, d, 64));
    const float w = ml.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
    float L = w * ml.y, o[N];
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) L += __shfl_xor(L, d, 64);
#pragma unroll
    for (int k = 0; k < N; ++k) o[k] = 0.f;
    for (int x = 0; x < parts; x += 4) {  // four parts' loads at a time (past the last one it is read again, with a weight of 0)
        float y[4][N];
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int k = 0; k < N; ++k) y[u][k] = from[min(x + u, parts - 1) * prompt_part_floats(ROWS, D) + at * D + N * lane + k];
#pragma unroll
        for (int u = 0; u < 4; ++u) {
            const float wx = x + u < parts ? __shfl(w, x + u, 64) : 0.f;
#pragma unroll
            for (int k = 0; k < N; ++k) o[k] = fmaf(wx, y[u][k], o[k]);
        }
    }
    const float inv = M == -INFINITY ? 0.f : 1.0f / L;
#pragma unroll
    for (int k = 0; k < N; ++k) reinterpret_cast<__bf16 *>(O)[(size_t)row * D + N * lane + k] = (__bf16)(o[k] * inv);
    if (lse != nullptr && lane == 0) lse[row] = M == -INFINITY ? -INFINITY : (M + log2f(L)) * LN2;
}

// How many workgroups share a block's keys: as many as fill the chip's 256 CUs once, each with eight tiles at least (of all keys: where
// a sequence has fewer than the batch, its parts are shorter).
constexpr int SPLIT_WAVES = 8;
static int prompt_parts(const PromptGeom &g)
{
    const long long blocks = g.Hkv * row_block_bound(g, 32 * SPLIT_WAVES), tiles = (g.Tk + KEY_TILE - 1) / KEY_TILE;
    return (int)std::max(1ll, std::min(std::min(256 / blocks, tiles / 8), 64ll));
}

static size_t prompt_partial_bytes(const PromptGeom &g, int D)
{
    const int parts = prompt_parts(g);
    return parts > 1 ? (size_t)g.Hkv * row_block_bound(g, 32 * SPLIT_WAVES) * parts * prompt_part_floats(32 * SPLIT_WAVES, D) * 4 : 0;
}
size_t prompt_workspace_bytes(const PromptGeom &g, int D) { return prompt_partial_bytes(g, D); }

template <int D, int WAVES, bool SPLIT>
static hipError_t launch_walk(const PromptGeom &g, int parts, const uint16_t *Q, const uint16_t *K, const uint16_t *V, uint16_t *O,
                              float *lse, float *partial, hipStream_t st)
{
    using C = Prompt<D, WAVES>;
    static LdsOptIn opted;  // one per kernel instantiation
    const hipError_t e = opted.ensure(reinterpret_cast<const void *>(&prompt_attn_kernel<D, WAVES, SPLIT>), C::BYTES);
    if (e != hipSuccess) return e;
    const int per_head = (int)row_block_bound(g, C::ROWS) * parts;
    hipLaunchKernelGGL((prompt_attn_kernel<D, WAVES, SPLIT>), dim3(head_grid(g.Hkv, per_head)), dim3(C::THREADS), C::BYTES, st, g, per_head,
                       parts, Q, K, V, O, lse, partial);
    return hipGetLastError();
}

template <int D>
static hipError_t launch_prompt_d(const PromptGeom &g, const uint16_t *Q, const uint16_t *K, const uint16_t *V, uint16_t *O, float *lse,
                                  float *partial, hipStream_t st)
{
    const int parts = prompt_parts(g);
    if (parts == 1) return getenv("W4") ? launch_walk<D, 4, false>(g, 1, Q, K, V, O, lse, nullptr, st) : launch_walk<D, 8, false>(g, 1, Q, K, V, O, lse, nullptr, st);
    const hipError_t e = launch_walk<D, SPLIT_WAVES, true>(g, parts, Q, K, V, O, lse, partial, st);
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((prompt_join_kernel<D, 32 * SPLIT_WAVES>), dim3((unsigned)(((long long)g.Tq * g.Hq + 3) / 4)), dim3(256), 0, st, g,
                       (int)row_block_bound(g, 32 * SPLIT_WAVES), parts, partial, O, lse);
    return hipGetLastError();
}

hipError_t launch_prompt_attn(const PromptGeom &g, int D, const uint16_t *Q, const uint16_t *K, const uint16_t *V, uint16_t *O,
                              float *lse, void *ws, hipStream_t st)
{
    float *partial = static_cast<float *>(ws);
    return D == 64 ? launch_prompt_d<64>(g, Q, K, V, O, lse, partial, st) : launch_prompt_d<128>(g, Q, K, V, O, lse, partial, st);
}

}  // namespace adaspark
