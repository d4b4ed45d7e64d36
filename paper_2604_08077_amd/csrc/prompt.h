// Attention over packed prompts: sequences of different lengths one behind the other, queries and keys each with their own
// starts.  What its kernels (prompt_attn.hip, prompt_bwd.hip) share: the sequences as the device sees them, and the order of the work.
//
// Token i of a sequence's n queries attends the keys j <= i + m - n of its m (causal; otherwise all m): the last query sees the
// last key, so that a follow-up turn's queries attend the history before them.  A KV head's rows are numbered token by token,
// row = token * G + head of the group: neighbouring rows reach equally far, and a token's G heads lie one behind the other in memory.
#pragma once
#include "rowtile.h"

namespace adaspark {

struct PromptGeom {
    const int32_t *q_start, *k_start;     // [B + 1]
    int B, Tq, Tk, Hq, Hkv, G, causal;
    uint32_t gmul, gshift, gnear;         // division of a row number by G (token_of_row, token_of_near_row)
    long long qs, ks, vs;                 // elements from one token of Q, K, V to the next
};

inline PromptGeom make_prompt_geom(const adaspark_prompts &p, const int32_t *q_start, const int32_t *k_start, int causal)
{
    PromptGeom g;
    g.q_start = q_start;
    g.k_start = k_start;
    g.B = p.sequences;
    g.Tq = p.q_tokens;
    g.Tk = p.k_tokens;
    g.Hq = p.q_heads;
    g.Hkv = p.kv_heads;
    g.G = p.q_heads / p.kv_heads;
    // floor(x / G) for x < 2^31 is the high word of x * gmul, shifted by gshift: gmul = floor(2^(31 + s) / G) + 1 with
    // 2^(s - 1) < G <= 2^s is off by less than 1 / 2^31 of a quotient
    int s = 1;
    while ((1ll << s) < g.G) ++s;
    g.gmul = g.G == 1 ? 0u : (uint32_t)((1ull << (31 + s)) / (unsigned long long)g.G + 1);
    g.gshift = (uint32_t)s - 1;
    g.gnear = 65536u / (uint32_t)g.G + 1;
    g.causal = causal != 0;
    g.qs = p.q_stride ? p.q_stride : (long long)p.q_heads * p.head_dim;
    g.ks = p.k_stride ? p.k_stride : (long long)p.kv_heads * p.head_dim;
    g.vs = p.v_stride ? p.v_stride : (long long)p.kv_heads * p.head_dim;
    return g;
}

// The token of row `row` (0 <= row < 2^31), counted from the sequence's first.
__device__ __forceinline__ int token_of_row(const PromptGeom &g, int row)
{
    return g.G == 1 ? row : (int)(__umulhi((uint32_t)row, g.gmul) >> g.gshift);
}

// The same for 0 <= x < 64 + G, G <= PROMPT_MAX_GROUP: gnear * G is over 65536 by at most G, and x * G < 65536.
constexpr int PROMPT_MAX_GROUP = 128;
__device__ __forceinline__ uint32_t token_of_near_row(const PromptGeom &g, uint32_t x) { return __umul24(x, g.gnear) >> 16; }

// A sequence: its first query and key token, and how many.  Starts that do not fit the tensors are cut to them: whatever the arrays hold,
// nothing outside is touched.
struct PromptSeq {
    int q0, n, k0, m;
};
__device__ __forceinline__ PromptSeq prompt_seq(const PromptGeom &g, int s)
{
    PromptSeq p;
    p.q0 = min(max(g.q_start[s], 0), g.Tq);
    p.n = min(max(g.q_start[s + 1], p.q0), g.Tq) - p.q0;
    p.k0 = min(max(g.k_start[s], 0), g.Tk);
    p.m = min(max(g.k_start[s + 1], p.k0), g.Tk) - p.k0;
    return p;
}

__device__ __forceinline__ PromptSeq seq_uniform(const PromptSeq &p)
{
    return {__builtin_amdgcn_readfirstlane(p.q0), __builtin_amdgcn_readfirstlane(p.n), __builtin_amdgcn_readfirstlane(p.k0),
            __builtin_amdgcn_readfirstlane(p.m)};
}

// Inclusive scan over a wavefront's lanes, without LDS: within rows of 16, then each row's sum carried on.
__device__ __forceinline__ int wave_scan(int x)
{
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast 15 into rows 1 and 3, 31 into rows 2 and 3
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
    return x;
}
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_scan(x), 63); }

// What a workgroup does follows from lengths that only the device knows, so every wavefront finds its own work: the w-th block of
// all.  A wavefront's lanes hold the lengths of 512 sequences, eight each; beyond, sequences are taken 512 at a time.
// count(n, m, t): blocks of a sequence (n queries, m keys) with a walk of at least t tiles (t = 0: all of them); they are the
// sequence's last ones (rows) or first ones (keys), and are numbered from the longest.
constexpr int PROMPT_SEQS = 512, PROMPT_CHUNKS = PROMPT_SEQS / 64;
struct PromptLengths {
    int q0[PROMPT_CHUNKS], n[PROMPT_CHUNKS], k0[PROMPT_CHUNKS], m[PROMPT_CHUNKS];
    int s0, chunks;
};
__device__ __forceinline__ PromptLengths prompt_lengths(const PromptGeom &g, int s0)
{
    PromptLengths l;
    l.s0 = s0;
    l.chunks = (min(g.B - s0, PROMPT_SEQS) + 63) >> 6;
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int c = 0; c < PROMPT_CHUNKS; ++c) {
        PromptSeq p = {0, 0, 0, 0};
        if (c < l.chunks && s0 + 64 * c + lane < g.B) p = prompt_seq(g, s0 + 64 * c + lane);
        l.q0[c] = p.q0;
        l.n[c] = p.n;
        l.k0[c] = p.k0;
        l.m[c] = p.m;
    }
    return l;
}

struct PromptBlock {
    PromptSeq p;
    int seq, block;  // block: counted from the sequence's longest
};
template <typename Count>
__device__ __forceinline__ int blocks_from(const PromptLengths &l, int t, Count count)
{
    int x = 0;
#pragma unroll
    for (int c = 0; c < PROMPT_CHUNKS; ++c)
        if (c < l.chunks) x += count(l.n[c], l.m[c], t);
    return wave_total(x);
}
// The r-th of the blocks with a walk of t0 .. t1 - 1 tiles (t1 < 0: or more).
template <typename Count>
__device__ __forceinline__ PromptBlock nth_block(const PromptLengths &l, int r, int t0, int t1, Count count)
{
    PromptBlock b = {{0, 0, 0, 0}, -1, 0};
#pragma unroll
    for (int c = 0; c < PROMPT_CHUNKS; ++c) {
        if (c >= l.chunks || b.seq >= 0) continue;
        const int longer = t1 < 0 ? 0 : count(l.n[c], l.m[c], t1), mine = count(l.n[c], l.m[c], t0) - longer, incl = wave_scan(mine);
        const unsigned long long hit = __ballot(r < incl);
        if (hit != 0ull) {
            const int src = __builtin_amdgcn_readfirstlane(__ffsll(hit) - 1);
            b.seq = l.s0 + 64 * c + src;
            b.block = __builtin_amdgcn_readlane(longer, src) + r - __builtin_amdgcn_readlane(incl - mine, src);
            b.p = {__builtin_amdgcn_readlane(l.q0[c], src), __builtin_amdgcn_readlane(l.n[c], src), __builtin_amdgcn_readlane(l.k0[c], src),
                   __builtin_amdgcn_readlane(l.m[c], src)};
        }
        r -= __builtin_amdgcn_readlane(incl, 63);
    }
    return b;
}

// Blocks dealt out longest first -- a launch ends when its last workgroup does, and a long walk begun late is the tail --, lengths
// told apart in half octaves (0, 1, 2, 3, 4, 6, 8, 12, ... tiles).  The w-th block; seq -1: there is none.
__device__ __forceinline__ int walk_level(int b)  // the b-th length
{
    return b < 2 ? b : (2 + (b & 1)) << ((b - 2) >> 1);
}
template <typename Count>
__device__ __forceinline__ PromptBlock longest_first(const PromptGeom &g, int w, int most_tiles, Count count)
{
    int top = 1;
    while (walk_level(top) <= most_tiles) ++top;  // (no block is that long)
    for (int s0 = 0; s0 < g.B; s0 += PROMPT_SEQS) {
        const PromptLengths l = prompt_lengths(g, s0);
        const int all = blocks_from(l, 0, count);
        if (w >= all) {
            w -= all;
            continue;
        }
        int lo = 0, hi = top, above = 0;  // the highest level with more than w blocks, and the blocks beyond it
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1, x = blocks_from(l, walk_level(mid), count);
            if (x > w) lo = mid;
            else hi = mid, above = x;
        }
        return nth_block(l, w - above, walk_level(lo), hi == top ? -1 : walk_level(hi), count);
    }
    return {{0, 0, 0, 0}, -1, 0};
}

// Blocks of R rows of a sequence and KV head whose walk over the keys has at least t tiles of 64; the last blocks walk farthest.
template <int R>
__device__ __forceinline__ int row_blocks(int n, int m, int G, int causal, int t)
{
    const int nb = (int)(((long long)n * G + R - 1) / R);
    if (t == 0) return nb;
    const int keys = 64 * (t - 1);  // a walk of t tiles needs more than so many
    if (!causal) return m > keys ? nb : 0;
    const int first = max(0, keys - (m - n));  // the first token that reaches that far
    return first < n ? nb - first * G / R : 0;
}

// Workgroups per KV head that hold every block of R rows, however the tokens are shared out.
inline long long row_block_bound(const PromptGeom &g, int R) { return (long long)g.Tq * g.G / R + g.B; }
// A number of its own for block i of a sequence whose first query token is q0, below that bound (if the starts ascend).
__device__ __forceinline__ int row_block_id(const PromptGeom &g, int R, int s, int q0, int i)
{
    return (int)((long long)q0 * g.G / R) + s + i;
}

size_t prompt_workspace_bytes(const PromptGeom &g, int D);
hipError_t launch_prompt_attn(const PromptGeom &g, int D, const uint16_t *Q, const uint16_t *K, const uint16_t *V, uint16_t *O,
                              float *lse, void *ws, hipStream_t st);
size_t prompt_bwd_workspace_bytes(const PromptGeom &g, int D);
hipError_t launch_prompt_bwd(const PromptGeom &g, int D, const uint16_t *Q, const uint16_t *K, const uint16_t *V, const uint16_t *O,
                             const float *lse, const uint16_t *dO, uint16_t *dQ, uint16_t *dK, uint16_t *dV, void *ws, hipStream_t st);

}  // namespace adaspark
