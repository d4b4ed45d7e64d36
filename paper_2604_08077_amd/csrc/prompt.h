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
    uint32_t gmul, gshift;                // division of a row number by G (token_of_row)
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

// Work is dealt out longest first: a launch ends when its last workgroup does, and a long walk begun late is the tail.  The
// lengths are on the device, so every wavefront finds its own: the w-th longest block, lengths told apart in half octaves
// (0, 1, 2, 3, 4, 6, 8, 12, ... tiles).  `count(n, m, t)`: blocks of a sequence (n queries, m keys) with a walk of at least t tiles, t = 0: all; they are
// the sequence's last ones (`from_end`) or first ones.  Sequences beyond 512 are dealt out 512 at a time.
constexpr int PROMPT_SEQS = 512;
__device__ __forceinline__ int walk_level(int b)  // the b-th length
{
    return b < 2 ? b : (2 + (b & 1)) << ((b - 2) >> 1);
}

__device__ __forceinline__ int wave_total(int x)
{
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d, 64);
    return __builtin_amdgcn_readfirstlane(x);
}

// The w-th block: its sequence, and its number among the sequence's blocks counted from the longest.  false: there is none.
template <typename Count>
__device__ __forceinline__ bool prompt_block(const PromptGeom &g, int w, int most_tiles, Count count, int &seq, int &block)
{
    const int lane = threadIdx.x & 63;
    for (int s0 = 0; s0 < g.B; s0 += PROMPT_SEQS) {
        const int chunks = (min(g.B - s0, PROMPT_SEQS) + 63) >> 6;
        int n[PROMPT_SEQS / 64], m[PROMPT_SEQS / 64];
#pragma unroll
        for (int c = 0; c < PROMPT_SEQS / 64; ++c) {
            n[c] = m[c] = 0;
            if (c < chunks && s0 + 64 * c + lane < g.B) {
                const PromptSeq p = prompt_seq(g, s0 + 64 * c + lane);
                n[c] = p.n;
                m[c] = p.m;
            }
        }
        auto total = [&](int t) -> int {
            int x = 0;
#pragma unroll
            for (int c = 0; c < PROMPT_SEQS / 64; ++c)
                if (c < chunks) x += count(n[c], m[c], t);
            return wave_total(x);
        };
        const int all = total(0);
        if (w >= all) {
            w -= all;
            continue;
        }
        // the highest level with more than w blocks
        int lo = 0, hi = 1;
        while (walk_level(hi) <= most_tiles) ++hi;  // (no block is that long)
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (total(walk_level(mid)) > w) lo = mid;
            else hi = mid;
        }
        const int above = walk_level(hi) <= most_tiles ? total(walk_level(hi)) : 0;
        int r = w - above;
        for (int c = 0; c < chunks; ++c) {
            int nn = 0, mm = 0;
#pragma unroll
            for (int k = 0; k < PROMPT_SEQS / 64; ++k)
                if (k == c) nn = n[k], mm = m[k];
            const int longer = walk_level(hi) <= most_tiles ? count(nn, mm, walk_level(hi)) : 0;
            const int mine = count(nn, mm, walk_level(lo)) - longer;
            int incl = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const int up = __shfl_up(incl, d, 64);
                if (lane >= d) incl += up;
            }
            const unsigned long long b = __ballot(r < incl);
            if (b != 0ull) {
                const int src = __builtin_amdgcn_readfirstlane(__ffsll(b) - 1);
                seq = s0 + 64 * c + src;
                block = __builtin_amdgcn_readlane(longer, src) + r - (__builtin_amdgcn_readlane(incl, src) - __builtin_amdgcn_readlane(mine, src));
                return true;
            }
            r -= __builtin_amdgcn_readlane(incl, 63);
        }
        return false;  // (not reached: the counts add up)
    }
    return false;
}

// Blocks of R rows of a sequence and KV head whose walk over the keys has at least t tiles of 64; the last blocks walk farthest.
template <int R>
__device__ __forceinline__ int row_blocks(int n, int m, int G, int causal, int t)
{
    const long long rows = (long long)n * G;
    const int nb = (int)((rows + R - 1) / R);
    if (t == 0) return nb;
    const long long keys = 64ll * (t - 1);  // a walk of t tiles needs more than so many
    if (!causal) return m > keys ? nb : 0;
    const long long first = max(0ll, keys - (m - n)) * G;  // the first row that reaches that far
    return first < rows ? nb - (int)(first / R) : 0;
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
