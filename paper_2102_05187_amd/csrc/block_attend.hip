// Attention over the blocks that are chosen for each query: which kernel, with what sizes.
#include "block_attend.hpp"

namespace comet {

namespace {

struct Plan { int wide, mt, tokens, chunk, chunks, splits, words, entries; int64_t tiles, bytes; };

Plan plan_of(const comet_cache &c, int64_t N, int64_t Q, int64_t B, int64_t M, int64_t K) {
    Plan p{};
    const int64_t G = Q / c.heads, each = B > 0 ? (N + B - 1) / B : 1;
    p.wide = c.size <= 64 ? 64 : c.size <= 128 ? 128 : 256;
    // rows of a workgroup: as many tokens as a request has on average, as far as the registers go
    const int64_t rows = each * G;
    p.mt = rows <= 16 ? 1 : attend_tiles(p.wide);
    p.chunk = (int)(G < 16 * p.mt ? G : 16 * p.mt);
    p.chunks = (int)((G + p.chunk - 1) / p.chunk);
    int64_t tokens = p.chunks > 1 ? 1 : 16 * p.mt / p.chunk;
    if (tokens > 32) tokens = 32;
    if (tokens * K > kMostEntries) tokens = kMostEntries / K;
    if (tokens > each) tokens = each;
    p.tokens = (int)tokens;
    p.tiles = N / tokens + (B < N ? B : N);
    if (p.tiles > N) p.tiles = N;
    p.words = (int)((M + 31) / 32);
    p.entries = (int)(tokens * K < M ? tokens * K : M > K ? M : K);           // a single token's choices are kept as they are
    // places are shared out where there are few tiles: to 512 workgroups, 64 KB of keys and values each or more (1 token, 2 x 64 KB: 14 us in two
    // workgroups, 18 in four and joined; 71 tokens, 141 x 410 KB: 44 us in 141, 38 in 423)
    const int64_t items = p.tiles * c.heads * p.chunks, most = K * c.block * c.size * (c.type == COMET_F32 ? 8 : 4) / 65536;
    int64_t splits = items > 0 ? 512 / items : 1;
    if (splits > most) splits = most;
    if (splits > kSplits) splits = kSplits;
    p.splits = (int)(splits < 1 ? 1 : splits);
    p.bytes = p.splits > 1 ? items * p.splits * 16 * p.mt * (p.wide + 4) * 4 : 0;
    return p;
}

}  // namespace

int64_t block_attend_work(const comet_cache &c, int64_t N, int64_t Q, int64_t B, int64_t M, int64_t K) { return plan_of(c, N, Q, B, M, K).bytes; }

hipError_t block_attend(const comet_cache &c, const Queries &q, const int32_t *sel, int64_t K, double scale, void *out, float *lse, void *work, hipStream_t st) {
    const Plan p = plan_of(c, q.N, q.Q, q.B, q.M, K);
    const int e = c.type == COMET_F32 ? 4 : 2;
    // 256 MB and more (64 tokens, 537 MB: 91 us past the last cache, 102 through it); the next token reads much of the same again, and less stays there
    const bool once = q.N * c.heads * K * c.block * c.size * 2 * e >= int64_t(256) << 20;
    AttendArgs a{q, (const char *)c.keys, (const char *)c.values, c.blocks, (int)c.block, (int)c.heads, (int)c.size, (int)(q.Q / c.heads), {}, {}, sel, (int)K,
                 (float)(scale * 1.4426950408889634), out, lse, p.tokens, p.chunk, p.chunks, p.tiles, p.splits, p.words, p.entries, once, (float *)work};
    for (int i = 0; i < 3; ++i) a.key_stride[i] = c.key_stride[i] * e, a.value_stride[i] = c.value_stride[i] * e;
    if (c.type == COMET_F32) return attend_f32(a, p.wide, p.mt, st);
    if (c.type == COMET_BF16) return attend_bf16(a, p.wide, p.mt, st);
    return attend_f16(a, p.wide, p.mt, st);
}

}  // namespace comet
