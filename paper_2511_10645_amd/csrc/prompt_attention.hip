// Calls of the prompts' attention: checks, workspace and the launch (kernel: prompt_kernel.h).
#include "prompt_common.h"

namespace paro {

// Scratch for the parts of any call of so many heads' tiles (of the least size) or fewer: fewer tiles are split more often, but a call has fewer parts
// than kSplitBlocks and its tiles together, and one that splits has fewer tiles than kSplitBlocks.
static size_t prompt_scratch_bytes(const paro_kv_cache &c, int64_t tiles)
{
    const int64_t heads = tiles * c.kv_heads, parts = heads * kMaxSplits < kMostParts ? heads * kMaxSplits : kMostParts;
    const int pairs = c.head_dim == 256 ? Shapes<256>::Many::Pairs : Shapes<128>::Many::Pairs;
    return (sizeof(float) * pairs * (c.head_dim + 2) * (size_t)parts + 255) / 256 * 256;
}
constexpr int kLeastPairs = 32;                  // of a tile in any shape

}  // namespace paro

extern "C" size_t paro_workspace_exchange_bytes_prompt(const paro_kv_cache *cache, int32_t q_heads, int32_t T, int32_t batch)
{
    using namespace paro;
    if (!cache || cache->kv_heads <= 0 || q_heads <= 0 || q_heads % cache->kv_heads || T <= 0 || batch <= 0) return 0;
    const size_t counters = (size_t)prompt_tiles(T, q_heads / cache->kv_heads, batch, kLeastPairs) * cache->kv_heads * sizeof(uint32_t);
    return kWsPartialOff + (counters + 255) / 256 * 256;
}

extern "C" size_t paro_workspace_bytes_prompt(const paro_kv_cache *cache, int32_t q_heads, int32_t T, int32_t batch)
{
    using namespace paro;
    const size_t e = paro_workspace_exchange_bytes_prompt(cache, q_heads, T, batch);
    return e && cache->head_dim > 0 ? e + prompt_scratch_bytes(*cache, prompt_tiles(T, q_heads / cache->kv_heads, batch, kLeastPairs)) : 0;
}

extern "C" paro_status paro_prompt_attention(const paro_kv_cache *cache, const paro_half_t *Q, int64_t ldq, int32_t q_heads, int32_t T,
                                             const int32_t *starts, const int32_t *block_table, int64_t ld_table, int32_t table_width,
                                             const int32_t *lengths, int32_t batch, float scale, int32_t window, const paro_scores_t *scores,
                                             const int32_t *prefix, const int32_t *first, paro_half_t *O, int64_t ldo, float *lse, void *ws,
                                             size_t ws_bytes, void *stream)
{
    using namespace paro;
    if (const paro_status st = check_cache(cache); st != PARO_OK) return st;
    if (!Q || !O || !starts || !block_table || !lengths) return PARO_ERR_NULL;
    const paro_kv_cache &c = *cache;
    if (T <= 0 || batch <= 0 || q_heads <= 0 || q_heads % c.kv_heads || table_width <= 0 || window < 0) return PARO_ERR_SHAPE;
    if ((ld_table != 0 && ld_table < table_width) || O == Q) return PARO_ERR_SHAPE;
    PromptArgs a;
    if (const paro_status st = check_scores(scores, scale, a.scores); st != PARO_OK) return st;
    if (const paro_status st = check_rows(Q, ldq, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
    if (const paro_status st = check_rows(O, ldo, (int64_t)q_heads * c.head_dim); st != PARO_OK) return st;
    if (!aligned(starts, 4) || !aligned(block_table, 4) || !aligned(lengths, 4) || !aligned(prefix, 4) || !aligned(first, 4) || !aligned(lse, 4)) return PARO_ERR_ALIGN;
    // a sequence's tokens and pairs, and the blocks of a launch, are numbered with 32 bits
    const int64_t tokens = (int64_t)table_width * c.page;
    if (q_heads > 65535 || tokens > (int64_t)1 << 30 || T > 1 << 24 || (int64_t)T * q_heads > (int64_t)1 << 30) return PARO_ERR_UNSUPPORTED;
    const int64_t tiles = prompt_tiles(T, q_heads / c.kv_heads, batch, kLeastPairs);
    if (tiles * c.kv_heads > (int64_t)1 << 23) return PARO_ERR_UNSUPPORTED;       // a launch holds fewer than 2^32 threads: T q_heads + 32 kv_heads min(batch, T) <= 2^28 do
    if (!ws || ws_bytes < paro_workspace_bytes_prompt(cache, q_heads, T, batch)) return PARO_ERR_WORKSPACE;
    if (!aligned(ws, 256)) return PARO_ERR_ALIGN;

    a.k = (const uint8_t *)c.k; a.v = (const uint8_t *)c.v; a.ks = c.k_scale; a.vs = c.v_scale;
    a.q = (const _Float16 *)Q; a.starts = starts; a.table = block_table; a.lengths = lengths; a.prefix = prefix; a.first = first;
    a.o = (_Float16 *)O; a.lse = lse;
    a.arrived = (uint32_t *)((char *)ws + kWsPartialOff);
    a.partial = (float *)((char *)ws + (ws_bytes & ~(size_t)255) - prompt_scratch_bytes(c, tiles));
    a.ldq = ldq; a.ldo = ldo; a.ld_table = ld_table;
    a.page_log = log2_of(c.page); a.n_pages = c.n_pages; a.kv_heads = c.kv_heads; a.group = q_heads / c.kv_heads; a.width = table_width;
    a.batch = batch; a.window = window < 1 << 30 ? window : 0; a.T = T;
    a.scale = scale * kLog2e;
    hipStream_t s = (hipStream_t)stream;
    const bool scored = a.scores.cap > 0 || a.scores.slopes;
    hipError_t e;
    switch (kernel_format(c.format)) {
    case kFp16: e = launch_prompt_fp16(c.head_dim, scored, a, s); break;
    case kE4m3: e = launch_prompt_e4m3(c.head_dim, scored, a, s); break;
    default: e = launch_prompt_mxfp4(c.head_dim, scored, a, s); break;
    }
    return e == hipSuccess ? PARO_OK : PARO_ERR_HIP;
}
