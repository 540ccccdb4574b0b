// extern "C" entry points that append to the decoder cache, attend over it with
// chunks of new tokens, add up its slots' attention weights and evict from it:
// argument checks and launch planning.
#include <algorithm>
#include <cmath>

#include "prcr_internal.h"

namespace prcr {
namespace {

int64_t cache_capacity(const prcr_cache_desc* c) {
    return c->kind == PRCR_CACHE_CONTIGUOUS ? int64_t(c->max_slots) : int64_t(c->bt_stride) * c->block_size;
}

CacheView cache_view(const prcr_cache_desc* c, int layer) {
    CacheView v = {};
    v.k = static_cast<uint16_t*>(c->k) + int64_t(layer) * c->layer_stride;
    v.v = static_cast<uint16_t*>(c->v) + int64_t(layer) * c->layer_stride;
    v.seq_stride = c->seq_stride;
    v.layer_stride = c->layer_stride;
    v.block_stride = c->block_stride;
    v.slot_stride = c->slot_stride;
    v.capacity = cache_capacity(c);
    v.block_table = c->block_table;
    v.bt_stride = c->bt_stride;
    v.block_size = c->kind == PRCR_CACHE_PAGED ? c->block_size : 1;
    v.n_blocks = c->n_blocks;
    v.kind = c->kind;
    // m = ceil(2^(31 + k) / d) with 2^k >= d: m d exceeds 2^(31 + k) by less than 2^k,
    // so that n m >> (31 + k) is n / d for every n below 2^31
    int k = 0;
    while ((int64_t(1) << k) < v.block_size) ++k;
    v.div_mul = uint32_t(((uint64_t(1) << (31 + k)) + v.block_size - 1) / v.block_size);
    v.div_shift = 31 + k;
    return v;
}

// query heads that the attention kernels take
bool heads_ok(const prcr_rope_cfg* cfg, int32_t n_q_heads) {
    const int D = cfg->head_dim;
    return (D == 64 || D == 128 || D == 256) && n_q_heads >= cfg->n_kv_heads &&
           n_q_heads % cfg->n_kv_heads == 0 && n_q_heads / cfg->n_kv_heads <= 8 &&
           int64_t(n_q_heads) * D <= PRCR_DECODE_MAX_Q_ELEMS;
}

// How a chunk call is cut into CTAs, one to an SM: units of the rows of a tile and a KV
// head, and parts of the slots that a unit sees. (items: at most; the lengths are
// on the device.)
//
// few: sequences of up to 160 rows (tokens by heads of a group) on average, in units of 128
// rows, whose next tile's products do not wait for the last one's softmax, instead
// of 256, which read the keys once. 16 sequences of up to 8198 slots, 8 heads of groups of 4:
// of up to 6 tokens 64 us | 69, 24 tokens 77 | 87, 40 tokens 77 | 100, 64 tokens 79 |
// 101, 100 tokens 120 | 100. (Every sequence there has new tokens. One without counts too,
// as the offsets are on the device: it lowers the average, and its item's CTAs end at once.)
//
// splits: as many as give every SM a CTA. Few rows are bound by the keys' and values'
// bytes, and their partials are small: where that is below 4, it is rounded up, and a
// second, partial wave evens out lengths that differ (sequences of 8 heads as above: 5 of
// them 31 us up | 34 down, 8 40 | 48, 12 62 | 72, 16 64 | 75; but 2 31 | 26, 4 35 | 31).
// With many rows the partials cost more than the idle SMs (D = 256: up 183, down 178).
// Up to 4 tiles of slots, or 12 with many rows, are not split: the kernel that joins the
// parts costs what they save (few rows, us split | not: 2 tiles 10.5 | 8.4, 4 10.9 | 10.1, 6
// 10.4 | 11.8; many: a prompt of 200 tokens 18.8 | 13.1, of 500 24 | 16, 300 tokens over 9
// tiles 24.5 | 22.3, 400 over 13 29.2 | 26.7, 256 over 17 25.8 | 31.3).
struct ChunkSplit {
    int64_t items, splits;
    bool few;
};
ChunkSplit chunk_split(const prcr_rope_cfg* cfg, int64_t n_seqs, int64_t n_q_heads, int64_t total_q, int64_t max_len, int sms) {
    const int64_t group = n_q_heads / cfg->n_kv_heads, seqs = std::min(n_seqs, total_q);
    ChunkSplit c;
    c.few = total_q * group <= 160 * seqs;
    c.items = total_q * group / chunk_rows(cfg->head_dim, c.few) + seqs;
    const int64_t units = c.items * cfg->n_kv_heads, tiles = std::max<int64_t>(1, (max_len + 127) / 128);
    const int64_t down = sms / units;
    c.splits = tiles <= (c.few ? 4 : 12) ? 1 : std::max<int64_t>(1, std::min(tiles, c.few && down < 4 ? (sms + units - 1) / units : down));
    return c;
}

size_t chunk_bytes(const prcr_rope_cfg* cfg, int64_t n_q_heads, int64_t rows) {  // of partials
    return size_t(rows) * n_q_heads * (cfg->head_dim + 2) * sizeof(float);
}

// The most that the partials of a call with up to total_q tokens and max_len slots
// take: for every number of splits, the most tokens that get so many (of one sequence;
// more of them have more items).
size_t chunk_most_bytes(const prcr_rope_cfg* cfg, int64_t n_q_heads, int64_t total_q, int64_t max_len, int sms) {
    const int64_t group = n_q_heads / cfg->n_kv_heads, rows = chunk_rows(cfg->head_dim, false), tiles = (max_len + 127) / 128;
    int64_t most = 0;
    for (int64_t s = 2; s <= std::min<int64_t>(tiles, sms); ++s) {
        const int64_t items = (sms - 1) / (s - 1) / cfg->n_kv_heads;  // (sms + units - 1) / units >= s
        if (items < 1) break;
        most = std::max(most, s * std::min(total_q, (items * rows - 1) / group));
    }
    return chunk_bytes(cfg, n_q_heads, most);
}

// CTAs of a cluster that takes one (sequence, layer, KV head), and its slots per
// CTA: the fewest whose logits leave room for two CTAs per SM (or, for long
// sequences, for one); more where there are SMs left for them and each keeps a tile of 16
// slots for every warp. 0 where no cluster's shared memory holds them.
int weights_cluster(const prcr_rope_cfg* cfg, int64_t n_seqs, int64_t n_q_heads, int64_t max_len, int sms, int* slots) {
    const int64_t units = n_seqs * cfg->n_layers * cfg->n_kv_heads;
    const int group = int(n_q_heads / cfg->n_kv_heads);
    auto per = [&](int c) { return ((max_len + 15) / 16 + c - 1) / c * 16; };
    for (const size_t room : {size_t(104) * 1024, size_t(208) * 1024}) {
        for (int c = 1; c <= 8; c *= 2) {
            if (max_len > (int64_t(1) << 20) || weights_smem(cfg->head_dim, group, int(per(c))) > room) continue;
            while (c < 8 && units * c * 2 <= 2 * int64_t(sms) && per(2 * c) >= 128) c *= 2;
            *slots = int(per(c));
            return c;
        }
    }
    return 0;
}

size_t weights_bytes(const prcr_rope_cfg* cfg, int64_t n_seqs, int64_t n_q_heads, int64_t max_len) {
    int slots;
    if (weights_cluster(cfg, n_seqs, n_q_heads, max_len, 1, &slots)) return 0;
    return size_t(n_seqs) * cfg->n_layers * n_q_heads * max_len * sizeof(float);
}

// CTAs that share the rows of one (sequence, layer, KV head), each with some of the
// dims: more than one while there are SMs left for them and a row's part is 64 bytes
// at least. (Head_dim 128, half of 8000 slots, 16 units: 1 CTA 75 us, 4 of 64 bytes 40, 8
// of 32 bytes 47; 144 units of 4096 to 1024: 1 CTA 46, 2 of 128 bytes 37.)
int evict_cluster(const prcr_rope_cfg* cfg, int64_t n_seqs, int sms) {
    const int64_t units = n_seqs * cfg->n_layers * cfg->n_kv_heads;
    int c = 1;
    while (c < 8 && cfg->head_dim % (64 * c) == 0 && units * c * 2 <= 2 * int64_t(sms)) c *= 2;
    return c;
}

// Whether two arrays of n lengths share an entry.
bool overlap(const int32_t* a, const int32_t* b, int64_t n) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return (x < y ? y - x : x - y) < uintptr_t(n) * sizeof(int32_t);
}

int status_of(cudaError_t e) { return e == cudaSuccess ? PRCR_OK : PRCR_ECUDA; }

}  // namespace
}  // namespace prcr

using namespace prcr;

extern "C" {

int prcr_append_kv(const prcr_rope_cfg* cfg, const prcr_cache_desc* cache, int32_t n_seqs, int32_t layer_begin,
                   int32_t n_layers, const void* k_src, const void* v_src, int64_t src_layer_stride,
                   int64_t src_token_stride, const int32_t* coords, const int32_t* tok_off, int32_t total,
                   const int32_t* cache_len_in, int32_t* cache_len_out, uint32_t* status, void* stream) {
    int rc = check_cfg(cfg);
    if (rc) return rc;
    if ((rc = check_cache(cfg, cache))) return rc;
    if (n_seqs < 0 || n_seqs > cache->n_seqs || layer_begin < 0 || n_layers < 1 ||
        layer_begin + int64_t(n_layers) > cfg->n_layers || total < 0)
        return PRCR_EINVAL;
    if (n_seqs == 0) return PRCR_OK;
    const int64_t row = int64_t(cfg->n_kv_heads) * cfg->head_dim;
    if (!tok_off || !cache_len_in || !cache_len_out || !status || overlap(cache_len_in, cache_len_out, n_seqs))
        return PRCR_EINVAL;
    if (total > 0 && (!k_src || !v_src || !coords || src_token_stride < row || src_layer_stride < 0))
        return PRCR_EINVAL;
    if (!aligned4(tok_off) || !aligned4(cache_len_in) || !aligned4(cache_len_out) || !aligned4(status))
        return PRCR_EALIGN;
    if (total > 0 && (!aligned16(k_src) || !aligned16(v_src) || !mult8(src_layer_stride) ||
                      !mult8(src_token_stride) || !aligned4(coords)))
        return PRCR_EALIGN;
    AppendArgs a = {};
    a.cache = cache_view(cache, layer_begin);
    a.src_k = static_cast<const uint16_t*>(k_src);
    a.src_v = static_cast<const uint16_t*>(v_src);
    a.src_layer_stride = src_layer_stride;
    a.src_token_stride = src_token_stride;
    a.coords = coords;
    a.tok_off = tok_off;
    a.len_in = cache_len_in;
    a.len_out = cache_len_out;
    a.status = status;
    a.n_seqs = n_seqs;
    a.total = total;
    a.n_layers = n_layers;
    a.head_dim = cfg->head_dim;
    a.layout = cfg->layout;
    a.sec_t = cfg->sections[0];
    a.sec_h = cfg->sections[1];
    a.sec_w = cfg->sections[2];
    copy_turn_freq(cfg, a.turn_freq);
    const int lanes = cfg->n_kv_heads * (cfg->head_dim / 16);
    const int T = std::max(1, kRebindTargetThreads / lanes);
    const int block = T * lanes;
    const size_t smem = size_t(T) * (cfg->head_dim * sizeof(float) + sizeof(int64_t));
    a.lanes = lanes;
    a.tok_per_cta = T;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PRCR_ECUDA;
    const int64_t tiles = std::max<int64_t>(1, (int64_t(total) + T - 1) / T);
    const int64_t slots = int64_t(sm_count(dev)) * blocks_per_sm(dev, block, smem, kAppend);
    const int G = stream_layers_per_cta(tiles, n_layers, slots, 8);
    a.layers_per_cta = G;
    const dim3 grid(unsigned(tiles), unsigned((n_layers + G - 1) / G), 1);
    return status_of(launch_append(a, grid, block, smem, static_cast<cudaStream_t>(stream)));
}

size_t prcr_chunk_workspace_size(const prcr_rope_cfg* cfg, int32_t n_seqs, int32_t n_q_heads, int32_t total_q,
                                 int64_t max_len) {
    if (check_cfg(cfg) || n_seqs < 1 || total_q < 1 || max_len < 1 || !heads_ok(cfg, n_q_heads)) return 0;
    int dev = 0, sms = 1;
    if (cudaGetDevice(&dev) == cudaSuccess) sms = sm_count(dev);
    return chunk_most_bytes(cfg, n_q_heads, total_q, max_len, sms);
}

int prcr_chunk_attention(const prcr_rope_cfg* cfg, const prcr_cache_desc* cache, int32_t n_seqs, int32_t layer,
                         int32_t n_q_heads, const void* q, int64_t q_token_stride, const int32_t* coords,
                         const int32_t* q_off, int32_t total_q, const int32_t* seq_len, int64_t max_len, void* out,
                         int64_t out_token_stride, uint32_t* status, void* workspace, size_t workspace_bytes,
                         void* stream) {
    int rc = check_cfg(cfg);
    if (rc) return rc;
    if ((rc = check_cache(cfg, cache))) return rc;
    if (!heads_ok(cfg, n_q_heads) || n_seqs < 0 || n_seqs > cache->n_seqs || layer < 0 || layer >= cfg->n_layers ||
        total_q < 0 || max_len < 0 || max_len > PRCR_CACHE_MAX_LEN || max_len > cache_capacity(cache))
        return PRCR_EINVAL;
    if (n_seqs == 0 || total_q == 0) return PRCR_OK;
    const int64_t row = int64_t(n_q_heads) * cfg->head_dim;
    if (!q || !coords || !q_off || !seq_len || !out || !status || q == out || q_token_stride < row || out_token_stride < row)
        return PRCR_EINVAL;
    if (!aligned16(q) || !aligned16(out) || !mult8(q_token_stride) || !mult8(out_token_stride) || !aligned4(coords) ||
        !aligned4(q_off) || !aligned4(seq_len) || !aligned4(status))
        return PRCR_EALIGN;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PRCR_ECUDA;
    const ChunkSplit split = chunk_split(cfg, n_seqs, n_q_heads, total_q, max_len, sm_count(dev));
    if (int64_t(total_q) * n_q_heads > INT32_MAX || split.items * cfg->n_kv_heads * split.splits > INT32_MAX)
        return PRCR_EINVAL;  // rows, grid x
    ChunkArgs a = {};
    if (split.splits > 1) {
        const int64_t rows = int64_t(total_q) * split.splits;
        if (!workspace || workspace_bytes < chunk_bytes(cfg, n_q_heads, rows)) return PRCR_EWORKSPACE;
        if (!aligned16(workspace)) return PRCR_EALIGN;
        a.partial = static_cast<float*>(workspace);
        a.partial_ml = reinterpret_cast<float2*>(a.partial + rows * n_q_heads * cfg->head_dim);
    }
    a.items = int32_t(split.items);
    a.splits = int32_t(split.splits);
    a.few = split.few;
    a.cache = cache_view(cache, layer);
    a.q = static_cast<const uint16_t*>(q);
    a.q_stride = q_token_stride;
    a.coords = coords;
    a.q_off = q_off;
    a.seq_len = seq_len;
    a.out = static_cast<uint16_t*>(out);
    a.out_stride = out_token_stride;
    a.status = status;
    a.top = int32_t(max_len);  // (at most the capacity)
    a.n_seqs = n_seqs;
    a.total_q = total_q;
    a.n_kv_heads = cfg->n_kv_heads;
    a.group = n_q_heads / cfg->n_kv_heads;
    a.head_dim = cfg->head_dim;
    a.layout = cfg->layout;
    a.sec_t = cfg->sections[0];
    a.sec_h = cfg->sections[1];
    a.sec_w = cfg->sections[2];
    a.scale_log2 = float(1.4426950408889634 / std::sqrt(double(cfg->head_dim)));
    copy_turn_freq(cfg, a.turn_freq);
    return status_of(launch_chunk(a, static_cast<cudaStream_t>(stream)));
}

size_t prcr_weights_workspace_size(const prcr_rope_cfg* cfg, int32_t n_seqs, int32_t n_q_heads, int64_t max_len) {
    if (check_cfg(cfg) || n_seqs < 1 || max_len < 1 || !heads_ok(cfg, n_q_heads)) return 0;
    return weights_bytes(cfg, n_seqs, n_q_heads, max_len);
}

int prcr_accumulate_weights(const prcr_rope_cfg* cfg, const prcr_cache_desc* cache, int32_t n_seqs, int32_t n_q_heads,
                            const void* q, const int64_t* q_pos, const int32_t* seq_len, int64_t max_len,
                            float* score, int64_t score_stride, float decay, uint32_t* status, void* workspace,
                            size_t workspace_size, void* stream) {
    int rc = check_cfg(cfg);
    if (rc) return rc;
    if ((rc = check_cache(cfg, cache))) return rc;
    if (!heads_ok(cfg, n_q_heads) || n_seqs < 0 || n_seqs > cache->n_seqs || max_len < 0 ||
        max_len > PRCR_CACHE_MAX_LEN || max_len > cache_capacity(cache) || score_stride < max_len ||
        !std::isfinite(decay))
        return PRCR_EINVAL;
    if (n_seqs == 0 || max_len == 0) return PRCR_OK;
    if (n_seqs > 65535 || int64_t(cfg->n_layers) * cfg->n_kv_heads > 65535) return PRCR_EINVAL;  // grid z and y
    if (!q || !q_pos || !seq_len || !score || !status) return PRCR_EINVAL;
    if (!aligned16(q) || !aligned8(q_pos) || !aligned4(seq_len) || !aligned4(score) || !aligned4(status))
        return PRCR_EALIGN;
    const size_t need = weights_bytes(cfg, n_seqs, n_q_heads, max_len);
    if (need > 0 && (!workspace || workspace_size < need)) return PRCR_EWORKSPACE;
    if (need > 0 && !aligned16(workspace)) return PRCR_EALIGN;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PRCR_ECUDA;
    WeightsArgs a = {};
    a.cluster = weights_cluster(cfg, n_seqs, n_q_heads, max_len, sm_count(dev), &a.slots_per_cta);
    if (a.cluster * int64_t(n_seqs) * cfg->n_layers * cfg->n_kv_heads > INT32_MAX) return PRCR_EINVAL;  // grid x
    a.cache = cache_view(cache, 0);
    a.q = static_cast<const uint16_t*>(q);
    a.q_pos = q_pos;
    a.seq_len = seq_len;
    a.score = score;
    a.logits = static_cast<float*>(workspace);
    a.status = status;
    a.max_len = max_len;
    a.score_stride = score_stride;
    a.decay = decay;
    a.n_seqs = n_seqs;
    a.n_layers = cfg->n_layers;
    a.n_kv_heads = cfg->n_kv_heads;
    a.group = n_q_heads / cfg->n_kv_heads;
    a.head_dim = cfg->head_dim;
    a.scale_log2 = float(1.4426950408889634 / std::sqrt(double(cfg->head_dim)));
    copy_turn_freq(cfg, a.turn_freq);
    return status_of(launch_weights(a, static_cast<cudaStream_t>(stream)));
}

int prcr_evict(const prcr_rope_cfg* cfg, const prcr_cache_desc* cache, const prcr_cache_desc* dst, int32_t n_seqs,
               const int32_t* seq_len, int64_t max_len, int32_t budget, int32_t n_sink, int32_t n_recent,
               const float* score, float* score_out, int64_t score_stride, int32_t* keep_out, int32_t* seq_len_out,
               uint32_t* status, void* stream) {
    int rc = check_cfg(cfg);
    if (rc) return rc;
    if ((rc = check_cache(cfg, cache))) return rc;
    if (dst && (rc = check_cache(cfg, dst))) return rc;
    if (n_seqs < 0 || n_seqs > cache->n_seqs || (dst && n_seqs > dst->n_seqs) || max_len < 0 ||
        max_len > PRCR_CACHE_MAX_LEN || max_len > cache_capacity(cache) || score_stride < max_len || budget < 1 ||
        budget > PRCR_CACHE_MAX_LEN || n_sink < 0 || n_recent < 0 || int64_t(n_sink) + n_recent > budget)
        return PRCR_EINVAL;
    if (dst && (dst->k == cache->k || dst->v == cache->v) &&  // (another part of a pool is another table's)
        (dst->kind == PRCR_CACHE_CONTIGUOUS || dst->block_table == cache->block_table))
        return PRCR_EINVAL;
    if (n_seqs == 0) return PRCR_OK;
    if (n_seqs > 65535 || cfg->n_layers > 65535) return PRCR_EINVAL;  // grid z and y
    if (!seq_len || !score || !score_out || !keep_out || !seq_len_out || !status ||
        overlap(seq_len, seq_len_out, n_seqs))
        return PRCR_EINVAL;
    if (!aligned4(seq_len) || !aligned4(score) || !aligned4(score_out) || !aligned4(keep_out) ||
        !aligned4(seq_len_out) || !aligned4(status))
        return PRCR_EALIGN;
    EvictArgs a = {};
    a.src = cache_view(cache, 0);
    a.dst = dst ? cache_view(dst, 0) : a.src;
    a.seq_len = seq_len;
    a.len_out = seq_len_out;
    a.score = score;
    a.score_out = score_out;
    a.keep = keep_out;
    a.status = status;
    a.max_len = max_len;
    a.score_stride = score_stride;
    a.budget = budget;
    a.n_sink = n_sink;
    a.n_recent = n_recent;
    a.n_layers = cfg->n_layers;
    a.n_kv_heads = cfg->n_kv_heads;
    a.head_dim = cfg->head_dim;
    a.in_place = dst == nullptr;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PRCR_ECUDA;
    a.cluster = evict_cluster(cfg, n_seqs, sm_count(dev));
    return status_of(launch_evict(a, n_seqs, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
