// extern "C" entry points of the quantised cache: argument checks and launch
// planning.
#include <algorithm>
#include <cmath>

#include "prcr_internal.h"

namespace prcr {
namespace {

int code_bytes(const prcr_qcache_desc* c, int head_dim) { return c->format == PRCR_QFMT_E4M3 ? head_dim : head_dim / 2; }
int scale_count(const prcr_qcache_desc* c, int head_dim) { return c->format == PRCR_QFMT_E4M3 ? 1 : head_dim / 32; }

int64_t qcache_capacity(const prcr_qcache_desc* c) {
    return c->kind == PRCR_CACHE_CONTIGUOUS ? int64_t(c->max_slots) : int64_t(c->bt_stride) * c->block_size;
}

bool aligned_to(const void* p, int64_t n) { return reinterpret_cast<uintptr_t>(p) % uintptr_t(n) == 0; }

int check_qcache(const prcr_rope_cfg* cfg, const prcr_qcache_desc* c) {
    if (!c || !c->k || !c->v || !c->k_scale || !c->v_scale || c->reserved != 0) return PRCR_EINVAL;
    const int D = cfg->head_dim;
    if (c->format != PRCR_QFMT_E4M3 && c->format != PRCR_QFMT_E2M1) return PRCR_EINVAL;
    if (c->format == PRCR_QFMT_E2M1 && D != 64 && D != 128 && D != 256) return PRCR_EINVAL;
    const int64_t row = int64_t(cfg->n_kv_heads) * code_bytes(c, D), n = scale_count(c, D), scales = cfg->n_kv_heads * n;
    if (c->slot_stride < row || c->scale_slot_stride < scales || c->layer_stride < 0 || c->scale_layer_stride < 0 || c->n_seqs < 1)
        return PRCR_EINVAL;
    auto strides_ok = [&](int64_t codes, int64_t s) { return codes % 16 == 0 && s % n == 0; };
    if (!aligned16(c->k) || !aligned16(c->v) || !aligned_to(c->k_scale, n) || !aligned_to(c->v_scale, n) ||
        !strides_ok(c->slot_stride, c->scale_slot_stride) || !strides_ok(c->layer_stride, c->scale_layer_stride))
        return PRCR_EALIGN;
    if (c->kind == PRCR_CACHE_CONTIGUOUS) {
        if (c->max_slots < 0 || c->seq_stride < 0 || c->scale_seq_stride < 0) return PRCR_EINVAL;
        if (!strides_ok(c->seq_stride, c->scale_seq_stride)) return PRCR_EALIGN;
    } else if (c->kind == PRCR_CACHE_PAGED) {
        if (!c->block_table || c->block_size < 1 || c->bt_stride < 0 || c->n_blocks < 0 || c->block_stride < 0 || c->scale_block_stride < 0)
            return PRCR_EINVAL;
        if (!aligned4(c->block_table) || !strides_ok(c->block_stride, c->scale_block_stride)) return PRCR_EALIGN;
    } else {
        return PRCR_EINVAL;
    }
    return PRCR_OK;
}

QCacheView qcache_view(const prcr_qcache_desc* c, int layer) {
    QCacheView v = {};
    v.k = static_cast<uint8_t*>(c->k) + layer * c->layer_stride;
    v.v = static_cast<uint8_t*>(c->v) + layer * c->layer_stride;
    v.k_scale = c->k_scale + layer * c->scale_layer_stride;
    v.v_scale = c->v_scale + layer * c->scale_layer_stride;
    v.seq_stride = c->seq_stride;
    v.layer_stride = c->layer_stride;
    v.block_stride = c->block_stride;
    v.slot_stride = c->slot_stride;
    v.scale_seq_stride = c->scale_seq_stride;
    v.scale_layer_stride = c->scale_layer_stride;
    v.scale_block_stride = c->scale_block_stride;
    v.scale_slot_stride = c->scale_slot_stride;
    v.capacity = qcache_capacity(c);
    v.block_table = c->block_table;
    v.bt_stride = c->bt_stride;
    v.block_size = c->kind == PRCR_CACHE_PAGED ? c->block_size : 1;
    v.n_blocks = c->n_blocks;
    v.kind = c->kind;
    fill_div(v.block_size, &v.div_mul, &v.div_shift);
    return v;
}

int power_of_two(int n) {
    int p = 1;
    while (p < n) p *= 2;
    return p;
}

// Layers that a CTA walks: as few as make at most `ctas` CTAs, else `most`, evened out; as
// many as the launch grid needs. Measured, us. Casts, 8 CTAs an SM, else 9 layers: E4M3, 36 layers of 16 sequences' up to 1024
// slots written in 341, read in 343 (one layer 531, 412; 36 layers 355, 345); E2M1, one sequence's 933 slots 35, 35 (of 2 CTAs
// an SM 37, 40; of 32 43, 42). Appends, 3 an SM, else 16: 28 layers of six prompts 158 (four layers 197, all 160); 24 layers
// of two prompts' pieces 26.5 (of one CTA an SM the same, of 12 30.8).
int layers_per_cta(int64_t tiles, int n_layers, int64_t ctas, int most) {
    int g = 1;
    while (g < most && tiles * ((n_layers + g - 1) / g) > ctas) ++g;
    const int groups = std::min(65535, (n_layers + g - 1) / g);
    return (n_layers + groups - 1) / groups;
}

// How a decode step's warps take its tiles: teams of warps with the same slots of as many neighbouring KV heads (four, or two
// that divide the heads; rows of less than 128 bytes by two even where that leaves a warp idle, since lines are fetched whole), as
// many teams as the SMs hold, unless there are fewer tiles.
struct DecodeQuantTeams {
    int team, head_sets;
    int64_t teams;
};
DecodeQuantTeams decode_quant_teams(int format, int head_dim, int n_kv_heads, int64_t seq_layers, int64_t max_len, int sms) {
    DecodeQuantTeams s;
    const int row = format == PRCR_QFMT_E4M3 ? head_dim : head_dim / 2;
    s.team = n_kv_heads % 4 == 0 ? 4 : n_kv_heads % 2 == 0 || (row < 128 && n_kv_heads > 1) ? 2 : 1;
    s.head_sets = (n_kv_heads + s.team - 1) / s.team;
    const int64_t tile = decode_quant_tile(format, head_dim), tiles = std::max<int64_t>(1, (max_len + tile - 1) / tile);
    const int64_t units = seq_layers * s.head_sets, most = int64_t(sms) * decode_quant_warps(head_dim) / s.team;
    s.teams = units > most / tiles ? most : units * tiles;
    return s;
}

size_t decode_quant_parts(const DecodeQuantTeams& s, int group, int head_dim) {
    return align256(size_t(s.teams) * 2 * s.team * group * (head_dim + 2) * sizeof(float));
}

// Fills what both directions share; *go is false where nothing is to be done.
int cast_setup(const prcr_rope_cfg* cfg, const prcr_cache_desc* wide, int32_t wide_layer, const prcr_qcache_desc* few, int32_t few_layer,
               int32_t n_layers, int32_t n_seqs, const int32_t* src_begin, const int32_t* dst_begin, const int32_t* count,
               int32_t max_count, uint32_t* status, bool quantise, CastArgs* a, dim3* grid, bool* go) {
    *go = false;
    int rc = check_cfg(cfg);
    if (rc) return rc;
    if ((rc = check_cache(cfg, wide))) return rc;
    if ((rc = check_qcache(cfg, few))) return rc;
    if (n_seqs < 0 || n_seqs > wide->n_seqs || n_seqs > few->n_seqs || n_seqs > 65535 || wide_layer < 0 || few_layer < 0 || n_layers < 1 ||
        wide_layer + int64_t(n_layers) > cfg->n_layers || few_layer + int64_t(n_layers) > cfg->n_layers || max_count < 0 ||
        max_count > PRCR_CACHE_MAX_LEN)
        return PRCR_EINVAL;
    if (n_seqs == 0) return PRCR_OK;
    if (!src_begin || !dst_begin || !count || !status) return PRCR_EINVAL;
    if (!aligned4(src_begin) || !aligned4(dst_begin) || !aligned4(count) || !aligned4(status)) return PRCR_EALIGN;
    *a = CastArgs{};
    a->wide = cache_view(wide, wide_layer);
    a->few = qcache_view(few, few_layer);
    a->src_begin = src_begin;
    a->dst_begin = dst_begin;
    a->count = count;
    a->status = status;
    a->max_count = max_count;
    a->n_layers = n_layers;
    a->head_dim = cfg->head_dim;
    a->format = few->format;
    a->n_scales = scale_count(few, cfg->head_dim);
    a->pad = quantise ? power_of_two(cfg->head_dim / 8) : cfg->head_dim / 8;
    a->lanes = cfg->n_kv_heads * a->pad;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PRCR_ECUDA;
    // A CTA takes two (reading: four) tokens of a thread's, or as much in few layers as make eight CTAs an SM, so that its look-ups
    // weigh less (one layer of four prompts of up to 16,384 slots, E4M3: written in 78 | 64 us, read in 62 | 56).
    int units = quantise ? 512 : 1024;
    const int most = units * 4 / n_layers;
    while (units * 2 <= most && int64_t(n_seqs) * max_count * a->lanes / (units * 2) >= int64_t(sm_count(dev)) * 8) units *= 2;
    a->tok_per_cta = std::max(1, std::min({64, int(max_count), units / a->lanes}));
    a->units = a->tok_per_cta * a->lanes;
    if (quantise) a->units = (a->units + 31) / 32 * 32;
    const int64_t tiles = std::max<int64_t>(1, (int64_t(max_count) + a->tok_per_cta - 1) / a->tok_per_cta);
    a->layers_per_cta = layers_per_cta(tiles * n_seqs, n_layers, int64_t(sm_count(dev)) * 8, 9);
    *grid = dim3(unsigned(tiles), unsigned((n_layers + a->layers_per_cta - 1) / a->layers_per_cta), unsigned(n_seqs));
    *go = true;
    return PRCR_OK;
}

int status_of(cudaError_t e) { return e == cudaSuccess ? PRCR_OK : PRCR_ECUDA; }

}  // namespace
}  // namespace prcr

using namespace prcr;

extern "C" {

int prcr_append_kv_quant(const prcr_rope_cfg* cfg, const prcr_qcache_desc* cache, int32_t n_seqs, int32_t layer_begin, int32_t n_layers,
                         const void* k_src, const void* v_src, int64_t src_layer_stride, int64_t src_token_stride, const int32_t* coords,
                         const int32_t* tok_off, int32_t total, const int32_t* cache_len_in, int32_t* cache_len_out, uint32_t* status,
                         void* stream) {
    int rc = check_cfg(cfg);
    if (rc) return rc;
    if ((rc = check_qcache(cfg, cache))) return rc;
    if (n_seqs < 0 || n_seqs > cache->n_seqs || layer_begin < 0 || n_layers < 1 || layer_begin + int64_t(n_layers) > cfg->n_layers || total < 0)
        return PRCR_EINVAL;
    if (n_seqs == 0) return PRCR_OK;
    const int64_t row = int64_t(cfg->n_kv_heads) * cfg->head_dim;
    if (!tok_off || !cache_len_in || !cache_len_out || !status || overlap(cache_len_in, cache_len_out, n_seqs)) return PRCR_EINVAL;
    if (total > 0 && (!k_src || !v_src || !coords || src_token_stride < row || src_layer_stride < 0)) return PRCR_EINVAL;
    if (!aligned4(tok_off) || !aligned4(cache_len_in) || !aligned4(cache_len_out) || !aligned4(status)) return PRCR_EALIGN;
    if (total > 0 && (!aligned16(k_src) || !aligned16(v_src) || !mult8(src_layer_stride) || !mult8(src_token_stride) || !aligned4(coords)))
        return PRCR_EALIGN;
    AppendQuantArgs a = {};
    a.cache = qcache_view(cache, layer_begin);
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
    a.format = cache->format;
    a.n_scales = scale_count(cache, cfg->head_dim);
    a.pad = power_of_two(cfg->head_dim / 16);
    a.n_kv_heads = cfg->n_kv_heads;
    const int heads = std::min(cfg->n_kv_heads, 256 / a.pad);
    a.lanes = heads * a.pad;
    a.tok_per_cta = 256 / a.lanes;
    a.layout = cfg->layout;
    a.sec_t = cfg->sections[0];
    a.sec_h = cfg->sections[1];
    a.sec_w = cfg->sections[2];
    copy_turn_freq(cfg, a.turn_freq);
    const int T = a.tok_per_cta, block = (T * a.lanes + 31) / 32 * 32;
    const size_t smem = size_t(T) * (2 * cfg->head_dim * sizeof(float) + 2 * sizeof(int64_t));
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PRCR_ECUDA;
    const int64_t tiles = std::max<int64_t>(1, (int64_t(total) + T - 1) / T);
    a.layers_per_cta = layers_per_cta(tiles, n_layers, int64_t(sm_count(dev)) * 3, 16);
    const dim3 grid(unsigned(tiles), unsigned((n_layers + a.layers_per_cta - 1) / a.layers_per_cta),
                    unsigned((cfg->n_kv_heads + heads - 1) / heads));
    return status_of(launch_append_quant(a, grid, block, smem, static_cast<cudaStream_t>(stream)));
}

int prcr_quantize_cache(const prcr_rope_cfg* cfg, const prcr_cache_desc* src, int32_t src_layer, const prcr_qcache_desc* dst,
                        int32_t dst_layer, int32_t n_layers, int32_t n_seqs, const int32_t* src_begin, const int32_t* dst_begin,
                        const int32_t* count, int32_t max_count, uint32_t* status, void* stream) {
    CastArgs a;
    dim3 grid;
    bool go;
    const int rc = cast_setup(cfg, src, src_layer, dst, dst_layer, n_layers, n_seqs, src_begin, dst_begin, count, max_count, status, true, &a,
                              &grid, &go);
    return rc || !go ? rc : status_of(launch_quantize(a, grid, static_cast<cudaStream_t>(stream)));
}

int prcr_dequantize_cache(const prcr_rope_cfg* cfg, const prcr_qcache_desc* src, int32_t src_layer, const prcr_cache_desc* dst,
                          int32_t dst_layer, int32_t n_layers, int32_t n_seqs, const int32_t* src_begin, const int32_t* dst_begin,
                          const int32_t* count, int32_t max_count, uint32_t* status, void* stream) {
    CastArgs a;
    dim3 grid;
    bool go;
    const int rc = cast_setup(cfg, dst, dst_layer, src, src_layer, n_layers, n_seqs, src_begin, dst_begin, count, max_count, status, false, &a,
                              &grid, &go);
    return rc || !go ? rc : status_of(launch_dequantize(a, grid, static_cast<cudaStream_t>(stream)));
}

size_t prcr_decode_quant_workspace_size(const prcr_rope_cfg* cfg, int32_t format, int32_t n_seqs, int32_t n_layers, int32_t n_q_heads,
                                        int64_t max_len) {
    if (check_cfg(cfg) || n_seqs < 1 || n_layers < 1 || max_len < 0 || max_len > PRCR_CACHE_MAX_LEN || !heads_ok(cfg, n_q_heads) ||
        (format != PRCR_QFMT_E4M3 && format != PRCR_QFMT_E2M1))
        return 0;
    int dev = 0, sms = 1;
    if (cudaGetDevice(&dev) == cudaSuccess) sms = sm_count(dev);
    const DecodeQuantTeams s = decode_quant_teams(format, cfg->head_dim, cfg->n_kv_heads, int64_t(n_seqs) * n_layers, max_len, sms);
    return decode_quant_parts(s, n_q_heads / cfg->n_kv_heads, cfg->head_dim);
}

int prcr_decode_attention_quant(const prcr_rope_cfg* cfg, const prcr_qcache_desc* cache, int32_t n_seqs, int32_t layer_begin, int32_t n_layers,
                                int32_t n_q_heads, const void* q, const int64_t* q_pos, const int32_t* seq_len, int64_t max_len, float* out,
                                uint32_t* status, void* workspace, size_t workspace_bytes, void* stream) {
    int rc = check_cfg(cfg);
    if (rc) return rc;
    if ((rc = check_qcache(cfg, cache))) return rc;
    if (!heads_ok(cfg, n_q_heads) || n_seqs < 0 || n_seqs > cache->n_seqs || layer_begin < 0 || n_layers < 1 ||
        layer_begin + int64_t(n_layers) > cfg->n_layers || max_len < 0 || max_len > PRCR_CACHE_MAX_LEN || max_len > qcache_capacity(cache))
        return PRCR_EINVAL;
    if (n_seqs == 0) return PRCR_OK;
    if (!q || !q_pos || !seq_len || !out || !status || q == out) return PRCR_EINVAL;
    if (!aligned4(q) || !aligned8(q_pos) || !aligned4(seq_len) || !aligned16(out) || !aligned4(status)) return PRCR_EALIGN;
    int dev = 0;
    if (cudaGetDevice(&dev) != cudaSuccess) return PRCR_ECUDA;
    const int64_t units = int64_t(n_seqs) * n_layers * cfg->n_kv_heads;
    if (units * (n_q_heads / cfg->n_kv_heads) > INT32_MAX) return PRCR_EINVAL;  // the join's grid x
    DecodeQuantArgs a = {};
    const DecodeQuantTeams s = decode_quant_teams(cache->format, cfg->head_dim, cfg->n_kv_heads, int64_t(n_seqs) * n_layers, max_len, sm_count(dev));
    const size_t parts = decode_quant_parts(s, n_q_heads / cfg->n_kv_heads, cfg->head_dim);
    if (!workspace || workspace_bytes < parts) return PRCR_EWORKSPACE;
    if (!aligned16(workspace)) return PRCR_EALIGN;
    a.team = s.team;
    a.head_sets = s.head_sets;
    a.teams = int32_t(s.teams);
    a.partial = static_cast<float*>(workspace);
    a.cache = qcache_view(cache, layer_begin);
    a.q = static_cast<const uint16_t*>(q);
    a.q_pos = q_pos;
    a.seq_len = seq_len;
    a.out = out;
    a.status = status;
    a.n_seqs = n_seqs;
    a.n_layers = n_layers;
    a.n_kv_heads = cfg->n_kv_heads;
    a.group = n_q_heads / cfg->n_kv_heads;
    a.head_dim = cfg->head_dim;
    a.format = cache->format;
    a.max_len = int32_t(max_len);
    a.scale_log2 = float(1.4426950408889634 / std::sqrt(double(cfg->head_dim)));
    copy_turn_freq(cfg, a.turn_freq);
    return status_of(launch_decode_quant(a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
