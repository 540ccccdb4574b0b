// Attention of a packed batch's new tokens over the decoder cache, one layer:
// query i of the n_b new tokens of sequence b sees the slots up to its own,
//   out = softmax(RoPE(q, (t, h, w)) K^T / sqrt(D)) V over slots [0, len_b - n_b + i].
//
// The query heads of a KV head's group share its keys, so a sequence's rows for
// one KV head are (token, head of the group) pairs, tokens first: row r is token
// r / group. A CTA takes 128 NQ consecutive rows of one sequence and KV head
// and walks the slots in tiles of 128:
//   S = Q K^T and O += P V on the tensor cores (tcgen05, 128 x 128 x 16 steps,
//   bf16 in, float32 out), the accumulators in tensor memory;
//   P = exp2(S scale - m) by one thread per row, written back over S as bf16.
// Roles: 4 warps of softmax per 128 rows, 4 warps that copy K and V rows, and one
// thread that issues the matrix instructions.
//  - NQ = 2 (head_dim 64 and 128): while the tensor cores work for one half of the
//    rows, the other half's softmax runs.
//  - NQ = 1 (head_dim 256, whose accumulator is 256 columns, and sequences of few
//    rows, which one half would hold): two S buffers; the next tile's S is made before
//    this tile's O.
// The running maximum m is only raised when it grows by more than 8 (in log2
// units): P then holds values up to 2^8, which bf16 represents as exactly as
// values up to 1, the sums are float32, and the accumulator is rarely read back
// to be scaled.
// Roundings to bf16: the rotated query and P are tensor-core operands. Each is
// off by at most 2^-8 of its value, unbiased, as much as the output's own.
//
// Slots that a row does not see are masked before the exponential, so P is 0
// there; 0 times an infinity or NaN of a hidden value row would still reach O.
// Rows behind the sequence's length are never loaded (zeros are); a row of
// later tokens can only matter if its value is not finite, and then the row's
// result is not finite: where that is so, a look at the values of the tile's hidden
// slots decides whether the row is computed again, in float32, from its own slots
// alone. (A row that sees an infinity or NaN keeps what the tensor cores make of it.)
// The same path serves the CTAs that meet an unmapped block.
//
// What bounds it, measured: with many rows the tensor cores. A tile of 128 slots costs
// 256 rows about 2600 clocks, 2048 of them matrix instructions, the rest the
// hand-overs between softmax and products; a CTA's start and end (its place in the
// batch, the queries' angles, the last products and the results' way out) about 17,000.
// One prompt of 8192 tokens, 32 heads of 128 over 8: 390 us, 1.43 PFLOP/s, 0.75 of a
// library product's rate; 1024 tokens each of four sequences of up to 16,384 slots:
// 416 us, 1.50 PFLOP/s (in a row, with queries in L2, 366 and 382); six prompts of up to
// 2116 tokens, few tiles per CTA: 150 us, 0.74 PFLOP/s; head_dim 256 (half as many rows per
// CTA), 1500 tokens each of two sequences of up to 3500 slots: 175 us, 0.98 PFLOP/s.
// With few rows the keys' and values' bytes: 6 tokens each of 16 sequences of up to
// 8198 slots 63 us, 5.1 TB/s (69 with NQ = 2); one token over 933 slots 12 us, all latency.
// Tiles and roles that were slower (that prompt in a row, then at 375 to 430 us, unless said): CTAs that
// stay and take runs of tiles 450 us, or whole units 490; queries in tensor memory with
// tiles of 64 slots 533; a thread of matrix instructions for each half, whose softmaxes
// then fall into step, 3970 clocks a tile; rows by TMA in boxes of 16 slots (a block of
// a paged cache) 260 clocks a tile more; CTAs of 128 rows, two per SM, 638 us (and six
// prompts 201, 6 tokens 73); two threads a row, 64 slots each, whose 24 warps leave 80
// registers a thread, 906 (at head_dim 256, where 16 warps are enough, 168 for 176).
#include "prcr_cache.cuh"
#include "prcr_chunk_phases.h"
#include "prcr_pdl.cuh"
#include "prcr_tc.cuh"

namespace prcr {
namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kTile = 128;  // slots a tile
constexpr float kRaise = 8.0f;

template <int D, int NQ>
struct ChunkShape {
    static constexpr int kDims = D < 128 ? D : 128;      // dims of a ring entry
    static constexpr int kParts = D / kDims;             // entries of a K (or V) tile
    static constexpr int kPanel = kTile * 128;           // bytes: 64 dims of 128 rows
    static constexpr int kEntry = kTile * kDims * 2;
    static constexpr int kQTile = 128 * D * 2;
    static constexpr int kStages = D == 64 || (D == 128 && NQ == 1) ? 6 : 5;  // what an SM holds (64: what is enough)
    static constexpr int kSoftWarps = 4 * NQ;
    static constexpr int kThreads = (kSoftWarps + 8) * 32;
    static constexpr int kRows = 128 * NQ;
    static constexpr size_t kSmem = 1024 + size_t(NQ) * kQTile + size_t(kStages) * kEntry;
};

// Byte offset of a row's 16-byte chunk in the CTA's query tiles: panels of 64
// dims, 128 bytes a row, chunks swizzled by the row.
template <class Sh>
__device__ __forceinline__ uint32_t chunk_at(int r, int c) {
    return uint32_t(r >> 7) * Sh::kQTile + uint32_t(c >> 3) * Sh::kPanel + uint32_t(r & 127) * 128 +
           uint32_t(((c & 7) ^ (r & 7)) * 16);
}
__device__ __forceinline__ void st_shared(uint32_t p, const uint4& v) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                 : "memory");
}
__device__ __forceinline__ uint4 ld_shared(uint32_t p) {
    uint4 v;
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "r"(p)
                 : "memory");
    return v;
}

// One query row by one warp in float32: online softmax over slots
// [lo, hi), E dims a lane (dims lane * E ..), the rows of eight slots in flight
// together. m is in units of log2.
template <int D>
__device__ __noinline__ void row_attention(const ChunkArgs& a, int b, int t, int hq, int64_t lo, int64_t hi,
                                           float& m, float& l, float (&o)[D / 32], uint32_t& err) {
    constexpr int E = D / 32, U = 8;
    const int lane = threadIdx.x & 31;
    const int kh = hq / a.group;
    const uint16_t* qr = a.q + int64_t(t) * a.q_stride + int64_t(hq) * D + lane * E;
    float q[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
        const float x = lo_f32(qr[e]), y = __shfl_xor_sync(kFull, x, 16);  // the pair's other half
        const int i = (lane & 15) * E + e;
        float s, c;
        sincos_turns(double(a.coords[3 * int64_t(t) + pair_axis(i, a.layout, a.sec_t, a.sec_h, a.sec_w)]),
                     a.turn_freq[i], &s, &c);
        q[e] = (lane < 16 ? fmaf(x, c, -y * s) : fmaf(x, c, y * s)) * a.scale_log2;
    }
    m = -INFINITY;
    l = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    const int64_t mine = int64_t(kh) * D + lane * E;
    for (int64_t s0 = lo; s0 < hi; s0 += 32) {
        const int64_t row = s0 + lane < hi ? slot_row(a.cache, b, s0 + lane, err) : int64_t(-1);
        for (int i0 = 0; i0 < min(int64_t(32), hi - s0); i0 += U) {
            uint32_t k[U][E / 2], v[U][E / 2];
            float x[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int64_t r = __shfl_sync(kFull, row, i0 + u);
                x[u] = r >= 0 ? 0.0f : -INFINITY;
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    k[u][e] = r >= 0 ? *reinterpret_cast<const uint32_t*>(a.cache.k + r + mine + 2 * e) : 0u;
                    v[u][e] = r >= 0 ? *reinterpret_cast<const uint32_t*>(a.cache.v + r + mine + 2 * e) : 0u;
                }
            }
            float mn = m;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                float y = 0.0f;
#pragma unroll
                for (int e = 0; e < E / 2; ++e) y = fmaf(q[2 * e + 1], hi_f32(k[u][e]), fmaf(q[2 * e], lo_f32(k[u][e]), y));
#pragma unroll
                for (int d = 16; d; d >>= 1) y += __shfl_xor_sync(kFull, y, d);
                x[u] += y;
                mn = fmaxf(mn, x[u]);
            }
            const float mu = mn == -INFINITY ? 0.0f : mn;
            const float r = exp2f(m - mu);
            m = mn;
            l *= r;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] *= r;
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float p = exp2f(x[u] - mu);
                l += p;
#pragma unroll
                for (int e = 0; e < E / 2; ++e) {
                    o[2 * e] = fmaf(p, lo_f32(v[u][e]), o[2 * e]);
                    o[2 * e + 1] = fmaf(p, hi_f32(v[u][e]), o[2 * e + 1]);
                }
            }
        }
    }
}

// The last of slots [lo, hi) whose value row (this KV head's) holds an infinity or
// NaN, or -1; by one warp, a slot a lane.
template <int D>
__device__ __noinline__ int64_t last_bad_value(const ChunkArgs& a, int b, int kh, int64_t lo, int64_t hi) {
    for (int64_t end = hi; end > lo; end -= 32) {
        const int64_t s = end - 1 - int64_t(threadIdx.x & 31);
        uint32_t err = 0;
        const int64_t row = s >= lo ? slot_row(a.cache, b, s, err) : int64_t(-1);
        bool bad = false;
        for (int i = 0; row >= 0 && i < D; i += 8) {
            const uint4 x = *reinterpret_cast<const uint4*>(a.cache.v + row + int64_t(kh) * D + i);
            for (const uint32_t w : {x.x, x.y, x.z, x.w})
                bad |= (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
        }
        const uint32_t who = __ballot_sync(kFull, bad);
        if (who) return end - 1 - (__ffs(int(who)) - 1);
    }
    return -1;
}

template <int N>
__device__ __forceinline__ void store_row(void* p, const uint32_t* v, bool wide) {
    char* c = static_cast<char*>(p);
    if (wide) {
#pragma unroll
        for (int i = 0; i < N; i += 8)
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(c + 4 * i), "r"(v[i]),
                         "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]),
                         "r"(v[i + 7])
                         : "memory");
    } else {
#pragma unroll
        for (int i = 0; i < N; i += 4)
            *reinterpret_cast<uint4*>(c + 4 * i) = make_uint4(v[i], v[i + 1], v[i + 2], v[i + 3]);
    }
}

struct ChunkSeq {
    int t0, n, len;  // its first token of the call, its new tokens, its slots
};
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkArgs& a, int b) {
    ChunkSeq s;
    s.t0 = a.q_off[b];
    s.n = a.q_off[b + 1] - s.t0;
    s.len = a.seq_len[b];
    return s;
}
// Tiles of each split of the slots that rows row0 .. of a sequence see.
__device__ __forceinline__ int split_tiles(const ChunkArgs& a, int64_t first, int row0, int rows) {
    const int64_t seen = min(int64_t(a.top), first + (row0 + rows - 1) / a.group + 1);
    const int tiles = seen > 0 ? int((seen + kTile - 1) / kTile) : 0;
    return (tiles + a.splits - 1) / a.splits;
}

// What a CTA works on, and the barriers of its roles.
struct ChunkWork {
    int b, row0, rows, t0;        // sequence, first row, rows, the sequence's first token
    int64_t first;                // slots that the sequence's token 0 sees - 1 (may be negative)
    int64_t lo, hi;               // slots of this CTA
    int tiles[2];                 // tiles of each 128 rows
    uint32_t tmem;
    int fail, unmapped;
};
struct ChunkBars {
    uint64_t full[6], empty[6], q, s[2], p[2][2], o[2], drain;  // p: halves of 64 slots
};

template <int D, int NQ>
__global__ void __launch_bounds__(ChunkShape<D, NQ>::kThreads, 1) chunk_kernel(const __grid_constant__ ChunkArgs a) {
    using Sh = ChunkShape<D, NQ>;
    constexpr int P = D / 2, ST = Sh::kStages, PARTS = Sh::kParts, DIMS = Sh::kDims;
    constexpr int kSoft = Sh::kSoftWarps;
    extern __shared__ unsigned char smem_raw[];
    __shared__ ChunkWork w;
    __shared__ __align__(8) ChunkBars bars;
    __shared__ uint64_t s_freq[P];
    __shared__ int s_axis[P];
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    // 1024-byte aligned: the swizzle goes by address bits
    const uint32_t base = (smem_u32(smem_raw) + 1023u) & ~1023u;
    const uint32_t q_s = base, ring = base + NQ * Sh::kQTile;
    const int G = a.group, H = a.n_kv_heads;
    const int kh = int(blockIdx.x % unsigned(H));
    const int rest = int(blockIdx.x / unsigned(H));
    const int split = rest % a.splits;
    const int item = rest / a.splits;

    pdl_allow();
    if (tid == 0) {
        for (int i = 0; i < ST; ++i) {
            mbar_init(smem_u32(&bars.full[i]), 128);  // every loading thread's copies
            mbar_init(smem_u32(&bars.empty[i]), 1);
        }
        mbar_init(smem_u32(&bars.q), kSoft);
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_u32(&bars.s[i]), 1);
            mbar_init(smem_u32(&bars.p[i][0]), 4);
            mbar_init(smem_u32(&bars.p[i][1]), 4);
            mbar_init(smem_u32(&bars.o[i]), 1);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        w.fail = 0;
        w.unmapped = 0;
    }
    if (warp == kSoft + 4) tmem_alloc(smem_u32(&w.tmem), 512);
    if (tid < P) {
        s_freq[tid] = a.turn_freq[tid];
        s_axis[tid] = pair_axis(tid, a.layout, a.sec_t, a.sec_h, a.sec_w);
    }
    pdl_wait();

    // This CTA's rows: an item is a sequence's rows of a tile; its last one, which sees
    // the most slots, first, and of up to 32 sequences the longest first, so that
    // the last CTAs to begin are short ones.
    if (warp == 0) {
        int b = -1;
        ChunkSeq seq = {};
        for (int b0 = 0, before = 0; b0 < a.n_seqs; b0 += 32) {
            ChunkSeq q = {};
            if (b0 + lane < a.n_seqs) q = chunk_seq(a, b0 + lane);
            const int c = q.n > 0 ? int((min(int64_t(q.n), int64_t(a.total_q)) * G + Sh::kRows - 1) / Sh::kRows) : 0;
            int first = before;
            if (a.n_seqs <= 32) {
                for (int o = 0; o < a.n_seqs; ++o) {
                    const int len = __shfl_sync(kFull, q.len, o), n = __shfl_sync(kFull, c, o);
                    if (len > q.len || (len == q.len && o < lane)) first += n;
                }
            } else {
                int upto = c;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int o = __shfl_up_sync(kFull, upto, d);
                    if (lane >= d) upto += o;
                }
                first += upto - c;
                before += __shfl_sync(kFull, upto, 31);
            }
            const uint32_t who = __ballot_sync(kFull, item >= first && item < first + c);
            if (who) {
                const int src = __ffs(int(who)) - 1;
                b = b0 + src;
                seq.t0 = __shfl_sync(kFull, q.t0, src);
                seq.n = __shfl_sync(kFull, q.n, src);
                seq.len = __shfl_sync(kFull, q.len, src);
                w.row0 = __shfl_sync(kFull, (c - 1 - (item - first)) * Sh::kRows, src);
                break;
            }
        }
        if (lane == 0) {
            w.b = b;
            if (b >= 0) {
                if (seq.len < 0 || seq.len > a.top) atomicOr(a.status, PRCR_ST_CAPACITY);
                w.t0 = seq.t0;
                w.rows = min(Sh::kRows, seq.n * G - w.row0);
                w.first = int64_t(seq.len) - seq.n;
                const int per = split_tiles(a, w.first, w.row0, w.rows);
                w.lo = int64_t(split) * per * kTile;
                int64_t hi = 0;
                for (int q = 0; q < 2; ++q) {
                    w.tiles[q] = 0;
                    if (q < NQ && q * 128 < w.rows) {
                        const int last = (w.row0 + min(w.rows, q * 128 + 128) - 1) / G;
                        hi = min(min(int64_t(a.top), w.first + last + 1), w.lo + int64_t(per) * kTile);
                        w.tiles[q] = hi > w.lo ? int((hi - w.lo + kTile - 1) / kTile) : 0;
                    }
                }
                w.hi = hi;
            }
        }
    }
    tc_fence_before();
    const bool bad = __syncthreads_or(bad_offsets(a.q_off, a.n_seqs, a.total_q));
    tc_fence_after();
    if (bad && blockIdx.x == 0 && tid == 0) atomicOr(a.status, PRCR_ST_CSR);
    const int nt = max(w.tiles[0], w.tiles[1]);
    const uint32_t tmem = w.tmem;
    const bool work = !bad && w.b >= 0 && w.rows > 0;
    uint16_t* const out = a.out + int64_t(w.t0) * a.out_stride + int64_t(kh) * G * D;
    bool failed = false;
    float m_run = -INFINITY, l_run = 0.0f;

    // Registers: 2 x 4 warps of 192 and 8 of 64 are the 16 of 128 that the CTA was
    // launched with (NQ = 1: 4 of 232 and 8 of 136 are the 12 of 168).
    // (Each role ends at the same two barriers, on its own way.)
    if (work) {
        if (warp < kSoft) {
            if constexpr (NQ == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 192;");
            else asm volatile("setmaxnreg.inc.sync.aligned.u32 232;");
          if (nt > 0) {
            // queries: rotated, rounded to bf16, into 128-byte rows of swizzled panels. A
            // thread takes eight pairs of a token for all heads of the group. The
            // angle is exact modulo one turn in integers; sin and cos are the fast
            // ones (2^-20, where bf16 keeps 2^-9).
            {
                const int tok0 = w.row0 / G, n_tok = (w.row0 + w.rows - 1) / G - tok0 + 1;
                constexpr int CH = P / 8, BATCH = 4;  // heads whose loads are in flight together
                struct Item {
                    int tok, pc, pos[3];
                    uint4 x[BATCH], y[BATCH];
                };
                auto load = [&](Item& m, int g0) {
                    const uint16_t* src = a.q + (int64_t(w.t0) + m.tok) * a.q_stride + (int64_t(kh) * G + g0) * D + m.pc * 8;
#pragma unroll
                    for (int g = 0; g < BATCH; ++g) {
                        const int r = m.tok * G + g0 + g - w.row0;
                        if (g0 + g < G && r >= 0 && r < w.rows) {
                            m.x[g] = ld_stream(src + g * D);
                            m.y[g] = ld_stream(src + g * D + P);
                        }
                    }
                };
                auto begin = [&](Item& m, int it) {
                    m.tok = tok0 + it / CH;
                    m.pc = it % CH;
                    const int32_t* c = a.coords + 3 * (int64_t(w.t0) + m.tok);
                    if (it < n_tok * CH) {
#pragma unroll
                        for (int x = 0; x < 3; ++x) m.pos[x] = c[x];
                        load(m, 0);
                    }
                };
                auto finish = [&](Item& m, int it) {
                    if (it >= n_tok * CH) return;
                    float c[8], s[8];
#pragma unroll
                    for (int u = 0; u < 8; ++u) {
                        const int i = m.pc * 8 + u;
                        const int ax = s_axis[i];
                        const int p = ax == 0 ? m.pos[0] : ax == 1 ? m.pos[1] : m.pos[2];
                        const int frac = int(uint32_t((uint64_t(int64_t(p)) * s_freq[i]) >> 32));
                        __sincosf(float(frac) * 1.46291807926715968e-09f, &s[u], &c[u]);
                    }
                    for (int g0 = 0; g0 < G; g0 += BATCH) {
                        if (g0) load(m, g0);
#pragma unroll
                        for (int g = 0; g < BATCH; ++g) {
                            const int r = m.tok * G + g0 + g - w.row0;
                            if (g0 + g >= G || r < 0 || r >= w.rows) continue;
                            uint4 xo, yo;
                            rotate_vec(m.x[g], m.y[g], c, s, xo, yo);
                            st_shared(q_s + chunk_at<Sh>(r, m.pc), xo);
                            st_shared(q_s + chunk_at<Sh>(r, m.pc + CH), yo);
                        }
                    }
                };
                Item m0, m1;
                for (int it = tid; it < n_tok * CH; it += 2 * kSoft * 32) {
                    begin(m0, it);
                    begin(m1, it + kSoft * 32);
                    finish(m0, it);
                    finish(m1, it + kSoft * 32);
                }
                // rows behind the last one: zeros
                for (int it = w.rows * (D / 8) + tid; it < Sh::kRows * (D / 8); it += kSoft * 32)
                    st_shared(q_s + chunk_at<Sh>(it / (D / 8), it % (D / 8)), make_uint4(0, 0, 0, 0));
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bars.q));
            }

            // softmax of row `tid & 127` of the 128 rows that this warp belongs to
            const int qi = warp >> 2;
            const int r = tid;  // row of the CTA
            const int64_t lim = min(w.hi, w.first + (w.row0 + min(r, w.rows - 1)) / G + 1);  // slots that the row sees
            const int64_t lim_lo = __shfl_sync(kFull, lim, 0);                    // the warp's least
            const uint32_t lanes = uint32_t(warp & 3) << 21;                      // TMEM lanes of this warp
            const uint32_t o_t = tmem + 256 + uint32_t(qi) * D + lanes;
            const float scale = a.scale_log2;
            for (int j = 0; j < w.tiles[qi]; ++j) {
                const ChunkPhase sc = chunk_scores(NQ, qi, j), before = chunk_products(NQ, qi, j - 1);
                const int buf = sc.bar;
                const uint32_t s_t = tmem + uint32_t(buf) * 128 + lanes;
                if (!mbar_wait(smem_u32(&bars.s[buf]), sc.parity)) {
                    failed = true;
                    break;
                }
                tc_fence_after();
                uint32_t s[128];
                float x[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) x[i] = tmem_ld32_max(s_t + 32 * i, s + 32 * i);
                tmem_wait_ld(s);
#pragma unroll
                for (int i = 0; i < 4; ++i) asm volatile("" : "+f"(x[i]));
                const int64_t at = w.lo + int64_t(j) * kTile;
                if (at + kTile > lim_lo) {  // some row of the warp does not see all of the tile
                    const int n = int(max(int64_t(0), min(int64_t(kTile), lim - at)));
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        x[k] = -INFINITY;
#pragma unroll
                        for (int i = 32 * k; i < 32 * k + 32; ++i) {
                            if (i >= n) s[i] = 0xff800000u;
                            x[k] = fmaxf(x[k], __uint_as_float(s[i]));
                        }
                    }
                }
                const float mt = fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) * scale;
                const bool raise = mt > m_run + kRaise;
                bool summed = j == 0;  // whether the last tile's products are known to be done
                if (j == 0) {
                    m_run = mt;
                } else if (__any_sync(kFull, raise)) {
                    // (NQ = 2: this S was made behind the last tile's products)
                    if (NQ == 1 && !mbar_wait(smem_u32(&bars.o[before.bar]), before.parity)) {
                        failed = true;
                        break;
                    }
                    summed = true;
                    tc_fence_after();
                    float f = 1.0f;
                    if (raise) {
                        f = exp2_fast(m_run - mt);
                        m_run = mt;
                    }
                    l_run *= f;
                    const uint64_t f2 = pair64(f, f);
#pragma unroll 1
                    for (int c = 0; c < D; c += 32) {
                        uint32_t o[32];
                        tmem_ld32(o_t + c, o);
                        tmem_wait_ld(o);
#pragma unroll
                        for (int i = 0; i < 32; i += 2) {
                            const uint64_t y = mul2(uint64_t(o[i]) | (uint64_t(o[i + 1]) << 32), f2);
                            o[i] = uint32_t(y);
                            o[i + 1] = uint32_t(y >> 32);
                        }
                        tmem_st32(o_t + c, o);
                    }
                }
                const float mu = m_run == -INFINITY ? 0.0f : m_run;
                const uint64_t c2 = pair64(scale, scale), m2 = pair64(-mu, -mu);
                // (three chains of sums: two leave the additions' latency on the way to the products,
                // one prompt of 8192 tokens 376 us for 366, calls in a row; four 368, eight 375)
                uint64_t sums[3] = {};
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t p[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int k = half * 64 + 2 * i;
                        const uint64_t x = fma2(uint64_t(s[k]) | (uint64_t(s[k + 1]) << 32), c2, m2);
                        const float e0 = exp2_fast(lo32(x)), e1 = exp2_fast(hi32(x));
                        const uint64_t e = pair64(e0, e1);
                        sums[i % 3] = add2(sums[i % 3], e);
                        p[i] = pack_bf16x2(e0, e1);
                    }
                    tmem_st32(s_t + 32 * half, p);
                    tmem_wait_st();
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_u32(&bars.p[buf][half]));
                }
                const uint64_t sum = add2(add2(sums[0], sums[1]), sums[2]);
                l_run += lo32(sum) + hi32(sum);
                // (each tile's phase is waited for before the next on its barrier can complete)
                if (NQ == 1 && !summed && !mbar_wait(smem_u32(&bars.o[before.bar]), before.parity)) {
                    failed = true;
                    break;
                }
            }
            // all of this half's products are done
            if (!failed && w.tiles[qi] > 0) {
                const ChunkPhase last = chunk_products(NQ, qi, w.tiles[qi] - 1);
                if (!mbar_wait(smem_u32(&bars.o[last.bar]), last.parity)) failed = true;
                tc_fence_after();
            }
          }
            if (failed) w.fail = 1;
            __syncthreads();
            if (w.fail) {
                if (tid == 0) atomicOr(a.status, PRCR_ST_TIMEOUT);
            } else {
        // results: a thread per row
        const int qi = warp >> 2, r = tid;
        const bool row_ok = r < w.rows;
        const int rr = w.row0 + min(r, w.rows - 1);
        const int tok = rr / G, g = rr - tok * G;
        const int64_t lim = min(w.first + tok + 1, w.hi);  // (rows of the other half see no more than w.hi)
        const uint32_t o_t = tmem + 256 + uint32_t(qi) * D + (uint32_t(warp & 3) << 21);
        const bool any = w.tiles[qi] > 0;  // this half's accumulator holds something
        const int64_t dst = int64_t(w.t0 + tok) * a.out_stride + (int64_t(kh) * G + g) * D;
        const int64_t prow = (int64_t(w.t0 + tok) * H + kh) * G + g;  // row of the partials
        float* po = a.splits > 1 ? a.partial + (prow * a.splits + split) * D : nullptr;
        const bool live = row_ok && lim > w.lo;
        const bool wide = (reinterpret_cast<uintptr_t>(a.partial) & 31) == 0;
        const float inv = l_run == 0.0f ? 0.0f : 1.0f / l_run;
        float odd[4] = {l_run * 0.0f, 0.0f, 0.0f, 0.0f};
        if (any) {
#pragma unroll 1
            for (int c = 0; c < D; c += 32) {
                uint32_t o[32];
                tmem_ld32(o_t + c, o);
                tmem_wait_ld(o);
#pragma unroll
                for (int i = 0; i < 32; ++i) odd[i & 3] = fmaf(__uint_as_float(o[i]), 0.0f, odd[i & 3]);
                if (a.splits == 1) {
#pragma unroll
                    for (int i = 0; i < 32; i += 8) {
                        uint4 v;
                        v.x = pack_bf16x2(__uint_as_float(o[i]) * inv, __uint_as_float(o[i + 1]) * inv);
                        v.y = pack_bf16x2(__uint_as_float(o[i + 2]) * inv, __uint_as_float(o[i + 3]) * inv);
                        v.z = pack_bf16x2(__uint_as_float(o[i + 4]) * inv, __uint_as_float(o[i + 5]) * inv);
                        v.w = pack_bf16x2(__uint_as_float(o[i + 6]) * inv, __uint_as_float(o[i + 7]) * inv);
                        st_shared(q_s + chunk_at<Sh>(r, (c + i) / 8), v);
                    }
                } else if (live) {
                    store_row<32>(po + c, o, wide);
                }
            }
        }
        if (a.splits == 1) {
            // the queries' place now holds the results (this half's products with
            // them are done): whole rows go out, 16 bytes a lane
            constexpr int CPR = D / 8, RPI = 32 / CPR;
            // (a row that sees no slot is zeros, also where a value hidden from it is not finite)
            const uint32_t seeing = __ballot_sync(kFull, live && any);
            __syncwarp();
#pragma unroll 4
            for (int i = 0; i < 32 / RPI; ++i) {
                const int src = i * RPI + lane / CPR;
                const int64_t to = __shfl_sync(kFull, row_ok ? dst : int64_t(-1), src);
                if (to >= 0)
                    st_row(a.out + to + (lane % CPR) * 8,
                           (seeing >> src) & 1u ? ld_shared(q_s + chunk_at<Sh>((r & ~31) + src, lane % CPR)) : make_uint4(0, 0, 0, 0));
            }
            __syncwarp();
        }
        if (a.splits > 1 && live) a.partial_ml[prow * a.splits + split] = make_float2(m_run, l_run);
        // rows to be computed again from their own slots: those that are not finite and
        // whose tiles held a value row that they do not see and that is not finite, and
        // all of a CTA with unmapped blocks
        const bool odd_row = live && any && odd[0] + odd[1] + (odd[2] + odd[3]) != 0.0f;
        uint32_t again = w.unmapped ? __ballot_sync(kFull, live && any) : 0u;
        if (!w.unmapped && __any_sync(kFull, odd_row)) {
            int64_t from = odd_row ? lim : w.hi;
#pragma unroll
            for (int d = 16; d; d >>= 1) from = min(from, __shfl_xor_sync(kFull, from, d));
            const int64_t bad = last_bad_value<D>(a, w.b, kh, from, min(w.hi, w.lo + int64_t(w.tiles[qi]) * kTile));
            again = __ballot_sync(kFull, odd_row && bad >= lim);
        }
        if (w.unmapped && tid == 0) atomicOr(a.status, PRCR_ST_NO_BLOCK);
        while (again) {
            const int src = __ffs(int(again)) - 1;
            again &= again - 1;
            const int tk = __shfl_sync(kFull, tok, src), gg = __shfl_sync(kFull, g, src);
            const int64_t lm = __shfl_sync(kFull, lim, src);
            float m, l, o[D / 32];
            uint32_t err = 0;
            row_attention<D>(a, w.b, w.t0 + tk, kh * G + gg, w.lo, lm, m, l, o, err);
            __syncwarp();
            constexpr int E = D / 32;
            if (a.splits == 1) {
                const float iv = l == 0.0f ? 0.0f : 1.0f / l;
                uint16_t* d = out + int64_t(tk) * a.out_stride + int64_t(gg) * D + lane * E;
#pragma unroll
                for (int i = 0; i < E; i += 2) *reinterpret_cast<uint32_t*>(d + i) = pack_bf16x2(o[i] * iv, o[i + 1] * iv);
            } else {
                const int64_t pr = (int64_t(w.t0 + tk) * H + kh) * G + gg;
                float* d = a.partial + (pr * a.splits + split) * D + lane * E;
#pragma unroll
                for (int i = 0; i < E; ++i) d[i] = o[i];
                if (lane == 0) a.partial_ml[pr * a.splits + split] = make_float2(m, l);
            }
        }
            }
        } else if (warp < kSoft + 4) {
            if constexpr (NQ == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
            else asm volatile("setmaxnreg.dec.sync.aligned.u32 136;");
          if (nt > 0) {
            // rows of K and V: warp lw copies slots 32 lw .. 32 lw + 31 of every tile,
            // 16 bytes a lane; slots without a row are zeros
            const int lw = warp - kSoft;
            const uint16_t* ck = a.cache.k + int64_t(kh) * D;
            const uint16_t* cv = a.cache.v + int64_t(kh) * D;
            constexpr int CPR = DIMS / 8, RPI = 32 / CPR;  // chunks a row, rows an instruction
            const int c = lane % CPR, rsub = lane / CPR;
            int e = 0;          // entries issued
            bool missing = false;
            // the block of this lane's slot of tile j, asked for a tile before it is needed
            const int32_t* bt = a.cache.block_table + int64_t(w.b) * a.cache.bt_stride;
            auto block_of_tile = [&](int j) -> int32_t {
                const int64_t slot = w.lo + int64_t(j) * kTile + lw * 32 + lane;
                if (a.cache.kind != PRCR_CACHE_PAGED || j >= nt || slot >= w.hi) return 0;
                return bt[block_index(a.cache, uint32_t(slot))];
            };
            auto row_of = [&](int j, int32_t blk) -> int64_t {
                const int64_t slot = w.lo + int64_t(j) * kTile + lw * 32 + lane;
                if (j >= nt || slot >= w.hi) return -1;
                const int64_t row = row_in_block(a.cache, w.b, uint32_t(slot), blk);
                missing |= row < 0;
                return row;
            };
            auto put = [&](const uint16_t* src, int64_t row, int part) -> bool {
                const int st = e % ST;
                if (e >= ST && !mbar_wait(smem_u32(&bars.empty[st]), uint32_t((e / ST - 1) & 1))) return false;
                const uint32_t dst = ring + uint32_t(st) * Sh::kEntry + uint32_t(c >> 3) * Sh::kPanel + uint32_t(lw * 32) * 128;
#pragma unroll
                for (int i = 0; i < 32 / RPI; ++i) {
                    const int r = i * RPI + rsub;
                    const int64_t rr = __shfl_sync(kFull, row, r);
                    const uint16_t* from = rr >= 0 ? src + rr + part * DIMS + c * 8 : src;
                    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(
                                     dst + uint32_t(r) * 128 + uint32_t(((c & 7) ^ (r & 7)) * 16)),
                                 "l"(from), "r"(rr >= 0 ? 16 : 0)
                                 : "memory");
                }
                mbar_arrive_copies(smem_u32(&bars.full[st]));
                ++e;
                return true;
            };
            // in the order of use: K0 V0 K1 V1 .., or with two S buffers K0 K1 V0 K2 V1 ..
            bool ok = true;
            int32_t blk = block_of_tile(1);
            int64_t row = row_of(0, block_of_tile(0)), next = 0;
            for (int p = 0; ok && p < PARTS; ++p) ok = put(ck, row, p);
            for (int j = 0; ok && j < nt; ++j) {
                next = row_of(j + 1, blk);
                blk = block_of_tile(j + 2);
                if (NQ == 1 && j + 1 < nt)
                    for (int p = 0; ok && p < PARTS; ++p) ok = put(ck, next, p);
                for (int p = 0; ok && p < PARTS; ++p) ok = put(cv, row, p);
                if (NQ == 2 && j + 1 < nt)
                    for (int p = 0; ok && p < PARTS; ++p) ok = put(ck, next, p);
                row = next;
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            if (missing) w.unmapped = 1;
            if (!ok) w.fail = 1;
          }
            __syncthreads();
        } else {
            if constexpr (NQ == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 64;");
            else asm volatile("setmaxnreg.dec.sync.aligned.u32 136;");
            if (warp == kSoft + 4 && nt > 0) {
                constexpr uint32_t id_qk = tc_idesc(kTile, false), id_pv = tc_idesc(DIMS, true);
                const uint32_t on = elect_lane();
                const uint64_t dq = tc_desc(q_s, 16, 1024), dk = tc_desc(ring, 16, 1024), dv = tc_desc(ring, Sh::kPanel, 1024);
                int e = 0;  // entries consumed
                // the entries' copies are in place, and visible to the tensor cores
                auto ready = [&](int e0) {
                    bool ok = true;
                    for (int i = e0; i < e0 + PARTS; ++i)
                        ok = ok && mbar_wait(smem_u32(&bars.full[i % ST]), uint32_t((i / ST) & 1));
                    fence_async_smem();
                    return ok;
                };
                // S of 128 rows: entries e0 .. hold the tile's keys
                auto qk = [&](int q, int j, int e0) {
                    const int buf = chunk_scores(NQ, q, j).bar;
                    tc_fence_after();
#pragma unroll
                    for (int part = 0; part < PARTS; ++part) {
                        const uint64_t da = dq + uint32_t(q) * (Sh::kQTile >> 4) + uint32_t(part) * ((DIMS / 64) * Sh::kPanel >> 4);
                        const uint64_t db = dk + uint32_t((e0 + part) % ST) * (Sh::kEntry >> 4);
#pragma unroll
                        for (int k = 0; k < DIMS / 16; ++k) {
                            const uint32_t step = (uint32_t(k >> 2) * Sh::kPanel + uint32_t(k & 3) * 32) >> 4;
                            tc_mma_ss(tmem + uint32_t(buf) * 128, da + step, db + step, id_qk, part + k > 0, on);
                        }
                    }
                    tc_commit(smem_u32(&bars.s[buf]), on);
                };
                // O += P V of 128 rows, each half of the slots as soon as its P is there
                auto pv = [&](int q, int j, int e0) -> bool {
                    const ChunkPhase sc = chunk_scores(NQ, q, j);
#pragma unroll
                    for (int half = 0; half < 2; ++half) {
                        if (!mbar_wait(smem_u32(&bars.p[sc.bar][half]), sc.parity)) return false;
                        tc_fence_after();
#pragma unroll
                        for (int part = 0; part < PARTS; ++part) {
                            const uint64_t db = dv + uint32_t((e0 + part) % ST) * (Sh::kEntry >> 4);
#pragma unroll
                            for (int k = half * 4; k < half * 4 + 4; ++k)
                                tc_mma_ts(tmem + 256 + uint32_t(q) * D + uint32_t(part) * DIMS, tmem + uint32_t(sc.bar) * 128 + uint32_t(k) * 8,
                                          db + uint32_t(k) * (2048 >> 4), id_pv, j > 0 || k > 0, on);
                        }
                    }
                    return true;
                };
                auto release = [&](int e0) {
                    for (int part = 0; part < PARTS; ++part) tc_commit(smem_u32(&bars.empty[(e0 + part) % ST]), on);
                };
                bool ok = mbar_wait(smem_u32(&bars.q), 0) && ready(0);
                if (ok) {
                    for (int q = 0; q < NQ; ++q)
                        if (w.tiles[q] > 0) qk(q, 0, 0);
                    release(0);
                    e = PARTS;
                }
                if constexpr (NQ == 2) {
                    const int n0 = w.tiles[0], n1 = w.tiles[1];
                    for (int j = 0; ok && j < nt; ++j) {
                        const int ev = e, ek = e + PARTS;
                        ok = ready(ev);
                        bool have = false;
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const int n = q ? n1 : n0;
                            if (!ok || j >= n) continue;
                            ok = pv(q, j, ev);
                            if (!ok) continue;
                            if (j + 1 < n) {
                                if (!have) ok = ready(ek);
                                have = true;
                                if (!ok) continue;
                                qk(q, j + 1, ek);
                            } else {
                                tc_commit(smem_u32(&bars.o[chunk_products(NQ, q, j).bar]), on);
                            }
                        }
                        if (ok && j + 1 < nt) {
                            release(ev);
                            release(ek);
                        }
                        e += 2 * PARTS;
                    }
                } else {
                    for (int j = 0; ok && j < nt; ++j) {
                        if (j + 1 < nt) {
                            ok = ready(e);
                            if (!ok) break;
                            qk(0, j + 1, e);
                            release(e);
                            e += PARTS;
                        }
                        ok = ready(e) && pv(0, j, e);
                        if (!ok) break;
                        if (j + 1 < nt) release(e);
                        tc_commit(smem_u32(&bars.o[chunk_products(NQ, 0, j).bar]), on);
                        e += PARTS;
                    }
                }
                if (!ok) {  // what was issued ends before the tensor memory is given back
                    if (lane == 0) {
                        w.fail = 1;
                        mbar_init(smem_u32(&bars.drain), 1);
                    }
                    __syncwarp();
                    tc_commit(smem_u32(&bars.drain), on);
                    mbar_wait(smem_u32(&bars.drain), 0);
                }
            }
            __syncwarp();
            __syncthreads();
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kSoft + 4) tmem_free(tmem, 512);
}

// Warps that join a row's splits: one for each four, up to a block's eight.
__host__ __device__ __forceinline__ int merge_warps(int splits) {
    return splits <= 4 ? 1 : splits <= 8 ? 2 : splits <= 16 ? 4 : 8;
}

// Joins the splits of a row: (max, sum, accumulator) of those that it sees. Latency:
// a lane reads a split's maximum and sum, and a row's warps take the accumulators in
// turn, all of them in flight together (9 tokens of 3 heads of groups of 8 over 9139 slots,
// 50 splits: one warp a row 18 us, eight 7.7).
template <int D, int NQ>
__global__ void __launch_bounds__(256) chunk_merge_kernel(const __grid_constant__ ChunkArgs a) {
    constexpr int E = D / 32, kRows = ChunkShape<D, NQ>::kRows;
    __shared__ __align__(16) float s_o[8][D];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, G = a.group, Hq = a.n_kv_heads * G;
    const int W = merge_warps(a.splits), part = warp % W;
    const int64_t row = int64_t(blockIdx.x) * (8 / W) + warp / W;
    pdl_allow();
    pdl_wait();
    if (__syncthreads_or(bad_offsets(a.q_off, a.n_seqs, a.total_q))) return;
    int n = 0, t = 0, hq = 0;
    bool live = false;  // (not behind the last sequence)
    if (row < int64_t(a.total_q) * Hq) {
        t = int(row / Hq);
        hq = int(row - int64_t(t) * Hq);
        const ChunkSeq q = chunk_seq(a, sequence_of(a.q_off, a.n_seqs, t));
        live = t < q.t0 + q.n;
        const int64_t first = int64_t(q.len) - q.n, lim = min(int64_t(a.top), first + (t - q.t0) + 1);
        const int row0 = ((t - q.t0) * G + hq % G) / kRows * kRows;
        const int per = split_tiles(a, first, row0, min(kRows, q.n * G - row0)) * kTile;
        n = live && lim > 0 ? int((lim + per - 1) / per) : 0;
    }
    const float2* const mls = a.partial_ml + row * a.splits;
    float m = -INFINITY, l = 0.0f, o[E];
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] = 0.0f;
    for (int s = lane; s < n; s += 32) m = fmaxf(m, mls[s].x);
#pragma unroll
    for (int d = 16; d; d >>= 1) m = fmaxf(m, __shfl_xor_sync(kFull, m, d));
    const float mu = m == -INFINITY ? 0.0f : m;
    for (int s0 = 0; s0 < n; s0 += 32) {
        float f = 0.0f;
        if (s0 + lane < n) {
            const float2 ml = mls[s0 + lane];
            f = exp2f(ml.x - mu);
            l = fmaf(f, ml.y, l);
        }
#pragma unroll 4
        for (int s = part; s < min(32, n - s0); s += W) {
            const float g = __shfl_sync(kFull, f, s);
            const float* p = a.partial + (row * a.splits + s0 + s) * D + lane * E;
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] = fmaf(g, p[e], o[e]);
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) l += __shfl_xor_sync(kFull, l, d);
    if (W > 1) {
        if (part) {
#pragma unroll
            for (int e = 0; e < E; ++e) s_o[warp][lane * E + e] = o[e];
        }
        __syncthreads();
        if (part) return;
        for (int x = 1; x < W; ++x)
#pragma unroll
            for (int e = 0; e < E; ++e) o[e] += s_o[warp + x][lane * E + e];
    }
    if (!live) return;
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    uint16_t* out = a.out + int64_t(t) * a.out_stride + int64_t(hq) * D + lane * E;
#pragma unroll
    for (int e = 0; e < E; e += 2) *reinterpret_cast<uint32_t*>(out + e) = pack_bf16x2(o[e] * inv, o[e + 1] * inv);
}

template <int D, int NQ>
cudaError_t launch_shape(const ChunkArgs& a, cudaStream_t stream) {
    using Sh = ChunkShape<D, NQ>;
    const cudaError_t e = raise_smem_limit(reinterpret_cast<const void*>(chunk_kernel<D, NQ>), Sh::kSmem);
    if (e != cudaSuccess) return e;
    const dim3 grid(unsigned(int64_t(a.items) * a.n_kv_heads * a.splits));
    const cudaError_t r = launch_pdl(chunk_kernel<D, NQ>, grid, dim3(Sh::kThreads), Sh::kSmem, stream, a);
    if (r != cudaSuccess || a.splits == 1) return r;
    const int64_t rows = int64_t(a.total_q) * a.n_kv_heads * a.group;
    return launch_pdl(chunk_merge_kernel<D, NQ>, dim3(unsigned((rows * merge_warps(a.splits) + 7) / 8)), dim3(256), 0, stream, a);
}

}  // namespace

int chunk_rows(int head_dim, bool few) { return head_dim == 256 || few ? 128 : 256; }

cudaError_t launch_chunk(const ChunkArgs& a, cudaStream_t stream) {
    if (a.head_dim == 64) return a.few ? launch_shape<64, 1>(a, stream) : launch_shape<64, 2>(a, stream);
    if (a.head_dim == 128) return a.few ? launch_shape<128, 1>(a, stream) : launch_shape<128, 2>(a, stream);
    return launch_shape<256, 1>(a, stream);
}

}  // namespace prcr
