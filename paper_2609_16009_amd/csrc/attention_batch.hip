// Latent attention of a decode batch over a paged cache whose sequences share a prefix (gfx950).
//
//   row r = (b T + t) H + h:   out_r = sum_j p_j v_j,  p = softmax_j(scale * q_r . k_j)
//   over the prefix's positions, shared by every row, and positions j < lens[b] - (T - 1 - t) of sequence b
//
// The prefix's keys are the same for every row, so it is one attention of all B T H rows over one cache,
// taken in tiles of 64 rows: its cache rows are read once per tile, where a pass per sequence would read
// them for each.  A sequence's own positions are attended by its T H rows in tiles of 16, 32 or 64.  Both
// kinds of tile are cut into spans of positions so that their workgroups fill the chip, run in one launch, and
// leave (reference, sum, unnormalised output) partials which a merge launch joins in a fixed order.
//
// A workgroup of 4 waves takes a tile over a span, chunk by chunk:
//  * Staging.  A chunk's rows lie in LDS as bf16, [9 column blocks][positions][8 pieces of 16 bytes]: the latents'
//    eight blocks of 64 columns, then RoPE's (columns that the cache lacks are zeros).  Piece c of row r sits in
//    slot c ^ f(r), which spreads the key reads (8 rows, one column) and the transposed value reads (4 rows, 2 pieces)
//    over all banks.  (By the counters 21 to 32 % of the cycles that LDS is busy are conflicts all the same; they have not been
//    traced to their accesses.)  bf16 rows come by LDS-direct loads of 8 rows x 128 bytes; 8-bit rows come into
//    registers a chunk ahead and are widened on their way to LDS (exact: a power of two per 32 values).  A wave's
//    lanes look up one position's page each, a chunk before its rows are loaded; rows that do not exist (past the end,
//    on a page outside the pool) read zeros and are masked.
//  * S^T = K Q^T, Q in registers as fragments; P = 2^(s - reference), the reference moved only when a chunk
//    exceeds it by 2^8; O^T = V^T P^T, a quarter of the columns a wave.
//    Scores, sums and outputs are fp32; P is rounded to bf16 for the matrix cores (2^-8 of each probability at most, as much as
//    the output's own rounding to bf16: against 64 bits 1.8e-3 to 2.0e-3 in all, 1.7e-3 with fp32 probabilities) and summed before
//    its rounding.
// Tiles of 16 and 32 rows (narrow_block) take chunks of 64 positions, 16 a wave; tiles of 64 (wide_block) chunks of 32 in
// a software pipeline.
//
// What bounds it.  64 sequences of 16 heads over 2049 .. 4097 own positions, 8-bit rows: 45 us for 130 MB (26 us at
// the rate of a large copy), 38 where all rows come from L2: two workgroups a CU spend more on widening the rows into LDS than on
// the products, each with one chunk's loads in flight.  16 sequences of 128 heads behind 8192 positions, bf16 rows: 67 us for
// 40 GFLOP (33 us at the rate
// of a large matrix product); 64 positions take 5300 cycles (6050 with 8-bit rows) where their MFMAs alone would take 2180: every
// key and value fragment is read from LDS by each of the four waves' quarters, and Q's start (7 us) and the fp32
// partials' end (4 us, and 8 us of the merge) are not hidden.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "attention_core.h"
#include "bf16_cast.h"
#include "latent_row.h"
#include "nmm_internal.h"

namespace nmm {
namespace {

using attn::as_bf16x8;
using attn::bf16x4;
using attn::cols4_max;
using attn::cols4_sum;
using attn::f32x4;
using attn::i32x4;
using attn::lds_bf16x4;
using attn::lds_sync;
using attn::lds_void;
using attn::wave_max;
using attn::wave_sum;

constexpr int kWavesB = 4, kThreadsB = 64 * kWavesB;
constexpr int kChunk = 64;                             // positions per chunk, rows of the largest tile
constexpr int kBlocks = 9;                             // column blocks of 64: 8 of latents, 1 of RoPE
constexpr int kBlockElems = kChunk * 64;               // elements of one column block of a chunk
constexpr int kSteps = 2 * kBlocks;                    // k-steps of 32 columns
constexpr int kTilesW = 8;                             // 16-column output tiles per wave
constexpr int kPPitchB = kChunk + 8;
constexpr float kLazy = 8.f;
constexpr int kMaxSlots = 64;                          // partials of a row: one lane of a wave each

struct BatchParams {
    const uint16_t* q;
    int64_t sqb, sqt, ldq;
    const uint8_t* cache;
    int64_t ld;
    int kv, rope;
    int page_shift, n_pages;
    const int32_t* prefix_pages;
    int prefix_len;
    const int32_t* pages;
    int64_t ld_pages;
    const int32_t* lens;
    int max_len;
    float scale_log2;
    uint16_t* out;
    int64_t sob, sot, ldo;
    float* part_o;           // [slots][rows][kv]
    float* part_ml;          // [slots][rows][2]
    int B, T, H, rows;
    int pre_tiles, pre_spans, pre_span, pre_items;
    int own_tiles, own_spans, own_span, own_items;
    int pre_grid;            // workgroups of the prefix: its items rounded up to a multiple of 8
    int direct;              // one slot: rows go straight to out
    uint32_t extent;         // bytes of a pool under 2 GB
};

// Cache rows that do not exist read zeros here.
__device__ __attribute__((aligned(128))) const uint8_t g_zero_row[2 * (kLatentMax + kLatentRopeMax)] = {};

struct Item {
    int r0, nrows;           // first row and rows of the tile
    int seq;                 // sequence of an own item, -1: the prefix
    const int32_t* table;
    int begin, end;          // positions of the span (end <= the length)
    int len;                 // own length of the sequence
    int slot;
    int tile, tiles;         // the tile among those that read the same rows
};

// Global memory, said so: a pointer that may also be the zero row's would otherwise be read by flat loads, which
// count as LDS operations too.
typedef const __attribute__((address_space(1))) uint8_t* gbytes;
typedef unsigned u32x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ u32x4 load16(gbytes p) { return *(const __attribute__((address_space(1))) u32x4*)p; }
// The zero row's address, its contents unknown to the compiler: knowing them it splits every select between
// a cache row and this one into branches.
__device__ __forceinline__ gbytes opaque_zero_row() {
    gbytes z = (gbytes)g_zero_row;
    asm("" : "+s"(z));
    return z;
}

// Two values rounded to bf16 (one conversion).
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    typedef float f32x2_t __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2_t{lo, hi}, bf16x2_t));
}

// The two halves of cols4_max: the maximum over rows 32 lanes apart, then 16.
__device__ __forceinline__ float rows_max32(float x) {
    const attn::u32x2 a = attn::swap32(__float_as_uint(x), __float_as_uint(x));
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}
__device__ __forceinline__ float rows_max16(float x) {
    const attn::u32x2 a = attn::swap16(__float_as_uint(x), __float_as_uint(x));
    return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

// f(r), from bits 1 to 3 of the row (bit 0 picks the half of LDS's 64 banks): LDS serves 256 bytes a cycle, 16 lanes of a
// key read (16 rows, one piece: every f differs) or 32 of a transposed value read (rows 8 g + 0 .. 3 of two g, two
// neighbouring pieces: f differs above bit 0).
__device__ __forceinline__ int swz(int row) { return ((row >> 1) & 4) | (row & 2) | ((row >> 2) & 1); }

__device__ __forceinline__ int64_t row_offset(int r, int T, int H, int64_t sb, int64_t st, int64_t ld) {
    const int bt = r / H, h = r - bt * H;
    const int b = bt / T, t = bt - b * T;
    return int64_t(b) * sb + int64_t(t) * st + int64_t(h) * ld;
}

// LDS-direct loads of 16-byte pieces of cache rows, a row per lane: with 32-bit offsets into the pool, a row that does
// not exist out of its range (zeros), or, for a pool of 2 GB and more, with 64-bit addresses and the zero row (the
// compiler takes those loads to count as LDS operations too, and so waits for every LDS read at once: 71 instead of
// 69 us for 16 x 128 heads behind 8192 positions).
template <bool BIG>
struct StageRows;
template <>
struct StageRows<false> {
    typedef uint32_t Row;
    __amdgpu_buffer_rsrc_t rsrc;
    uint32_t ld;
    __device__ __forceinline__ explicit StageRows(const BatchParams& p)
        : rsrc(attn::make_rsrc(p.cache, p.extent)), ld(static_cast<uint32_t>(p.ld)) {}
    __device__ __forceinline__ Row row(int rows, int lane_of) const {
        const int r = __builtin_amdgcn_ds_bpermute(lane_of << 2, rows);
        return r < 0 ? attn::kOutOfRange : uint32_t(r) * ld;
    }
    __device__ __forceinline__ void load(Row row, uint32_t off, uint16_t* dst) const {
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_void*)dst, 16, row + off, 0, 0, 0);
    }
};
template <>
struct StageRows<true> {
    typedef gbytes Row;
    gbytes cache, zero_row;
    int64_t ld;
    __device__ __forceinline__ explicit StageRows(const BatchParams& p)
        : cache((gbytes)p.cache), zero_row(opaque_zero_row()), ld(p.ld) {}
    __device__ __forceinline__ Row row(int rows, int lane_of) const {
        const int r = __builtin_amdgcn_ds_bpermute(lane_of << 2, rows);
        return r < 0 ? zero_row : cache + int64_t(r) * ld;
    }
    __device__ __forceinline__ void load(Row row, uint32_t off, uint16_t* dst) const {
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)(row + off), (lds_void*)dst, 16, 0, 0);
    }
};

// Row 16 t + j of a tile: normalised to out, or as the span's partial (reference, sum, unnormalised output).
template <int HT>
__device__ __forceinline__ void store_row(const BatchParams& p, const Item& it, int row, int pw, int g, const f32x4 (&o)[kTilesW][HT],
                                          int t, float m, float lsum) {
    if (row >= it.nrows) return;
    const int r = it.r0 + row;
    if (p.direct) {
        // a row that sees nothing is zeros
        const float scl = lsum == 0.f ? 0.f : 1.f / lsum;
        uint16_t* dst = p.out + row_offset(r, p.T, p.H, p.sob, p.sot, p.ldo) + 4 * g;
#pragma unroll
        for (int i = 0; i < kTilesW; ++i) {
            const int c = 16 * (pw + 4 * i);
            const f32x4 v = o[i][t] * scl;
            if (c < p.kv) *reinterpret_cast<uint2*>(dst + c) = uint2{pack2(v[0], v[1]), pack2(v[2], v[3])};
        }
    } else {
        const int64_t at = int64_t(it.slot) * p.rows + r;
        float* const dst = p.part_o + at * p.kv + 4 * g;
#pragma unroll
        for (int i = 0; i < kTilesW; ++i) {
            const int c = 16 * (pw + 4 * i);
            if (c < p.kv) __builtin_nontemporal_store(o[i][t], reinterpret_cast<f32x4*>(dst + c));
        }
        if (pw == 0 && g == 0) *reinterpret_cast<float2*>(p.part_ml + at * 2) = float2{m, lsum};
    }
}

// One (tile, span).  kv_a, kv_b: chunk buffers; pbuf: P [16 HT][kPPitchB]; red: [4][16 HT].
template <int HT, bool E4M3, bool BIG>
__device__ __forceinline__ void narrow_block(const BatchParams& p, const Item it, uint16_t* const kv_a, uint16_t* const kv_b,
                                            uint16_t* const pbuf, float* const red, int* const flags) {
    constexpr int HB = 16 * HT;
    // K and V fragments read ahead of their MFMAs: LDS takes about 130 cycles, a step's HT MFMAs 16 HT.  (16 rows: two
    // workgroups a CU have half the registers each, and hide the rest for each other: 47.3 us with 9 and 8 ahead, 45.5 with 4.)
    static_assert(HT == 1 || HT == 2, "16 or 32 rows");
    constexpr int kAhead = HT == 2 ? 6 : 4, kAheadV = HT == 2 ? 8 : 4;
    // 16 rows: one chunk buffer (kv_b is kv_a), so that two workgroups share a CU and one's loads run beside the
    // other's work; a chunk is staged between two others' work instead of beside it (64 x 16 heads over 4097 positions: 53
    // to 48.5 us with 8-bit rows, 68 to 62 with bf16 ones)
    constexpr bool SINGLE = HT == 1;
    const int tid = threadIdx.x, lane = tid & 63;
    const int pw = __builtin_amdgcn_readfirstlane(tid >> 6) & (kWavesB - 1);
    const int g = lane >> 4, j = lane & 15;
    const int nchunks = (it.end - it.begin + kChunk - 1) / kChunk;
    const gbytes cache = (gbytes)p.cache;
    const gbytes zero_row = opaque_zero_row();

    // Chunk ck of the walk.  The tiles that read the same rows start their walks at different chunks, so that each
    // row comes from memory once, for one of them, and from L2 for the others.
    const int first = nchunks ? int(uint64_t(it.tile) * uint64_t(nchunks) / uint64_t(it.tiles)) : 0;
    auto start_of = [&](int ck) {
        int c = ck + first;
        c = c >= nchunks ? c - nchunks : c;
        return ck < nchunks ? it.begin + c * kChunk : it.end;      // past the last: no positions
    };

    // ---- staging.  The page of position c0 + lane (past the end, the last position's) and its cache row, or -1.
    // Two steps: memory operations complete in order, so waiting for a page also waits for every older load, and
    // is left until those are wanted anyway.
    auto page_of = [&](int c0) { return it.table[min(c0 + lane, max(it.end - 1, 0)) >> p.page_shift]; };
    auto row_at = [&](int page, int c0) {
        const int pos = c0 + lane;
        const int r = (page << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
        return pos < it.end && uint32_t(page) < uint32_t(p.n_pages) ? r : -1;
    };
    auto row_of = [&](int c0) { return row_at(page_of(c0), c0); };
    auto ptr_of = [&](int rows, int row) {
        const int r = __builtin_amdgcn_ds_bpermute(row << 2, rows);
        return r < 0 ? zero_row : cache + int64_t(r) * p.ld;
    };
    // Columns that the cache lacks read the last ones that it has: Q is zero there, and their outputs are not stored.
    // 8 rows x 128 bytes per LDS-direct load; the wave's rows are 16 pw .. 16 pw + 15
    const uint32_t lat_last = uint32_t(2 * p.kv - 16);
    const StageRows<BIG> stage(p);
    auto stage_bf16 = [&](const typename StageRows<BIG>::Row& row, uint16_t* buf, int cb, int half) {
        const int c_st = (lane & 7) ^ swz(8 * half + (lane >> 3));
        const uint32_t off = cb < 8 ? min(uint32_t(cb * 128 + c_st * 16), lat_last)
                                    : p.rope ? uint32_t(2 * p.kv + min(16 * c_st, 2 * p.rope - 16)) : 0u;
        stage.load(row, off, buf + cb * kBlockElems + (16 * pw + 8 * half) * 64);
    };
    // 8-bit rows, half a chunk at a time: a thread takes pieces 8 i + (tid & 7) of 16 codes of row tid / 8 (+ 32),
    // the row's scales and one piece of RoPE
    constexpr int kHalves = SINGLE ? 2 : 1;        // halves of a chunk held in registers
    u32x4 code[kHalves][4], code_scale[kHalves], code_rope[kHalves];
    const int l8 = tid & 7;
    const uint32_t rope8 = p.rope ? uint32_t(p.kv + kScaleBytes + min(16 * l8, 2 * p.rope - 16)) : 0u;
    auto load_raw = [&](int rows, int ps) {
        const gbytes src = ptr_of(rows, (tid >> 3) + 32 * ps);
        const uint32_t last = uint32_t(p.kv - 16);
        const int k = SINGLE ? ps : 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) code[k][i] = load16(src + min(uint32_t(16 * l8 + 128 * i), last));
        code_scale[k] = load16(src + p.kv);
        code_rope[k] = load16(src + rope8);
    };
    // part i < 4: piece l8 + 8 i, which is pieces 2 (l8 % 4) and + 1 of column block 2 i + l8 / 4; part 4: RoPE's
    const int f8 = swz(tid >> 3), hi8 = l8 >> 2;
    const int w8_first = (tid >> 3) * 64 + hi8 * kBlockElems + (((2 * (l8 & 3) + hi8) ^ f8) << 3);
    const int w8_second = (tid >> 3) * 64 + hi8 * kBlockElems + (((2 * (l8 & 3) + 1 - hi8) ^ f8) << 3);
    const int w8_rope = (tid >> 3) * 64 + 8 * kBlockElems + ((l8 ^ f8) << 3);
    auto commit_part = [&](uint16_t* buf, int ps, int i) {         // ps and i constants where it is called
        uint16_t* const dst = buf + 32 * 64 * ps;
        const int k = SINGLE ? ps : 0;
        if (i == 4) {
            *reinterpret_cast<u32x4*>(dst + w8_rope) = code_rope[k];
        } else {
            const u32x4 q = code[k][i];
            const float s = 16 * (l8 + 8 * i) < p.kv ? scale_of(code_scale[k][i] >> (8 * (l8 >> 1))) : 0.f;
            const uint2 a = dequant4(q[0], s), b = dequant4(q[1], s), c = dequant4(q[2], s), d = dequant4(q[3], s);
            const u32x4 lo{a.x, a.y, b.x, b.y}, up{c.x, c.y, d.x, d.y};
            // lanes 4 to 7 write their upper half first: the eight lanes of a row then hit eight slots
            *reinterpret_cast<u32x4*>(dst + 2 * i * kBlockElems + w8_first) = hi8 ? up : lo;
            *reinterpret_cast<u32x4*>(dst + 2 * i * kBlockElems + w8_second) = hi8 ? lo : up;
        }
    };

    // ---- Q rows to buffer b, in the chunk's layout (rows past the tile's and columns past the cache's: zeros)
    {
        int64_t qo = -1;
        if (lane < it.nrows && lane < HB) qo = row_offset(it.r0 + lane, p.T, p.H, p.sqb, p.sqt, p.ldq);
        for (int ins = pw; ins < 2 * HT * kBlocks; ins += kWavesB) {
            const int cb = ins / (2 * HT), grp = ins - cb * 2 * HT;
            const int row = 8 * grp + (lane >> 3);
            const int c = (lane & 7) ^ swz(row);
            const uint32_t lo = __builtin_amdgcn_ds_bpermute(row << 2, int(uint32_t(qo)));
            const uint32_t hi = __builtin_amdgcn_ds_bpermute(row << 2, int(uint32_t(uint64_t(qo) >> 32)));
            const int64_t o = int64_t((uint64_t(hi) << 32) | lo);
            const bool ok = o >= 0 && (cb < 8 ? 64 * cb + 8 * c < p.kv : 8 * c < p.rope);
            const gbytes src = ok ? (gbytes)(p.q + o + (cb < 8 ? 64 * cb : p.kv) + 8 * c) : zero_row;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                             (lds_void*)(kv_b + cb * kBlockElems + 8 * grp * 64), 16, 0, 0);
        }
    }
    int rows_cur = row_of(start_of(0));
    // (rows_after: 16 rows, 8 bits: what is loaded next)
    auto stage_chunk = [&](int rows, uint16_t* buf, int rows_after) {
        if constexpr (E4M3) {
#pragma unroll
            for (int ps = 0; ps < 2; ++ps) {
                if constexpr (!SINGLE) load_raw(rows, ps);
#pragma unroll
                for (int i = 0; i < 5; ++i) commit_part(buf, ps, i);
                if constexpr (SINGLE) load_raw(rows_after, ps);
            }
        } else {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                const auto rp = stage.row(rows, 16 * pw + 8 * half + (lane >> 3));
#pragma unroll
                for (int cb = 0; cb < kBlocks; ++cb) stage_bf16(rp, buf, cb, half);
            }
        }
    };
    if constexpr (E4M3 && SINGLE) {
        load_raw(rows_cur, 0);
        load_raw(rows_cur, 1);
    }
    if constexpr (!SINGLE) stage_chunk(rows_cur, kv_a, -1);
    int rows_next = row_of(start_of(1));
    __builtin_amdgcn_s_waitcnt(0);
    lds_sync();
    // fragment addresses: row j of a 16-row tile, piece 4 (u & 1) + g of column block u / 2
    const int fj = swz(j);
    const int fr0 = j * 64 + ((g ^ fj) << 3), fr1 = j * 64 + (((4 + g) ^ fj) << 3);
    i32x4 qf[HT][kSteps];
#pragma unroll
    for (int t = 0; t < HT; ++t)
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
            qf[t][u] = *reinterpret_cast<const i32x4*>(kv_b + (u >> 1) * kBlockElems + 16 * t * 64 + (u & 1 ? fr1 : fr0));
    lds_sync();
    // Q in the accumulation half of the register file, which MFMA operands may come from
#pragma unroll
    for (int t = 0; t < HT; ++t)
#pragma unroll
        for (int u = 0; u < kSteps; ++u)
            asm("" : "+a"(qf[t][u]));
    if constexpr (SINGLE) {
        stage_chunk(rows_cur, kv_a, rows_next);
        if constexpr (!E4M3) __builtin_amdgcn_s_waitcnt(0);
        lds_sync();
    } else if constexpr (E4M3) {
        load_raw(rows_next, 0);
    }

    // positions that a row sees: those below its limit
    int limit[HT];
    const int all_see = it.seq >= 0 ? it.len - (p.T - 1) : it.end;    // positions below it are seen by every row
#pragma unroll
    for (int t = 0; t < HT; ++t) {
        limit[t] = it.end;
        if (it.seq >= 0 && p.T > 1) {
            const int tok = (it.r0 + 16 * t + j - it.seq * p.T * p.H) / p.H;
            limit[t] = min(it.end, it.len - (p.T - 1 - tok));
        }
    }

    f32x4 o[kTilesW][HT];     // O^T: lane (g, j) holds columns 16 (pw + 4 i) + 4 g .. + 3 of row 16 t + j
#pragma unroll
    for (int i = 0; i < kTilesW; ++i)
#pragma unroll
        for (int t = 0; t < HT; ++t) o[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_ref[HT], l_acc[HT];
#pragma unroll
    for (int t = 0; t < HT; ++t) {
        m_ref[t] = -INFINITY;
        l_acc[t] = 0.f;
    }
    const int a4 = j >> 2, b4 = j & 3;
    // value fragments: rows 8 g + a4 and + 4 of a k-step, piece 2 pw + b4 / 2 of column block i
    const int vrow = 8 * g + a4;
    const int v_lo = vrow * 64 + (((2 * pw + (b4 >> 1)) ^ swz(vrow)) << 3) + 4 * (b4 & 1);
    const int v_hi = (vrow + 4) * 64 + (((2 * pw + (b4 >> 1)) ^ swz(vrow + 4)) << 3) + 4 * (b4 & 1);

    auto chunk = [&](const uint16_t* cur, uint16_t* nxt, int ck) {
        const int c0 = start_of(ck);
        const uint64_t present = __builtin_amdgcn_ballot_w64(rows_cur >= 0);
        // the next chunk (behind the last: rows of zeros, which nothing reads)
        typename StageRows<BIG>::Row rp[2];
        if constexpr (!E4M3 && !SINGLE) {
            rp[0] = stage.row(rows_next, 16 * pw + (lane >> 3));
            rp[1] = stage.row(rows_next, 16 * pw + 8 + (lane >> 3));
        }
        const int page_after = page_of(start_of(ck + 2));
        int rows_after = -1;

        // ---- S^T, K fragments read kAhead steps ahead, the next chunk's loads between the steps
        f32x4 s[HT];
#pragma unroll
        for (int t = 0; t < HT; ++t) s[t] = f32x4{0.f, 0.f, 0.f, 0.f};
        const uint16_t* krow = cur + 16 * pw * 64;
        auto k_frag = [&](int u) {
            return *reinterpret_cast<const i32x4*>(krow + (u >> 1) * kBlockElems + (u & 1 ? fr1 : fr0));
        };
        i32x4 kf[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) kf[u] = k_frag(u);
#pragma unroll
        for (int u = 0; u < kSteps; ++u) {
#pragma unroll
            for (int t = 0; t < HT; ++t)
                s[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[u % kAhead]), as_bf16x8(qf[t][u]), s[t], 0, 0, 0);
            if (u + kAhead < kSteps) kf[u % kAhead] = k_frag(u + kAhead);
            if constexpr (SINGLE) {
            } else if constexpr (E4M3) {
                // the first half of the next chunk's rows, in the MFMAs' shadow
                if (u % 3 == 2 && u < 15) commit_part(nxt, 0, u / 3);
                if (u == 15) load_raw(rows_next, 1);
            } else {
                stage_bf16(rp[u & 1], nxt, u >> 1, u & 1);
            }
            __builtin_amdgcn_sched_barrier(0);
        }

        // ---- scores in log2 units, masked where some row does not see all 64 positions, and the wave's maximum
        // per row
        const int at = 16 * pw + 4 * g;
        float mx[HT];
        bool need = false;
#pragma unroll
        for (int t = 0; t < HT; ++t) s[t] *= p.scale_log2;
        if (present != ~uint64_t(0) || c0 + kChunk > all_see) {
            const uint32_t here = uint32_t(present >> at);
#pragma unroll
            for (int t = 0; t < HT; ++t)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[t][i] = ((here >> i) & 1u) && c0 + at + i < limit[t] ? s[t][i] : -INFINITY;
        }
#pragma unroll
        for (int t = 0; t < HT; ++t) {
            mx[t] = cols4_max(fmaxf(fmaxf(s[t][0], s[t][1]), fmaxf(s[t][2], s[t][3])));
            need |= !(mx[t] <= m_ref[t] + kLazy);
        }
        float lc[HT];
        auto write_p = [&]() {
#pragma unroll
            for (int t = 0; t < HT; ++t) {
                // (a row that has seen nothing yet: 2^(-inf - 0) = 0)
                const float m = m_ref[t] == -INFINITY ? 0.f : m_ref[t];
                float pv[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) pv[i] = __builtin_amdgcn_exp2f(s[t][i] - m);
                lc[t] = (pv[0] + pv[1]) + (pv[2] + pv[3]);
                *reinterpret_cast<uint2*>(pbuf + (16 * t + j) * kPPitchB + at) =
                    uint2{pack2(pv[0], pv[1]), pack2(pv[2], pv[3])};
            }
        };
        if (g == 0) {
#pragma unroll
            for (int t = 0; t < HT; ++t) red[pw * HB + 16 * t + j] = mx[t];
        }
        bool any = ck == 0;
        if (ck > 0) {
            write_p();
            const bool wave_needs = __builtin_amdgcn_ballot_w64(need) != 0;
            if (lane == 0) flags[pw] = wave_needs ? 1 : 0;
        }
        lds_sync();
        if (ck > 0) {
            const i32x4 f0 = *reinterpret_cast<const i32x4*>(flags);
            any = (f0[0] | f0[1] | f0[2] | f0[3]) != 0;
        }
        // a reference moves (every wave reads the same maxima): the output rescaled, P written again
        if (any) {
            bool resc = false;
            float alpha[HT];
#pragma unroll
            for (int t = 0; t < HT; ++t) {
                const int hh = 16 * t + j;
                const float mc = fmaxf(fmaxf(red[hh], red[HB + hh]), fmaxf(red[2 * HB + hh], red[3 * HB + hh]));
                alpha[t] = 1.f;
                if (mc > m_ref[t] + kLazy) {
                    alpha[t] = (m_ref[t] == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m_ref[t] - mc);
                    m_ref[t] = mc;
                    l_acc[t] *= alpha[t];
                    resc = true;
                }
            }
            if (__builtin_amdgcn_ballot_w64(resc)) {
#pragma unroll
                for (int i = 0; i < kTilesW; ++i)
#pragma unroll
                    for (int t = 0; t < HT; ++t) o[i][t] *= alpha[t];
            }
            write_p();
            lds_sync();
        }
#pragma unroll
        for (int t = 0; t < HT; ++t) l_acc[t] += lc[t];

        // ---- O^T += V^T P^T: step v is column tile v % 8 of positions 32 (v / 8) .. + 31
        auto p_frag = [&](int t, int kk) {
            return *reinterpret_cast<const i32x4*>(pbuf + (16 * t + j) * kPPitchB + 32 * kk + 8 * g);
        };
        auto v_frag = [&](int v) {
            const uint16_t* base = cur + (v % kTilesW) * kBlockElems + 32 * (v / kTilesW) * 64;
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(base + v_lo));
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(base + v_hi));
            const uint2 ulo = __builtin_bit_cast(uint2, lo), uhi = __builtin_bit_cast(uint2, hi);
            return i32x4{int(ulo.x), int(ulo.y), int(uhi.x), int(uhi.y)};
        };
        i32x4 pf[HT], vf[kAheadV];
#pragma unroll
        for (int t = 0; t < HT; ++t) pf[t] = p_frag(t, 0);
#pragma unroll
        for (int v = 0; v < kAheadV; ++v) vf[v] = v_frag(v);
#pragma unroll
        for (int v = 0; v < 2 * kTilesW; ++v) {
            const int i = v % kTilesW;
#pragma unroll
            for (int t = 0; t < HT; ++t) {
                o[i][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[v % kAheadV]), as_bf16x8(pf[t]), o[i][t], 0, 0, 0);
                if (v == kTilesW - 1) pf[t] = p_frag(t, 1);
            }
            if (v + kAheadV < 2 * kTilesW) vf[v % kAheadV] = v_frag(v + kAheadV);
            if constexpr (E4M3 && !SINGLE) {
                // the second half of the next chunk's rows; then the loads of the one after it
                if (v % 3 == 2 && v < 15) commit_part(nxt, 1, v / 3);
                if (v == 15) {
                    rows_after = row_at(page_after, start_of(ck + 2));
                    load_raw(rows_after, 0);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (SINGLE) {
            // every wave is done with this chunk: the next one takes its place, and as its registers fall free the one
            // after it is loaded
            lds_sync();
            rows_after = row_at(page_after, start_of(ck + 2));
            stage_chunk(rows_next, nxt, rows_after);
        }
        // the next chunk has landed, and every wave is done with this one and with P
        if constexpr (!E4M3) __builtin_amdgcn_s_waitcnt(0);
        if constexpr (!E4M3 && !SINGLE) rows_after = row_at(page_after, start_of(ck + 2));
        rows_cur = rows_next;
        rows_next = rows_after;
        lds_sync();
    };
    for (int ck = 0; ck < nchunks; ck += 2) {
        chunk(kv_a, kv_b, ck);
        if (ck + 1 < nchunks) chunk(kv_b, kv_a, ck + 1);
    }

    // ---- the rows' sums: the wave's four lanes of a row, then the waves in order
#pragma unroll
    for (int t = 0; t < HT; ++t) {
        const float lw = cols4_sum(l_acc[t]);
        if (g == 0) red[pw * HB + 16 * t + j] = lw;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < HT; ++t) {
        const int row = 16 * t + j;
        const float lsum = ((red[row] + red[HB + row]) + red[2 * HB + row]) + red[3 * HB + row];
        store_row<HT>(p, it, row, pw, g, o, t, m_ref[t], lsum);
    }
}

// A tile of 64 rows over a span, in chunks of 32 positions, software-pipelined: while chunk i's scores go through
// the softmax (vector units), the matrix cores work on chunk i + 1's, and chunk i + 3 is on its way into a ring of four
// buffers [9 column blocks][32 rows][8 pieces].
//  * S^T of a chunk: wave w takes positions 16 (w % 2) .. + 15 and half of the columns (9 of 18 steps), for all 64
//    rows: half of Q in its registers (64 rows x 288 columns), every key fragment read from LDS once and used by four MFMAs.
//    The two halves of a sum meet through LDS: each wave finishes two of the four row tiles.
//  * Per chunk: QK(i + 1) with softmax(i), barrier (P, maxima, half sums and chunk i + 2 are there), PV(i),
//    barrier (chunk i's buffer is free).
template <bool E4M3, bool BIG>
__device__ __forceinline__ void wide_block(const BatchParams& p, const Item it, uint16_t* const b0, uint16_t* const b1,
                                           uint16_t* const b2, uint16_t* const b3, uint16_t* const pbuf, float* const xbuf,
                                           float* const red, int* const flags) {
    constexpr int kPos = 32, kBlk = kPos * 64;
    constexpr int kHalf = kSteps / 2, kAheadK = 4, kAheadV = 4, kPitch = kPos + 8;
    const int tid = threadIdx.x, lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6) & 3;
    const int pg = wave & 1, dh = wave >> 1;
    const int g = lane >> 4, j = lane & 15;
    const int n = (it.end - it.begin + kPos - 1) / kPos;
    const gbytes cache = (gbytes)p.cache;
    const gbytes zero_row = opaque_zero_row();

    // the walk, as in narrow_block
    const int first = n ? int(uint64_t(it.tile) * uint64_t(n) / uint64_t(it.tiles)) : 0;
    auto start_of = [&](int ck) {
        int c = ck + first;
        c = c >= n ? c - n : c;
        return ck < n ? it.begin + c * kPos : it.end;
    };
    auto page_of = [&](int c0) { return it.table[min(c0 + (lane & 31), max(it.end - 1, 0)) >> p.page_shift]; };
    auto row_at = [&](int page, int c0) {
        const int pos = c0 + (lane & 31);
        const int r = (page << p.page_shift) + (pos & ((1 << p.page_shift) - 1));
        return pos < it.end && uint32_t(page) < uint32_t(p.n_pages) ? r : -1;
    };
    auto row_of = [&](int c0) { return row_at(page_of(c0), c0); };
    auto ptr_of = [&](int rows, int row) {
        const int r = __builtin_amdgcn_ds_bpermute(row << 2, rows);
        return r < 0 ? zero_row : cache + int64_t(r) * p.ld;
    };
    auto present_of = [&](int rows) { return uint32_t(__builtin_amdgcn_ballot_w64(rows >= 0)); };
    // bf16 rows: wave w stages rows 8 w .. 8 w + 7, a column block a load
    const int c_st = (lane & 7) ^ swz(8 * wave + (lane >> 3));
    const uint32_t lat_last = uint32_t(2 * p.kv - 16);
    const uint32_t rope_off = p.rope ? uint32_t(2 * p.kv + min(16 * c_st, 2 * p.rope - 16)) : 0u;
    const StageRows<BIG> stage(p);
    auto stage_bf16 = [&](const typename StageRows<BIG>::Row& row, uint16_t* buf, int cb) {
        const uint32_t off = cb < 8 ? min(uint32_t(cb * 128 + (c_st ^ (cb & 1)) * 16), lat_last) : rope_off;
        stage.load(row, off, buf + cb * kBlk + 8 * wave * 64);
    };
    // 8-bit rows: a thread takes pieces 8 i + (tid & 7) of row tid / 8
    u32x4 code0, code1, code2, code3, code_scale, code_rope;
    const int l8 = tid & 7, r8 = tid >> 3, f8 = swz(r8), hi8 = l8 >> 2;
    const uint32_t rope8 = p.rope ? uint32_t(p.kv + kScaleBytes + min(16 * l8, 2 * p.rope - 16)) : 0u;
    auto load_part = [&](gbytes src, int i) {
        const uint32_t last = uint32_t(p.kv - 16);
        if (i == 0) code0 = load16(src + min(uint32_t(16 * l8), last));
        if (i == 1) code1 = load16(src + min(uint32_t(16 * l8 + 128), last));
        if (i == 2) code2 = load16(src + min(uint32_t(16 * l8 + 256), last));
        if (i == 3) code3 = load16(src + min(uint32_t(16 * l8 + 384), last));
        if (i == 4) code_scale = load16(src + p.kv);
        if (i == 5) code_rope = load16(src + rope8);
    };
    auto load_raw = [&](int rows) {
        const gbytes src = ptr_of(rows, r8);
#pragma unroll
        for (int i = 0; i < 6; ++i) load_part(src, i);
    };
    // Piece l8 + 8 i is pieces 2 (l8 % 4) and + 1 of column block 2 i + l8 / 4; with the odd blocks' slots the eight
    // lanes of a row write eight different ones.
    const int w8_lo = r8 * 64 + hi8 * kBlk + (((2 * (l8 & 3) + hi8) ^ f8) << 3), w8_up = w8_lo ^ 8;
    const int w8_rope = r8 * 64 + 8 * kBlk + ((l8 ^ f8) << 3);
    float c_scale = 0.f;
    uint2 c_a, c_b, c_c, c_d;
    // part i, in five slices; part 4 (RoPE's) in one
    auto commit = [&](uint16_t* dst, auto part, int slice) {
        constexpr int i = decltype(part)::value;
        if constexpr (i == 4) {
            if (slice == 0) *reinterpret_cast<u32x4*>(dst + w8_rope) = code_rope;
        } else {
            const u32x4 q = i == 0 ? code0 : i == 1 ? code1 : i == 2 ? code2 : code3;
            if (slice == 0) c_scale = 16 * (l8 + 8 * i) < p.kv ? scale_of(code_scale[i] >> (8 * (l8 >> 1))) : 0.f;
            if (slice == 1) {
                c_a = dequant4(q[0], c_scale);
                c_b = dequant4(q[1], c_scale);
            }
            if (slice == 2) *reinterpret_cast<u32x4*>(dst + 2 * i * kBlk + w8_lo) = u32x4{c_a.x, c_a.y, c_b.x, c_b.y};
            if (slice == 3) {
                c_c = dequant4(q[2], c_scale);
                c_d = dequant4(q[3], c_scale);
            }
            if (slice == 4) *reinterpret_cast<u32x4*>(dst + 2 * i * kBlk + w8_up) = u32x4{c_c.x, c_c.y, c_d.x, c_d.y};
        }
    };
    auto commit_at = [&](uint16_t* buf, int part, int slice) {       // constants where it is called
        if (part == 0) commit(buf, std::integral_constant<int, 0>{}, slice);
        if (part == 1) commit(buf, std::integral_constant<int, 1>{}, slice);
        if (part == 2) commit(buf, std::integral_constant<int, 2>{}, slice);
        if (part == 3) commit(buf, std::integral_constant<int, 3>{}, slice);
        if (part == 4) commit(buf, std::integral_constant<int, 4>{}, slice);
    };
    auto stage_all = [&](int rows, uint16_t* buf) {
        if constexpr (E4M3) {
            load_raw(rows);
#pragma unroll
            for (int i = 0; i < 25; ++i) commit_at(buf, i / 5, i % 5);
        } else {
            const auto rp = stage.row(rows, 8 * wave + (lane >> 3));
#pragma unroll
            for (int cb = 0; cb < kBlocks; ++cb) stage_bf16(rp, buf, cb);
        }
    };

    // ---- chunks 0 and 1 to buffers 0 and 1; Q's rows to buffers 2 (rows 0 to 31) and 3, in the same layout
    const int rows0 = row_of(start_of(0)), rows1 = row_of(start_of(1)), rows2 = row_of(start_of(2));
    int page3 = page_of(start_of(3));
    {
        int64_t qo = -1;
        if (lane < it.nrows) qo = row_offset(it.r0 + lane, p.T, p.H, p.sqb, p.sqt, p.ldq);
        for (int ins = wave; ins < 8 * kBlocks; ins += kWavesB) {
            const int cb = ins >> 3, grp = ins & 7;
            const int row = 8 * grp + (lane >> 3);
            const int c = (lane & 7) ^ swz(row) ^ (cb & 1);
            const uint32_t lo = __builtin_amdgcn_ds_bpermute(row << 2, int(uint32_t(qo)));
            const uint32_t hi = __builtin_amdgcn_ds_bpermute(row << 2, int(uint32_t(uint64_t(qo) >> 32)));
            const int64_t o = int64_t((uint64_t(hi) << 32) | lo);
            const bool ok = o >= 0 && (cb < 8 ? 64 * cb + 8 * c < p.kv : 8 * c < p.rope);
            const gbytes src = ok ? (gbytes)(p.q + o + (cb < 8 ? 64 * cb : p.kv) + 8 * c) : zero_row;
            __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)src,
                                             (lds_void*)((grp < 4 ? b2 : b3) + cb * kBlk + 8 * (grp & 3) * 64), 16, 0, 0);
        }
    }
    stage_all(rows0, b0);
    stage_all(rows1, b1);
    uint32_t here0 = present_of(rows0), here1 = present_of(rows1), here2 = present_of(rows2), here3 = 0;
    __builtin_amdgcn_s_waitcnt(0);
    lds_sync();
    // The wave's k-steps are 9 dh + u: row j of a 16-row tile, piece 4 (step % 2) + g of column block step / 2, which is
    // (u / 2) + (0 or, with dh, 4 for even u and 5 for odd); odd blocks have the other slots.
    const int fj = swz(j);
    const int fr0 = j * 64 + ((g ^ fj) << 3), fr1 = j * 64 + (((4 + g) ^ fj) << 3);
    const int fr_even = dh ? fr1 + 4 * kBlk : fr0, fr_odd = dh ? (fr0 ^ 8) + 5 * kBlk : fr1;
    auto frag = [&](const uint16_t* rows16, int u) {
        const int at = u & 1 ? fr_odd : fr_even;
        return *reinterpret_cast<const i32x4*>(rows16 + ((u >> 1) & 1 ? at ^ 8 : at) + (u >> 1) * kBlk);
    };
    i32x4 qf[4][kHalf];
    // local tile t is row tile (t + 2 dh) % 4: the wave finishes its local tiles 0 and 1
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < kHalf; ++u) qf[t][u] = frag(((t < 2) == (dh == 0) ? b2 : b3) + 1024 * (t & 1), u);
    lds_sync();
    // Q in the accumulation half of the register file, which MFMA operands may come from (said so: the compiler
    // keeps it there as spills otherwise, with a copy before every use)
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
        for (int u = 0; u < kHalf; ++u) asm("" : "+a"(qf[t][u]));
    stage_all(rows2, b2);
    if constexpr (E4M3) {
        const int rows3 = row_at(page3, start_of(3));
        here3 = present_of(rows3);
        load_raw(rows3);
    }

    const int all_see = it.seq >= 0 ? it.len - (p.T - 1) : it.end;    // positions below it are seen by every row
    int limit[2];                                                     // of the wave's own two row tiles
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        limit[k] = it.end;
        if (it.seq >= 0 && p.T > 1) {
            const int tok = (it.r0 + 32 * dh + 16 * k + j - it.seq * p.T * p.H) / p.H;
            limit[k] = min(it.end, it.len - (p.T - 1 - tok));
        }
    }

    f32x4 o[kTilesW][4];      // O^T: lane (g, j) holds columns 16 (wave + 4 i) + 4 g .. + 3 of row 16 t + j
#pragma unroll
    for (int i = 0; i < kTilesW; ++i)
#pragma unroll
        for (int t = 0; t < 4; ++t) o[i][t] = f32x4{0.f, 0.f, 0.f, 0.f};
    float m_ref[4], l_acc[2] = {0.f, 0.f};     // references of every row tile, sums of the wave's own
#pragma unroll
    for (int t = 0; t < 4; ++t) m_ref[t] = -INFINITY;
    const int a4 = j >> 2, b4 = j & 3;
    const int vrow = 8 * g + a4;
    const int v_lo = vrow * 64 + (((2 * wave + (b4 >> 1)) ^ swz(vrow)) << 3) + 4 * (b4 & 1);
    const int v_hi = (vrow + 4) * 64 + (((2 * wave + (b4 >> 1)) ^ swz(vrow + 4)) << 3) + 4 * (b4 & 1);
    float* const x_mine = xbuf + (wave * 2 * 64 + lane) * 4;
    const float* const x_other = xbuf + ((wave ^ 2) * 2 * 64 + lane) * 4;

    f32x4 sp[4], s[2];
    // QK of a chunk: one step of the wave's nine
    auto k_frag = [&](const uint16_t* buf, int u) { return frag(buf + 1024 * pg, u); };
    auto qk_mfma = [&](const i32x4 (&kf)[kAheadK], int u, int t) {
        sp[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kf[u % kAheadK]), as_bf16x8(qf[t][u]),
                                                        u ? sp[t] : f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
    };
    auto x_write = [&]() {
        *reinterpret_cast<f32x4*>(x_mine) = sp[2];
        *reinterpret_cast<f32x4*>(x_mine + 256) = sp[3];
    };
    // The finished scores of the wave's own two tiles in log2 units, masked where some row does not see every position.
    auto x_load = [&](f32x4 (&x)[2]) {
        // local tiles 0 and 1 of this wave are tiles 2 and 3 of the other
        x[0] = *reinterpret_cast<const f32x4*>(x_other);
        x[1] = *reinterpret_cast<const f32x4*>(x_other + 256);
    };
    const int at = 16 * pg + 4 * g;
    auto scale_scores = [&](const f32x4 (&x)[2], int k) { s[k] = (sp[k] + x[k]) * p.scale_log2; };
    auto mask_scores = [&](uint32_t here, int c0) {
        if (here != ~0u || c0 + kPos > all_see) {
            const uint32_t bits = here >> at;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int e = 0; e < 4; ++e) s[k][e] = ((bits >> e) & 1u) && c0 + at + e < limit[k] ? s[k][e] : -INFINITY;
        }
    };
    i32x4 kf[kAheadK];        // the next chunk's first key fragments
    if (n > 0) {
#pragma unroll
        for (int u = 0; u < kAheadK; ++u) kf[u] = k_frag(b0, u);
#pragma unroll
        for (int u = 0; u < kHalf; ++u) {
#pragma unroll
            for (int t = 0; t < 4; ++t) qk_mfma(kf, u, t);
            if (u + kAheadK < kHalf) kf[u % kAheadK] = k_frag(b0, u + kAheadK);
        }
        x_write();
        lds_sync();
        f32x4 x[2];
        x_load(x);
        scale_scores(x, 0);
        scale_scores(x, 1);
        mask_scores(here0, start_of(0));
#pragma unroll
        for (int u = 0; u < kAheadK; ++u) kf[u] = k_frag(b1, u);
        if constexpr (!E4M3) __builtin_amdgcn_s_waitcnt(0);     // (chunk 2)
        lds_sync();
    }

    // chunk i lies in cur, i + 1 in next, i + 2 in after; fill, chunk i - 1's, takes chunk i + 3
    auto step = [&](auto last_c, int i, const uint16_t* const cur, const uint16_t* const next, const uint16_t* const after,
                    uint16_t* const fill) {
        constexpr bool LAST = decltype(last_c)::value;
        gbytes rp = zero_row;
        typename StageRows<BIG>::Row row3{};
        if constexpr (!E4M3) {
            const int rows3 = row_at(page3, start_of(i + 3));
            here3 = present_of(rows3);
            row3 = stage.row(rows3, 8 * wave + (lane >> 3));
        }
        const int page4 = page_of(start_of(i + 4));
        uint32_t here4 = 0;
        auto v_frag = [&](int v) {
            const uint16_t* base = cur + v * kBlk;
            const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(base + (v & 1 ? v_lo ^ 8 : v_lo)));
            const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(base + (v & 1 ? v_hi ^ 8 : v_hi)));
            const uint2 ulo = __builtin_bit_cast(uint2, lo), uhi = __builtin_bit_cast(uint2, hi);
            return i32x4{int(ulo.x), int(ulo.y), int(uhi.x), int(uhi.y)};
        };
        auto p_frag = [&](int t) { return *reinterpret_cast<const i32x4*>(pbuf + (16 * t + j) * kPitch + 8 * g); };

        // ---- softmax(i) beside QK(i + 1).  An MFMA takes the matrix core 16 cycles, three vector instructions' time,
        // and a wave issues in order: the softmax is cut into slices, one after each MFMA, kept there by scheduling
        // barriers (left to itself the compiler runs one after the other).
        float mx[2], mr[2], lc[2], pv[2][4];
        bool need = false;
        auto soft_max = [&](int k, int slice) {
            if (slice == 0) mx[k] = fmaxf(fmaxf(s[k][0], s[k][1]), fmaxf(s[k][2], s[k][3]));
            if (slice == 1) mx[k] = rows_max32(mx[k]);
            if (slice == 2) mx[k] = rows_max16(mx[k]);
        };
        auto reference = [&](int k) {
            const float m = dh ? m_ref[2 + k] : m_ref[k];
            need |= !(mx[k] <= m + kLazy);
            mr[k] = m == -INFINITY ? 0.f : m;      // (a row that has seen nothing: 2^(-inf - 0) = 0)
        };
        auto put_p = [&](int k) {
            *reinterpret_cast<uint2*>(pbuf + (32 * dh + 16 * k + j) * kPitch + at) =
                uint2{pack2(pv[k][0], pv[k][1]), pack2(pv[k][2], pv[k][3])};
        };
        i32x4 pf[4], vf[kAheadV];
        auto soft = [&](int m) {
            if (m < 6) soft_max(m & 1, m >> 1);
            if (m == 6 || m == 7) reference(m - 6);
            if (m >= 8 && m < 16) pv[(m - 8) / 4][m % 4] = __builtin_amdgcn_exp2f(s[(m - 8) / 4][m % 4] - mr[(m - 8) / 4]);
            if (m == 16 || m == 18) lc[(m - 16) / 2] = (pv[(m - 16) / 2][0] + pv[(m - 16) / 2][1]) + (pv[(m - 16) / 2][2] + pv[(m - 16) / 2][3]);
            if (m == 17 || m == 19) put_p((m - 17) / 2);
            // (every lane of a row writes the same maximum, every lane of a wave the same flag: no branch)
            if (m == 20 || m == 21) red[pg * 64 + 32 * dh + 16 * (m - 20) + j] = mx[m - 20];
            if (m == 22) flags[wave] = __builtin_amdgcn_ballot_w64(need) != 0 ? 1 : 0;
            if (m >= 28 && m % 2 == 0 && (m - 28) / 2 < kAheadV) vf[(m - 28) / 2] = v_frag((m - 28) / 2);
        };
#pragma unroll
        for (int m = 0; m < 4 * kHalf; ++m) {
            // (the other wave's tiles first: they go to LDS behind the last step)
            const int u = m / 4, t = (m + 2) % 4;
            if constexpr (!LAST) {
                qk_mfma(kf, u, t);
                if (m % 4 == 3 && u + kAheadK < kHalf) kf[u % kAheadK] = k_frag(next, u + kAheadK);
                if constexpr (!E4M3) {
                    if (m % 8 == 3) stage_bf16(row3, fill, m / 8);
                }
            }
            soft(m);
            if constexpr (!LAST) __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!LAST) {
            x_write();
            // chunk i + 2 has landed once at most this phase's loads are on their way
            if constexpr (!E4M3) attn::wait_vm<(4 * kHalf + 4) / 8>();
        }
        lds_sync();
        const i32x4 f0 = *reinterpret_cast<const i32x4*>(flags);
#pragma unroll
        for (int t = 0; t < 4; ++t) pf[t] = p_frag(t);
        f32x4 x[2];
        if constexpr (!LAST) x_load(x);
        if ((f0[0] | f0[1] | f0[2] | f0[3]) != 0) {
            // a reference moves (every wave reads the same maxima): the output rescaled, P written again
            float alpha[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) {
                const float mc = fmaxf(red[16 * t + j], red[64 + 16 * t + j]);
                alpha[t] = 1.f;
                if (mc > m_ref[t] + kLazy) {
                    alpha[t] = (m_ref[t] == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(m_ref[t] - mc);
                    m_ref[t] = mc;
                }
            }
#pragma unroll
            for (int k = 0; k < 2; ++k) l_acc[k] *= dh ? alpha[2 + k] : alpha[k];
#pragma unroll
            for (int q = 0; q < kTilesW; ++q)
#pragma unroll
                for (int t = 0; t < 4; ++t) o[q][t] *= alpha[t];
            lds_sync();                  // (every wave has read the P that is written again)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                reference(k);
#pragma unroll
                for (int e = 0; e < 4; ++e) pv[k][e] = __builtin_amdgcn_exp2f(s[k][e] - mr[k]);
                lc[k] = (pv[k][0] + pv[k][1]) + (pv[k][2] + pv[k][3]);
                put_p(k);
            }
            lds_sync();
#pragma unroll
            for (int t = 0; t < 4; ++t) pf[t] = p_frag(t);
        }
        l_acc[0] += lc[0];
        l_acc[1] += lc[1];

        // ---- PV(i), and (the rest of) the staging of chunk i + 3 in slices beside it
#pragma unroll
        for (int m = 0; m < 4 * kTilesW; ++m) {
            const int v = m / 4, t = m % 4;
            if constexpr (!LAST && E4M3) {
                // (the first slices before the first MFMA, which waits for P)
                if (m == 0) {
                    commit_at(fill, 0, 0);
                    commit_at(fill, 0, 1);
                    commit_at(fill, 0, 2);
                    commit_at(fill, 0, 3);
                }
            }
            o[v][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(vf[v % kAheadV]), as_bf16x8(pf[t]), o[v][t], 0, 0, 0);
            if (t == 3 && v + kAheadV < kTilesW) vf[v % kAheadV] = v_frag(v + kAheadV);
            if constexpr (!LAST) {
                if (m >= 22 && m < 30 && m % 2 == 0) kf[(m - 22) / 2] = k_frag(after, (m - 22) / 2);
                if (m == 29 || m == 30) scale_scores(x, m - 29);
                if constexpr (E4M3) {
                    if (m == 0) commit_at(fill, 0, 4);
                    if (m >= 2 && m < 17) commit_at(fill, 1 + (m - 2) / 5, (m - 2) % 5);
                    if (m == 17) commit_at(fill, 4, 0);
                    // chunk i + 4's loads, as chunk i + 3's registers come free
                    if (m == 6) {
                        const int rows4 = row_at(page4, start_of(i + 4));
                        here4 = present_of(rows4);
                        rp = ptr_of(rows4, r8);
                    }
                    if (m == 9 || m == 13) load_part(rp, (m - 9) / 4);
                    if (m == 18 || m == 21 || m == 24 || m == 27) load_part(rp, 2 + (m - 18) / 3);
                } else if (m % 7 == 4) {
                    stage_bf16(row3, fill, 5 + m / 7);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        if constexpr (!LAST) mask_scores(here1, start_of(i + 1));
        here0 = here1;
        here1 = here2;
        here2 = here3;
        here3 = here4;
        page3 = page4;
        if constexpr (!LAST) lds_sync();      // every wave is done with chunk i, and its part of chunk i + 3 is written
    };
    // (four buffers by name, so that the compiler sees which of them a staging load writes)
    for (int i = 0; i + 1 < n; i += 4) {
        step(std::false_type{}, i, b0, b1, b2, b3);
        if (i + 2 < n) step(std::false_type{}, i + 1, b1, b2, b3, b0);
        if (i + 3 < n) step(std::false_type{}, i + 2, b2, b3, b0, b1);
        if (i + 4 < n) step(std::false_type{}, i + 3, b3, b0, b1, b2);
    }
    if (n > 0) {
        const int last = (n - 1) & 3;
        step(std::true_type{}, n - 1, last == 0 ? b0 : last == 1 ? b1 : last == 2 ? b2 : b3, nullptr, nullptr, nullptr);
    }

    // (the loads of the chunks behind the last, and of a span without positions: none may write LDS after the workgroup has left)
    if constexpr (!E4M3) __builtin_amdgcn_s_waitcnt(0);

    // ---- the rows' sums: a wave's four lanes of a row, then the two position groups
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const float lw = cols4_sum(l_acc[k]);
        if (g == 0) red[128 + pg * 64 + 32 * dh + 16 * k + j] = lw;
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < 4; ++t) {
        const int row = 16 * t + j;
        store_row<4>(p, it, row, wave, g, o, t, m_ref[t], red[128 + row] + red[192 + row]);
    }
}

// Workgroup ids go round the 8 XCDs: id b of a range of items padded to a multiple of 8 takes an item such that
// each XCD gets a run of consecutive ones, which read the same cache rows through its L2.  -1: padding.
__device__ __forceinline__ int xcd_run(int b, int items) {
    const int per = (items + 7) >> 3;
    const int v = (b & 7) * per + (b >> 3);
    return v < items ? v : -1;
}

// The item of a workgroup, in tiles of TR rows; false: none.
template <int TR>
__device__ __forceinline__ bool item_of(const BatchParams& p, Item* out) {
    const int bid = static_cast<int>(blockIdx.x);
    Item it;
    if (bid < p.pre_grid) {
        const int v = xcd_run(bid, p.pre_items);
        if (v < 0) return false;
        const int sp = v / p.pre_tiles, tile = v - sp * p.pre_tiles;
        it.r0 = tile * TR;
        it.nrows = min(TR, p.rows - it.r0);
        it.seq = -1;
        it.table = p.prefix_pages;
        it.begin = sp * p.pre_span;
        it.end = min(p.prefix_len, it.begin + p.pre_span);
        it.len = 0;
        it.slot = sp;
        it.tile = tile;
        it.tiles = p.pre_tiles;
    } else {
        const int v = xcd_run(bid - p.pre_grid, p.own_items);
        if (v < 0) return false;
        const int unit = v / p.own_tiles, tile = v - unit * p.own_tiles;
        const int b = unit / p.own_spans, sp = unit - b * p.own_spans;
        const int th = p.T * p.H;
        it.r0 = b * th + tile * TR;
        it.nrows = min(TR, th - tile * TR);
        it.seq = b;
        it.table = p.pages + b * p.ld_pages;
        it.len = max(0, min(p.lens[b], p.max_len));
        it.begin = sp * p.own_span;
        it.end = min(it.len, it.begin + p.own_span);
        it.slot = p.pre_spans + sp;
        it.tile = tile;
        it.tiles = p.own_tiles;
        if (it.begin >= it.end && !p.direct) return false;     // the merge knows how many spans a sequence has
        it.end = max(it.end, it.begin);
    }
    *out = it;
    return true;
}

template <int HT, bool E4M3, bool BIG>
__global__ __launch_bounds__(kThreadsB, HT == 1 ? 2 : 1) void attention_batch_kernel(const BatchParams p) {
    __shared__ __attribute__((aligned(128))) uint16_t kv_a[kBlocks * kBlockElems];
    __shared__ __attribute__((aligned(128))) uint16_t kv_b[HT == 1 ? 64 : kBlocks * kBlockElems];
    __shared__ __attribute__((aligned(16))) uint16_t pbuf[16 * HT * kPPitchB];
    __shared__ __attribute__((aligned(16))) float red[kWavesB * 16 * HT];
    __shared__ __attribute__((aligned(16))) int flags[4];
    Item it;
    if (item_of<16 * HT>(p, &it)) narrow_block<HT, E4M3, BIG>(p, it, kv_a, HT == 1 ? kv_a : kv_b, pbuf, red, flags);
}

template <bool E4M3, bool BIG>
__global__ __launch_bounds__(kThreadsB) void attention_batch_wide_kernel(const BatchParams p) {
    constexpr int kElems = kBlocks * 32 * 64;
    __shared__ __attribute__((aligned(128))) uint16_t b0[kElems];
    __shared__ __attribute__((aligned(128))) uint16_t b1[kElems];
    __shared__ __attribute__((aligned(128))) uint16_t b2[kElems];
    __shared__ __attribute__((aligned(128))) uint16_t b3[kElems];
    __shared__ __attribute__((aligned(16))) uint16_t pbuf[64 * (32 + 8)];
    __shared__ __attribute__((aligned(16))) float xbuf[4 * 2 * 64 * 4];
    __shared__ __attribute__((aligned(16))) float red[256];
    __shared__ __attribute__((aligned(16))) int flags[4];
    Item it;
    if (item_of<64>(p, &it)) wide_block<E4M3, BIG>(p, it, b0, b1, b2, b3, pbuf, xbuf, red, flags);
}

// out = sum_s w_s O_s / sum_s w_s l_s, w_s = 2^(m_s - max m), the prefix's spans, then the sequence's own.  A block
// takes a row, a thread four columns; lane s of each wave weighs slot s.
constexpr int kMergeT = 128;
// BATCH: slots loaded at once, before the sequence's length is known; what a slot that was not written holds is dropped
template <int BATCH>
__global__ __launch_bounds__(kMergeT) void attention_batch_merge_kernel(const BatchParams p) {
    const int r = static_cast<int>(blockIdx.x), lane = threadIdx.x & 63;
    const int b = r / (p.T * p.H);
    const int c = 4 * static_cast<int>(threadIdx.x);
    const bool has = c < p.kv;
    const int slots = p.pre_spans + p.own_spans;
    const float* src = p.part_o + int64_t(r) * p.kv + (has ? c : 0);
    const int64_t step = int64_t(p.rows) * p.kv;
    f32x4 v[BATCH];
#pragma unroll
    for (int u = 0; u < BATCH; ++u) v[u] = *reinterpret_cast<const f32x4*>(src + int64_t(min(u, slots - 1)) * step);
    float2 ml = *reinterpret_cast<const float2*>(p.part_ml + (int64_t(min(lane, slots - 1)) * p.rows + r) * 2);
    int n = p.pre_spans;
    if (p.own_spans) {
        const int len = max(0, min(p.lens[b], p.max_len));
        n += (len + p.own_span - 1) / p.own_span;
    }
    n = __builtin_amdgcn_readfirstlane(n);
    if (lane >= n) ml = float2{-INFINITY, 0.f};
    const float top = wave_max(ml.x);
    // a NaN reference cannot occur (a maximum skips NaN); a NaN sum stays one
    const float w = (ml.x == -INFINITY) ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
    const float total = wave_sum(w * ml.y);
    f32x4 acc{0.f, 0.f, 0.f, 0.f};
    for (int s0 = 0; s0 < n; s0 += BATCH) {
        if (s0 > 0) {
#pragma unroll
            for (int u = 0; u < BATCH; ++u) v[u] = *reinterpret_cast<const f32x4*>(src + int64_t(min(s0 + u, slots - 1)) * step);
        }
#pragma unroll
        for (int u = 0; u < BATCH; ++u) {
            if (s0 + u < n) {
                const float wu = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), s0 + u));
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[e] = __builtin_fmaf(wu, v[u][e], acc[e]);
            }
        }
    }
    if (!has) return;
    const float scl = total == 0.f ? 0.f : 1.f / total;
    uint16_t* dst = p.out + row_offset(r, p.T, p.H, p.sob, p.sot, p.ldo) + c;
    *reinterpret_cast<uint2*>(dst) = uint2{pack2(acc[0] * scl, acc[1] * scl), pack2(acc[2] * scl, acc[3] * scl)};
}

// No position anywhere: zeros.
__global__ __launch_bounds__(kMergeT) void attention_batch_zero_kernel(const BatchParams p) {
    const int c = 4 * static_cast<int>(threadIdx.x);
    if (c < p.kv)
        *reinterpret_cast<uint2*>(p.out + row_offset(static_cast<int>(blockIdx.x), p.T, p.H, p.sob, p.sot, p.ldo) + c) = uint2{0, 0};
}

// ---------------------------------------------------------------------------------------------
// The partition.
// ---------------------------------------------------------------------------------------------
struct BatchPlan {
    int ht = 1;                        // 16-row tiles per workgroup: 1, 2 or 4
    int pre_tiles = 0, pre_spans = 0, pre_span = kChunk;
    int own_tiles = 1, own_spans = 0, own_span = kChunk;
    int64_t pre_items = 0, own_items = 0, grid = 0;
    size_t ws_bytes = 0;
};

int64_t cdiv(int64_t a, int64_t b) { return (a + b - 1) / b; }

// Time of a chunk in a tile of 16 ht rows, relative to 16 rows (measured, per 64 positions).
int chunk_cost(int ht) { return ht == 4 ? 16 : ht == 2 ? 11 : 10; }

// The partition in tiles of 16 ht rows, and an estimate of its time.
int64_t plan_tiles(const nmm_latent_attn_batch& a, int ht, BatchPlan* out) {
    // workgroups that run at once (16 rows, two a CU: 50.0 us with spans for 256, 48.5 for 512, 62 for 768 at 64 x 16 heads
    // over 4097 positions)
    const int64_t kCus = ht == 1 ? 512 : 256;
    BatchPlan q;
    q.ht = ht;
    const int64_t th = a.tokens * a.heads, rows = a.batch * th;
    q.own_tiles = static_cast<int>(cdiv(th, 16 * ht));
    const int64_t pc = cdiv(a.prefix_len, kChunk), oc = cdiv(a.max_len, kChunk);
    q.pre_tiles = pc ? static_cast<int>(cdiv(rows, 16 * ht)) : 0;
    const int64_t own_groups = oc ? a.batch * q.own_tiles : 0;
    const int cost = chunk_cost(ht);
    // For each number of prefix spans, own spans of about the same time; the pair with the least estimated
    // time: the longest item where one round of the CUs holds all, else the CUs' share and a last item, and
    // the merge's reads.
    int64_t best = -1, best_ps = 0, best_os = 0;
    const int64_t ps_max = pc ? std::min<int64_t>(pc, kMaxSlots - (oc ? 1 : 0)) : 0;
    const int64_t tries = pc ? ps_max : std::min<int64_t>(oc, kMaxSlots);
    for (int64_t i = 1; i <= tries; ++i) {
        int64_t ps = 0, os = 0;
        if (pc) {
            ps = cdiv(pc, cdiv(pc, i));
            if (oc) os = std::min<int64_t>({oc, kMaxSlots - ps, cdiv(oc, cdiv(pc, ps))});
        } else {
            os = i;
        }
        if (os) os = cdiv(oc, cdiv(oc, os));
        const int64_t ip = ps ? cdiv(pc, ps) * cost : 0, io = os ? cdiv(oc, os) * cost : 0;
        const int64_t items = ps * q.pre_tiles + os * own_groups;
        const int64_t work = ps * q.pre_tiles * ip + os * own_groups * io;
        int64_t t = items <= kCus ? std::max(ip, io) : work / kCus + std::max(ip, io);
        t = t * 16 + (ps + os > 1 ? 64 + (ps + os) * rows / 64 : 0);
        if (best < 0 || t < best) {
            best = t;
            best_ps = ps;
            best_os = os;
        }
    }
    if (pc) {
        q.pre_span = static_cast<int>(cdiv(pc, best_ps) * kChunk);
        q.pre_spans = static_cast<int>(cdiv(a.prefix_len, q.pre_span));
    }
    if (oc) {
        q.own_span = static_cast<int>(cdiv(oc, best_os) * kChunk);
        q.own_spans = static_cast<int>(cdiv(a.max_len, q.own_span));
    }
    q.pre_items = int64_t(q.pre_tiles) * q.pre_spans;
    q.own_items = own_groups * q.own_spans;
    q.grid = (cdiv(q.pre_items, 8) + cdiv(q.own_items, 8)) * 8;
    const int64_t slots = q.pre_spans + q.own_spans;
    if (slots > 1) q.ws_bytes = size_t(kTicketBytes) + size_t(slots) * size_t(rows) * (size_t(a.cache.kv_lora) + 2) * 4;
    *out = q;
    return best;
}

// A sequence's own positions take the smallest tile that holds its rows (16 heads, 64 sequences over 4097 positions: 48.9 us
// in tiles of 16, 55.8 of 32, 60.1 of 64; 32 heads, 16 over 2000: 21.4 in tiles of 32, 25.2 of 64); with a prefix, whose rows
// are all sequences', tiles of 64 for both where that is estimated to be faster (32 x 2 x 16 behind 16000: 70.8 us against
// 85.0; 8 x 16 behind 2000 stays at 16: 16.9 against 22.3).
void plan_batch(const nmm_latent_attn_batch& a, BatchPlan* out) {
    const int64_t th = a.tokens * a.heads;
    const int ht = th <= 16 ? 1 : th <= 32 ? 2 : 4;
    const int64_t t = plan_tiles(a, ht, out);
    if (ht == 4 || a.prefix_len == 0 || a.batch * th <= 16 * ht) return;
    BatchPlan wide;
    if (plan_tiles(a, 4, &wide) < t) *out = wide;
}

constexpr int64_t kLim = int64_t(1) << 31;
constexpr int64_t kMaxPositions = int64_t(1) << 30;

bool aligned(const void* p, uintptr_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

// The sizes that the partition depends on.
nmm_status validate_sizes(const nmm_latent_attn_batch& a) {
    const nmm_status st = validate_latent_cache(a.cache);
    if (st != NMM_OK) return st;
    if (a.batch < 0 || a.tokens < 0 || a.heads < 0 || a.batch >= (1 << 20) || a.tokens >= (1 << 16) || a.heads >= (1 << 16))
        return NMM_ERR_SHAPE;
    if (a.batch * a.tokens * a.heads >= (1 << 24)) return NMM_ERR_SHAPE;
    if (a.prefix_len < 0 || a.max_len < 0 || a.prefix_len >= kMaxPositions || a.max_len >= kMaxPositions) return NMM_ERR_SHAPE;
    if (a.page_size < 1 || a.page_size > 65536 || (a.page_size & (a.page_size - 1))) return NMM_ERR_SHAPE;
    return NMM_OK;
}

template <bool E4M3, bool BIG>
void launch_tiles(int ht, const BatchParams& p, dim3 grid, dim3 block, hipStream_t s) {
    if (ht == 1) hipLaunchKernelGGL((attention_batch_kernel<1, E4M3, BIG>), grid, block, 0, s, p);
    else if (ht == 2) hipLaunchKernelGGL((attention_batch_kernel<2, E4M3, BIG>), grid, block, 0, s, p);
    else hipLaunchKernelGGL((attention_batch_wide_kernel<E4M3, BIG>), grid, block, 0, s, p);
}

}  // namespace
}  // namespace nmm

using namespace nmm;

extern "C" {

size_t nmm_latent_attention_batch_workspace_size(const nmm_latent_attn_batch* attn) {
    if (!attn || validate_sizes(*attn) != NMM_OK || attn->batch * attn->tokens * attn->heads == 0) return 0;
    BatchPlan q;
    plan_batch(*attn, &q);
    return q.ws_bytes;
}

nmm_status nmm_latent_attention_batch(const nmm_latent_attn_batch* attn, void* workspace, size_t workspace_bytes,
                                      void* stream) {
    if (!attn) return NMM_ERR_NULL;
    const nmm_latent_attn_batch& a = *attn;
    nmm_status st = validate_sizes(a);
    if (st != NMM_OK) return st;
    if (!std::isfinite(a.scale)) return NMM_ERR_ARG;
    const int64_t d = a.cache.kv_lora + a.cache.rope;
    if (a.ldq < d || a.ldo < a.cache.kv_lora || a.ldq >= kLim || a.ldo >= kLim) return NMM_ERR_SHAPE;
    const int64_t strides[] = {a.stride_qb, a.stride_qt, a.stride_ob, a.stride_ot};
    for (int64_t v : strides)
        if (v < 0 || v >= (int64_t(1) << 40)) return NMM_ERR_SHAPE;
    if (a.max_len > 0 && (a.ld_pages < cdiv(a.max_len, a.page_size) || a.ld_pages >= kLim)) return NMM_ERR_SHAPE;
    const int64_t rows = a.batch * a.tokens * a.heads;
    if (rows == 0) return NMM_OK;
    // (rows of out over each other would be written by several workgroups)
    if ((a.batch > 1 && a.stride_ob < a.cache.kv_lora) || (a.tokens > 1 && a.stride_ot < a.cache.kv_lora)) return NMM_ERR_SHAPE;
    if (!a.q || !a.out) return NMM_ERR_NULL;
    if (a.prefix_len > 0 && !a.prefix_pages) return NMM_ERR_NULL;
    if (a.max_len > 0 && (!a.pages || !a.lens)) return NMM_ERR_NULL;
    if (!a.cache.data && a.cache.rows > 0) return NMM_ERR_NULL;
    if (!aligned(a.q, 16) || a.ldq % 8 || a.stride_qb % 8 || a.stride_qt % 8 || !aligned(a.out, 8) || a.ldo % 4 ||
        a.stride_ob % 4 || a.stride_ot % 4 || !aligned(a.prefix_pages, 4) || !aligned(a.pages, 4) || !aligned(a.lens, 4))
        return NMM_ERR_ALIGN;
    BatchPlan q;
    plan_batch(a, &q);
    if (q.grid >= (int64_t(1) << 32) / kThreadsB) return NMM_ERR_SHAPE;
    st = validate_workspace(workspace, workspace_bytes, q.ws_bytes);
    if (st != NMM_OK) return st;

    BatchParams p{};
    p.q = static_cast<const uint16_t*>(a.q);
    p.sqb = a.stride_qb; p.sqt = a.stride_qt; p.ldq = a.ldq;
    p.cache = static_cast<const uint8_t*>(a.cache.data);
    p.ld = a.cache.ld;
    p.kv = static_cast<int>(a.cache.kv_lora);
    p.rope = static_cast<int>(a.cache.rope);
    while ((int64_t(1) << p.page_shift) < a.page_size) ++p.page_shift;
    p.n_pages = static_cast<int>(a.cache.rows / a.page_size);
    p.prefix_pages = a.prefix_pages;
    p.prefix_len = static_cast<int>(a.prefix_len);
    p.pages = a.pages;
    p.ld_pages = a.ld_pages;
    p.lens = a.lens;
    p.max_len = static_cast<int>(a.max_len);
    p.scale_log2 = a.scale * 1.4426950408889634f;
    p.out = static_cast<uint16_t*>(a.out);
    p.sob = a.stride_ob; p.sot = a.stride_ot; p.ldo = a.ldo;
    if (q.ws_bytes) {
        p.part_o = reinterpret_cast<float*>(static_cast<uint8_t*>(workspace) + kTicketBytes);
        p.part_ml = p.part_o + size_t(q.pre_spans + q.own_spans) * size_t(rows) * size_t(a.cache.kv_lora);
    }
    p.B = static_cast<int>(a.batch);
    p.T = static_cast<int>(a.tokens);
    p.H = static_cast<int>(a.heads);
    p.rows = static_cast<int>(rows);
    p.pre_tiles = q.pre_tiles; p.pre_spans = q.pre_spans; p.pre_span = q.pre_span;
    p.pre_items = static_cast<int>(q.pre_items);
    p.pre_grid = static_cast<int>(cdiv(q.pre_items, 8) * 8);
    p.own_items = static_cast<int>(q.own_items);
    p.own_tiles = q.own_tiles; p.own_spans = q.own_spans; p.own_span = q.own_span;
    p.direct = q.pre_spans + q.own_spans == 1 ? 1 : 0;
    const int64_t extent = a.cache.rows * a.cache.ld;
    const bool big = extent >= kLim;
    p.extent = big ? 0u : static_cast<uint32_t>(extent);
    hipStream_t s = static_cast<hipStream_t>(stream);
    if (q.grid > 0) {
        const dim3 grid(static_cast<uint32_t>(q.grid)), block(kThreadsB);
        if (a.cache.format == NMM_CACHE_E4M3) launch_tiles<true, false>(q.ht, p, grid, block, s);
        else if (big) launch_tiles<false, true>(q.ht, p, grid, block, s);
        else launch_tiles<false, false>(q.ht, p, grid, block, s);
    }
    const int slots = q.pre_spans + q.own_spans;
    const dim3 rgrid(static_cast<uint32_t>(rows)), rblock(kMergeT);
    if (slots == 0) hipLaunchKernelGGL(attention_batch_zero_kernel, rgrid, rblock, 0, s, p);
    else if (slots > 8) hipLaunchKernelGGL(attention_batch_merge_kernel<16>, rgrid, rblock, 0, s, p);
    else if (slots > 4) hipLaunchKernelGGL(attention_batch_merge_kernel<8>, rgrid, rblock, 0, s, p);
    else if (slots > 1) hipLaunchKernelGGL(attention_batch_merge_kernel<4>, rgrid, rblock, 0, s, p);
    return hipGetLastError() == hipSuccess ? NMM_OK : NMM_ERR_HIP;
}

}  // extern "C"
