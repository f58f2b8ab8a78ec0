// cp_shared_prefix: attention of groups of requests that share cached pages (see the header).
//
// For a row (token, q head) of request r in group g, with the keys cut into ranges c:
//     m_c = max s_j, l_c = sum exp2(s_j - m_c), O_c = sum exp2(s_j - m_c) v_j        over the keys j of range c
//     out = sum_c 2^(m_c - m) O_c / sum_c 2^(m_c - m) l_c,  m = max m_c              (s in the log2 domain)
// Two kinds of range: of the group's S_g shared keys, which every row of the group sees whole, and of the request's
// own keys, causal at the end.  One launch has both:
//   row tiles   up to 256 rows of a (group, KV head), token by token, whatever request they are of, against a range of shared
//               keys.  Eight wavefronts share tiles of 64 keys in LDS: each has 32 rows, and those behind the last row only
//               load
//   own keys    32 rows of a (request, KV head) against a range of its own keys by one to eight wavefronts (cp_decode.h)
// and a second one joins them.  Where no request of a group has cached tokens of its own, what is left are the new tokens, which
// lie side by side: the row tiles of the last range go on over those of their requests, with a mask, and nothing is left
// to join if there is one range.
//
// Measured, both launches: 64/8 heads, 128 requests with a new token on 131072 shared ones 522 us, bound by the matrix pipe (1.05
// PFLOP/s; 3360 us request by request); 32/8 heads, 32 requests on 10240 24 us, bound by the chains start - tiles - join (12 us
// of reading; 98 us); 48 in six groups with up to 1500 tokens of their own 60 us, 188 MB (183 us).
#include <hip/hip_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>
#include <vector>

#include "cp_checks.h"
#include "cp_decode.h"
#include "cp_device.h"
#include "cp_shared_prefix.h"

namespace {

constexpr int kBM = 256; // rows of a tile
constexpr int kBN = 64;  // keys of a tile
constexpr int kThreads = 512;
constexpr int kWaves = kThreads / 64;
constexpr int kLoadRows = kWaves * 4;
constexpr int kNKB = kBN / 32;
static_assert(kBM == kWaves * 32 && kBN == 2 * kLoadRows, "tile shape");

constexpr int kMaxRanges = 64; // of a group's shared keys, and of a request's own

// A group whose shared keys are read once.  They travel in the kernel's arguments, one for each lane of a wavefront; a batch
// with more groups takes several launches.
constexpr int kMaxGroups = 64;
struct Group {
    int32_t first_item; // in the list of a KV head's row tiles
    int32_t request, requests;
    int32_t token, tokens; // packed rows of q
    int32_t keys, ranges, per_range; // S; ranges of so many tiles of keys
    int32_t part_row; // first row of its partial results, [ranges][tokens]
    int32_t new_tiles; // of those, for a row tile, at most (host)
    int32_t new_keys; // the last range goes on over the new tokens: the requests have no other keys of their own
};

struct SharedParams : AttnParams {
    int32_t groups;
    int32_t tile_items, tile_per_xcd; // row tiles of a KV head; list positions of an XCD
    int32_t own_items, own_per_xcd;   // workgroups of own keys of a KV head
    int32_t own_blocks;               // own keys of an item in blocks of 32, at most
    int32_t own_waves;                // wavefronts that share them: 1, 2, 4 or 8
    int32_t own_part_row;             // partial results of own keys begin here
    int32_t same_extend, same_ranges; // one group, and every request has so many new tokens and ranges of own keys; else 0
    Group group[kMaxGroups];
};

// Ranges of a request's own keys.
__host__ __device__ inline int own_ranges(int keys, int own_blocks) { return ((keys + 31) / 32 + own_blocks - 1) / own_blocks; }

// Every lane reads one group at once and keeps it: a chain of scalar reads, one behind the other, costs 0.4 us each.
__device__ __forceinline__ Group lane_group(const SharedParams &p, int lane)
{
    Group g{INT32_MAX, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
    if (lane < p.groups) g = p.group[lane];
    return g;
}
__device__ __forceinline__ Group group_of_lane(const Group &mine, int lane)
{
    Group g;
    g.first_item = __builtin_amdgcn_readlane(mine.first_item, lane);
    g.request = __builtin_amdgcn_readlane(mine.request, lane);
    g.requests = __builtin_amdgcn_readlane(mine.requests, lane);
    g.token = __builtin_amdgcn_readlane(mine.token, lane);
    g.tokens = __builtin_amdgcn_readlane(mine.tokens, lane);
    g.keys = __builtin_amdgcn_readlane(mine.keys, lane);
    g.ranges = __builtin_amdgcn_readlane(mine.ranges, lane);
    g.per_range = __builtin_amdgcn_readlane(mine.per_range, lane);
    g.part_row = __builtin_amdgcn_readlane(mine.part_row, lane);
    g.new_keys = __builtin_amdgcn_readlane(mine.new_keys, lane);
    return g;
}

// Position in a list of `items` per KV head of which every XCD takes a contiguous part, -1: none.
__device__ __forceinline__ int position(int xcd, int at, int per_xcd, int items, int heads, int &kvh)
{
    const int item = xcd * per_xcd + at;
    kvh = item / items;
    return kvh < heads ? item - kvh * items : -1;
}

// ---- results of wavefronts -------------------------------------------------------------------
// Of own keys a wavefront leaves 32 rows of O with their (m, l) in an area of LDS; what goes out is then added up over the areas
// that have the same rows and written a whole row of 512 bytes at a time.  Row tiles have nothing to add up: they write from
// the accumulators, 32 bytes of each of 32 rows a store (1.7 us of a tile's end; through LDS 2.8).
constexpr int kPitchO = kD + 4; // floats
constexpr int kArea = kDecLdsPerWave;
static_assert((32 * kPitchO + 64) * 4 <= kArea, "an area holds a wavefront's result");

__device__ __forceinline__ void put_result(char *area, int lane, const f32x16 (&o)[4], float m, float l_tot)
{
    const int j = lane & 31, h = lane >> 5;
    float *const mine = reinterpret_cast<float *>(area);
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
            const f32x4 x = {o[db][4 * gq], o[db][4 * gq + 1], o[db][4 * gq + 2], o[db][4 * gq + 3]};
            *reinterpret_cast<f32x4 *>(mine + j * kPitchO + db * 32 + 8 * gq + 4 * h) = x;
        }
    if (h == 0) *reinterpret_cast<f32x2 *>(mine + 32 * kPitchO + 2 * j) = f32x2{m, l_tot};
}

// Row i of kParts areas, `step` bytes apart: four d of the sum, and the row's (m, l).
template <int kParts>
__device__ __forceinline__ f32x4 take_row(const char *area, int step, int i, int d4, f32x2 &ml)
{
    f32x2 part[kParts];
    f32x4 x[kParts];
#pragma unroll
    for (int w = 0; w < kParts; ++w) {
        const float *const from = reinterpret_cast<const float *>(area + w * step);
        part[w] = *reinterpret_cast<const f32x2 *>(from + 32 * kPitchO + 2 * i);
        x[w] = *reinterpret_cast<const f32x4 *>(from + i * kPitchO + d4);
    }
    if (kParts == 1) {
        ml = part[0];
        return x[0];
    }
    float m = -INFINITY;
#pragma unroll
    for (int w = 0; w < kParts; ++w) m = fmaxf(m, part[w][1] != 0.f ? part[w][0] : -INFINITY);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
    float l = 0.f;
#pragma unroll
    for (int w = 0; w < kParts; ++w) {
        // a sum of 0: no keys, or none that the row sees, and x is 0; NaN goes through
        const float f = part[w][1] != 0.f ? fast_exp2(part[w][0] - m) : 0.f;
        acc += x[w] * f;
        l = fmaf(part[w][1], f, l);
    }
    ml = f32x2{m, l};
    return acc;
}

__device__ __forceinline__ void write_partial(const SharedParams &p, int64_t prow, int d4, f32x4 x, f32x2 ml)
{
    *reinterpret_cast<f32x4 *>(p.part_o + prow * kD + d4) = x;
    if (d4 == 0) *reinterpret_cast<f32x2 *>(p.part_ml + prow * 2) = ml;
}

// ---- row tiles -------------------------------------------------------------------------------
// K tiles in four buffers, V tiles in five, 256 bytes a row, filled by direct loads from global memory (lane i of a wavefront
// writes 16 bytes at slot i of 1 KiB).  The 16-byte chunks of a row are swizzled on the source side: chunk c of K row r at slot
// c ^ (r & 15), of V row r at c ^ ((r & 3) << 2), so that neither the reads of 16 rows at one column nor the transposing
// reads of four rows meet in a bank.
constexpr int kPitch = 256;
constexpr int kTileBytes = kBN * kPitch;
constexpr int kBufsK = 4, kBufsV = 5;
constexpr int kLdsBytes = std::max((kBufsK + kBufsV) * kTileBytes, kWaves * kArea);

typedef __attribute__((address_space(3))) const char *lptr;
typedef const __attribute__((address_space(1))) char *gptr;
typedef f32x16 STile[kNKB];     // scores: 32-key blocks x 32 query rows
typedef bf16x8 PTile[2 * kNKB]; // probabilities: an operand per 16 keys

__device__ __forceinline__ void row_tile_item(const SharedParams &p, char *lds, int wave, int lane, int item, int kvh)
{
    Group grp = p.group[0]; // comes with the other arguments
    if (p.groups > 1) {
        const Group mine = lane_group(p, lane);
        grp = group_of_lane(mine, __popcll(__builtin_amdgcn_ballot_w64(mine.first_item <= item)) - 1);
    }
    item -= grp.first_item;
    const int rows = grp.tokens * p.G;
    const int tiles = (rows + kBM - 1) / kBM;
    const int range = item / tiles, tile = item - range * tiles;
    const int key_tiles = (grp.keys + kBN - 1) / kBN;
    const int kt0 = range * grp.per_range;
    const int n_shared = min(key_tiles - kt0, grp.per_range);
    const int j = lane & 31, h = lane >> 5;
    const int wave_row0 = tile * kBM + wave * 32;
    const bool no_rows = wave_row0 >= rows;
    const int row = min(wave_row0 + j, rows - 1);
    const int tok = over_heads(row, p), head = kvh * p.G + row - tok * p.G;

    // New tokens: those from `lo` on, where the first row's request begins, to the last row's; a row sees the ones from
    // its own request's first (row_lo) to itself.
    int lo = 0, row_lo = 0, n_it = n_shared;
    if (grp.new_keys && range == grp.ranges - 1) {
        const int tok0 = over_heads(tile * kBM, p), tok1 = over_heads(min(rows, (tile + 1) * kBM) - 1, p);
        int cu = 0;
        for (int base = 0; base < grp.requests && cu <= tok1; base += 64) {
            const int e = base + lane < grp.requests ? p.extend_lens[grp.request + base + lane] : 0;
            const int end = cu + wave_scan(e), begin = end - e;
            // requests that have a row of the tile
            for (uint64_t some = __builtin_amdgcn_ballot_w64(end > tok0 && begin <= tok1 && e > 0); some != 0; some &= some - 1) {
                const int first = __builtin_amdgcn_readlane(begin, __builtin_ctzll(some));
                if (first <= tok0) lo = first;
                if (first <= tok) row_lo = first;
            }
            cu = __builtin_amdgcn_readlane(end, 63);
        }
        n_it += (tok1 - lo) / kBN + 1;
    }

    // ---- loads: key rows wave * 4 + lane / 16 and that + 32 of a tile, chunk lane % 16
    const int ld_row = wave * 4 + (lane >> 4), ld_chunk = lane & 15;
    const __attribute__((address_space(4))) int32_t *table =
        (const __attribute__((address_space(4))) int32_t *)(p.block_table + (int64_t)grp.request * p.max_pages);
    const uint64_t page_bytes = (uint64_t)p.Hkv * (2u * kPS * kD * 2u);
    const uint32_t lane_k = (uint32_t)(((ld_row & 15) * kD + (ld_chunk ^ (ld_row & 15)) * 8) * 2);
    const uint32_t lane_v = (uint32_t)(((ld_row & 15) * kD + (ld_chunk ^ ((ld_row & 3) << 2)) * 8) * 2) +
                            (uint32_t)p.Hkv * (kPS * kD * 2u);
    const gptr pages_head = (gptr)p.kv_pages + (int64_t)kvh * (kPS * kD * 2);
    const uint32_t lds_k0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds;
    const uint32_t lds_v0 = lds_k0 + kBufsK * kTileBytes;
    const int last_page = grp.keys / kPS - 1;
    const int tsel = wave >> 2;
    // Pages of the wavefront's rows of the next tile to be requested, read a step ahead (in front of the loads their latency
    // is part of every step).  Those behind the last shared one are replaced by it; their scores are masked.
    uint32_t pg0, pg1;
    auto read_pages = [&](int t) {
        pg0 = (uint32_t)table[min((kt0 + t) * (kBN / kPS) + tsel, last_page)];
        pg1 = (uint32_t)table[min((kt0 + t) * (kBN / kPS) + 2 + tsel, last_page)];
    };
    auto load_tile = [&](int t, int kbuf, int vbuf, auto shared) { // shared: surely one of those
        gptr k0, v0, k1, v1;
        if (decltype(shared)::value || t < n_shared) {
            const gptr b0 = pages_head + (uint64_t)pg0 * page_bytes, b1 = pages_head + (uint64_t)pg1 * page_bytes;
            k0 = b0 + lane_k;
            v0 = b0 + lane_v;
            k1 = b1 + lane_k;
            v1 = b1 + lane_v;
        } else { // rows behind the group's last one are replaced by it, and masked
            const int at = lo + (t - n_shared) * kBN + ld_row;
            const int64_t row0 = ((int64_t)(grp.token + min(at, grp.tokens - 1)) * p.Hkv + kvh) * kD;
            const int64_t row1 = ((int64_t)(grp.token + min(at + kLoadRows, grp.tokens - 1)) * p.Hkv + kvh) * kD;
            const int ck = (ld_chunk ^ (ld_row & 15)) * 8, cv = (ld_chunk ^ ((ld_row & 3) << 2)) * 8;
            k0 = (gptr)(p.k_new + row0 + ck);
            v0 = (gptr)(p.v_new + row0 + cv);
            k1 = (gptr)(p.k_new + row1 + ck);
            v1 = (gptr)(p.v_new + row1 + cv);
        }
        const uint32_t dk0 = __builtin_amdgcn_readfirstlane(lds_k0 + kbuf * kTileBytes + wave * (4 * kPitch));
        const uint32_t dv0 = __builtin_amdgcn_readfirstlane(lds_v0 + vbuf * kTileBytes + wave * (4 * kPitch));
        const uint32_t dk1 = dk0 + kLoadRows * kPitch, dv1 = dv0 + kLoadRows * kPitch;
        // as assembly: for the builtin the compiler waits for every direct load in flight before the next LDS read
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %4, off\n\t"
                     "s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %5, off\n\t"
                     "s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %6, off\n\t"
                     "s_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %7, off"
                     :
                     : "s"(dk0), "s"(dv0), "s"(dk1), "s"(dv1), "v"(k0), "v"(v0), "v"(k1), "v"(v1)
                     : "memory");
        read_pages(t + 1);
    };
    auto meet = [&]() {
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
        __syncthreads();
    };
    read_pages(0);
    load_tile(0, 0, 0, std::true_type{});
    if (n_it > 1) load_tile(1, 1, 1, std::false_type{});

    // query rows, B operand of S^T = K Q^T: lane (j, h) holds q[row j][16 kk + 8 h .. + 8)
    bf16x8 qf[8];
    {
        const uint16_t *qp = p.q + ((int64_t)(grp.token + tok) * p.Hq + head) * kD + 8 * h;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk) qf[kk] = __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(qp + 16 * kk));
    }
    const float c = p.scale_log2;
    const int k_lane = j * kPitch + ((h ^ (j & 15)) << 4);
    const int v_lane = (4 * h + ((lane & 15) >> 2)) * kPitch + (((lane >> 2) & 3) << 6) + ((lane >> 4) & 1) * 32 + (lane & 3) * 8;

    f32x16 o[4];
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
    float m_ref = -INFINITY, l_run = 0.f; // reference of the exponentials (log2 domain), sum over this half-wave's keys
    const bf16x2 ones = {(__bf16)1.0f, (__bf16)1.0f};

    auto qk_tile = [&](int kbuf, STile &s) {
        const uint32_t kb = lds_k0 + kbuf * kTileBytes + k_lane;
        const f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int b = 0; b < kNKB; ++b) s[b] = zero;
#pragma unroll
        for (int kk = 0; kk < 8; ++kk)
#pragma unroll
            for (int b = 0; b < kNKB; ++b) {
                const u32x4 a = *reinterpret_cast<__attribute__((address_space(3))) const u32x4 *>((lptr)(uintptr_t)(kb ^ (kk << 5)) + b * 32 * kPitch);
                s[b] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), qf[kk], s[b], 0, 0, 0);
            }
        // eight operands requested before the first MFMA, one more behind each
        constexpr int kAhead = 8;
        __builtin_amdgcn_sched_group_barrier(0x100, kAhead, 0);
#pragma unroll
        for (int i = 0; i < 8 * kNKB - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x008, kAhead, 0);
    };
    auto mask_tile = [&](int t, STile &s) {
        // the last shared tile and new tokens: accumulator element v of block b is key 32 b + 8 (v / 4) + 4 h + v % 4
        int to = grp.keys - (kt0 + t) * kBN;
        if (t >= n_shared) to = tok + 1 - lo - (t - n_shared) * kBN;
        if (t >= n_shared || to < kBN) {
#pragma unroll
            for (int b = 0; b < kNKB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (b * 32 + 8 * (v >> 2) + (v & 3) >= to - 4 * h) s[b][v] = -INFINITY;
        }
        // another request's tokens in front of the row's own
        const int from = t >= n_shared ? row_lo - lo - (t - n_shared) * kBN : 0;
        if (__builtin_amdgcn_ballot_w64(from > 0) != 0) {
#pragma unroll
            for (int b = 0; b < kNKB; ++b)
#pragma unroll
                for (int v = 0; v < 16; ++v)
                    if (b * 32 + 8 * (v >> 2) + (v & 3) < from - 4 * h) s[b][v] = -INFINITY;
        }
    };
    auto pv_tile = [&](int vbuf, const PTile &pb) {
        const uint32_t vb = lds_v0 + vbuf * kTileBytes + v_lane;
#pragma unroll
        for (int ks = 0; ks < 2 * kNKB; ++ks)
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                const lptr a = (lptr)(uintptr_t)(vb ^ (db << 6)) + ks * 16 * kPitch;
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(a));
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(a + 8 * kPitch));
                const s16x8 vv = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
                o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vv), pb[ks], o[db], 0, 0, 0);
            }
        // operands five MFMAs ahead, the next tile's exponentials behind them
        constexpr int kAhead = 5;
        __builtin_amdgcn_sched_group_barrier(0x100, 2 * kAhead, 0);
#pragma unroll
        for (int i = 0; i < 8 * kNKB; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < 8 * kNKB - kAhead) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
            __builtin_amdgcn_sched_group_barrier(0x400, 4, 0);
        }
    };
    // New tokens lie next to those of other requests, and 0 times a value that is not finite is not 0.  A tile with such a
    // value of V takes its rows token by token here, where the values of keys that a token does not see are 0; false: it has
    // none, and pv_tile does it.
    auto pv_tokens = [&](int t, const PTile &pb) {
        if (t < n_shared) return false;
        const uint32_t v0 = lds_v0 + t % kBufsV * kTileBytes, vb = v0 + v_lane;
        u16x2 top = {0, 0};
#pragma unroll
        for (int i = 0; i < kTileBytes / 1024; ++i) {
            const u32x4 x = *reinterpret_cast<__attribute__((address_space(3))) const u32x4 *>((lptr)(uintptr_t)(v0 + lane * 16) + i * 1024);
#pragma unroll
            for (int e = 0; e < 4; ++e) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, x[e] & 0x7fff7fffu));
        }
        if (__builtin_amdgcn_ballot_w64(top[0] >= 0x7f80 || top[1] >= 0x7f80) == 0) return false;
        const int at = lo + (t - n_shared) * kBN; // new token that is key 0 of the tile
        for (uint64_t left = ~UINT64_C(0); left != 0;) {
            const int one = __builtin_amdgcn_readlane(tok, __builtin_ctzll(left));
            const int from = __builtin_amdgcn_readlane(row_lo, __builtin_ctzll(left)) - at - 4 * h, to = one + 1 - at - 4 * h;
            left &= ~__builtin_amdgcn_ballot_w64(tok == one);
#pragma unroll
            for (int db = 0; db < 4; ++db) {
                f32x16 x = o[db];
#pragma unroll
                for (int ks = 0; ks < 2 * kNKB; ++ks) {
                    const lptr a = (lptr)(uintptr_t)(vb ^ (db << 6)) + ks * 16 * kPitch;
                    s16x8 vv;
#pragma unroll
                    for (int u = 0; u < 2; ++u) {
                        const s16x4 part = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(a + u * 8 * kPitch));
#pragma unroll
                        for (int e = 0; e < 4; ++e) { // key + 4 h
                            const int key = 16 * ks + 8 * u + e;
                            vv[4 * u + e] = key >= from && key < to ? part[e] : (short)0;
                        }
                    }
                    x = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, vv), pb[ks], x, 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                }
                if (tok == one) o[db] = x;
            }
        }
        return true;
    };
    // Probabilities against the reference m, rounded to bf16 for the second product; the sum is of the rounded ones.
    // The sums come after all conversions (the empty statement says so): between the MFMAs they wait for each other.
    auto exp_tile = [&](const STile &s, PTile &pb, float m) -> float {
        u32x4 w[2 * kNKB];
#pragma unroll
        for (int t = 0; t < 2 * kNKB; ++t)
#pragma unroll
            for (int e = 0; e < 8; e += 2) {
                f32x2 x;
                x[0] = fast_exp2(fmaf(s[t >> 1][8 * (t & 1) + e], c, -m));
                x[1] = fast_exp2(fmaf(s[t >> 1][8 * (t & 1) + e + 1], c, -m));
                w[t][e / 2] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
            }
        asm("" : "+v"(w[0]), "+v"(w[1]), "+v"(w[2]), "+v"(w[3]));
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int t = 0; t < 2 * kNKB; ++t) sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)w[t][e]), ones, sum, false);
#pragma unroll
        for (int t = 0; t < 2 * kNKB; ++t) pb[t] = __builtin_bit_cast(bf16x8, w[t]);
        return sum;
    };
    // Reference from the tile's row maximum; O and l follow.
    auto first_tile = [&](const STile &s, PTile &pb) -> float {
        float mx = s[0][0];
#pragma unroll
        for (int i = 1; i < 16 * kNKB; ++i) mx = fmaxf(mx, s[i >> 4][i & 15]);
        const float m_new = fmaxf(m_ref, halfwave_max(mx) * c);
        const float m_use = m_new == -INFINITY ? 0.f : m_new;
        const float alpha = fast_exp2(m_ref - m_use);
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int v = 0; v < 16; ++v) o[db][v] *= alpha;
        l_run *= alpha;
        m_ref = m_new;
        return exp_tile(s, pb, m_use);
    };
    // Against the reference that there is; it is taken anew where a row has none or its sum says that it is stale by 2^80.
    constexpr float kStale = 1.2089258196146292e24f; // 2^80
    auto stale = [&](float sum) { return __builtin_amdgcn_ballot_w64(!(sum < kStale) || m_ref == -INFINITY) != 0; };

    // A tile is requested two steps before it is used, V of tile t is read one step after K, and a barrier comes after every
    // second step.
    meet();
    PTile pb, pb_next;
    if (2 < n_it) load_tile(2, 2, 2, std::false_type{});
    if (!no_rows) {
        STile s;
        qk_tile(0, s);
        mask_tile(0, s);
        l_run = first_tile(s, pb);
    }
    meet();
    auto step = [&](int it, auto plain) { // plain: tile it + 2 is one of the shared keys, and this one is not their last
        if (decltype(plain)::value || it + 2 < n_it) load_tile(it + 2, (it + 2) % kBufsK, (it + 2) % kBufsV, plain);
        if (!no_rows) {
            const bool by_token = !decltype(plain)::value && pv_tokens(it - 1, pb);
            STile s;
            qk_tile(it % kBufsK, s);
            if (!decltype(plain)::value) mask_tile(it, s);
            float sum = exp_tile(s, pb_next, m_ref == -INFINITY ? 0.f : m_ref);
            if (decltype(plain)::value || !by_token) pv_tile((it - 1) % kBufsV, pb);
            if (stale(sum)) sum = first_tile(s, pb_next);
            l_run += sum;
#pragma unroll
            for (int t = 0; t < 2 * kNKB; ++t) pb[t] = pb_next[t];
        }
        if (!(it & 1)) meet();
    };
    int it = 1;
    for (; it + 2 < n_shared; ++it) step(it, std::true_type{});
    for (; it < n_it; ++it) step(it, std::false_type{});
    if (no_rows) return;
    if (!pv_tokens(n_it - 1, pb)) pv_tile((n_it - 1) % kBufsV, pb);

    // ---- partial result: o[db][v] is O^T[d = db * 32 + 8 (v / 4) + 4 h + v % 4][row j]
    const float l_tot = halfwave_sum(l_run);
    if (wave_row0 + j >= rows) return;
    if (grp.new_keys && grp.ranges == 1) { // these were all keys
        const float inv = 1.f / l_tot;
        uint16_t *const out = p.out + ((int64_t)(grp.token + tok) * p.Hq + head) * kD;
#pragma unroll
        for (int db = 0; db < 4; ++db)
#pragma unroll
            for (int gq = 0; gq < 4; ++gq) {
                bf16x4 x;
#pragma unroll
                for (int e = 0; e < 4; ++e) x[e] = (__bf16)(o[db][4 * gq + e] * inv);
                *reinterpret_cast<bf16x4 *>(out + db * 32 + 8 * gq + 4 * h) = x;
            }
        return;
    }
    const int64_t prow = ((int64_t)grp.part_row + (int64_t)range * grp.tokens + tok) * p.Hq + head;
    float *const po = p.part_o + prow * kD;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
        for (int gq = 0; gq < 4; ++gq) {
            const f32x4 x = {o[db][4 * gq], o[db][4 * gq + 1], o[db][4 * gq + 2], o[db][4 * gq + 3]};
            *reinterpret_cast<f32x4 *>(po + db * 32 + 8 * gq + 4 * h) = x;
        }
    if (h == 0) *reinterpret_cast<f32x2 *>(p.part_ml + prow * 2) = f32x2{m_ref, l_tot};
}

// ---- own keys --------------------------------------------------------------------------------
struct Request {
    int r, E, P, S, cu, ranges, shared_ranges, group, part;
};
// The request with new token `at` (kUnits: with unit `at` of a KV head's own keys: requests in order, a request's row blocks, and
// of each its key ranges).  `at` becomes the place in the request; false if there is none.
template <bool kUnits>
__device__ __forceinline__ bool find_request(const SharedParams &p, const Group &mine, int lane, int &at, Request &q)
{
    if (p.same_extend > 0) { // nothing to look for, and no loads to wait for
        q.E = p.same_extend;
        q.ranges = p.same_ranges;
        const int size = kUnits ? (q.E * p.G + kDecRows - 1) / kDecRows * q.ranges : q.E;
        q.r = at / size;
        if (q.r >= p.batch) return false;
        at -= q.r * size;
        q.group = 0;
        q.S = p.group[0].keys;
        q.shared_ranges = p.group[0].ranges;
        q.cu = q.r * q.E;
        q.part = p.own_part_row + q.cu * q.ranges; // a group has a shared range: every own one leaves a partial result
        q.P = kUnits ? p.prefix_lens[q.r] : 0;
        return true;
    }
    q.cu = 0;
    q.part = p.own_part_row;
    for (int base = 0; base < p.batch; base += 64) {
        const int rr = base + lane;
        const int e = rr < p.batch ? p.extend_lens[rr] : 0;
        const int pl = rr < p.batch ? p.prefix_lens[rr] : 0;
        // The lane's group: groups lie one behind the other, so it is the last one that begins at the lane's request or in
        // front of it, if it goes so far.  There is a bit for each of the 64 requests with which a group begins, and the bits up to
        // the lane's are counted.  A look at every group, for every 64 requests, took longer than the keys: 32/8 heads, on 1024
        // tokens and 40 of their own, 64 groups of 8 requests 222 us, 96 this way; 8 groups 18.6 and 17.8, one group the same.
        const int begin = lane < p.groups ? mine.request - base : 64;
        const uint32_t low = (uint32_t)__builtin_amdgcn_readlane(wave_scan(begin >= 0 && begin < 32 ? 1 << begin : 0), 63);
        const uint32_t high = (uint32_t)__builtin_amdgcn_readlane(wave_scan(begin >= 32 && begin < 64 ? 1 << (begin - 32) : 0), 63);
        const int before = __popcll(__builtin_amdgcn_ballot_w64(begin < 0));
        const int here = (lane < 32 ? low >> lane : high >> (lane - 32)) & 1;
        int group = before - 1 + here + (int)__builtin_amdgcn_mbcnt_hi(high, __builtin_amdgcn_mbcnt_lo(low, 0));
        const int of = max(group, 0);
        int sl = __shfl(mine.keys, of, 64), sr = __shfl(mine.ranges, of, 64); // S and ranges of the lane's request
        bool own = !__shfl(mine.new_keys, of, 64);
        const int end = __shfl(mine.request + mine.requests, of, 64);
        if (group < 0 || rr >= end) {
            sl = sr = 0;
            group = -1;
            own = true;
        }
        const int n = e > 0 && own ? own_ranges(pl - sl + e, p.own_blocks) : 0;
        const int parts = n + sr > 1 ? e * n : 0;
        const int size = kUnits ? (e * p.G + kDecRows - 1) / kDecRows * n : e;
        const int incl = wave_scan(size);
        const int incl_e = kUnits ? wave_scan(e) : incl;
        const int incl_p = wave_scan(parts);
        const int total = __builtin_amdgcn_readlane(incl, 63);
        if (at < total) {
            const int first = __builtin_ctzll(__builtin_amdgcn_ballot_w64(incl > at));
            at -= __builtin_amdgcn_readlane(incl - size, first);
            q.cu += __builtin_amdgcn_readlane(incl_e - e, first);
            q.part += __builtin_amdgcn_readlane(incl_p - parts, first);
            q.r = base + first;
            q.E = __builtin_amdgcn_readlane(e, first);
            q.P = __builtin_amdgcn_readlane(pl, first);
            q.S = __builtin_amdgcn_readlane(sl, first);
            q.ranges = __builtin_amdgcn_readlane(n, first);
            q.shared_ranges = __builtin_amdgcn_readlane(sr, first);
            q.group = __builtin_amdgcn_readlane(group, first);
            return true;
        }
        at -= total;
        q.cu += __builtin_amdgcn_readlane(incl_e, 63);
        q.part += __builtin_amdgcn_readlane(incl_p, 63);
    }
    return false;
}

// A workgroup has kWaves / own_waves units; the wavefronts of a unit take the key blocks of its range in turn.
__device__ __forceinline__ void own_item(const SharedParams &p, char *lds, int wave, int lane, int item, int kvh)
{
    const int waves = p.own_waves, in_unit = wave & (waves - 1), unit0 = wave & ~(waves - 1);
    int unit = item * (kWaves / waves) + wave / waves;
    Request q;
    const bool found = find_request<true>(p, p.same_extend > 0 ? Group{} : lane_group(p, lane), lane, unit, q);
    int rb = 0, range = 0;
    if (found) {
        rb = unit / q.ranges;
        range = unit - rb * q.ranges;
        AttnParams own = p; // the request as one whose cached tokens begin behind the shared ones
        own.block_table += q.S / kPS;
        const int P = q.P - q.S;
        // no row of the block sees keys behind its last token
        const int end = min(rb * kDecRows % q.E + kDecRows, q.E);
        const int blocks = (P + end + 31) / 32;
        const int per = ((P + q.E + 31) / 32 + q.ranges - 1) / q.ranges;
        DecResult res[1];
        decode_keys<1>(own, lds + wave * kArea, lane, q.r, kvh, P, q.E, q.cu, rb, range * per + in_unit,
                       min(blocks, range * per + per), waves, res);
        put_result(lds + wave * kArea, lane, res[0].o, res[0].m, halfwave_sum(res[0].l));
    }
    __syncthreads();
    if (!found) return;
    const int d4 = (lane & 31) * 4, rows = q.E * p.G - rb * kDecRows;
    const bool alone = q.ranges + q.shared_ranges == 1;
    for (int i = in_unit * 2 + (lane >> 5); i < min(kDecRows, rows); i += 2 * waves) {
        f32x2 ml;
        f32x4 x;
        const char *const areas = lds + unit0 * kArea;
        if (waves == 8) x = take_row<8>(areas, kArea, i, d4, ml);
        else if (waves == 4) x = take_row<4>(areas, kArea, i, d4, ml);
        else if (waves == 2) x = take_row<2>(areas, kArea, i, d4, ml);
        else x = take_row<1>(areas, kArea, i, d4, ml);
        const int row = rb * kDecRows + i, hg = row / q.E, e = row - hg * q.E, head = kvh * p.G + hg;
        if (alone) {
            const float inv = 1.f / ml[1]; // every row sees its own key
            bf16x4 y;
#pragma unroll
            for (int k = 0; k < 4; ++k) y[k] = (__bf16)(x[k] * inv);
            *reinterpret_cast<bf16x4 *>(p.out + ((int64_t)(q.cu + e) * p.Hq + head) * kD + d4) = y;
        } else {
            write_partial(p, ((int64_t)q.part + (int64_t)range * q.E + e) * p.Hq + head, d4, x, ml);
        }
    }
}

__global__ __launch_bounds__(kThreads) void shared_attn_kernel(const SharedParams p)
{
    __shared__ __attribute__((aligned(256))) char lds[kLdsBytes];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int lane = threadIdx.x & 63;
    const int xcd = blockIdx.x % kXcds, at = blockIdx.x / kXcds;
    int kvh;
    if (at < p.tile_per_xcd) {
        const int item = position(xcd, at, p.tile_per_xcd, p.tile_items, p.Hkv, kvh);
        if (item >= 0) row_tile_item(p, lds, wave, lane, item, kvh);
    } else {
        const int item = position(xcd, at - p.tile_per_xcd, p.own_per_xcd, p.own_items, p.Hkv, kvh);
        if (item >= 0) own_item(p, lds, wave, lane, item, kvh);
    }
}

// ---- join ------------------------------------------------------------------------------------
// kGroups groups of 32 threads have a (token, head), each up to kParts of its partial results, four d a thread.  The time is a
// chain of loads: the lengths, then all (m, l) and all O of a thread at once; the groups' sums are added up in order.
constexpr int kJoinThreads = 256, kJoinFew = 4, kJoinParts = 16;
template <int kGroups, int kParts>
__global__ __launch_bounds__(kJoinThreads) void join_kernel(const SharedParams p)
{
    constexpr int kHeads = kJoinThreads / 32 / kGroups, kMls = (kGroups * kParts + 31) / 32;
    __shared__ f32x4 sums[kJoinThreads];
    const int head_blocks = (p.Hq + kHeads - 1) / kHeads;
    const int token = blockIdx.x / head_blocks;
    const int unit = threadIdx.x >> 5, gr = unit % kGroups;
    const int head = (int)(blockIdx.x - token * head_blocks) * kHeads + unit / kGroups;
    const int lane = threadIdx.x & 63, t = threadIdx.x & 31;
    int e_at = token;
    Request q;
    const Group mine = p.same_extend > 0 ? Group{} : lane_group(p, lane);
    if (!find_request<false>(p, mine, lane, e_at, q)) return; // the same for the whole workgroup
    int shared_row = 0, shared_step = 0;
    if (q.group >= 0) {
        const Group grp = p.same_extend > 0 ? p.group[0] : group_of_lane(mine, q.group);
        shared_row = grp.part_row + token - grp.token;
        shared_step = grp.tokens;
    }
    const int n = q.shared_ranges + q.ranges;
    if (n <= 1) return; // written already
    const int use = min(head, p.Hq - 1);
    // partial result i: the shared ranges first
    auto row_of = [&](int i) {
        const int64_t at = i < q.shared_ranges ? (int64_t)shared_row + (int64_t)i * shared_step
                                               : (int64_t)q.part + (int64_t)(i - q.shared_ranges) * q.E + e_at;
        return at * p.Hq + use;
    };
    f32x2 ml[kMls];
#pragma unroll
    for (int i = 0; i < kMls; ++i)
        ml[i] = t + 32 * i < n ? *reinterpret_cast<const f32x2 *>(p.part_ml + row_of(t + 32 * i) * 2) : f32x2{0.f, 0.f};
    f32x4 x[kParts];
#pragma unroll
    for (int i = 0; i < kParts; ++i)
        x[i] = gr + i * kGroups < n ? *reinterpret_cast<const f32x4 *>(p.part_o + row_of(gr + i * kGroups) * kD + t * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < kMls; ++i)
        if (ml[i][1] != 0.f) m = fmaxf(m, ml[i][0]);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) m = fmaxf(m, __shfl_xor(m, off, 32));
    float w[kMls], denom = 0.f;
#pragma unroll
    for (int i = 0; i < kMls; ++i) {
        w[i] = ml[i][1] != 0.f ? fast_exp2(ml[i][0] - m) : -1.f; // -1: no keys, and no values left
        denom += ml[i][1] * w[i];
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) denom += __shfl_xor(denom, off, 32);
    f32x4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < kParts; ++i) {
        const float ws = __shfl(w[i * kGroups / 32], (gr + i * kGroups) & 31, 32);
        if (!(ws < 0.f)) acc += x[i] * ws; // a weight that is not a number counts; past the end x is 0 and the weight -1
    }
    if (kGroups > 1) {
        sums[threadIdx.x] = acc;
        __syncthreads();
        if (gr != 0) return;
#pragma unroll
        for (int i = 1; i < kGroups; ++i) acc += sums[threadIdx.x + 32 * i];
    }
    if (head >= p.Hq) return;
    const float inv = 1.f / denom;
    bf16x4 y;
#pragma unroll
    for (int e = 0; e < 4; ++e) y[e] = (__bf16)(acc[e] * inv);
    *reinterpret_cast<bf16x4 *>(p.out + ((int64_t)token * p.Hq + head) * kD + t * 4) = y;
}

// Groups of threads for a head, and workgroups for a token.
int join_groups(int most_parts) { return most_parts <= kJoinParts ? 1 : most_parts <= 2 * kJoinParts ? 2 : most_parts <= 4 * kJoinParts ? 4 : 8; }
int64_t join_blocks(int heads, int most_parts)
{
    const int each = kJoinThreads / 32 / join_groups(most_parts);
    return ((int64_t)heads + each - 1) / each;
}
void launch_join(const SharedParams &p, int most_parts, hipStream_t hs)
{
    const dim3 grid((unsigned)(p.T * join_blocks(p.Hq, most_parts)));
    auto go = [&](auto groups, auto parts) {
        hipLaunchKernelGGL((join_kernel<decltype(groups)::value, decltype(parts)::value>), grid, dim3(kJoinThreads), 0, hs, p);
    };
    const std::integral_constant<int, kJoinParts> many;
    if (most_parts <= kJoinFew) go(std::integral_constant<int, 1>{}, std::integral_constant<int, kJoinFew>{});
    else if (join_groups(most_parts) == 1) go(std::integral_constant<int, 1>{}, many);
    else if (join_groups(most_parts) == 2) go(std::integral_constant<int, 2>{}, many);
    else if (join_groups(most_parts) == 4) go(std::integral_constant<int, 4>{}, many);
    else go(std::integral_constant<int, 8>{}, many);
}
static_assert(2 * kMaxRanges <= 8 * kJoinParts, "every partial result has a thread");

// ---- host ------------------------------------------------------------------------------------
int validate_sharing(const cp_shape *s, const cp_sharing *sharing)
{
    if (!sharing || !sharing->h_group_sizes || !sharing->h_shared_lens) return CP_ERR_NULL;
    if (sharing->num_groups < 1 || sharing->num_groups > s->batch) return CP_ERR_SHAPE;
    int64_t r = 0;
    for (int g = 0; g < sharing->num_groups; ++g) {
        const int32_t size = sharing->h_group_sizes[g], keys = sharing->h_shared_lens[g];
        if (size < 1 || r + size > s->batch || keys < 0 || keys % kPS != 0) return CP_ERR_SHAPE;
        for (int64_t i = r; i < r + size; ++i)
            if (keys > s->h_prefix_lens[i]) return CP_ERR_SHAPE;
        r += size;
    }
    return r == s->batch ? CP_OK : CP_ERR_SHAPE;
}

// A run of whole groups, at most kMaxGroups of them shared, that is one launch (and its join).
struct Part {
    int request = 0, requests = 0;
    int64_t token = 0, tokens = 0;
    std::vector<Group> groups;
    int64_t tile_items = 0, own_units = 0; // per KV head
    int64_t own_part_row = 0, part_rows = 0;
    double us = -1.0;    // estimated
    double range_us = 0.0; // of a row tile's range, about
    int own_blocks = 1, own_waves = 1;
    int most_parts = 0; // of a row
    int same_extend = 0, same_ranges = 0;
};
struct Plan {
    bool shared = false;
    std::vector<Part> parts;
    int64_t part_rows = 0; // of the part that has most
    int ranges = 0;
};

size_t part_bytes(int64_t rows, int heads)
{
    const size_t rh = (size_t)rows * (size_t)heads;
    return ((rh * kD * sizeof(float) + 255) / 256) * 256 + rh * 2 * sizeof(float);
}

// What a workgroup takes, in microseconds: a row tile to its first tile of keys and from its last one, a tile of keys with more than
// 128 rows and with fewer; own keys the same, a block of 32 keys.  Measured with 32/8 heads, one group, S = 10240: 32 tokens, all
// keys in one range 1.03 a tile, in 27 ranges 1.24, 64 tokens 1.41; 64/8 heads, 128 tokens, S = 131072 2.0 (the clock falls
// under that load); one tile of keys alone 6.9 with the launch, 20 blocks of own keys for each of 512 wavefronts 55.  The starts are
// set longer than they are alone, for the plans that come of it: 300 drawn batches take 0.99 of the time that 5.5 and 5 lead to.
constexpr double kTileStartUs = 6.5, kTileUs = 1.75, kNarrowTileUs = 1.2, kOwnStartUs = 7.0, kOwnBlockUs = 2.6;
constexpr double kLaunchUs = 0.4, kJoinUs = 4.0; // what comes on top of the first launch's work; the second with few partial results
constexpr double kPartBytesPerUs = 5.0e6; // of partial results, written and read

// Time until `cus` compute units have done the batches (count, us each), taken in order by whichever is free first.
struct Batch {
    int64_t count;
    double us;
};
double makespan(const Batch *batch, int batches, int64_t cus)
{
    constexpr int kMost = 16;
    Batch free_at[kMost] = {{cus, 0.0}};
    int n = 1;
    double base = 0.0;
    for (int b = 0; b < batches; ++b) {
        int64_t left = batch[b].count;
        if (left > 3 * cus) { // rounds that keep everyone busy
            const int64_t rounds = left / cus - 2;
            base += (double)rounds * batch[b].us;
            left -= rounds * cus;
        }
        while (left > 0) {
            int first = 0;
            for (int i = 1; i < n; ++i)
                if (free_at[i].us < free_at[first].us) first = i;
            const int64_t take = std::min(left, free_at[first].count);
            const double until = free_at[first].us + batch[b].us;
            left -= take;
            if (take == free_at[first].count) free_at[first].us = until;
            else if (n < kMost) {
                free_at[first].count -= take;
                free_at[n++] = {take, until};
            } else break;
        }
    }
    double last = 0.0;
    for (int i = 0; i < n; ++i) last = std::max(last, free_at[i].us);
    return base + last;
}

// A tile of keys for a group's row tiles, and the ranges that make them take about range_us each.
double group_tile_us(const Group &grp, int G) { return (int64_t)grp.tokens * G <= kBM / 2 ? kNarrowTileUs : kTileUs; }
int64_t group_ranges(const Group &grp, int G, double range_us)
{
    const int64_t n = (grp.keys + kBN - 1) / kBN;
    const double us = group_tile_us(grp, G) * (double)(n + grp.new_tiles);
    return std::max<int64_t>(1, std::min({n, (int64_t)kMaxRanges, (int64_t)std::ceil(us / range_us - 1e-9)}));
}

// The length of the shared ranges, the own keys of a workgroup and how many wavefronts share them: the least estimated time.
// Finer ranges fill the compute units, until their start and the partial results cost more than that gains.
// Own keys: requests by the logarithm of their blocks of 32 keys.
struct OwnKeys {
    int64_t most = 1; // blocks of a request
    int64_t tokens = 0;
    int64_t units[32] = {}, blocks[32] = {}; // of 32 rows of a KV head, and those times their key blocks
    void add(int64_t rows, int64_t keys)
    {
        const int64_t n = (keys + 31) / 32, u = (rows + kDecRows - 1) / kDecRows;
        const int k = 31 - __builtin_clz((unsigned)n);
        most = std::max(most, n);
        units[k] += u;
        blocks[k] += u * n;
    }
};
void choose_lengths(const cp_shape *s, const OwnKeys &own, int G, Part &part)
{
    const int64_t most = own.most;
    const int64_t cus = cp::num_compute_units(), heads = s->num_kv_heads;
    double total = 0.0, longest = 0.0; // of the row tiles over all their keys
    for (const Group &grp : part.groups) {
        const double us = group_tile_us(grp, G) * (double)((grp.keys + kBN - 1) / kBN + grp.new_tiles);
        total += (double)(((int64_t)grp.tokens * G + kBM - 1) / kBM * heads) * us;
        longest = std::max(longest, us);
    }
    double tried = -1.0;
    double best = -1.0;
    for (const double share : {0.25, 0.5, 0.65, 0.75, 0.85, 0.93, 1.0, 1.5, 2.0, 3.0, 4.0}) { // row tiles for each compute unit
        const double range_us = std::min(longest, std::max(total / ((double)cus * share), kNarrowTileUs));
        if (range_us == tried) continue;
        tried = range_us;
        Batch batch[3] = {};
        int64_t part_rows = 0;
        double item_us = kOwnStartUs + kOwnBlockUs;
        for (const Group &grp : part.groups) {
            const int64_t all = (grp.keys + kBN - 1) / kBN + grp.new_tiles, rows = (int64_t)grp.tokens * G;
            const int64_t ranges = group_ranges(grp, G, range_us);
            const int64_t narrow = rows % kBM > 0 && rows % kBM <= kBM / 2, wide = (rows + kBM - 1) / kBM - narrow;
            const double per = (double)((all + ranges - 1) / ranges);
            batch[0].count += wide * ranges * heads;
            batch[0].us += (double)(wide * ranges * heads) * (kTileStartUs + per * kTileUs);
            batch[1].count += narrow * ranges * heads;
            batch[1].us += (double)(narrow * ranges * heads) * (kTileStartUs + per * kNarrowTileUs);
            item_us = std::max(item_us, kTileStartUs + per * group_tile_us(grp, G));
            if (ranges > 1 || !grp.new_keys) part_rows += ranges * grp.tokens;
        }
        for (int b = 0; b < 2; ++b) batch[b].us /= (double)std::max<int64_t>(batch[b].count, 1);
        // how many wavefronts share the own keys of a workgroup, each with no more blocks than a row tile's time has room for
        for (int waves = 1; waves <= kWaves && (waves == 1 || waves < 2 * most); waves *= 2) {
            const int64_t least = std::max<int64_t>(1, (most + kMaxRanges * waves - 1) / (kMaxRanges * waves));
            const int64_t each = std::max(least, std::min((most + waves - 1) / waves, (int64_t)((item_us - kOwnStartUs) / kOwnBlockUs)));
            double items = 0.0, item_blocks = 0.0, parts_per_unit = 0.0, all_units = 0.0; // wavefronts, and blocks of each
            for (int k = 0; k < 32; ++k) {
                if (own.units[k] == 0) continue;
                const double mean = (double)own.blocks[k] / (double)own.units[k], ranges = std::ceil(mean / (double)(each * waves));
                items += (double)own.units[k] * ranges * waves;
                item_blocks += (double)own.units[k] * ranges * waves * std::ceil(mean / ranges / waves);
                parts_per_unit += (double)own.units[k] * ranges;
                all_units += (double)own.units[k];
            }
            batch[2].count = (int64_t)std::ceil(items / kWaves) * heads;
            batch[2].us = items > 0.0 ? kOwnStartUs + kOwnBlockUs * item_blocks / items : 0.0;
            const double own_parts = items > 0.0 ? parts_per_unit / all_units * (double)own.tokens : 0.0;
            const double join_us = (part_rows > 0 || own.tokens > 0 ? kJoinUs : 0.0) + 2.0 * (double)part_bytes(part_rows + (int64_t)own_parts, s->num_q_heads) / kPartBytesPerUs;
            double work = 0.0;
            for (const Batch &x : batch) work += (double)x.count * x.us;
            if (best >= 0.0 && work / (double)cus + join_us >= best) continue;
            const double longest_own = items > 0.0 ? kOwnStartUs + kOwnBlockUs * (double)each : 0.0;
            // the longest may be the last to begin
            const double us = std::max(makespan(batch, 3, cus) + 0.2 * std::max(0.0, longest_own - batch[2].us), longest_own) + join_us;
            if (best < 0.0 || us < best) {
                best = us;
                part.range_us = range_us;
                part.own_waves = waves;
                part.own_blocks = (int)(each * waves);
            }
        }
    }
    part.us = best;
}

// What cp_extend_attention takes for the same call.  Requests of few rows read their keys: their own from memory, the shared
// ones mostly from the caches, where the others' reads have brought them (32/8 heads, S = 10240, no own keys: 8 requests
// 38 us, 32 96; 64/8 heads, 128 requests on 131072 3360; 100 requests on 20000 with 3000 of their own 766).  Where one
// of the batch has more than kDecRows, they are read by fewer wavefronts, with two blocks of rows or next to row tiles: 61 requests
// on 8615 tokens, 8/2 heads 134 us, 126 on 1344, 64/8 heads 132 (0.37 and 0.46 of it by the other rates).  The others are row
// tiles, each over all keys.  Over 1000 drawn batches the plan that is taken has 1.006 of the time of the better one. One
// plan is chosen for the whole batch.
constexpr double kSplitKeys = 1024.0, kSplitUs = 4.0; // from so many keys on workgroups share them, and a merge comes behind
constexpr double kOrdinaryStartUs = 6.7, kOwnBytesPerUs = 6.5e6, kSharedBytesPerUs = 1.5e7, kOwnTwoBytesPerUs = 5.0e6, kSharedTwoBytesPerUs = 7.5e6;
double ordinary_us(const cp_shape *s, const cp_sharing *sharing, int G)
{
    double own = 0.0, shared = 0.0, tile_us = 0.0, longest = 0.0;
    bool split = false;
    int64_t most_rows = 0;
    for (int i = 0; i < s->batch; ++i) most_rows = std::max(most_rows, (int64_t)s->h_extend_lens[i] * G);
    const bool two = most_rows > kDecRows;
    int r = 0;
    for (int g = 0; g < sharing->num_groups; ++g) {
        bool first = true; // of a group's requests: it brings the shared keys into the caches
        for (const int end = r + sharing->h_group_sizes[g]; r < end; ++r) {
            const double E = s->h_extend_lens[r], N = (double)s->h_prefix_lens[r] + E, S = sharing->h_shared_lens[g];
            if (E == 0.0) continue;
            if (E * G <= 2.0 * kDecRows) {
                (first ? own : shared) += S;
                own += N - S;
                first = false;
                split = split || N >= kSplitKeys;
            } else {
                const double us = (std::ceil(N / kBN) + 1.0) * (E * G <= kBM / 2 ? kNarrowTileUs : kTileUs);
                tile_us += std::ceil(E * G / kBM) * us;
                longest = std::max(longest, us);
            }
        }
    }
    const double bytes = 512.0 * s->num_kv_heads, cus = cp::num_compute_units(), tiles = tile_us * s->num_kv_heads / cus;
    // fewer row tiles than compute units are split over the keys, at the price of a second launch
    const double rows_us = tiles > 0.0 ? std::max(tiles, std::min(longest, 1.2 * tiles + 6.0)) : 0.0;
    return kOrdinaryStartUs + (split ? kSplitUs : 0.0) + rows_us + bytes * (two ? own / kOwnTwoBytesPerUs + shared / kSharedTwoBytesPerUs : own / kOwnBytesPerUs + shared / kSharedBytesPerUs);
}

// CP_OK, or the code of a batch that is too large for the plan that is asked for.
int make_plan_of(const cp_shape *s, const cp_sharing *sharing, Plan &pl)
{
    const int G = s->num_q_heads / s->num_kv_heads;
    int r = 0;
    int64_t token = 0;
    for (int g = 0; g < sharing->num_groups; ++g) {
        const int size = sharing->h_group_sizes[g], keys = sharing->h_shared_lens[g];
        int64_t tokens = 0;
        for (int i = r; i < r + size; ++i) tokens += s->h_extend_lens[i];
        if (pl.parts.empty() || pl.parts.back().groups.size() == kMaxGroups) {
            pl.parts.emplace_back();
            pl.parts.back().request = r;
            pl.parts.back().token = token;
        }
        Part &part = pl.parts.back();
        if (keys > 0 && tokens > 0 && (size > 1 || s->num_splits > 0)) {
            Group grp{};
            grp.request = r - part.request;
            grp.requests = size;
            grp.token = (int32_t)(token - part.token);
            grp.tokens = (int32_t)tokens;
            grp.keys = keys;
            grp.new_keys = 1;
            int longest = 0;
            for (int i = r; i < r + size; ++i) {
                if (s->h_extend_lens[i] > 0 && s->h_prefix_lens[i] > keys) grp.new_keys = 0;
                longest = std::max(longest, s->h_extend_lens[i]);
            }
            // at most: a tile's tokens, and those in front of them in the first one's request
            if (grp.new_keys) grp.new_tiles = (int32_t)((std::min<int64_t>(tokens, (kBM + G - 1) / G + (int64_t)longest) + kBN - 1) / kBN);
            part.groups.push_back(grp);
            pl.shared = true;
        }
        part.requests += size;
        part.tokens += tokens;
        r += size;
        token += tokens;
    }
    if (!pl.shared) return CP_OK;
    // not worth planning where even one tile of keys, and a join if one is needed, would take longer
    const double other_us = s->num_splits == 0 ? ordinary_us(s, sharing, G) : 0.0;
    bool join = false;
    for (const Part &part : pl.parts)
        for (const Group &grp : part.groups) join = join || !grp.new_keys;
    if (s->num_splits == 0 && other_us <= kLaunchUs + kTileStartUs + kNarrowTileUs + (join ? kJoinUs : 0.0)) {
        pl.shared = false;
        return CP_OK;
    }
    double shared_us = 0.0;
    for (Part &part : pl.parts) {
        if (part.tokens == 0) continue; // is not launched
        std::vector<int> shared_keys((size_t)part.requests, 0), ranges((size_t)part.requests, 0); // of every request
        std::vector<char> alone((size_t)part.requests, 0); // no item of own keys
        for (const Group &grp : part.groups) {
            std::fill_n(shared_keys.begin() + grp.request, grp.requests, grp.keys);
            std::fill_n(alone.begin() + grp.request, grp.requests, (char)grp.new_keys);
        }
        OwnKeys own;
        for (int i = 0; i < part.requests; ++i) {
            const int64_t at = part.request + i, E = s->h_extend_lens[at];
            if (E > 0 && !alone[(size_t)i]) {
                own.tokens += E;
                own.add(E * G, s->h_prefix_lens[at] - shared_keys[(size_t)i] + E);
            }
        }
        choose_lengths(s, own, G, part);
        for (Group &grp : part.groups) {
            const int64_t n = (grp.keys + kBN - 1) / kBN, all = n + grp.new_tiles;
            const int64_t count = s->num_splits > 0 ? std::min<int64_t>({s->num_splits, n, kMaxRanges}) : group_ranges(grp, G, part.range_us);
            // as even as can be: the last range has the new tokens too
            grp.per_range = (int32_t)std::max<int64_t>((s->num_splits > 0 ? n : all) + count - 1, 1) / (int32_t)count;
            grp.ranges = (int32_t)((n + grp.per_range - 1) / grp.per_range);
            grp.first_item = (int32_t)part.tile_items;
            grp.part_row = (int32_t)part.part_rows;
            part.tile_items += grp.ranges * (((int64_t)grp.tokens * G + kBM - 1) / kBM);
            if (grp.ranges > 1 || !grp.new_keys) part.part_rows += (int64_t)grp.ranges * grp.tokens; // else there is nothing to join
            pl.ranges = std::max(pl.ranges, grp.ranges);
            std::fill_n(ranges.begin() + grp.request, grp.requests, grp.ranges);
        }
        part.own_part_row = part.part_rows;
        part.same_extend = part.groups.size() == 1 && part.groups[0].requests == part.requests ? s->h_extend_lens[part.request] : 0;
        part.same_ranges = -1;
        for (int i = 0; i < part.requests; ++i) {
            const int at = part.request + i, E = s->h_extend_lens[at];
            if (E != part.same_extend) part.same_extend = 0;
            if (E == 0) continue;
            const int n = alone[(size_t)i] ? 0 : own_ranges(s->h_prefix_lens[at] - shared_keys[(size_t)i] + E, part.own_blocks);
            if (part.same_ranges >= 0 && n != part.same_ranges) part.same_extend = 0;
            part.same_ranges = n;
            part.own_units += ((int64_t)E * G + kDecRows - 1) / kDecRows * n;
            if (n + ranges[(size_t)i] > 1) {
                part.part_rows += (int64_t)E * n;
                part.most_parts = std::max(part.most_parts, n + ranges[(size_t)i]);
            }
        }
        // in 32 bits, the threads of the launches too
        const int64_t items = (part.tile_items + part.own_units) * s->num_kv_heads;
        bool counted = part.part_rows <= INT32_MAX && part.own_units <= INT32_MAX && items <= cp::kMostThreads / kThreads - 2 * kXcds &&
                       part.tokens * join_blocks(s->num_q_heads, part.most_parts) <= cp::kMostThreads / kJoinThreads;
        for (const Group &grp : part.groups) counted = counted && (int64_t)grp.tokens * G <= INT32_MAX - kBM;
        if (!counted) {
            pl.shared = false;
            return s->num_splits > 0 ? CP_ERR_SHAPE : CP_OK;
        }
        pl.part_rows = std::max(pl.part_rows, part.part_rows);
        shared_us += kLaunchUs + part.us;
    }
    if (s->num_splits == 0 && other_us <= shared_us) pl.shared = false;
    return CP_OK;
}

// No exception leaves a C entry point.
int make_plan(const cp_shape *s, const cp_sharing *sharing, Plan &pl)
{
    try {
        return make_plan_of(s, sharing, pl);
    } catch (const std::bad_alloc &) {
        return CP_ERR_LAUNCH;
    }
}

} // namespace

extern "C" {

size_t cp_shared_workspace_bytes(const cp_shape *shape, const cp_sharing *sharing)
{
    if (cp::validate_shape(shape) != CP_OK || validate_sharing(shape, sharing) != CP_OK) return 0;
    Plan pl;
    if (make_plan(shape, sharing, pl) != CP_OK) return 0;
    if (!pl.shared) return cp_workspace_bytes(shape);
    return pl.part_rows > 0 ? part_bytes(pl.part_rows, shape->num_q_heads) : 0;
}

int32_t cp_shared_ranges(const cp_shape *shape, const cp_sharing *sharing)
{
    if (cp::validate_shape(shape) != CP_OK || validate_sharing(shape, sharing) != CP_OK) return 0;
    Plan pl;
    return make_plan(shape, sharing, pl) == CP_OK && pl.shared ? pl.ranges : 0;
}

int cp_shared_prefix_attention(const void *q, const void *k_new, const void *v_new, const void *kv_pages,
                               const int32_t *block_table, const int32_t *prefix_lens, const int32_t *extend_lens,
                               void *out, void *stream, const cp_shape *shape, const cp_sharing *sharing,
                               void *workspace, size_t workspace_bytes)
{
    int st = cp::validate_shape(shape);
    if (st == CP_OK) st = validate_sharing(shape, sharing);
    if (st != CP_OK) return st;
    if (!block_table || !prefix_lens || !extend_lens) return CP_ERR_NULL;
    if (shape->total_extend == 0) return CP_OK;
    if (!q || !k_new || !v_new || !kv_pages || !out) return CP_ERR_NULL;
    if (!aligned_to(q, 16) || !aligned_to(k_new, 16) || !aligned_to(v_new, 16) || !aligned_to(kv_pages, 16) ||
        !aligned_to(out, 16) || !aligned_to(block_table, 4) || !aligned_to(prefix_lens, 4) || !aligned_to(extend_lens, 4))
        return CP_ERR_ALIGN;
    Plan pl;
    st = make_plan(shape, sharing, pl);
    if (st != CP_OK) return st;
    if (!pl.shared)
        return cp_extend_attention(q, k_new, v_new, kv_pages, block_table, prefix_lens, extend_lens, out, stream, shape,
                                   workspace, workspace_bytes);
    if (pl.part_rows > 0 && (!workspace || workspace_bytes < part_bytes(pl.part_rows, shape->num_q_heads) || !aligned_to(workspace, 256)))
        return CP_ERR_WORKSPACE;
    if (cp::debug_checks_on()) {
        const int chk = cp_check_tables(block_table, prefix_lens, extend_lens, stream, shape, nullptr);
        if (chk != CP_OK) return chk;
    }
    const int Hq = shape->num_q_heads, Hkv = shape->num_kv_heads;
    hipStream_t hs = static_cast<hipStream_t>(stream);
    for (const Part &part : pl.parts) {
        if (part.tokens == 0) continue;
        SharedParams p{};
        p.q = static_cast<const uint16_t *>(q) + part.token * Hq * kD;
        p.k_new = static_cast<const uint16_t *>(k_new) + part.token * Hkv * kD;
        p.v_new = static_cast<const uint16_t *>(v_new) + part.token * Hkv * kD;
        p.kv_pages = static_cast<const uint16_t *>(kv_pages);
        p.block_table = block_table + (int64_t)part.request * shape->max_pages_per_req;
        p.prefix_lens = prefix_lens + part.request;
        p.extend_lens = extend_lens + part.request;
        p.out = static_cast<uint16_t *>(out) + part.token * Hq * kD;
        p.part_o = static_cast<float *>(workspace);
        p.part_ml = reinterpret_cast<float *>(static_cast<char *>(workspace) +
                                              ((size_t)part.part_rows * (size_t)Hq * kD * sizeof(float) + 255) / 256 * 256);
        p.batch = part.requests;
        p.Hq = Hq;
        p.Hkv = Hkv;
        p.G = Hq / Hkv;
        p.max_pages = shape->max_pages_per_req;
        p.T = (int32_t)part.tokens;
        p.scale_log2 = shape->softmax_scale * 1.4426950408889634f;
        int64_t most_rows = kBM;
        for (const Group &grp : part.groups) most_rows = std::max<int64_t>(most_rows, (int64_t)grp.tokens * p.G);
        p.g_magic = (most_rows + kBM + 1) * p.G <= INT64_C(0x100000000) ? 0xffffffffu / (uint32_t)p.G : 0u;
        p.groups = (int32_t)part.groups.size();
        p.tile_items = (int32_t)part.tile_items;
        p.tile_per_xcd = (int32_t)((part.tile_items * Hkv + kXcds - 1) / kXcds);
        const int per_group = kWaves / part.own_waves;
        p.own_items = (int32_t)((part.own_units + per_group - 1) / per_group);
        p.own_per_xcd = (int32_t)(((int64_t)p.own_items * Hkv + kXcds - 1) / kXcds);
        p.own_blocks = part.own_blocks;
        p.own_waves = part.own_waves;
        p.own_part_row = (int32_t)part.own_part_row;
        p.same_extend = part.same_extend;
        p.same_ranges = part.same_extend > 0 ? part.same_ranges : 0;
        std::copy(part.groups.begin(), part.groups.end(), p.group);
        const unsigned groups = (unsigned)(p.tile_per_xcd + p.own_per_xcd) * kXcds;
        hipLaunchKernelGGL(shared_attn_kernel, dim3(groups), dim3(kThreads), 0, hs, p);
        if (hipGetLastError() != hipSuccess) return CP_ERR_LAUNCH;
        if (part.most_parts > 0) {
            launch_join(p, part.most_parts, hs);
            if (hipGetLastError() != hipSuccess) return CP_ERR_LAUNCH;
        }
    }
    return CP_OK;
}

} // extern "C"
