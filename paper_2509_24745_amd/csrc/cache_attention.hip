// Attention of a batch's newest tokens over the paged cache.
//
// The rows of a (sequence, KV head) are its new tokens' query heads, 16 NR of
// them to a workgroup; a wave walks its share of the cached keys in steps of
// 16 KT:
//   S^T = K Q^T    (16x16 MFMA, keys by rows)
//   P^T = exp2(S^T - reference), the sums and the largest score beside it
//   O^T += V^T P^T (16x16 MFMA, values of a head by rows)
// Lane l holds row n = l % 16 of every tile (g = l / 16).  S^T leaves it the
// scores of keys KT (4 g + r) + t of the step (tile t < KT, r < 4): 4 KT
// consecutive keys, and just those that the second product wants from it, so
// P never leaves its lane.  K comes as one 16-byte piece of a key per lane and
// product, V as the 4 KT keys of the lane's group, D/16 values of each, and both go from
// memory to registers: no other wave wants them.  What the MFMAs take for a
// key's index or a value's is free as long as both operands agree, which is
// what picks the orders here (see Rows).
//
// Work is dealt flat: every (sequence, KV head, row tile) is a run of units of
// 64 KT keys (four waves' steps), all runs lie end to end, and workgroup w of W takes the w-th
// equal part, whatever the lengths are.  A run cut between workgroups leaves
// partial rows (reference, sum, output) in the workspace, added up in order by
// a second launch.
//
// Bound: the cache's bytes.  A key and its value take 4 D bytes in bf16 and
// 17/16 D in 4 bits, for 4 D products a row; at 16 rows that is 16 and 60
// products a byte, where the card's rates balance at 250.
#include <algorithm>
#include <type_traits>

#include "cache.h"
#include "cache_device.h"
#include "common.h"
#include "proxyattn.h"

namespace pa {

constexpr int kAttnThreads = 256;   // 4 waves
constexpr int kCus = 256, kCuShift = 8;
constexpr int kCacheGroups = 2 * kCus;   // workgroups at most
// Below any score that a finite row gives: the reference before the first key.
constexpr float kNoScore = -1e30f;
// Scores above the reference by this much (log2) move it: the sums grow by
// 2^kSlack at most.
constexpr float kSlack = 8.f;

typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));

// 16-key tiles of a step: 32 keys in 4 bits with one row tile, 64 with several,
// 32 in bf16 and in fp32 up to 64 values, 16 otherwise, so that two steps' keys and
// values fit beside the rows.  (4 bits, 64 and 32 keys, us: 64 sequences to 32K 34.9,
// 33.6, one of 128K 36.9, 36.5; 8 to 60K with 36 rows 61, 75.)
constexpr int key_tiles(bool fp4, int esz, int d, int nr) {
    return fp4 ? (nr == 1 ? 2 : 4) : esz * d > 256 ? 1 : 2;
}

// Workgroups that a CU holds: as many as the registers allow.
constexpr int groups_per_cu(bool fp4, int esz, int d, int nr) {
    return nr == 1 || (nr == 2 && (fp4 || d == 64)) || (nr == 3 && !fp4 && d == 64) ? 2 : 1;
}

// Units that a run's start counts for when the work is dealt: a workgroup's
// time goes by the runs it starts as well as by the keys it reads.  They lie
// before the run's first keys.  With 0, 1, 2, 3 and 4 of them (us): 64 sequences of up to
// 32K tokens in 4 bits 44.7, 37.1, 36.0, 37.4, 37.2; 64 to 8K in bf16 -, 87.8, 88.7, 92.7,
// 94.7, 4 to 24K with 9 new tokens 47.1, 45.2, 43.1, 41.1, 43.4.
constexpr int start_units(bool fp4, int nr) { return fp4 ? 2 : nr == 1 ? 1 : 3; }

// Up to so many units a run is a workgroup's own, by the number of runs: one
// launch, and nobody looks up who has what.  Calls in a graph, 32 query heads on 8,
// d 128, whole against cut (us): 1 sequence (8 runs) of 512 keys in bf16 (4 units)
// 8.5 / 8.8, of 1024 12.7 / 8.7; 8 sequences of 1024 13.6 / 15.7, in 4 bits (8 units
// too) 9.1 / 11.1; 64 of 1024 44.2 / 47.6.  Longer runs of many sequences gain as
// much where their lengths are equal, but lose more where they are not.
static int whole_units(int64_t runs) { return runs >= 64 ? 8 : 4; }

// A sequence of the batch as the header reads its arrays.
struct Seq {
    int len, row, fresh;   // cached tokens, first row, new tokens
};
__device__ __forceinline__ Seq seq_at(const CacheShape& s, const int* lens, const int* starts,
                                      int b) {
    Seq q;
    q.len = min(max(lens[b], 0), s.max_len);
    q.row = b;
    q.fresh = 1;
    if (starts) {
        q.row = min(max(starts[b], 0), s.t);
        q.fresh = min(max(min(starts[b + 1], s.t) - q.row, 0), s.max_new);
    }
    return q;
}

// Row tiles of a KV head and units of a row tile.
template <int ROWS, int UNIT, int START> struct Runs {
    int tiles, units;
    __device__ __forceinline__ Runs(const CacheShape& s, const Seq& q)
        : tiles((q.fresh * s.rep + ROWS - 1) / ROWS), units(max(1, (q.len + UNIT - 1) / UNIT)) {}
    __device__ __forceinline__ int flat() const { return units + START; }
};

__device__ __forceinline__ int wave_uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }

// Sums of x over the lanes up to each (within rows of 16 lanes, then across).
__device__ __forceinline__ int wave_sums(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr 1, 2, 4, 8
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // lane 15 of a row to the next
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);   // lane 31 to the upper half
    return x;
}

// Which sequence a flat unit lies in, its first unit, and the number of all
// units.  A block of 256 threads.  plan (not NULL): every sequence's first unit
// is left there, the total behind them.  seqs: the sequences, up to 256 of them.
struct Found {
    int begin, end, b, base;   // the workgroup's units; the sequence that begin lies in
};
// Workgroup w's first unit of `total`, and the workgroup that unit f is with.
// Fewer than kCus or twice kCus workgroups are as many as there can be units,
// and have one each (or none).
__device__ __forceinline__ int first_unit(int total, int groups, int w) {
    if (total <= groups) return min(w, total);
    return (int)((int64_t)w * total >> (groups == kCus ? kCuShift : kCuShift + 1));
}
__device__ __forceinline__ int group_of(int total, int groups, int f) {
    if (total <= groups) return f;
    // in doubles: the quotient is at least 1 / total off every whole number above it
    return (int)((((double)f + 1) * groups - 1) / total);
}
template <int ROWS, int UNIT, int START>
__device__ __forceinline__ Found find_unit(const CacheShape& s, const int* lens, const int* starts,
                                           int* plan, int groups, int group, Seq* seqs) {
    __shared__ int wave_total[4];
    __shared__ int found[2];
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int chunk = (s.b + kAttnThreads - 1) / kAttnThreads;
    const int b0 = min(tid * chunk, s.b), b1 = min(b0 + chunk, s.b);
    auto count = [&](const Seq& q) {
        const Runs<ROWS, UNIT, START> r(s, q);
        return s.hkv * r.tiles * r.flat();
    };
    if (s.b <= 64) {   // every wave for itself: no barriers (0.85 us less before the first load)
        const Seq q = seq_at(s, lens, starts, min(lane, s.b - 1));
        const int n = lane < s.b ? count(q) : 0, incl = wave_sums(n);
        seqs[lane] = q;   // the same by all four
        const int all = __builtin_amdgcn_readlane(incl, 63);
        const int want = first_unit(all, groups, group), end = first_unit(all, groups, group + 1);
        if (plan && wave == 0) {
            if (lane < s.b) plan[lane] = incl - n;
            if (lane == 0) plan[s.b] = all;
        }
        const int b = want < end ? __popcll(__ballot(incl <= want)) : 0;
        return {want, end, b, __builtin_amdgcn_readlane(incl - n, b)};
    }
    int mine = 0;
    for (int b = b0; b < b1; ++b) {
        const Seq q = seq_at(s, lens, starts, b);
        if (chunk == 1) seqs[tid] = q;
        mine += count(q);
    }
    const int incl = wave_sums(mine);
    if (lane == 63) wave_total[wave] = incl;
    __syncthreads();
    int before = incl - mine, all = 0;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        if (w < wave) before += wave_total[w];
        all += wave_total[w];
    }
    const int want = first_unit(all, groups, group), end = first_unit(all, groups, group + 1);
    if (plan || (want >= before && want < before + mine)) {
        int at = before;
        for (int b = b0; b < b1; ++b) {
            const int n = chunk == 1 ? mine : count(seq_at(s, lens, starts, b));
            if (plan) plan[b] = at;
            if (want >= at && want < at + n) {
                found[0] = b;
                found[1] = at;
            }
            at += n;
        }
    }
    if (plan && tid == 0) plan[s.b] = all;
    __syncthreads();
    const bool any = want < end;
    return {want, end, any ? wave_uniform(found[0]) : 0, any ? wave_uniform(found[1]) : 0};
}

// ---------------------------------------------------------------------------
// K and V of a step, from memory to registers
// ---------------------------------------------------------------------------
template <typename T, bool FP4, int D, int TILES> struct KeyStep;

// A load, past the caches or not (see CacheShape::past).
template <bool PAST, typename V> __device__ __forceinline__ V fetch(const void* p) {
    if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const V*>(p));
    return *reinterpret_cast<const V*>(p);
}

// The problem's own type.  Chunk i of a key is its values 16 B of which lane
// group g holds: for bf16 8 values 32 i + 8 g, for fp32 4 values 16 i + 4 g.
template <typename T, int D, int TILES> struct KeyStep<T, false, D, TILES> {
    static constexpr int KT = TILES, N = 16 / sizeof(T);
    static constexpr int KC = D / 4 / N;              // 16-byte pieces of a key for a lane
    static constexpr int VW = D / 16 * sizeof(T) / 4; // words of a value row for a lane
    u32x4 k[KT][KC];
    uint32_t v[4 * KT][VW];

    template <bool PAST>
    __device__ __forceinline__ void load(const CacheShape& s, const PagePtrs& pg, int kpage,
                                         int vpage, int head, int kpos, int vpos, int lane) {
        const int g = lane >> 4, m = lane & 15, mask = (1 << s.page_shift) - 1;
        const T* kp = (const T*)pg.k +
                      ((((int64_t)kpage * s.hkv + head) << s.page_shift) + (kpos & mask)) * D + N * g;
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int i = 0; i < KC; ++i)
                k[t][i] = fetch<PAST, u32x4>(kp + t * D + 4 * N * i);
        const T* vp = (const T*)pg.v +
                      ((((int64_t)vpage * s.hkv + head) << s.page_shift) + (vpos & mask)) * D +
                      D / 16 * m;
#pragma unroll
        for (int x = 0; x < 4 * KT; ++x) {
            if constexpr (VW % 4 == 0) {
#pragma unroll
                for (int i = 0; i < VW; i += 4) {
                    const u32x4 w = fetch<PAST, u32x4>(vp + x * D + i * 4 / sizeof(T));
#pragma unroll
                    for (int j = 0; j < 4; ++j) v[x][i + j] = w[j];
                }
            } else {
                const u32x2 w = fetch<PAST, u32x2>(vp + x * D);
                v[x][0] = w[0];
                v[x][1] = w[1];
            }
        }
    }
    // Values from key `from` of the lane's on are none: a probability of 0 times
    // what an unwritten slot holds has to be 0.
    __device__ __forceinline__ void drop_values(int from) {
#pragma unroll
        for (int x = 0; x < 4 * KT; ++x)
#pragma unroll
            for (int i = 0; i < VW; ++i) v[x][i] = x < from ? v[x][i] : 0u;
    }
};

// 4 bits.  A lane holds the D/4 values (D/4) g .. of each of its keys, D/16 of
// each of its values, and their scales.
template <typename T, int D, int TILES> struct KeyStep<T, true, D, TILES> {
    static constexpr int KT = TILES;
    static constexpr int KC = D / 32;   // words of a key for a lane
    uint32_t k[KT][KC];
    uint32_t ks;        // scales of the lane's KT keys, a byte each
    uint32_t v[4 * KT]; // D = 64: the low half
    uint32_t vs[KT];    // scales of the lane's 4 KT values

    template <bool PAST>
    __device__ __forceinline__ void load(const CacheShape& s, const PagePtrs& pg, int kpage,
                                         int vpage, int head, int kpos, int vpos, int lane) {
        const int g = lane >> 4, m = lane & 15, mask = (1 << s.page_shift) - 1;
        const int64_t kh = (int64_t)kpage * s.hkv + head, vh = (int64_t)vpage * s.hkv + head;
        const uint8_t* kp = (const uint8_t*)pg.k +
                            ((kh << s.page_shift) + (kpos & mask)) * (D / 2) + D / 8 * g;
#pragma unroll
        for (int t = 0; t < KT; ++t) {
            if constexpr (KC == 4) {
                const u32x4 w = fetch<PAST, u32x4>(kp + t * (D / 2));
#pragma unroll
                for (int j = 0; j < 4; ++j) k[t][j] = w[j];
            } else {
                const u32x2 w = fetch<PAST, u32x2>(kp + t * (D / 2));
                k[t][0] = w[0];
                k[t][1] = w[1];
            }
        }
        const uint8_t* ksp = (const uint8_t*)pg.ks +
                             ((kh * (D / 32) + g * (D / 4) / 32) << s.page_shift) + (kpos & mask);
        if constexpr (KT == 4)
            ks = fetch<PAST, uint32_t>(ksp);
        else
            ks = fetch<PAST, uint16_t>(ksp);
        const uint8_t* vp = (const uint8_t*)pg.v +
                            ((vh << s.page_shift) + (vpos & mask)) * (D / 2) + D / 32 * m;
#pragma unroll
        for (int x = 0; x < 4 * KT; ++x) {
            if constexpr (D == 128)
                v[x] = fetch<PAST, uint32_t>(vp + x * (D / 2));
            else
                v[x] = fetch<PAST, uint16_t>(vp + x * (D / 2));
        }
        const uint8_t* vsp = (const uint8_t*)pg.vs +
                             ((vh * (D / 32) + m * (D / 16) / 32) << s.page_shift) + (vpos & mask);
        if constexpr (KT == 4) {
            const u32x4 w = fetch<PAST, u32x4>(vsp);
#pragma unroll
            for (int j = 0; j < KT; ++j) vs[j] = w[j];
        } else {
            const u32x2 w = fetch<PAST, u32x2>(vsp);
            vs[0] = w[0];
            vs[1] = w[1];
        }
    }
    // A scale of an unwritten slot may be no number; 0 times a value is 0.
    __device__ __forceinline__ void drop_values(int from) {
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            const int keep = min(max(from - 4 * j, 0), 4);
            vs[j] = keep == 4 ? vs[j] : vs[j] & ((1u << (8 * keep)) - 1u);
        }
    }
    __device__ __forceinline__ float kscale(int t) const {
        return __uint_as_float((ks >> (8 * t) & 255u) << 23);
    }
    __device__ __forceinline__ float vscale(int x) const {
        return __uint_as_float((vs[x / 4] >> (8 * (x % 4)) & 255u) << 23);
    }
};

// ---------------------------------------------------------------------------
// products
// ---------------------------------------------------------------------------
__device__ __forceinline__ f32x4 mma16(const bf16x8& a, const bf16x8& b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x4 mma16(float a, float b, const f32x4& c) {
    return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ uint32_t fp4_pair_bf16(uint32_t w, float scale, int byte) {
    switch (byte) {   // the byte is an immediate
        case 0: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 0));
        case 1: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 1));
        case 2: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 2));
        default: return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, 3));
    }
}
__device__ __forceinline__ bf16x8 as_frag(const u32x4& w) { return __builtin_bit_cast(bf16x8, w); }

// fp32 values as TERMS bf16 values that add up to them: each the rounding of
// what those before leave (three hold all 24 bits).
template <int TERMS>
__device__ __forceinline__ void split_pair(float a, float b, uint32_t (&w)[TERMS]) {
#pragma unroll
    for (int i = 0; i < TERMS; ++i) {
        w[i] = pack_rne(a, b);
        if (i + 1 < TERMS) {
            a -= __uint_as_float(w[i] << 16);
            b -= __uint_as_float(w[i] & 0xffff0000u);
        }
    }
}

// The queries of NR tiles of 16 rows, as 16-byte pieces for the MFMAs.  Piece i
// of a row for lane group g is what meets the group's part of a key.  Queries in fp32
// over 4-bit keys, which are bf16 values, go as three bf16 terms of 8 values, else a
// piece holds values as they are.  One tile's pieces stay in registers; several
// tiles' lie in LDS, lines padded by 16 bytes so that 16 rows meet all banks, and are
// read in every step: the registers hold the outputs and the next keys.
template <typename T, bool FP4, int D, int NR> struct Queries {
    static constexpr int TERMS = FP4 && sizeof(T) == 4 ? 3 : 1;
    typedef typename std::conditional<TERMS == 3, bf16, T>::type E;
    static constexpr int N = 16 / sizeof(E), QC = D / 4 / N;   // pieces of a term
    static constexpr int LINE = TERMS * D + N;
    static constexpr int LDS = NR == 1 ? 4 : 16 * NR * LINE;   // elements
    static constexpr bool kept = NR == 1;
    static __device__ __forceinline__ int piece_at(int i, int g) {
        return FP4 ? D / 4 * g + N * i : 4 * N * i + N * g;
    }
    u32x4 reg[kept ? TERMS * QC : 1];
    const E* lds;

    // N values of a row as their terms
    static __device__ __forceinline__ void terms(const T* p, u32x4 (&w)[TERMS]) {
        if constexpr (TERMS == 1) {
            w[0] = *reinterpret_cast<const u32x4*>(p);
        } else {
            const f32x4 x[2] = {*reinterpret_cast<const f32x4*>(p),
                                *reinterpret_cast<const f32x4*>(p + 4)};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                uint32_t z[TERMS];
                split_pair(x[j / 2][2 * (j % 2)], x[j / 2][2 * (j % 2) + 1], z);
#pragma unroll
                for (int k = 0; k < TERMS; ++k) w[k][j] = z[k];
            }
        }
    }
    // row(n): row n of the tiles, or NULL for none
    template <typename F> __device__ __forceinline__ void load(E* buf, int lane, F row) {
        lds = buf;
        if constexpr (kept) {
            const T* p = row(lane & 15);
#pragma unroll
            for (int i = 0; i < QC; ++i) {
                u32x4 w[TERMS];
#pragma unroll
                for (int k = 0; k < TERMS; ++k) w[k] = zero_u32x4();
                if (p) terms(p + piece_at(i, lane >> 4), w);
#pragma unroll
                for (int k = 0; k < TERMS; ++k) reg[k * QC + i] = w[k];
            }
        } else {
            for (int x = threadIdx.x; x < 16 * NR * (D / N); x += kAttnThreads) {
                const int n = x / (D / N), c = x % (D / N);
                const T* p = row(n);
                u32x4 w[TERMS];
#pragma unroll
                for (int k = 0; k < TERMS; ++k) w[k] = zero_u32x4();
                if (p) terms(p + N * c, w);
#pragma unroll
                for (int k = 0; k < TERMS; ++k)
                    *reinterpret_cast<u32x4*>(buf + n * LINE + k * D + N * c) = w[k];
            }
            __syncthreads();
        }
    }
    __device__ __forceinline__ u32x4 piece(int nr, int i, int lane, int term = 0) const {
        if constexpr (kept) return reg[term * QC + i];
        return *reinterpret_cast<const u32x4*>(lds + (16 * nr + (lane & 15)) * LINE + term * D +
                                               piece_at(i, lane >> 4));
    }
};

// The rows' side of the products for NR tiles of 16 rows, and a step.  Keys and
// values that are bf16 values: MFMAs of 32 products.  For the scores, product i of
// lane group g takes the values that chunk i of KeyStep holds; for the outputs,
// product (u, i) takes the keys of tiles 2 u and 2 u + 1 and value D/16 m + i of row m.
// Probabilities go as a bf16 and the bf16 of what that rounds off, so that the
// output's own rounding is the only one that shows (error against 64 bits 1.66e-3,
// 2.07e-3 with the one bf16); the MFMAs of the second wait beside the loads.  Not so
// with several row tiles over 4-bit values, which carry errors of some percent
// themselves: one bf16 there (8 sequences to 60K with 36 rows 72 -> 65 us, 16 to 20K
// with 64 rows 75 -> 67).  fp32 rows take three terms of the queries and of the
// probabilities: exact products as with fp32 MFMAs, in a fifth of their cycles.
template <typename T, bool FP4, int D, int NR> struct Rows {
    typedef KeyStep<T, FP4, D, key_tiles(FP4, sizeof(T), D, NR)> Keys;
    typedef Queries<T, FP4, D, NR> Q;
    static constexpr int KT = Keys::KT, QC = D / 32, OC = D / 16;
    static constexpr int PT = Q::TERMS == 3 ? 3 : FP4 && NR > 1 ? 1 : 2;   // terms of a probability
    // With two and four row tiles the scheduler would spread a step's conversions
    // until registers spill (16 sequences to 20K in 4 bits, 64 rows: 96 instead of 67 us);
    // three fit, and gain 3-6 % from the overlap.
    static constexpr bool kApart = NR == 2 || NR == 4;
    Q q;
    f32x4 o[NR][OC];

    __device__ __forceinline__ void scores(const Keys& ks, int lane, f32x4 (&x)[NR][KT]) const {
#pragma unroll
        for (int t0 = 0; t0 < KT; t0 += 2) {
            if constexpr (kApart) __builtin_amdgcn_sched_barrier(0);
            bf16x8 kf[2][QC];
#pragma unroll
            for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int i = 0; i < QC; ++i) {
                    if constexpr (FP4) {
                        u32x4 w;
                        const float sc = ks.kscale(t0 + t);
#pragma unroll
                        for (int j = 0; j < 4; ++j) w[j] = fp4_pair_bf16(ks.k[t0 + t][i], sc, j);
                        kf[t][i] = as_frag(w);
                    } else {
                        kf[t][i] = as_frag(ks.k[t0 + t][i]);
                    }
                }
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
#pragma unroll
                for (int t = 0; t < 2; ++t) x[nr][t0 + t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int k = Q::TERMS - 1; k >= 0; --k)   // smallest first
#pragma unroll
                    for (int i = 0; i < QC; ++i) {
                        const bf16x8 qf = as_frag(q.piece(nr, i, lane, k));
#pragma unroll
                        for (int t = 0; t < 2; ++t)
                            x[nr][t0 + t] = mma16(kf[t][i], qf, x[nr][t0 + t]);
                    }
            }
        }
    }
    __device__ __forceinline__ void outputs(const Keys& ks, const f32x4 (&p)[NR][KT]) {
#pragma unroll
        for (int u = 0; u < KT / 2; ++u) {
            if constexpr (kApart) __builtin_amdgcn_sched_barrier(0);
            bf16x8 pf[NR][PT];
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
                u32x4 f[PT];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    uint32_t z[PT];
                    split_pair(p[nr][2 * u + w / 2][2 * (w % 2)],
                               p[nr][2 * u + w / 2][2 * (w % 2) + 1], z);
#pragma unroll
                    for (int k = 0; k < PT; ++k) f[k][w] = z[k];
                }
#pragma unroll
                for (int k = 0; k < PT; ++k) pf[nr][k] = as_frag(f[k]);
            }
            // slots 2 w, 2 w + 1 of the fragment: keys KT r + 2 u + w / 2, r = 2 (w % 2) and the next
#pragma unroll
            for (int c = 0; c < OC / 2; ++c) {   // values 2 c and 2 c + 1 of the lane's
                u32x4 even, odd;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int x0 = KT * 2 * (w % 2) + 2 * u + w / 2, x1 = x0 + KT;
                    uint32_t a, b;
                    if constexpr (FP4) {
                        a = fp4_pair_bf16(ks.v[x0], ks.vscale(x0), c);
                        b = fp4_pair_bf16(ks.v[x1], ks.vscale(x1), c);
                    } else {
                        a = ks.v[x0][c];
                        b = ks.v[x1][c];
                    }
                    even[w] = __builtin_amdgcn_perm(b, a, 0x05040100u);
                    odd[w] = __builtin_amdgcn_perm(b, a, 0x07060302u);
                }
#pragma unroll
                for (int k = PT - 1; k >= 0; --k)
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr) {
                        o[nr][2 * c] = mma16(as_frag(even), pf[nr][k], o[nr][2 * c]);
                        o[nr][2 * c + 1] = mma16(as_frag(odd), pf[nr][k], o[nr][2 * c + 1]);
                    }
            }
        }
    }
};

// fp32 keys and values: MFMAs of 4 products, one value of each lane group, exact as
// fp32 products are.  Their rate, 1/16 of bf16's, still outruns the cache's bytes
// four times.
template <int D, int NR> struct Rows<float, false, D, NR> {
    typedef KeyStep<float, false, D, key_tiles(false, 4, D, NR)> Keys;
    static constexpr int KT = Keys::KT, QC = D / 16, OC = D / 16;
    Queries<float, false, D, NR> q;
    f32x4 o[NR][OC];

    __device__ __forceinline__ void scores(const Keys& ks, int lane, f32x4 (&x)[NR][KT]) const {
#pragma unroll
        for (int nr = 0; nr < NR; ++nr)
#pragma unroll
            for (int t = 0; t < KT; ++t) x[nr][t] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < QC; ++i) {
            if constexpr (NR > 1) __builtin_amdgcn_sched_barrier(0);
            u32x4 qf[NR];
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) qf[nr] = q.piece(nr, i, lane);
#pragma unroll
            for (int t = 0; t < KT; ++t)
#pragma unroll
                for (int j = 0; j < 4; ++j)
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr)
                        x[nr][t] = mma16(__uint_as_float(ks.k[t][i][j]), __uint_as_float(qf[nr][j]),
                                         x[nr][t]);
        }
    }
    __device__ __forceinline__ void outputs(const Keys& ks, const f32x4 (&p)[NR][KT]) {
#pragma unroll
        for (int t = 0; t < KT; ++t)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (NR > 1) __builtin_amdgcn_sched_barrier(0);
                const int x = KT * r + t;
#pragma unroll
                for (int i = 0; i < OC; ++i)
#pragma unroll
                    for (int nr = 0; nr < NR; ++nr)
                        o[nr][i] = mma16(__uint_as_float(ks.v[x][i]), p[nr][t][r], o[nr][i]);
            }
    }
};

// Over the four lane groups, which hold the same rows.
__device__ __forceinline__ float groups_max(float x) {
    x = fmaxf(x, __shfl_xor(x, 16));
    return halves_max(x);
}
__device__ __forceinline__ float groups_sum(float x) {
    x += __shfl_xor(x, 16);
    return halves_sum(x);
}

template <typename T> __device__ __forceinline__ void store8(T* p, const float (&x)[8]);
template <> __device__ __forceinline__ void store8<bf16>(bf16* p, const float (&x)[8]) {
    u32x4 w;
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = pack_rne(x[2 * j], x[2 * j + 1]);
    *reinterpret_cast<u32x4*>(p) = w;
}
template <> __device__ __forceinline__ void store8<float>(float* p, const float (&x)[8]) {
    *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
    *reinterpret_cast<f32x4*>(p + 4) = f32x4{x[4], x[5], x[6], x[7]};
}

template <typename T, bool FP4, int D, int NR, bool PAST>
__global__ __launch_bounds__(kAttnThreads, groups_per_cu(FP4, sizeof(T), D, NR)) void
cache_attn_kernel(
    CacheShape s, const T* qp, const int* table, const int* lens, const int* starts, PagePtrs pg,
    T* out, float* lse, int max_tiles, int* plan, float2* stat, float* part) {
    typedef typename Rows<T, FP4, D, NR>::Keys Keys;
    constexpr int KT = Keys::KT, SK = 16 * KT, UNIT = 4 * SK, ROWS = 16 * NR, OC = D / 16;
    constexpr int START = start_units(FP4, NR);
    constexpr int LINE = D + 4;   // a row's outputs in LDS, padded by a bank group
    // all row tiles at once where their outputs and another workgroup fit into LDS
    constexpr int MT = sizeof(T) == 2 ? NR : 1;
    __shared__ __align__(16) float merge[4][16 * MT][LINE];
    __shared__ float2 wstat[4][ROWS];
    __shared__ __align__(16) typename Queries<T, FP4, D, NR>::E queries[Queries<T, FP4, D, NR>::LDS];
    const int lane = threadIdx.x & 63, wave = wave_uniform(threadIdx.x >> 6);
    const int g = lane >> 4, n = lane & 15;
    const int group = blockIdx.x;

    auto uniform = [](Seq q) {
        return Seq{wave_uniform(q.len), wave_uniform(q.row), wave_uniform(q.fresh)};
    };
    __shared__ Seq seqs[kAttnThreads];
    const bool own = !plan;   // a workgroup to a run
    Found found = {0, 1, 0, 0};
    if (own)
        found.b = group / (s.hkv * max_tiles);
    else
        found = find_unit<ROWS, UNIT, START>(s, lens, starts, group == 0 ? plan : nullptr,
                                             gridDim.x, group, seqs);
    int f = found.begin, b = found.b, base = found.base;
    while (f < found.end) {
        const Seq sq = uniform(!own && s.b <= kAttnThreads ? seqs[b] : seq_at(s, lens, starts, b));
        const Runs<ROWS, UNIT, START> run(s, sq);
        // units u0 .. u1 - 1 of a run; if these are not all, partial rows go to slot
        int head, row0, u0, u1, slot = 0;
        if (own) {
            const int item = group - b * s.hkv * max_tiles;
            head = item / max_tiles;
            row0 = (item - head * max_tiles) * ROWS;
            u0 = 0;
            u1 = run.units;
            f = 1;
            if (row0 >= run.tiles * ROWS) break;
        } else {
            const int past = base + s.hkv * run.tiles * run.flat();
            if (f >= past) {   // on to the next sequence
                base = past;
                ++b;
                continue;
            }
            const int at = f - base, item = at / run.flat(), u = at - item * run.flat();
            const int ahead = min(run.flat(), u + (found.end - f));
            head = run.tiles == 1 ? item : item / run.tiles;
            row0 = (item - head * run.tiles) * ROWS;
            u0 = max(u - START, 0);
            u1 = ahead - START;
            // a run that goes on from the workgroup before, or starts here
            slot = 2 * group + (f - u + START > found.begin ? 1 : 0);
            f += ahead - u;
            if (u1 <= 0) continue;
        }

        // rows: (new token, query head of the KV head); row n of tile nr sees keys up to limit
        const int rows = sq.fresh * s.rep, newest = sq.len - sq.fresh;
        auto token_of = [&](int row) { return sq.fresh == 1 ? 0 : row / s.rep; };
        Rows<T, FP4, D, NR> r;
        int limit[NR];
        float ref[NR], sum[NR];
        r.q.load(queries, lane, [&](int i) -> const T* {
            const int row = row0 + i, j = token_of(row);
            return row < rows ? qp + (int64_t)(sq.row + j) * s.q_tok +
                                    (int64_t)(head * s.rep + row - j * s.rep) * s.q_head
                              : nullptr;
        });
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            const int row = row0 + 16 * nr + n;
            limit[nr] = row < rows ? newest + token_of(row) : sq.len - 1;
            ref[nr] = kNoScore;
            sum[nr] = 0.f;
#pragma unroll
            for (int i = 0; i < OC; ++i) r.o[nr][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
        const int all_see = newest + token_of(row0);   // keys up to here: every row
        const int some_see = newest + token_of(min(row0 + ROWS, rows) - 1);
        const int key0 = u0 * UNIT, key1 = min(u1 * UNIT, some_see + 1);

        // page of a step's keys for this lane, inside the sequence
        const int* pages = table + (int64_t)b * s.width;
        const int klast = (sq.len - 1) & ~(KT - 1), vlast = (sq.len - 1) & ~(4 * KT - 1);
        auto kpos = [&](int s0) { return min(s0 + KT * n, klast); };
        auto vpos = [&](int s0) { return min(s0 + 4 * KT * g, vlast); };
        auto page = [&](int pos) { return pages[pos >> s.page_shift]; };
        auto clamp_page = [&](int p) { return min(max(p, 0), s.num_pages - 1); };

        auto step = [&](Keys& ks, int s0) {
            f32x4 x[NR][KT];
            r.scores(ks, lane, x);
            if (s0 + SK > sq.len) ks.drop_values(sq.len - (s0 + 4 * KT * g));
            if (s0 + SK - 1 > all_see) {   // some row does not see all of the step
#pragma unroll
                for (int nr = 0; nr < NR; ++nr)
#pragma unroll
                    for (int t = 0; t < KT; ++t)
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (s0 + KT * (4 * g + c) + t > limit[nr]) x[nr][t][c] = kNegInf;
            }
#pragma unroll
            for (int nr = 0; nr < NR; ++nr) {
                float top = x[nr][0][0];
#pragma unroll
                for (int t = 0; t < KT; ++t)
#pragma unroll
                    for (int c = 0; c < 4; ++c) top = fmaxf(top, x[nr][t][c]);
                top *= s.scale2;
                if (__any(top > ref[nr] + kSlack)) {
                    const float next = fmaxf(ref[nr], groups_max(top));
                    const float shrink = fast_exp2(ref[nr] - next);
                    ref[nr] = next;
                    sum[nr] *= shrink;
#pragma unroll
                    for (int i = 0; i < OC; ++i) r.o[nr][i] *= shrink;
                }
#pragma unroll
                for (int t = 0; t < KT; ++t) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) {
                        // fp32: the scale's rounding would show, a score of 20 by 1e-6
                        float less = -ref[nr];
                        if constexpr (sizeof(T) == 4) less = fmaf(x[nr][t][c], s.scale2_rest, less);
                        x[nr][t][c] = fast_exp2(fmaf(x[nr][t][c], s.scale2, less));
                    }
                    sum[nr] += (x[nr][t][0] + x[nr][t][1]) + (x[nr][t][2] + x[nr][t][3]);
                }
            }
            r.outputs(ks, x);
        };

        // Steps key0 + SK (wave + 4 j).  Two register sets: one step's loads
        // run beside the other's products; pages are looked up a step further
        // ahead (their loads come first, so that waiting for them waits for
        // nothing else).
        int s0 = key0 + SK * wave;
        if (s0 < key1) {
            Keys ka, kb;
            int kp = page(kpos(s0)), vp = page(vpos(s0));
            auto read = [&](Keys& ks, int at_key) {   // at_key's pages are in kp, vp
                const int kc = clamp_page(kp), vc = clamp_page(vp);
                const int ahead = at_key + 4 * SK;
                kp = page(kpos(ahead));
                vp = page(vpos(ahead));
                ks.template load<PAST>(s, pg, kc, vc, head, kpos(at_key), vpos(at_key), lane);
            };
            read(ka, s0);
            while (true) {
                const int s1 = s0 + 4 * SK, s2 = s1 + 4 * SK;
                if (s1 < key1) read(kb, s1);
                step(ka, s0);
                if (s1 >= key1) break;
                if (s2 < key1) read(ka, s2);
                step(kb, s1);
                if (s2 >= key1) break;
                s0 = s2;
            }
        }

        // the four waves' rows together, MT row tiles at a time
        const bool whole = u0 == 0 && u1 == run.units;
#pragma unroll
        for (int nr = 0; nr < NR; ++nr) {
            sum[nr] = groups_sum(sum[nr]);
            if (g == 0) wstat[wave][16 * nr + n] = float2{ref[nr], sum[nr]};
        }
#pragma unroll
        for (int m0 = 0; m0 < NR; m0 += MT) {
#pragma unroll
            for (int nr = m0; nr < m0 + MT; ++nr)
#pragma unroll
                for (int c = 0; c < 4; ++c)   // values OC (4 g + c) ..
#pragma unroll
                    for (int i = 0; i < OC; i += 4)
                        *reinterpret_cast<f32x4*>(
                            &merge[wave][16 * (nr - m0) + n][OC * (4 * g + c) + i]) =
                            f32x4{r.o[nr][i][c], r.o[nr][i + 1][c], r.o[nr][i + 2][c],
                                  r.o[nr][i + 3][c]};
            __syncthreads();
            // rows of D/8 pieces of 8 values
            const int piece = threadIdx.x % (D / 8);
            for (int line = threadIdx.x / (D / 8); line < 16 * MT;
                 line += kAttnThreads / (D / 8)) {
                const int at = 16 * m0 + line, row = row0 + at;
                if (row >= rows) break;
                float2 st[4];
                float hi = kNoScore, l = 0.f, z[8];
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    st[w] = wstat[w][at];
                    hi = fmaxf(hi, st[w].x);
                }
#pragma unroll
                for (int j = 0; j < 8; ++j) z[j] = 0.f;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const float k = fast_exp2(st[w].x - hi);
                    l += st[w].y * k;
                    const float* m = &merge[w][line][8 * piece];
#pragma unroll
                    for (int j = 0; j < 8; ++j) z[j] += m[j] * k;
                }
                if (whole) {
                    const int j = token_of(row);
                    const int64_t t = sq.row + j, i = head * s.rep + row - j * s.rep;
                    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
                    for (int e = 0; e < 8; ++e) z[e] *= inv;
                    store8<T>(out + t * s.o_tok + i * s.o_head + 8 * piece, z);
                    if (lse && piece == 0)
                        lse[i * s.t + t] = l > 0.f ? (hi + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
                } else {
                    store8<float>(part + ((int64_t)slot * ROWS + at) * D + 8 * piece, z);
                    if (piece == 0) stat[(int64_t)slot * ROWS + at] = float2{hi, l};
                }
            }
            __syncthreads();
        }
    }
}

// Rows cut between workgroups: their partial rows added up in the order of
// the keys.  TEAM threads (a workgroup or a wave) to a row, the workgroup's rows all of
// one run (sequence, head, tile) blockIdx.x.  D/4 threads hold a partial row, the
// team reads TEAM / (D/4) partial rows side by side, the first EARLY of each thread
// before anything is known of their references.  Whole workgroups are for few rows
// of many parts (8 runs of 4 rows in 64 parts: 4.1 us), waves for many rows, of which
// most were not cut (128 runs of 64 rows: 14.1 -> 6.6 us).
template <typename T, int D, int NR, int UNIT, int START, int TEAM>
__global__ __launch_bounds__(256) void cache_join_kernel(CacheShape s, const int* lens,
                                                         const int* starts, int max_tiles,
                                                         int groups, const int* plan,
                                                         const float2* stat, const float* part,
                                                         T* out, float* lse) {
    constexpr int ROWS = 16 * NR, L4 = D / 4, SIDE = TEAM / L4, EARLY = 4;
    constexpr bool WAVE = TEAM == 64;
    __shared__ float2 piece[WAVE ? 1 : kCacheGroups];
    __shared__ float top[4];
    __shared__ __align__(16) float side[WAVE ? 1 : SIDE][D];
    __shared__ float side_sum[WAVE ? 1 : SIDE];
    const int tid = threadIdx.x % TEAM, e = tid % L4, k = tid / L4;
    const int line = blockIdx.y * (256 / TEAM) + threadIdx.x / TEAM;
    const int per_seq = s.hkv * max_tiles;
    const int b = blockIdx.x / per_seq, item = blockIdx.x - b * per_seq;
    const int head = max_tiles == 1 ? item : item / max_tiles, tile = item - head * max_tiles;
    const Seq sq = seq_at(s, lens, starts, b);
    const int total = plan[s.b], base = plan[b];
    const Runs<ROWS, UNIT, START> run(s, sq);
    const int row = tile * ROWS + line;
    if (tile >= run.tiles || line >= ROWS || row >= sq.fresh * s.rep) return;
    const int f0 = base + (head * run.tiles + tile) * run.flat() + START;
    const int w0 = group_of(total, groups, f0), w1 = group_of(total, groups, f0 + run.units - 1);
    if (w0 == w1) return;
    const int n = w1 - w0 + 1, first = 2 * w0 + (f0 > first_unit(total, groups, w0) ? 1 : 0);
    auto slot = [&](int i) { return (int64_t)(i ? 2 * (w0 + i) : first) * ROWS + line; };
    auto values = [&](int i) {
        return *reinterpret_cast<const f32x4*>(part + slot(i) * D + 4 * e);
    };
    f32x4 early[EARLY];
#pragma unroll
    for (int i = 0; i < EARLY; ++i) early[i] = values(min(k + i * SIDE, n - 1));
    float hi = kNoScore;
    for (int i = tid; i < n; i += TEAM) {
        const float2 st = stat[slot(i)];
        if constexpr (!WAVE) piece[i] = st;
        hi = fmaxf(hi, st.x);
    }
    hi = wave_max(hi);
    if constexpr (!WAVE) {
        if ((tid & 63) == 0) top[tid >> 6] = hi;
        __syncthreads();
        hi = fmaxf(fmaxf(top[0], top[1]), fmaxf(top[2], top[3]));
    }
    auto stat_of = [&](int i) { return WAVE ? stat[slot(i)] : piece[i]; };
    float l = 0.f;
    f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < EARLY; ++i)
        if (k + i * SIDE < n) {
            const float2 st = stat_of(k + i * SIDE);
            const float x = fast_exp2(st.x - hi);
            l += st.y * x;
            z += early[i] * x;
        }
#pragma unroll 4
    for (int i = k + EARLY * SIDE; i < n; i += SIDE) {
        const float2 st = stat_of(i);
        const float x = fast_exp2(st.x - hi);
        l += st.y * x;
        z += values(i) * x;
    }
    const int j = sq.fresh == 1 ? 0 : row / s.rep;
    const int64_t t = sq.row + j, i = head * s.rep + row - j * s.rep;
    T* const o = out + t * s.o_tok + i * s.o_head;
    if constexpr (WAVE) {
#pragma unroll
        for (int x = L4; x < 64; x *= 2) {
            l += __shfl_xor(l, x);
#pragma unroll
            for (int c = 0; c < 4; ++c) z[c] += __shfl_xor(z[c], x);
        }
        const float inv = l > 0.f ? 1.f / l : 0.f;
        if (k == 0) {
            if constexpr (sizeof(T) == 2) {
                u32x2 w = {pack_rne(z[0] * inv, z[1] * inv), pack_rne(z[2] * inv, z[3] * inv)};
                *reinterpret_cast<u32x2*>(o + 4 * e) = w;
            } else {
                *reinterpret_cast<f32x4*>(o + 4 * e) = z * inv;
            }
        }
    } else {
        *reinterpret_cast<f32x4*>(&side[k][4 * e]) = z;
        if (e == 0) side_sum[k] = l;
        __syncthreads();
        if (tid >= D) return;
        float v = 0.f;
        l = 0.f;
#pragma unroll
        for (int x = 0; x < SIDE; ++x) {
            l += side_sum[x];
            v += side[x][tid];
        }
        o[tid] = from_f32_rne<T>(l > 0.f ? v / l : 0.f);
    }
    if (lse && tid == 0)
        lse[i * s.t + t] = l > 0.f ? (hi + __builtin_amdgcn_logf(l)) * kLn2 : kNegInf;
}

// 16-row tiles of a workgroup's rows.  As few row tiles of at most 64 rows as
// there can be, equally full, where the keys' bytes bound the time.  4-bit keys cost more
// to unpack than to read: past 48 rows, two workgroups of 32 rows on a CU beat one of
// 64 (us, 12 sequences of up to 20K, d 128, most tiles 2, 3, 4: bf16 with 36 rows 122, 75,
// 75; 64 rows 119, 125, 82; 96 rows 174, 129, 144; 4 bits 59, 53, 53; 61, 90, 69; 82, 93,
// 118).  fp32 rows fill the registers with two.
static int row_tiles(int64_t rows, bool fp4, int esz) {
    const int64_t n = (rows + 15) / 16;
    if (esz == 4) return (int)std::min<int64_t>(n, 2);
    if (fp4) return n <= 3 ? (int)n : 2;
    const int64_t parts = (n + 3) / 4;
    return (int)((n + parts - 1) / parts);
}

static int max_row_tiles(const CacheShape& s, int tiles) {
    return (int)(((int64_t)s.rep * s.max_new + 16 * tiles - 1) / (16 * tiles));
}

bool cache_ws(const CacheShape& s, CacheWs* w) {
    const int64_t rows = (int64_t)s.rep * s.max_new;
    const int esz = s.dtype == PROXYATTN_BF16 ? 2 : 4;
    w->tiles = row_tiles(rows, s.fp4, esz);
    const int unit = 64 * key_tiles(s.fp4, esz, s.d, w->tiles);
    const int64_t units = (s.max_len + unit - 1) / unit, flat = units + start_units(s.fp4, w->tiles);
    const int64_t runs = (int64_t)s.b * s.hkv * max_row_tiles(s, w->tiles);
    // a workgroup of 256 threads to each run in the second launch
    if (rows > INT32_MAX || runs > INT32_MAX / 256 || runs * flat > INT32_MAX) return false;
    w->joined = units > whole_units(runs);
    if (!w->joined) {
        w->groups = (int)runs;
        w->total = 0;
        return true;
    }
    w->groups = (int)std::max<int64_t>(1, std::min<int64_t>(kCus * groups_per_cu(s.fp4, esz, s.d, w->tiles), runs * flat));
    auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    const size_t parts = (size_t)2 * w->groups * 16 * w->tiles;
    size_t off = 0;
    w->plan = off, off = up(off + (size_t)(s.b + 1) * 4);
    w->stat = off, off = up(off + parts * 8);
    w->part = off, off = up(off + parts * s.d * 4);
    w->total = off;
    return true;
}

// Rows past which a wave, not a workgroup, adds a row's parts up: more would not be
// on the GPU at once.
constexpr int kJoinWaves = 2048;

template <typename T, int D, bool FP4, int NR>
static void attention_as(const CacheShape& s, const void* q, const int* table, const int* lens,
                         const int* starts, const PagePtrs& pg, void* out, float* lse, char* ws,
                         const CacheWs& w, hipStream_t st) {
    const int mt = max_row_tiles(s, NR);
    int* plan = w.joined ? (int*)(ws + w.plan) : nullptr;
    float2* stat = (float2*)(ws + w.stat);
    float* part = (float*)(ws + w.part);
    if (s.past)
        cache_attn_kernel<T, FP4, D, NR, true><<<w.groups, kAttnThreads, 0, st>>>(
            s, (const T*)q, table, lens, starts, pg, (T*)out, lse, mt, plan, stat, part);
    else
        cache_attn_kernel<T, FP4, D, NR, false><<<w.groups, kAttnThreads, 0, st>>>(
            s, (const T*)q, table, lens, starts, pg, (T*)out, lse, mt, plan, stat, part);
    if (!w.joined) return;
    constexpr int UNIT = 64 * key_tiles(FP4, sizeof(T), D, NR);
    const int rows = std::min(16 * NR, s.rep * s.max_new);
    const unsigned runs = (unsigned)s.b * s.hkv * mt;
    if ((int64_t)runs * rows > kJoinWaves)
        cache_join_kernel<T, D, NR, UNIT, start_units(FP4, NR), 64>
            <<<dim3(runs, (rows + 3) / 4), 256, 0, st>>>(s, lens, starts, mt, w.groups, plan, stat,
                                                         part, (T*)out, lse);
    else
        cache_join_kernel<T, D, NR, UNIT, start_units(FP4, NR), 256>
            <<<dim3(runs, rows), 256, 0, st>>>(s, lens, starts, mt, w.groups, plan, stat, part,
                                               (T*)out, lse);
}

hipError_t launch_cache_attention(const CacheShape& s, const void* q, const int* table,
                                  const int* lens, const int* starts, const PagePtrs& pg,
                                  void* out, float* lse, char* ws, const CacheWs& w,
                                  hipStream_t st) {
    by_cache_type(s, [&](auto t, auto d, auto fp4) {
        typedef typename decltype(t)::type T;
        constexpr int D = decltype(d)::value;
        constexpr bool F = decltype(fp4)::value;
        auto run = [&](auto nr) {
            attention_as<T, D, F, decltype(nr)::value>(s, q, table, lens, starts, pg, out, lse, ws,
                                                       w, st);
        };
        if (w.tiles == 1)
            run(std::integral_constant<int, 1>());
        else if (w.tiles == 2)
            run(std::integral_constant<int, 2>());
        else if constexpr (sizeof(T) == 2) {
            if constexpr (F) {
                run(std::integral_constant<int, 3>());
            } else {
                if (w.tiles == 3)
                    run(std::integral_constant<int, 3>());
                else
                    run(std::integral_constant<int, 4>());
            }
        }
    });
    return hipGetLastError();
}

}  // namespace pa
