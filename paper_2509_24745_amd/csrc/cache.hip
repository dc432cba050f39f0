// Norm and rotation of query and key heads, and the paged cache's writes and
// reads (see the header for the formulas and layouts).
//
// All four are passes over rows (one head of one token, d values) bound by the
// memory system.  A row is held by d/16 lanes, 16 values each, as the two
// 8-value chunks that the rotation pairs with one another, so that no value
// leaves its lane: rows are 4 or 8 lanes wide and a wave holds 16 or 8 of them.
#include "cache.h"
#include "cache_device.h"
#include "common.h"
#include "internal.h"
#include "proxyattn.h"

namespace pa {

constexpr int kRowThreads = 256;   // 4 waves

template <int D> struct RowLanes {
    static constexpr int per_row = D / 16;
    static constexpr int rows = 64 / per_row;   // rows of a wave
};

// How a pass goes about the caches, by the bytes it writes.  More than L2 holds
// (8 x 4 MB) would not stay there for its reader anyway and is stored past the
// caches; where it is more than the MALL holds too, the rows are also loaded past them.
// Neither, stores, both (us): 4K tokens, 40 heads of 128 rotated 24.0, 21.5, 27 (the
// input still lies in the MALL); 128K tokens 588, 575, 565; 80K tokens appended in 4
// bits and read back 485, 463, 439.  128K tokens read back from 4 bits: 160, 151.
enum { kCached = 0, kStorePast = 1, kAllPast = 2 };
static int how_past(int64_t bytes) {
    return bytes > (int64_t)kMallBytes ? kAllPast : bytes > ((int64_t)32 << 20) ? kStorePast
                                                                               : kCached;
}
template <int HOW> __device__ __forceinline__ void put16(void* p, const u32x4& x) {
    if constexpr (HOW >= kStorePast)
        __builtin_nontemporal_store(x, reinterpret_cast<u32x4*>(p));
    else
        *reinterpret_cast<u32x4*>(p) = x;
}
template <int HOW> __device__ __forceinline__ u32x4 get16(const void* p) {
    if constexpr (HOW == kAllPast)
        return __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p));
    else
        return *reinterpret_cast<const u32x4*>(p);
}
// Calls f with `how` as a type.
template <typename F> static void by_how(int how, F f) {
    if (how == kAllPast)
        f(std::integral_constant<int, kAllPast>());
    else if (how == kStorePast)
        f(std::integral_constant<int, kStorePast>());
    else
        f(std::integral_constant<int, kCached>());
}

// Eight consecutive values.
template <typename T> struct Chunk;
template <> struct Chunk<bf16> {
    u32x4 w;
    template <int HOW = kCached> __device__ __forceinline__ void load(const bf16* p) {
        w = get16<HOW>(p);
    }
    template <int HOW> __device__ __forceinline__ void store(bf16* p) const { put16<HOW>(p, w); }
    __device__ __forceinline__ float at(int e) const { return get_elem<bf16>(w, e); }
    __device__ __forceinline__ void from(const float (&x)[8]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = pack_rne(x[2 * j], x[2 * j + 1]);
    }
};
template <> struct Chunk<float> {
    f32x4 a, b;
    template <int HOW = kCached> __device__ __forceinline__ void load(const float* p) {
        a = __builtin_bit_cast(f32x4, get16<HOW>(p));
        b = __builtin_bit_cast(f32x4, get16<HOW>(p + 4));
    }
    template <int HOW> __device__ __forceinline__ void store(float* p) const {
        put16<HOW>(p, __builtin_bit_cast(u32x4, a));
        put16<HOW>(p + 4, __builtin_bit_cast(u32x4, b));
    }
    __device__ __forceinline__ float at(int e) const { return e < 4 ? a[e & 3] : b[e & 3]; }
    __device__ __forceinline__ void from(const float (&x)[8]) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            a[j] = x[j];
            b[j] = x[4 + j];
        }
    }
};

// 1 / sqrt(a) in 64 bits: the hardware's estimate (relative error e0 below
// 2^-14) and two Newton steps of third order, each e -> (5/16) e^3 at most.
__device__ __forceinline__ double rsqrt64(double a) {
    double y = __builtin_amdgcn_rsq(a);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const double e = fma(-a * y, y, 1.0);
        y = fma(y * e, fma(0.375, e, 0.5), y);
    }
    return y;
}

// The two chunks that a lane holds of its row: those that the rotation pairs,
// c and c + rot/16 for the first rot values, and two of the rest.
struct LaneChunks {
    int c0, c1;
    bool turned;
};
template <int D>
__device__ __forceinline__ LaneChunks lane_chunks(int rot, int lane_in_row) {
    const int half = rot / 16, rest = D / 16 - half;
    const bool turned = lane_in_row < half;
    const int c0 = turned ? lane_in_row : half + lane_in_row;
    return {c0, c0 + (turned ? half : rest), turned};
}

// Normed (weight not NULL) and rotated values of the lane's chunks.  In 64
// bits: the products of a bf16 or fp32 value and a table entry are exact and
// the sums nearly so, so that what is stored does not hang on the order of an
// fp32 evaluation (4-bit codes change by a whole step at their borders).  The
// pass stays at the copy's rate with it (128K tokens: VALU busy in 68 % of cycles).
template <typename T, int D>
__device__ __forceinline__ void turn_row(const Chunk<T>& a, const Chunk<T>& b,
                                         const LaneChunks& lc, const T* weight, double eps,
                                         const float* cos, const float* sin, int interleaved,
                                         float (&z0)[8], float (&z1)[8]) {
    double x[2][8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        x[0][j] = a.at(j);
        x[1][j] = b.at(j);
    }
    if (weight) {
        double ss = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) ss = fma(x[0][j], x[0][j], fma(x[1][j], x[1][j], ss));
#pragma unroll
        for (int o = 1; o < RowLanes<D>::per_row; o *= 2) ss += __shfl_xor(ss, o);
        const double inv = rsqrt64(ss * (1.0 / D) + eps);
        Chunk<T> w0, w1;
        w0.load(weight + 8 * lc.c0);
        w1.load(weight + 8 * lc.c1);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[0][j] = x[0][j] * inv * (double)w0.at(j);
            x[1][j] = x[1][j] * inv * (double)w1.at(j);
        }
    }
    if (lc.turned) {
        if (interleaved) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
                const int at = 4 * (k ? lc.c1 : lc.c0);
                const f32x4 c = *reinterpret_cast<const f32x4*>(cos + at);
                const f32x4 s = *reinterpret_cast<const f32x4*>(sin + at);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const double u = x[k][2 * j], v = x[k][2 * j + 1];
                    x[k][2 * j] = fma(u, (double)c[j], -(v * (double)s[j]));
                    x[k][2 * j + 1] = fma(v, (double)c[j], u * (double)s[j]);
                }
            }
        } else {
            Chunk<float> c, s;
            c.load(cos + 8 * lc.c0);
            s.load(sin + 8 * lc.c0);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double u = x[0][j], v = x[1][j], cj = c.at(j), sj = s.at(j);
                x[0][j] = fma(u, cj, -(v * sj));
                x[1][j] = fma(v, cj, u * sj);
            }
        }
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        z0[j] = (float)x[0][j];
        z1[j] = (float)x[1][j];
    }
}

// ---------------------------------------------------------------------------
// norm and rotation of a prompt's Q and K
// ---------------------------------------------------------------------------
// A workgroup takes 2^shift tokens, all heads; consecutive rows of a wave are
// consecutive tokens of one head.
template <typename T, int D, int HOW>
__global__ __launch_bounds__(kRowThreads) void norm_rotate_kernel(RotateRows w, RotaryArgs r,
                                                                  int shift) {
    constexpr int RW = RowLanes<D>::rows, LR = RowLanes<D>::per_row;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int in_row = lane % LR;
    const LaneChunks lc = lane_chunks<D>(r.rot, in_row);
    const int t0 = blockIdx.x << shift;
    const int nq = w.q ? w.hq : 0, nk = w.k ? w.hkv : 0;
    const int rows = (nq + nk) << shift;
    for (int base = (blockIdx.y * 4 + wave) * RW; base < rows; base += gridDim.y * 4 * RW) {
        const int row = base + lane / LR;
        const int t = t0 + (row & ((1 << shift) - 1)), h = row >> shift;
        const bool live = row < rows && t < w.n;
        const int tc = live ? t : t0, hc = live ? h : 0;
        const bool is_k = hc >= nq;
        const T* x = is_k ? (const T*)w.k + tc * w.k_tok + (hc - nq) * w.k_head
                          : (const T*)w.q + tc * w.q_tok + hc * w.q_head;
        T* y = is_k ? (T*)w.ko + tc * w.ko_tok + (hc - nq) * w.ko_head
                    : (T*)w.qo + tc * w.qo_tok + hc * w.qo_head;
        Chunk<T> a, b;
        a.template load<HOW>(x + 8 * lc.c0);
        b.template load<HOW>(x + 8 * lc.c1);
        int pos = 0;
        if (r.rot) {
            pos = w.positions ? w.positions[tc] : w.first + tc;
            pos = min(max(pos, 0), r.table_len - 1);
        }
        float z0[8], z1[8];
        turn_row<T, D>(a, b, lc, (const T*)(is_k ? r.kw : r.qw), r.eps,
                       r.cos + (int64_t)pos * (r.rot / 2), r.sin + (int64_t)pos * (r.rot / 2),
                       r.interleaved, z0, z1);
        if (live) {
            a.from(z0);
            b.from(z1);
            a.template store<HOW>(y + 8 * lc.c0);
            b.template store<HOW>(y + 8 * lc.c1);
        }
    }
}

// Tokens to a workgroup (as a power of two, at most four) and workgroups along
// a token's rows, `fill` workgroups in all where there is work for them.
// 128K tokens, 40 heads: rotated in 645, 602, 565, 570 and 586 us with 1, 2, 4,
// 8 and 16 tokens; 4K tokens 24.2 us with 1044 workgroups, 21.5 with 4176 (but 80K
// tokens appended 473 us with one workgroup to four tokens, 596 with four, which
// each look the slots up).
static void row_grid(int tokens, int row_steps, int fill, int* shift, dim3* grid) {
    const int sh = tokens >= 2048 ? 2 : tokens >= 1024 ? 1 : 0;
    const int gx = (tokens + (1 << sh) - 1) >> sh;
    const int steps = row_steps << sh;   // rounds of four waves, about
    int gy = 1;
    while (gy < steps && gx * gy < fill) gy *= 2;
    *shift = sh;
    *grid = dim3(gx, gy);
}

template <typename T>
static void norm_rotate_d(const RotateRows& w, const RotaryArgs& r, hipStream_t st) {
    const int rows = (w.q ? w.hq : 0) + (w.k ? w.hkv : 0);
    int shift;
    dim3 grid;
    const int rw = 4 * 1024 / w.d;   // rows of a workgroup's round
    row_grid(w.n, (rows + rw - 1) / rw, 4096, &shift, &grid);
    by_how(how_past((int64_t)w.n * rows * w.d * (int)sizeof(T)), [&](auto how) {
        constexpr int HOW = decltype(how)::value;
        if (w.d == 64)
            norm_rotate_kernel<T, 64, HOW><<<grid, kRowThreads, 0, st>>>(w, r, shift);
        else
            norm_rotate_kernel<T, 128, HOW><<<grid, kRowThreads, 0, st>>>(w, r, shift);
    });
}

hipError_t launch_norm_rotate(const RotateRows& w, const RotaryArgs& r, hipStream_t st) {
    if (w.dtype == PROXYATTN_BF16)
        norm_rotate_d<bf16>(w, r, st);
    else
        norm_rotate_d<float>(w, r, st);
    return hipGetLastError();
}

// ---------------------------------------------------------------------------
// the paged cache
// ---------------------------------------------------------------------------
// Where a token's keys and values go: page -1 for none.
struct Slot {
    int pos, page, slot;
};

// Looked up by a whole wave, the same in every lane.  LIMIT: a sequence's
// new tokens past max_new are tokens of no sequence.
template <bool LIMIT>
__device__ __forceinline__ Slot find_slot(const CacheShape& s, const int* table, const int* lens,
                                          const int* starts, int t) {
    Slot at{-1, -1, 0};
    if (t >= s.t) return at;
    int b = t, j = 0, n = 1;
    if (starts) {
        b = seq_of_token(starts, s.b, t);
        if (b >= s.b) return at;
        const int first = max(starts[b], 0);
        j = t - first;
        n = min(starts[b + 1], s.t) - first;
        if (j < 0 || j >= n) return at;
        if (LIMIT) {
            n = min(n, s.max_new);
            if (j >= n) return at;
        }
    } else if (b >= s.b) {
        return at;
    }
    const int pos = min(max(lens[b], 0), s.max_len) - n + j;
    if (pos < 0) return at;
    const int page = table[(int64_t)b * s.width + (pos >> s.page_shift)];
    at.pos = pos;
    at.page = (unsigned)page < (unsigned)s.num_pages ? page : -1;
    at.slot = pos & ((1 << s.page_shift) - 1);
    return at;
}

// The workgroup's place in the row of token blocks when reading back: each XCD
// (workgroups go to them in turn) takes a run of blocks, so that the cache lines that
// neighbouring blocks share, a page's scales above all, pass through one L2 (80K tokens
// of 4 bits read back 65 -> 59 us, 128K 142.4 -> 141.2; appending takes the same time
// either way).
__device__ __forceinline__ int token_block() {
    const int x = blockIdx.x % kNumXcd, n = gridDim.x / kNumXcd, rest = gridDim.x % kNumXcd;
    return x * n + min(x, rest) + blockIdx.x / kNumXcd;
}

// Slots of a workgroup's tokens, in LDS.
template <bool LIMIT>
__device__ __forceinline__ void find_slots(Slot* slots, const CacheShape& s, const int* table,
                                           const int* lens, const int* starts, int t0, int shift) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int j = wave; j < 1 << shift; j += kRowThreads / 64) {
        const Slot at = find_slot<LIMIT>(s, table, lens, starts, t0 + j);
        if (lane == 0) slots[j] = at;
    }
    __syncthreads();
}

// 16 consecutive values as 4-bit codes and their group's scale (32 values, two
// neighbouring lanes): 8 bytes of codes, and the scale's byte.
__device__ __forceinline__ uint64_t quantise16(const float (&x)[16], uint32_t* scale_byte) {
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 16; ++j) top = max(top, __float_as_uint(x[j]) & 0x7fffffffu);
    top = max(top, (uint32_t)__shfl_xor((int)top, 1));
    // the smallest e with top <= 7 * 2^e, top = 1.f * 2^E: E - 2 up to 1.75, else E - 1
    int e = (int)((top + 0x1fffffu) >> 23) - 127 - 2;
    e = min(max(e, -110), 125);
    const float scale = __uint_as_float((uint32_t)(e + 127) << 23);
    uint32_t w[2] = {0, 0};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const float* y = x + 8 * j;
        w[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[j], y[0], y[1], scale, 0);
        w[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[j], y[2], y[3], scale, 1);
        w[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[j], y[4], y[5], scale, 2);
        w[j] = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w[j], y[6], y[7], scale, 3);
    }
    *scale_byte = (uint32_t)(e + 127);
    return (uint64_t)w[1] << 32 | w[0];
}

template <int D>
__device__ __forceinline__ void store_fp4(uint8_t* codes, uint8_t* scales, const CacheShape& s,
                                          const Slot& at, int head, int in_row,
                                          const float (&x)[16], bool live) {
    uint32_t sb;
    const uint64_t w = quantise16(x, &sb);
    if (!live) return;
    const int64_t page_head = (int64_t)at.page * s.hkv + head;
    const int64_t row = (page_head << s.page_shift) + at.slot;
    *reinterpret_cast<uint64_t*>(codes + row * (D / 2) + 8 * in_row) = w;
    if ((in_row & 1) == 0)
        scales[((page_head * (D / 32) + in_row / 2) << s.page_shift) + at.slot] = (uint8_t)sb;
}

// Queries to q_out, keys and values into their pages.  Units of a workgroup:
// RW rows of queries, of keys or of values; consecutive rows are consecutive
// tokens of a head, whose codes and scales are neighbours in a page.
template <typename T, int D, bool FP4, int HOW>
__global__ __launch_bounds__(kRowThreads) void cache_append_kernel(
    CacheShape s, RotaryArgs r, AppendArgs a, const int* table, const int* lens, const int* starts,
    PagePtrs pg, int shift) {
    constexpr int RW = RowLanes<D>::rows, LR = RowLanes<D>::per_row;
    constexpr int LINE = D + 4;   // a row's values in LDS, padded by a bank group
    __shared__ Slot slots[4];
    __shared__ __align__(16) float stage[FP4 ? 4 * RW * LINE : 4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int in_row = lane % LR, row_in_wave = lane / LR;
    const LaneChunks lc = lane_chunks<D>(r.rot, in_row);
    const int t0 = blockIdx.x << shift, mask = (1 << shift) - 1;
    find_slots<true>(slots, s, table, lens, starts, t0, shift);
    const int qrows = a.q ? s.hq << shift : 0, krows = s.hkv << shift;
    const int qu = (qrows + RW - 1) / RW, ku = (krows + RW - 1) / RW;
    for (int u = blockIdx.y * 4 + wave; u < qu + 2 * ku; u += gridDim.y * 4) {
        const int part = u < qu ? 0 : u < qu + ku ? 1 : 2;   // queries, keys, values
        const int row = (u - (part == 0 ? 0 : part == 1 ? qu : qu + ku)) * RW + row_in_wave;
        const int head = row >> shift;
        const Slot at = slots[row & mask];
        const bool live = row < (part ? krows : qrows) && (part ? at.page >= 0 : at.pos >= 0);
        const int64_t t = live ? t0 + (row & mask) : 0;
        const int h = live ? head : 0;
        const T* x = part == 0   ? (const T*)a.q + t * s.q_tok + h * s.q_head
                     : part == 1 ? (const T*)a.k + t * s.kv_tok + h * s.kv_head
                                 : (const T*)a.v + t * s.kv_tok + h * s.kv_head;
        const bool turn = part < 2 && a.norm_rotate;
        // rows that are not turned: 16 values in a row to each lane for the
        // codes, else chunks that make a wave's accesses run on
        const int c0 = turn ? lc.c0 : FP4 ? 2 * in_row : in_row;
        const int c1 = turn ? lc.c1 : FP4 ? 2 * in_row + 1 : in_row + LR;
        Chunk<T> lo, hi;
        lo.template load<HOW>(x + 8 * c0);
        hi.template load<HOW>(x + 8 * c1);
        float z[16];
        if (turn) {
            const int64_t at_pos = (int64_t)max(at.pos, 0) * (r.rot / 2);
            float z0[8], z1[8];
            turn_row<T, D>(lo, hi, lc, (const T*)(part ? r.kw : r.qw), r.eps, r.cos + at_pos,
                           r.sin + at_pos, r.interleaved, z0, z1);
            lo.from(z0);
            hi.from(z1);
        }
        if (part == 0) {
            if (live) {
                T* y = (T*)a.qo + t * a.qo_tok + h * a.qo_head;
                lo.template store<HOW>(y + 8 * c0);
                hi.template store<HOW>(y + 8 * c1);
            }
            continue;
        }
        if constexpr (FP4) {
            // what the problem's dtype would hold is what is quantised
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                z[j] = lo.at(j);
                z[8 + j] = hi.at(j);
            }
            if (turn) {   // back to 16 values in a row to each lane
                float* line = stage + (wave * RW + row_in_wave) * LINE;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    *reinterpret_cast<f32x4*>(line + 8 * c0 + 4 * j) =
                        f32x4{z[4 * j], z[4 * j + 1], z[4 * j + 2], z[4 * j + 3]};
                    *reinterpret_cast<f32x4*>(line + 8 * c1 + 4 * j) =
                        f32x4{z[8 + 4 * j], z[9 + 4 * j], z[10 + 4 * j], z[11 + 4 * j]};
                }
                wave_lds_fence();
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const f32x4 v = *reinterpret_cast<const f32x4*>(line + 16 * in_row + 4 * j);
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[4 * j + i] = v[i];
                }
                wave_lds_fence();
            }
            store_fp4<D>((uint8_t*)(part == 1 ? pg.k : pg.v), (uint8_t*)(part == 1 ? pg.ks : pg.vs),
                         s, at, h, in_row, z, live);
        } else if (live) {
            T* y = (T*)(part == 1 ? pg.k : pg.v) +
                   ((((int64_t)at.page * s.hkv + h) << s.page_shift) + at.slot) * D;
            lo.template store<HOW>(y + 8 * c0);
            hi.template store<HOW>(y + 8 * c1);
        }
    }
}

// Rows of the pages back in the problem's dtype.
template <typename T, int D, bool FP4, int HOW>
__global__ __launch_bounds__(kRowThreads) void cache_read_kernel(CacheShape s, const int* table,
                                                                 const int* lens,
                                                                 const int* starts, PagePtrs pg,
                                                                 T* ko, T* vo, int shift) {
    constexpr int RW = RowLanes<D>::rows, LR = RowLanes<D>::per_row;
    __shared__ Slot slots[4];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int in_row = lane % LR, row_in_wave = lane / LR;
    const int t0 = token_block() << shift, mask = (1 << shift) - 1;
    find_slots<false>(slots, s, table, lens, starts, t0, shift);
    const int rows = s.hkv << shift, ru = (rows + RW - 1) / RW;
    for (int u = blockIdx.y * 4 + wave; u < 2 * ru; u += gridDim.y * 4) {
        const bool is_v = u >= ru;
        T* const out = is_v ? vo : ko;
        if (!out) continue;
        const int row = (is_v ? u - ru : u) * RW + row_in_wave;
        const Slot at = slots[row & mask];
        if (row >= rows || at.page < 0) continue;
        const int h = row >> shift;
        const int64_t page_head = (int64_t)at.page * s.hkv + h;
        const int64_t line = (page_head << s.page_shift) + at.slot;
        Chunk<T> lo, hi;   // chunks in_row and in_row + LR: a wave's stores run on
        if constexpr (FP4) {
            const uint8_t* codes = (const uint8_t*)(is_v ? pg.v : pg.k) + line * (D / 2) + 4 * in_row;
            const uint8_t* scales = (const uint8_t*)(is_v ? pg.vs : pg.ks) +
                                    ((page_head * (D / 32) + in_row / 4) << s.page_shift) + at.slot;
            const uint32_t w0 = *reinterpret_cast<const uint32_t*>(codes);
            const uint32_t w1 = *reinterpret_cast<const uint32_t*>(codes + 4 * LR);
            const uint32_t s0 = scales[0], s1 = scales[(LR / 4) << s.page_shift];
            float z0[8], z1[8];
            fp4_values(w0, __uint_as_float(s0 << 23), z0);
            fp4_values(w1, __uint_as_float(s1 << 23), z1);
            lo.from(z0);
            hi.from(z1);
        } else {
            const T* x = (const T*)(is_v ? pg.v : pg.k) + line * D + 8 * in_row;
            lo.load(x);
            hi.load(x + 8 * LR);
        }
        T* y = out + (int64_t)(t0 + (row & mask)) * s.kv_tok + h * s.kv_head + 8 * in_row;
        lo.template store<HOW>(y);
        hi.template store<HOW>(y + 8 * LR);
    }
}

template <typename T, int D, bool FP4>
static void append_as(const CacheShape& s, const RotaryArgs& r, const AppendArgs& a,
                      const int* table, const int* lens, const int* starts, const PagePtrs& pg,
                      hipStream_t st) {
    int shift;
    dim3 grid;
    const int rw = 4 * 1024 / D;
    row_grid(s.t, ((a.q ? s.hq : 0) + 2 * s.hkv + rw - 1) / rw, 1024, &shift, &grid);
    const int64_t rows = (int64_t)s.t * ((a.q ? s.hq : 0) + (FP4 ? 0 : 2 * s.hkv));
    by_how(how_past(rows * D * (int)sizeof(T)), [&](auto how) {
        cache_append_kernel<T, D, FP4, decltype(how)::value>
            <<<grid, kRowThreads, 0, st>>>(s, r, a, table, lens, starts, pg, shift);
    });
}
template <typename T, int D, bool FP4>
static void read_as(const CacheShape& s, const int* table, const int* lens, const int* starts,
                    const PagePtrs& pg, void* ko, void* vo, hipStream_t st) {
    int shift;
    dim3 grid;
    const int rw = 4 * 1024 / D;
    row_grid(s.t, (2 * s.hkv + rw - 1) / rw, 1024, &shift, &grid);
    by_how(how_past((int64_t)s.t * 2 * s.hkv * D * (int)sizeof(T)), [&](auto how) {
        cache_read_kernel<T, D, FP4, decltype(how)::value><<<grid, kRowThreads, 0, st>>>(
            s, table, lens, starts, pg, (T*)ko, (T*)vo, shift);
    });
}

hipError_t launch_cache_append(const CacheShape& s, const RotaryArgs& r, const AppendArgs& a,
                               const int* table, const int* lens, const int* starts,
                               const PagePtrs& pg, hipStream_t st) {
    by_cache_type(s, [&](auto t, auto d, auto fp4) {
        append_as<typename decltype(t)::type, decltype(d)::value, decltype(fp4)::value>(
            s, r, a, table, lens, starts, pg, st);
    });
    return hipGetLastError();
}

hipError_t launch_cache_read(const CacheShape& s, const int* table, const int* lens,
                             const int* starts, const PagePtrs& pg, void* ko, void* vo,
                             hipStream_t st) {
    by_cache_type(s, [&](auto t, auto d, auto fp4) {
        read_as<typename decltype(t)::type, decltype(d)::value, decltype(fp4)::value>(
            s, table, lens, starts, pg, ko, vo, st);
    });
    return hipGetLastError();
}

}  // namespace pa
