// sk_experts.hip -- the experts' products: each expert's rows times that expert's matrix, and both gradients.
//
//   forward   y[r, n]     = sum_k x[src(r), k] w[e, n, k]                 offsets[e] <= r < offsets[e + 1]
//   input     gr[r, k]    = sum_n gy[r, n] w[e, n, k]                     gx[t] = sum_s gr[slots[t, s]]
//   weight    gw[e, n, k] = sum_r gy[r, n] x[src(r), k]
//
// src(r) = tokens[r] where the rows are gathered from the tokens, else r.  Products of 16-bit factors on the matrix
// cores, sums in 32 bits, one rounding at the end.
#include "sk_experts.h"

namespace sk {
namespace {

constexpr int kThreads = 256;

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

// Two neighbouring whole numbers of 8 bits: where the factors are these, the kernels below move them as they move
// 16-bit factors, and only the products and what becomes of the sums differ.
using Pair = int16_t;
template <class T>
constexpr bool kPairs = std::is_same_v<T, Pair>;
template <class T>
using Sum4 = std::conditional_t<kPairs<T>, i32x4, f32x4>;

template <class T>
__device__ __forceinline__ Sum4<T> mfma16(const Frag8<T> &a, const Frag8<T> &b, Sum4<T> c) {
    if constexpr (kPairs<T>)
        return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0,
                                                     0);
    else if constexpr (std::is_same_v<T, __bf16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// ---- tiles: columns in whole chunks of eight, every pointer aligned to 16 bytes ----
//
// A work-group computes BM x BN results; its wavefronts, WM x WN of them, a part of BM / WM x BN / WN each, held in
// registers.  The contraction goes in steps of 64 (128 bytes of a row, a whole cache line).  Operands are copied to LDS
// by the memory pipe itself, 16 bytes a lane, into the next of BUFFERS buffers, so many steps less one ahead of the
// products, with one barrier a step.  Two buffers where several work-groups a CU cover each other's waits, more where one
// or two have the CU to themselves (Cut, below).  The copies are issued one by one among the products, since the pipe takes few at a time and a wavefront
// whose copy is not taken cannot issue its products; they are addressed by a scalar base and an offset of 32 bits a
// lane, which the pipe takes a tenth faster than addresses of 64 bits.
//
// An operand whose rows run along the contraction ("along": x, w in forward, gy in input) lies in LDS as rows of 64,
// and a lane's eight elements are one 16-byte read.  An operand whose rows run across it ("across": w in input, gy
// and x in weight) lies as 64 rows of the tile's width and is read through the transposing LDS read, so no copy is
// transposed in memory.  LDS takes a copy in lane order, so the places that keep the reads off each other's banks are
// reached by permuting the lanes' sources: chunk c of row r lies at c ^ (r & 7) ("along", 16-byte chunks), granule q
// of row d at q ^ spread(d) ("across", 32-byte granules).
//
// Elements past the end of the contraction come from a page of zeros; rows and columns past the tile's end repeat the
// last one and are not stored.
//
// 65536 rows of 64 experts of 2048 x 2048, bf16, equal shares: forward 487 us (1130 TFLOP/s), the input gradient's rows in
// 32 bits 475 (1160), weight gradient 514 (1070); a library product of 65536 x 2048 x 2048 reaches 1410 TFLOP/s here.  Of
// a step's 1.55 us the products alone take 0.95 and the copies alone 1.28.  The LDS reads are not what bounds a step: 16-byte reads
// alone reach 248 bytes a cycle a CU, transposing ones 173, which for the weight gradient's 192 KB is a quarter of a step.
// Rows that are no whole 16 bytes take 2 times as long forward and 3 to 4 times in the gradients.
//
// Rows in 8 bits: the same bytes hold twice the products.  65536 rows of 64 experts of 2048 x 2048 272 us with equal shares
// (2020 TOP/s), of 4096 x 2048 (K = 4096) 490 (2240); a library product of 8192^3 in 8 bits reaches 2090 here.  Of a tile's
// 31 us its 16 steps take 27.

constexpr int kDeep = 64;

__device__ __attribute__((aligned(16))) uint32_t zero_page[4];

using LdsByte = __attribute__((address_space(3))) char;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
using LdsShort4 = __attribute__((address_space(3))) s16x4;

// Copies 16 bytes a lane to LDS: from base + each lane's offset to `to` (one for the wavefront) + 16 lane.  WIDE: the
// offset is a whole address.  Written out, since the compiler puts a wait for every copy under way before each
// transposing read that follows it.  It has no result in registers, and the place is not read before copies_landed.
template <bool WIDE>
using Offset = std::conditional_t<WIDE, const char *, uint32_t>;

template <bool WIDE>
__device__ __forceinline__ void copy16(const char *base, Offset<WIDE> from, char *to) {
    const uint32_t place = (uint32_t)(uintptr_t)(LdsByte *)to;
    if constexpr (WIDE)
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off"
                     :
                     : "v"(from), "s"(place)
                     : "m0", "memory");
    else
        asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %2"
                     :
                     : "v"(from), "s"(place), "s"(base)
                     : "m0", "memory");
}
// Every copy of the work-group has landed but the last `later` steps' ones, of EACH a wavefront (each wavefront waits for
// its own; loads land in order), and every LDS read is done.  later <= MOST.
template <int EACH, int MOST>
__device__ __forceinline__ void copies_landed(int later) {
    __builtin_amdgcn_sched_barrier(0);
    if (MOST == 0 || later == MOST)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(EACH * MOST) : "memory");
    else if constexpr (MOST > 0)
        copies_landed<EACH, MOST - 1>(later);
    __builtin_amdgcn_sched_barrier(0);
}

// The 16 rows that one transposing read takes (bits 0, 1, 3, 4 of d) fall on as many granules as a row of G has.
template <int G>
__device__ __forceinline__ int spread(int d) {
    if constexpr (G >= 16) return (d & 3) | ((d >> 3) & 3) << 2;
    if constexpr (G == 8) return (d & 3) | ((d >> 3) & 1) << 2;
    return d & 3;
}

// One operand: BR rows (or columns) of the tile, copied by WAVES wavefronts, read as F fragments by each.
template <class T, bool ACROSS, int BR, int WAVES, int F>
struct Operand {
    static constexpr int kBytes = BR * kDeep * 2;
    static constexpr int kRounds = kBytes / (WAVES * 1024);
    static_assert(kRounds * WAVES * 1024 == kBytes);
    static constexpr int kRowBytes = ACROSS ? BR * 2 : kDeep * 2, kGranules = BR / 16;
    int part[ACROSS ? F : kDeep / 32];  // LDS places of the lane's parts of fragments

    // Round q of the copies fills 1024 bytes a wavefront in lane order.  The lane's row (along: of the tile, across:
    // of the step) and its first element in the row.
    __device__ __forceinline__ static int copy_row(int q, int wave, int lane) {
        return (q * WAVES + wave) * (1024 / kRowBytes) + lane / (kRowBytes / 16);
    }
    __device__ __forceinline__ static int copy_element(int q, int wave, int lane) {
        const int r = copy_row(q, wave, lane), p = lane % (kRowBytes / 16);
        if constexpr (!ACROSS) return (p ^ (r & 7)) * 8;
        return ((p / 2) ^ spread<kGranules>(r)) * 16 + (p & 1) * 8;
    }
    // Whether the lane's chunk of round q lies past the end of the contraction, of which `left` places are left.
    __device__ __forceinline__ static bool past(int q, int wave, int lane, int left) {
        return (ACROSS ? copy_row(q, wave, lane) : copy_element(q, wave, lane)) >= left;
    }
    // The wavefront's fragments begin at row `first` of the tile, a multiple of 16 F.
    __device__ __forceinline__ void start_read(int first, int lane) {
        if constexpr (!ACROSS) {
#pragma unroll
            for (int kk = 0; kk < kDeep / 32; ++kk)
                part[kk] = (first + (lane & 15)) * kRowBytes + ((kk * 4 + (lane >> 4)) ^ (lane & 7)) * 16;
        } else {
            const int d = (lane >> 4) * 8 + ((lane >> 2) & 3);
#pragma unroll
            for (int i = 0; i < F; ++i)
                part[i] = d * kRowBytes + ((first / 16 + i) ^ spread<kGranules>(d)) * 32 + (lane & 3) * 8;
        }
    }
    // The i-th fragment, part kk of the step.
    __device__ __forceinline__ Frag8<T> frag(const char *lds, int i, int kk) const {
        if constexpr (!ACROSS) {
            return *reinterpret_cast<const Frag8<T> *>(lds + part[kk] + i * 16 * kRowBytes);
        } else {
            s16x4 half[2];
#pragma unroll
            for (int h = 0; h < 2; ++h)
                half[h] = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (LdsShort4 *)(lds + part[i] + (kk * 32 + h * 4) * kRowBytes));
            const s16x8 all = __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7);
            return __builtin_bit_cast(Frag8<T>, all);
        }
    }
};

// `count` elements from p, at any alignment, zeros after them; count may be anything.
template <class T>
__device__ __forceinline__ Frag8<T> load_chunk(const T *p, int count) {
    Frag8<T> v = {};
    if (count >= 8) {
        __builtin_memcpy(&v, p, 16);
    } else {
#pragma unroll
        for (int i = 0; i < 7; ++i)
            if (i < count) v[i] = p[i];
    }
    return v;
}

// GATHERED: x's rows are looked up in tokens.  WIDE: x has 2^32 bytes or more.  STAGED: rows that are no whole chunks of
// 16 bytes, or pointers that are not aligned to them: the chunks come through registers, loaded at the start of a step
// and written to LDS at its end.
template <class T, int MODE, int BM, int BN, int WM, int WN, bool GATHERED, bool WIDE, bool STAGED, int BUFFERS = 2>
__global__ __launch_bounds__(WM *WN * 64) __attribute__((amdgpu_waves_per_eu(2))) void sk_experts_tile(ExpertArgs A) {
    constexpr int WAVES = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16;
    using OpA = Operand<T, MODE == kWeight, BM, WAVES, FM>;
    using OpB = Operand<T, MODE != kForward, BN, WAVES, FN>;
    constexpr int kStep = OpA::kBytes + OpB::kBytes;
    constexpr bool kWideA = WIDE && MODE == kForward, kWideB = WIDE && MODE == kWeight;
    constexpr int kOut = BM * (BN * 2 + 32);  // the results, below
    static_assert(BM / WM * (BN * 4 + 32) <= kOut);
    constexpr int kLds = BUFFERS * kStep;
    static_assert(BUFFERS == 2 || (!STAGED && MODE != kWeight));  // those have one step's chunks or rows at hand
    __shared__ __attribute__((aligned(1024))) char lds[kLds > kOut ? kLds : kOut];

    __shared__ __attribute__((aligned(16))) float scales[kPairs<T> ? BM + BN : 1];  // of the tile's rows and columns

    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int K = A.K, N = A.N, cols = MODE == kForward ? N : K;
    const T *x = static_cast<const T *>(A.x), *w = static_cast<const T *>(A.w), *gy = static_cast<const T *>(A.gy);

    // The tile: rows [m0, m1) of the result, columns from c0, of expert e, with `deep` products to a sum (weight: over
    // the rows from r0).
    int e, m0, m1, c0, deep, r0 = 0, part = 0;
    if constexpr (MODE == kWeight) {
        const int tn = (N + BM - 1) / BM, tk = (K + BN - 1) / BN;
        const int t = xcd_order(blockIdx.x, A.E * tn * tk * A.parts);
        if (t < 0) return;
        const int tile = t / A.parts;
        part = t - tile * A.parts;
        e = tile / (tn * tk);
        const int i = tile - e * (tn * tk);
        m0 = i / tk * BM, m1 = N;
        c0 = i % tk * BN;
        // this part's share of the expert's rows, in whole steps
        const RowRange rr = expert_rows(A, e);
        const int steps = (rr.end - rr.begin + kDeep - 1) / kDeep, share = (steps + A.parts - 1) / A.parts * kDeep;
        r0 = min(rr.begin + part * share, rr.end);
        deep = min(share, rr.end - r0);
    } else {
        const Tile t = find_tile(A, BM, (cols + BN - 1) / BN, blockIdx.x);
        if (t.expert < 0) return;
        e = t.expert, m0 = t.begin, m1 = t.end;
        c0 = t.column * BN;
        deep = e >= A.E ? 0 : MODE == kForward ? K : N;
    }
    // one answer for the work-group: kept in scalar registers
    e = __builtin_amdgcn_readfirstlane(e), m0 = __builtin_amdgcn_readfirstlane(m0);
    m1 = __builtin_amdgcn_readfirstlane(m1), c0 = __builtin_amdgcn_readfirstlane(c0);
    r0 = __builtin_amdgcn_readfirstlane(r0), deep = __builtin_amdgcn_readfirstlane(deep);

    // A scale a thread, under way with the first copies.
    [[maybe_unused]] float scale = 0.f;
    if constexpr (kPairs<T>) {
        static_assert(BM + BN <= WM * WN * 64);
        const int i = threadIdx.x;
        if (deep > 0 && i < BM) {
            const int r = min(m0 + i, m1 - 1);
            int t = GATHERED ? A.tokens[r] : r;
            if (GATHERED && (t < 0 || t >= A.T)) t = 0;
            scale = A.x_scale[t];
        } else if (deep > 0 && i < BM + BN) {
            scale = A.w_scale[(int64_t)e * N + min(c0 + i - BM, N - 1)];
        }
    }
    Sum4<T> acc[FM][FN] = {};
    const int wm = wave / WN * (BM / WM), wn = wave % WN * (BN / WN);
    const bool idle = m0 + wm >= m1 || c0 + wn >= cols;  // the wavefront's part lies past the edge: it copies only
    if (deep > 0) {
        OpA oa;
        OpB ob;
        oa.start_read(wm, lane);
        ob.start_read(wn, lane);

        // Where the copies of a step come from: a base that moves on with the steps and the lane's offsets from it.  x's
        // rows in "weight" are looked up anew for every step, a step before their copies.
        constexpr bool kLookUp = MODE == kWeight && GATHERED;
        const char *base_a, *base_b;
        Offset<kWideA> from_a[OpA::kRounds];
        Offset<kWideB> from_b[OpB::kRounds];
        int token[kLookUp ? OpB::kRounds : 1];
        if constexpr (MODE == kForward) {
            base_a = reinterpret_cast<const char *>(x + (GATHERED ? 0 : (int64_t)m0 * K));
#pragma unroll
            for (int q = 0; q < OpA::kRounds; ++q) {
                const int r = min(m0 + OpA::copy_row(q, wave, lane), m1 - 1);
                int t = GATHERED ? A.tokens[r] : r - m0;
                if (GATHERED && (t < 0 || t >= A.T)) t = 0;
                if constexpr (kWideA)
                    from_a[q] = base_a + ((int64_t)t * K + OpA::copy_element(q, wave, lane)) * 2;
                else
                    from_a[q] = ((uint32_t)t * K + OpA::copy_element(q, wave, lane)) * 2;
            }
        } else {
            const int64_t first = MODE == kInput ? (int64_t)m0 * N : (int64_t)r0 * N + m0;
            base_a = reinterpret_cast<const char *>(gy + first);
#pragma unroll
            for (int q = 0; q < OpA::kRounds; ++q) {
                const int r = OpA::copy_row(q, wave, lane), c = OpA::copy_element(q, wave, lane);
                from_a[q] = MODE == kInput ? (uint32_t)(min(r, m1 - 1 - m0) * N + c) * 2
                                           : (uint32_t)(r * N + (STAGED ? c : min(c, N - 8 - m0))) * 2;
            }
        }
        if constexpr (MODE == kWeight) {
            base_b = reinterpret_cast<const char *>(x + c0 + (GATHERED ? 0 : (int64_t)r0 * K));
        } else {
            base_b = reinterpret_cast<const char *>(w + (int64_t)e * N * K + (MODE == kForward ? (int64_t)c0 * K : c0));
        }
#pragma unroll
        for (int q = 0; q < OpB::kRounds; ++q) {
            const int r = OpB::copy_row(q, wave, lane), c = OpB::copy_element(q, wave, lane);
            if constexpr (!kLookUp)
                from_b[q] = MODE == kForward ? (uint32_t)(min(r, N - 1 - c0) * K + c) * 2
                                             : (uint32_t)(r * K + (STAGED ? c : min(c, K - 8 - c0))) * 2;
        }
        auto look_up = [&](int d0) {
            if constexpr (kLookUp) {
#pragma unroll
                for (int q = 0; q < OpB::kRounds; ++q)
                    token[q] = A.tokens[r0 + min(d0 + OpB::copy_row(q, wave, lane), deep - 1)];
            }
        };
        auto take_rows = [&] {
            if constexpr (kLookUp) {
#pragma unroll
                for (int q = 0; q < OpB::kRounds; ++q) {
                    // To the compiler, a wait for the look-up: here, where no copy is under way.
                    asm volatile("" : "+v"(token[q]));
                    const int t = token[q] >= 0 && token[q] < A.T ? token[q] : 0;
                    const int e8 = OpB::copy_element(q, wave, lane), c = STAGED ? e8 : min(e8, K - 8 - c0);
                    if constexpr (kWideB)
                        from_b[q] = base_b + ((int64_t)t * K + c) * 2;
                    else
                        from_b[q] = ((uint32_t)t * K + c) * 2;
                }
            }
        };
        // Copy c of the step at d0.  PARTIAL: the contraction ends within the step, zeros from there.
        constexpr int kCopies = OpA::kRounds + OpB::kRounds;
        Frag8<T> held[STAGED ? kCopies : 1];
        auto place = [&](int c) {
            return c < OpA::kRounds ? (c * WAVES + wave) * 1024
                                    : OpA::kBytes + ((c - OpA::kRounds) * WAVES + wave) * 1024;
        };
        auto copy = [&](auto partial, int c, int d0, char *to) {
            const bool is_a = c < OpA::kRounds;
            const int q = is_a ? c : c - OpA::kRounds;
            to += place(c);
            if constexpr (STAGED) {
                // How many of the chunk's elements there are, along the contraction or across the tile.
                const int left = deep - d0;
                const char *from;
                int count;
                if (is_a) {
                    const int r = OpA::copy_row(q, wave, lane), el = OpA::copy_element(q, wave, lane);
                    count = MODE != kWeight ? left - el : r < left ? N - m0 - el : 0;
                    if constexpr (kWideA) from = from_a[q];
                    else from = base_a + from_a[q];
                } else {
                    const int r = OpB::copy_row(q, wave, lane), el = OpB::copy_element(q, wave, lane);
                    count = MODE == kForward ? left - el : r < left ? K - c0 - el : 0;
                    if constexpr (kWideB) from = from_b[q];
                    else from = base_b + from_b[q];
                }
                held[c] = load_chunk(reinterpret_cast<const T *>(from), count);
            } else if constexpr (decltype(partial)::value) {
                const char *from;
                if (is_a) {
                    if constexpr (kWideA) from = from_a[q];
                    else from = base_a + from_a[q];
                    if (OpA::past(q, wave, lane, deep - d0)) from = reinterpret_cast<const char *>(zero_page);
                } else {
                    if constexpr (kWideB) from = from_b[q];
                    else from = base_b + from_b[q];
                    if (OpB::past(q, wave, lane, deep - d0)) from = reinterpret_cast<const char *>(zero_page);
                }
                copy16<true>(nullptr, from, to);
            } else if (is_a) {
                copy16<kWideA>(base_a, from_a[q], to);
            } else {
                copy16<kWideB>(base_b, from_b[q], to);
            }
        };
        // STAGED: the chunks of the step's copies, to their places in LDS.
        auto put = [&](char *to) {
            if constexpr (STAGED) {
#pragma unroll
                for (int c = 0; c < kCopies; ++c) *reinterpret_cast<Frag8<T> *>(to + place(c) + lane * 16) = held[c];
            }
        };
        // On to the next step's places.
        auto advance = [&] {
            const int64_t on_a = (MODE == kWeight ? (int64_t)N : 1) * kDeep * 2;
            const int64_t on_b = kLookUp ? 0 : (MODE == kForward ? 1 : (int64_t)K) * kDeep * 2;
            base_a += on_a, base_b += on_b;
            if constexpr (kWideA) {
#pragma unroll
                for (int q = 0; q < OpA::kRounds; ++q) from_a[q] += on_a;
            }
        };
        // The step at d0 in `here`: FN products to a turn.  A turn reads the rows' fragment of two turns on and, towards
        // the end of the first half, a fragment of the second half's columns, and issues its share of the next step's
        // copies, if there is one: all in the first half, so that they land during the second (over all turns: 4 %
        // slower).  The compiler may not move anything across turns, or it would read each fragment right before its
        // use and wait for it.
        constexpr int kAhead = (BUFFERS - 1) * kDeep;
        auto step = [&](auto next, auto partial, int later, int d0, const char *here, char *there) {
            constexpr int kTurns = kDeep / 32 * FM, kLead = 2, kEach = kCopies / (kTurns / 2);
            static_assert(kEach * (kTurns / 2) == kCopies && FM >= FN);
            copies_landed<kCopies, BUFFERS - 2>(later);
            take_rows();
            look_up(d0 + 2 * kDeep);
            const char *la = here, *lb = here + OpA::kBytes;
            Frag8<T> fb[kDeep / 32][FN], fa[kTurns];
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[0][j] = ob.frag(lb, j, 0);
#pragma unroll
            for (int i = 0; i < kLead; ++i) fa[i] = oa.frag(la, i % FM, i / FM);
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < kTurns; ++i) {
                if (i + kLead < kTurns) fa[i + kLead] = oa.frag(la, (i + kLead) % FM, (i + kLead) / FM);
                const int j0 = i - (FM - FN);
                if (j0 >= 0 && j0 < FN) fb[1][j0] = ob.frag(lb, j0, 1);
                if constexpr (decltype(next)::value) {
                    if (i < kTurns / 2) {
#pragma unroll
                        for (int c = i * kEach; c < (i + 1) * kEach; ++c) copy(partial, c, d0 + kAhead, there);
                    }
                }
                __builtin_amdgcn_s_setprio(1);  // before the other wavefront's reads and copies
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i % FM][j] = mfma16<T>(fb[i / FM][j], fa[i], acc[i % FM][j]);
                __builtin_amdgcn_s_setprio(0);
                __builtin_amdgcn_sched_barrier(0);
            }
            if constexpr (decltype(next)::value) put(there);
            advance();
        };
        constexpr std::true_type yes{};
        constexpr std::false_type no{};
        look_up(0);
        take_rows();
#pragma unroll
        for (int b = 0; b < BUFFERS - 1; ++b) {
            if (b && b * kDeep >= deep) break;
#pragma unroll
            for (int c = 0; c < kCopies; ++c) copy(yes, c, b * kDeep, lds + b * kStep);
            put(lds);
            advance();
        }
        look_up(kDeep);
        auto run = [&](auto one_step) {
            int d0 = 0, here = 0, there = (BUFFERS - 1) * kStep;
            auto on = [&] {
                d0 += kDeep;
                there = here;
                here = here + kStep == kLds ? 0 : here + kStep;
            };
            for (; d0 + kAhead + kDeep <= deep; on()) one_step(yes, no, BUFFERS - 2, d0, lds + here, lds + there);
            if (d0 + kAhead < deep) {
                one_step(yes, yes, BUFFERS - 2, d0, lds + here, lds + there);
                on();
            }
            if constexpr (BUFFERS == 2) {
                one_step(no, no, 0, d0, lds + here, lds);
            } else {
                for (; d0 < deep; on())
                    one_step(no, no, min((deep - d0 - 1) / kDeep, BUFFERS - 2), d0, lds + here, lds);
            }
        };
        if (idle)
            run([&](auto next, auto partial, int later, int d0, const char *, char *there) {
                copies_landed<kCopies, BUFFERS - 2>(later);
                take_rows();
                look_up(d0 + 2 * kDeep);
                if constexpr (decltype(next)::value) {
#pragma unroll
                    for (int c = 0; c < kCopies; ++c) copy(partial, c, d0 + kAhead, there);
                    put(there);
                }
                advance();
            });
        else
            run(step);
    }
    // The results go through LDS, so that whole lines are written: a lane holds four neighbouring columns of a row (row
    // lane % 16, columns (lane / 16) * 4 of a 16 x 16 block), 32 bytes a row of a block.  Written straight from there the
    // products took 6 % longer.  Results in 32 bits go in WM passes, of BM / WM rows.
    if constexpr (kPairs<T>) {
        if (threadIdx.x < BM + BN) scales[threadIdx.x] = scale;
    }
    __syncthreads();  // nobody reads the last step's operands any more
    [[maybe_unused]] float x_scale[kPairs<T> ? FM : 1], w_scale[kPairs<T> ? FN : 1][4];
    if constexpr (kPairs<T>) {
        static_assert(MODE == kForward && !STAGED);
#pragma unroll
        for (int i = 0; i < FM; ++i) x_scale[i] = scales[wm + i * 16 + (lane & 15)];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            const f32x4 w4 = *reinterpret_cast<const f32x4 *>(&scales[BM + wn + j * 16 + (lane >> 4) * 4]);
#pragma unroll
            for (int v = 0; v < 4; ++v) w_scale[j][v] = w4[v];
        }
    }
    // Whether results are stored in whole 16 bytes: rows in 8 bits are, whatever the results' columns.
    const bool whole_out = !STAGED && (!kPairs<T> || A.whole_out);
    const int64_t row0 = MODE == kWeight ? ((int64_t)part * A.E + e) * N : 0;
    auto pass = [&](auto type, int rows0, int rows, bool mine) {
        using O = decltype(type);
        constexpr int kPitch = BN * (int)sizeof(O) + 32, kEach = 16 / (int)sizeof(O), kChunks = BN / kEach;
        if (mine) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    typedef O O4 __attribute__((ext_vector_type(4)));
                    O4 o;
#pragma unroll
                    for (int v = 0; v < 4; ++v) {
                        if constexpr (kPairs<T>)
                            o[v] = (O)((float)acc[i][j][v] * x_scale[i] * w_scale[j][v]);
                        else
                            o[v] = (O)acc[i][j][v];
                    }
                    *reinterpret_cast<O4 *>(lds + (wm - rows0 + i * 16 + (lane & 15)) * kPitch +
                                            (wn + j * 16 + (lane >> 4) * 4) * (int)sizeof(O)) = o;
                }
        }
        __syncthreads();
        for (int c = threadIdx.x; c < rows * kChunks; c += WAVES * 64) {
            const int r = c / kChunks, row = m0 + rows0 + r, col = c0 + c % kChunks * kEach;
            if (row >= m1 || col >= cols) continue;
            const Words4 v = *reinterpret_cast<const Words4 *>(lds + r * kPitch + c % kChunks * 16);
            char *out = sizeof(O) == 4 ? reinterpret_cast<char *>(A.out32) : static_cast<char *>(A.out);
            out += ((row0 + row) * cols + col) * (int)sizeof(O);
            if (whole_out && MODE == kWeight && A.out32) {
                *reinterpret_cast<Words4 *>(out) = v;  // parts, which are read again at once (32768 x 128 x 128: 19 / 26 us)
            } else if (whole_out) {
                // Not kept in L2, where a round's results would push out the operands.  Kept / not, in us: 65536 rows of
                // 64 experts of 2048 x 1024 in 8 bits 188 / 160; 32768 of 16 of 2048 x 1024 in 16 bits forward 153 / 142,
                // input gradient 166 / 141; weight gradient of 65536 of 64 of 2048 x 2048 546 / 514.
                __builtin_nontemporal_store(__builtin_bit_cast(i32x4, v), reinterpret_cast<i32x4 *>(out));
            } else if (cols - col >= kEach) {
                __builtin_memcpy(out, &v, 16);
            } else {
                for (int i = 0; i < cols - col; ++i)
                    reinterpret_cast<O *>(out)[i] = reinterpret_cast<const O *>(lds + r * kPitch + c % kChunks * 16)[i];
            }
        }
    };
    if ((MODE != kForward || kPairs<T>) && A.out32) {
#pragma unroll
        for (int q = 0; q < WM; ++q) {
            if (q) __syncthreads();
            pass(float{}, q * (BM / WM), BM / WM, wm == q * (BM / WM));
        }
    } else if constexpr (kPairs<T>) {
        if (A.dtype == SK_BF16)
            pass(__bf16{}, 0, BM, true);
        else
            pass(_Float16{}, 0, BM, true);
    } else {
        pass(T{}, 0, BM, true);
    }
}

// ---- few rows: single tokens ----
//
// Forward for up to 16 rows of an expert at a time: what counts is that the weights are read at the memory's rate, so
// many wavefronts have to ask for them at once.  A work-group takes kFewCols columns, and its four wavefronts a quarter
// of the contraction each, straight from memory to registers; their sums meet in LDS.  A lane's 32 bytes of a row's 128
// are two fragments: the products' order along the contraction is free as long as both factors have the same.  16 rows
// of 14 of 64 experts of 1024 x 2048: 59 MB in 12.5 us (4.7 TB/s), in tiles of 64 with four buffers 11.0; in 8 bits 7.9
// and 7.2.

constexpr int kFewRows = 16, kFewCols = 32, kFewChunk = 64, kFewAtOnce = 4;

template <class T, bool GATHERED>
__global__ __launch_bounds__(kThreads) void sk_experts_few(ExpertArgs A) {
    constexpr int NC = kFewCols / 16, kWaves = kThreads / 64, kPitch = kFewCols + 4;
    using Sum = std::conditional_t<kPairs<T>, int, float>;
    __shared__ __attribute__((aligned(16))) Sum part[kWaves][kFewRows][kPitch];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int K = A.K, N = A.N;
    const Tile t = find_tile(A, kFewRows, (N + kFewCols - 1) / kFewCols, blockIdx.x);
    if (t.expert < 0) return;
    const int c0 = t.column * kFewCols, row = min(t.begin + (lane & 15), t.end - 1);
    Sum4<T> acc[NC] = {};
    if (t.expert < A.E) {
        int64_t from = row;
        if (GATHERED) {
            const int token = A.tokens[row];
            from = token >= 0 && token < A.T ? token : 0;
        }
        const int mine = (lane >> 4) * 16;  // the lane's first element of a chunk
        const T *x = static_cast<const T *>(A.x) + from * K + mine;
        const T *w[NC];
#pragma unroll
        for (int j = 0; j < NC; ++j)
            w[j] = static_cast<const T *>(A.w) + ((int64_t)t.expert * N + min(c0 + j * 16 + (lane & 15), N - 1)) * K + mine;
        const int chunks = (K + kFewChunk - 1) / kFewChunk;
        for (int first = wave; first < chunks; first += kWaves * kFewAtOnce) {
            Frag8<T> fx[kFewAtOnce][2], fw[kFewAtOnce][NC][2];
#pragma unroll
            for (int i = 0; i < kFewAtOnce; ++i) {
                const int d = (first + i * kWaves) * kFewChunk;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const bool in = d + mine + h * 8 < K;
                    fx[i][h] = in ? *reinterpret_cast<const Frag8<T> *>(x + d + h * 8) : Frag8<T>{};
#pragma unroll
                    for (int j = 0; j < NC; ++j)
                        fw[i][j][h] = in ? *reinterpret_cast<const Frag8<T> *>(w[j] + d + h * 8) : Frag8<T>{};
                }
            }
#pragma unroll
            for (int i = 0; i < kFewAtOnce; ++i)
#pragma unroll
                for (int h = 0; h < 2; ++h)
#pragma unroll
                    for (int j = 0; j < NC; ++j) acc[j] = mfma16<T>(fw[i][j][h], fx[i][h], acc[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < NC; ++j)
        *reinterpret_cast<Sum4<T> *>(&part[wave][lane & 15][j * 16 + (lane >> 4) * 4]) = acc[j];
    __syncthreads();
    const int r = threadIdx.x / (kFewCols / 2), c = threadIdx.x % (kFewCols / 2) * 2;
    if (t.begin + r >= t.end || c0 + c >= N) return;
    Sum sum[2] = {};
#pragma unroll
    for (int q = 0; q < kWaves; ++q) sum[0] += part[q][r][c], sum[1] += part[q][r][c + 1];
    if constexpr (kPairs<T>) {
        int from = t.begin + r;
        if (GATHERED && t.expert < A.E) from = A.tokens[from];
        if (from < 0 || (GATHERED && from >= A.T)) from = 0;
        const int64_t to = (int64_t)(t.begin + r) * N + c0 + c;
        float y[2] = {};
        if (t.expert < A.E) {
#pragma unroll
            for (int v = 0; v < 2; ++v)
                if (c0 + c + v < N)
                    y[v] = (float)sum[v] * A.x_scale[from] * A.w_scale[(int64_t)t.expert * N + c0 + c + v];
        }
#pragma unroll
        for (int v = 0; v < 2; ++v) {
            if (c0 + c + v >= N) break;
            if (A.out32)
                A.out32[to + v] = y[v];
            else if (A.dtype == SK_BF16)
                static_cast<__bf16 *>(A.out)[to + v] = (__bf16)y[v];
            else
                static_cast<_Float16 *>(A.out)[to + v] = (_Float16)y[v];
        }
    } else {
        typedef T T2 __attribute__((ext_vector_type(2)));
        const T2 out = {(T)sum[0], (T)sum[1]};
        *reinterpret_cast<T2 *>(static_cast<T *>(A.out) + (int64_t)(t.begin + r) * N + c0 + c) = out;
    }
}

// gx[t] = sum over the token's slots of the rows' gradients, kept in 32 bits until here; eight columns to a thread.
// Memory: 65536 rows of 2048 in 118 us (5.1 TB/s).
template <class T>  // the result's
__global__ __launch_bounds__(kThreads) void sk_experts_sum_slots(ExpertArgs A, const float *rows, T *gx) {
    const int64_t chunks = (A.K + 7) / 8, all = (int64_t)A.T * A.k;
    const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
    const int64_t t = i / chunks, c = (i - t * chunks) * 8;
    if (t >= A.T) return;
    const bool whole = c + 8 <= A.K;
    const int left = whole ? 8 : (int)(A.K - c);
    float sum[8] = {};
    for (int s = 0; s < A.k; ++s) {
        const int32_t r = A.slots[t * A.k + s];
        if (r < 0 || r >= all) continue;
        const float *from = rows + (int64_t)r * A.K + c;
        float v[8];
        if (whole)
            load8(from, v);
        else
            load_some(from, 0, left, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
    }
    if (whole)
        store8(gx + t * A.K + c, sum);
    else
        store_some(gx + t * A.K + c, 0, left, sum);
}

// The parts of a weight gradient, summed in order; n elements, eight to a thread.
template <class T>
__global__ __launch_bounds__(kThreads) void sk_experts_sum_parts(const float *part, T *out, int64_t n, int parts) {
    const int64_t i = ((int64_t)blockIdx.x * kThreads + threadIdx.x) * 8;
    if (i >= n) return;
    const bool whole = i + 8 <= n;
    const int left = whole ? 8 : (int)(n - i);
    float sum[8] = {};
    for (int q = 0; q < parts; ++q) {
        float v[8];
        if (whole)
            load8(part + q * n + i, v);
        else
            load_some(part + q * n + i, 0, left, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) sum[j] += v[j];
    }
    if (whole)
        store8(out + i, sum);
    else
        store_some(out + i, 0, left, sum);
}

template <class F>
hipError_t with_half(int dtype, F f) {
    return dtype == SK_BF16 ? f(__bf16{}) : f(_Float16{});
}

int64_t parts_of(int64_t n, int64_t of) { return (n + of - 1) / of; }

// Row tiles that E experts' rows and the rows of none can take at most.
int64_t most_row_tiles(const ExpertArgs &a, int tile) {
    const int64_t rows = (int64_t)a.T * a.k;
    return rows / tile + (rows < a.E + 1 ? rows : a.E + 1);
}

// How a product is cut: tiles of `tile` squared with `buffers` steps of operands in LDS, the weight gradient's rows in
// `parts`.
struct Cut {
    int tile, parts, buffers;
};

// Rows' products.  The expected number of tiles (half a tile of each of several experts is empty) decides.  256: one
// work-group a CU; wherever its last round is filled it halves what the tiles read.  128: two a CU, which cover each
// other's first copies and last writes, or one with another step of copies under way.  64: too few tiles of 128 to go
// round.  What is under way bounds those, so they have as many buffers as let all tiles run at once: four up to two a CU,
// three up to three.  128 with three has a CU to itself, so one tile past 256 doubles its time: it is taken where there are
// no more whatever the shares (a last tile for each expert).  1760 rows of 16 of 1536 x 2048, 288 tiles, with two 26 us,
// with three 43; 1648 of 8 of 2048 x 512, 272 tiles, 11.5 / 16.3, in 8 bits 8.3 / 12.1.
// Measured, 256 / 128 / 64, in us: 65536 rows of 64 experts of 2048 x 2048 (9.0 rounds) 535 / 611 / 916; 8192 rows of 8 of
// 4096 x 2048 (2.3 rounds) 161 / 159 / 223; 8000 rows of 2 of 2048 x 1024 (1.0) 32 / 39 / 53.  Equal shares of whole tiles
// come out even better in 256 (8192 rows of 8: 118 / 147), but how the shares are is known on the device alone.
// 128 with two buffers / with three / 64 with four: in 8 bits, rows of one of 8192 x 8192: 256 49 / 35 / 30, 512 53 / 39 / 57,
// 1024 65 / 74 / 107; 1024 rows of one of 4096 x 4096 26 / 21 / 31, 512 of it 23 / 18 / 17; 2331 rows of 12 of 520 x 1008
// 9.8 / 9.0 / 8.0, 5000 10.3 / 9.9 / 11.6; in 16 bits, 512 rows of one of 8192 x 8192 112 / 88 / 115; 600 rows of 4 of
// 2048 x 2048 22 / 23 / 14.  64 with two / four: 8 bits, 256 rows of one of 4096 x 4096 17 / 9.6; 16 bits, 256 of one of
// 2048 x 2048 16 / 8.8, 128 of one of 8192 x 8192 93 / 43; two / three / four, 8 bits, 4000 rows of 64 of 512 x 512 (2.9 a
// CU) 6.9 / 7.0 / 8.4.  128 with three in the input gradient, two / three: 1024 rows of one of 4096 x 4096 45 / 50, 512 of
// 8192 x 8192 105 / 96: two.
// Where most experts have less than a tile of 64 (up to 32 rows an expert), the weights' reading is all the time, and small
// tiles with much under way read fastest; four buffers where a row is 4 KB or more.  64 with three / four / 128 / 256: 8 bits,
// 500 rows of 64 of 2048 x 2048 52 / 56 / 52 / 59, 64 rows 32 / 33 / 41 / 52, 64 of 16 of 4096 x 4096 61 / 57 / 68 / 70, 256
// of 32 of 4096 x 1024 29 / 30 / 31 / 36; 16 bits, 500 of 64 of 2048 x 2048 107 / 101 / 125 / 132, 1000 of 64 of 1024 x 2048
// 61 / 57 / 68 / 69, 500 of 32 of 4096 x 1024 52 / 53 / 52 / 58.  The input gradient,
// whose copies of w are as wide as the tile, has 128 there: 500 of 64 of 2048 x 2048 100 / 97 / 93 / 108, 64 of 16 of
// 4096 x 4096 104 / 108 / 87 / 97.
// Rows that are no whole chunks have two buffers, in tiles of 64 or 128: 64 where the larger ones do not go round, and
// forward where experts have few rows.  64 / 128, in us: forward, 500 rows of 64 of 1003 x 1001 31 / 34, 1000 of them
// 37 / 34, 1000 of 64 of 2050 x 517 37 / 56, 256 of 32 of 1999 x 2041 62 / 58; input gradient, 1780 of 4 of 1021 x 2041
// 34 / 51, 2700 of 16 of 2045 x 1017 64 / 92.
Cut cut_rows(const ExpertArgs &a, bool input, bool whole) {
    const int cols = input ? a.K : a.N;
    const int64_t rows = (int64_t)a.T * a.k, half = (a.E + 1) / 2;
    auto tiles = [&](int64_t tile, int64_t last) {
        return (a.E == 1 ? parts_of(rows, tile) : rows / tile + last) * parts_of(cols, tile);
    };
    const int64_t large = tiles(256, half), rounds = parts_of(large, 256), mid = tiles(128, half), small = tiles(64, half);
    const bool sparse = rows <= 32 * (int64_t)a.E, few = mid < 256 && small <= 512;
    if (!whole) return {mid < 256 || (sparse && !input) ? 64 : 128, 1, 2};
    if (!sparse && large >= 256 && large * 20 >= rounds * 256 * 17) return {256, 1, 2};
    if (sparse && !input) return {64, 1, few || a.K >= 2048 ? 4 : 3};
    if (mid < 256 && small <= 768) return {64, 1, few ? 4 : 3};
    return {128, 1, tiles(128, a.E) <= 256 && !input ? 3 : 2};
}

// Weight gradients.  256 where there are two rounds of it and its edges waste no more than 128's would; else 128, or 64
// where that makes too few work-groups.  Few tiles over many rows are cut along the rows, into parts of eight steps or
// more, until there are two work-groups a CU.  Measured, in us: 256 / 128: 8192 rows of 8 of 4096 x 2048 121 / 140,
// 24000 rows of 32 of 2048 x 1024 98 / 106; 128 / 64: 9620 rows of 14 of 96 x 80 8.7 / 6.4; whole / in parts: 65536
// rows of 16 experts of 512 x 512 46 / 46, 32768 rows of 2 of 128 x 128 81 / 19, of 128 x 127 786 / 43.
Cut cut_weight(const ExpertArgs &a) {
    auto tiles = [&](int64_t tile) { return a.E * parts_of(a.N, tile) * parts_of(a.K, tile); };
    if (tiles(256) >= 512 && tiles(256) * 4 * 20 <= tiles(128) * 23) return {256, 1, 2};
    const int64_t steps = parts_of((int64_t)a.T * a.k, (int64_t)a.E * kDeep);
    auto cut = [&](int tile) {
        int64_t parts = parts_of(512, tiles(tile));
        if (parts > steps / 8) parts = steps / 8;
        return Cut{tile, (int)(parts < 1 ? 1 : parts), 2};
    };
    const Cut c = cut(128);
    return tiles(128) * c.parts >= 256 ? c : cut(64);
}

// Whether rows can be copied in chunks of 16 bytes.
bool chunks(const ExpertArgs &a) {
    return a.K % 8 == 0 && a.N % 8 == 0 && (!a.x || aligned16(a.x)) && (!a.w || aligned16(a.w)) &&
           (!a.gy || aligned16(a.gy)) && aligned16(a.out) && aligned16(a.out32);
}

template <int MODE, int TILE, int WM, int WN, bool STAGED = false, int BUFFERS = 2>
hipError_t launch_tile(const ExpertArgs &a, hipStream_t st) {
    const int64_t tiles = MODE == kWeight ? a.E * parts_of(a.N, TILE) * parts_of(a.K, TILE) * a.parts
                                          : most_row_tiles(a, TILE) * parts_of(MODE == kForward ? a.N : a.K, TILE);
    return with_half(a.dtype, [&](auto type) {
        using T = decltype(type);
        auto go = [&](auto kernel) {
            hipLaunchKernelGGL(kernel, dim3((unsigned)(parts_of(tiles, 8) * 8)), dim3(WM * WN * 64), 0, st, a);
            return hipGetLastError();
        };
        constexpr bool kGathers = MODE != kInput;
        if constexpr (STAGED) {
            if (a.tokens && kGathers) return go(sk_experts_tile<T, MODE, TILE, TILE, WM, WN, kGathers, kGathers, true>);
            return go(sk_experts_tile<T, MODE, TILE, TILE, WM, WN, false, false, true>);
        } else {
            if (a.tokens && kGathers)
                return (int64_t)a.T * a.K * 2 >= (int64_t(1) << 32)
                           ? go(sk_experts_tile<T, MODE, TILE, TILE, WM, WN, kGathers, kGathers, false, BUFFERS>)
                           : go(sk_experts_tile<T, MODE, TILE, TILE, WM, WN, kGathers, false, false, BUFFERS>);
            return go(sk_experts_tile<T, MODE, TILE, TILE, WM, WN, false, false, false, BUFFERS>);
        }
    });
}

hipError_t launch_few(const ExpertArgs &a, hipStream_t st) {
    const int64_t tiles = most_row_tiles(a, kFewRows) * parts_of(a.N, kFewCols);
    return with_half(a.dtype, [&](auto type) {
        using T = decltype(type);
        const dim3 grid((unsigned)(parts_of(tiles, 8) * 8));
        if (a.tokens)
            hipLaunchKernelGGL((sk_experts_few<T, true>), grid, dim3(kThreads), 0, st, a);
        else
            hipLaunchKernelGGL((sk_experts_few<T, false>), grid, dim3(kThreads), 0, st, a);
        return hipGetLastError();
    });
}

// Rows in 8 bits, which are whole chunks always.
template <int TILE, int WM, int WN, int BUFFERS = 2>
hipError_t launch_pairs(const ExpertArgs &a, hipStream_t st) {
    const int64_t tiles = most_row_tiles(a, TILE) * parts_of(a.N, TILE);
    auto go = [&](auto kernel) {
        hipLaunchKernelGGL(kernel, dim3((unsigned)(parts_of(tiles, 8) * 8)), dim3(WM * WN * 64), 0, st, a);
        return hipGetLastError();
    };
    if (!a.tokens) return go(sk_experts_tile<Pair, kForward, TILE, TILE, WM, WN, false, false, false, BUFFERS>);
    return (int64_t)a.T * a.K * 2 >= (int64_t(1) << 32)
               ? go(sk_experts_tile<Pair, kForward, TILE, TILE, WM, WN, true, true, false, BUFFERS>)
               : go(sk_experts_tile<Pair, kForward, TILE, TILE, WM, WN, true, false, false, BUFFERS>);
}

template <int MODE>
hipError_t launch_product(const ExpertArgs &a, const Cut &c, hipStream_t st) {
    if (!chunks(a))
        return c.tile == 64 ? launch_tile<MODE, 64, 2, 2, true>(a, st) : launch_tile<MODE, 128, 2, 2, true>(a, st);
    if (c.tile == 256) return launch_tile<MODE, 256, 2, 4>(a, st);
    if constexpr (MODE != kWeight) {
        if (c.tile == 64)
            return c.buffers == 4 ? launch_tile<MODE, 64, 2, 2, false, 4>(a, st) : launch_tile<MODE, 64, 2, 2, false, 3>(a, st);
    } else if (c.tile == 64) {
        return launch_tile<MODE, 64, 2, 2>(a, st);
    }
    if constexpr (MODE == kForward) {
        if (c.buffers == 3) return launch_tile<MODE, 128, 2, 2, false, 3>(a, st);
    }
    return launch_tile<MODE, 128, 2, 2>(a, st);
}

hipError_t launch_rows_input(const ExpertArgs &a, hipStream_t st) {
    return launch_product<kInput>(a, cut_rows(a, true, chunks(a)), st);
}

}  // namespace

size_t experts_workspace_bytes(int T, int k, int K) { return (size_t)T * k * K * 4; }

size_t experts_weight_workspace_bytes(const ExpertArgs &a) {
    const Cut c = cut_weight(a);
    return c.parts > 1 ? (size_t)c.parts * a.E * a.N * a.K * 4 : 0;
}

hipError_t launch_experts_forward(const ExpertArgs &a, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    // The weights are read once for each 16 rows of an expert.  Few / tiles, in us: 256 rows, 64 experts of 2048 x 2048
    // 98 / 99, 64 rows 66 / 73; 512 rows, 64 of 1024 x 2048 60 / 57; 64 rows of one of 2048 x 2048 8.6 / 8.7, of 512 x 512
    // 5.2 / 5.1, 16 of one of 8192 x 8192 33 / 38; 16 rows of 64 of 1024 x 2048 12.5 / 11.0.  For 17 to 64 rows of one of
    // 4096 x 4096 (25 / 15) and more the tiles are much faster, but they sum in another order, and results there would not
    // stay the same to the last bit.
    const int64_t rows = (int64_t)a.T * a.k;
    if (chunks(a) && (rows <= 64 || rows <= 4 * a.E)) return launch_few(a, st);
    return launch_product<kForward>(a, cut_rows(a, false, chunks(a)), st);
}

hipError_t launch_experts_packed(const ExpertArgs &p, hipStream_t st) {
    ExpertArgs a = p;
    a.whole_out = aligned16(a.out) && (int64_t)a.N * (a.dtype == SK_F32 ? 4 : 2) % 16 == 0;
    a.out32 = a.dtype == SK_F32 ? static_cast<float *>(a.out) : nullptr;
    // Few / tiles, in us: 1 row of one of 8192 x 8192 14.5 / 15.7, 8 15.0 / 16.0, 16 16.3 / 16.4, 64 47 / 19; 4 rows of 64
    // of 1024 x 2048 5.0 / 5.8, 16 7.9 / 7.1, 32 12.2 / 11.0, 96 22 / 23; 512 33 / 29.
    if ((int64_t)a.T * a.k <= 8) {
        const dim3 grid((unsigned)(parts_of(most_row_tiles(a, kFewRows) * parts_of(a.N, kFewCols), 8) * 8));
        if (a.tokens)
            hipLaunchKernelGGL((sk_experts_few<Pair, true>), grid, dim3(kThreads), 0, st, a);
        else
            hipLaunchKernelGGL((sk_experts_few<Pair, false>), grid, dim3(kThreads), 0, st, a);
        return hipGetLastError();
    }
    const Cut c = cut_rows(a, false, true);
    if (c.tile == 256) return launch_pairs<256, 2, 4>(a, st);
    if (c.tile == 64) return c.buffers == 4 ? launch_pairs<64, 2, 2, 4>(a, st) : launch_pairs<64, 2, 2, 3>(a, st);
    return c.buffers == 3 ? launch_pairs<128, 2, 2, 3>(a, st) : launch_pairs<128, 2, 2>(a, st);
}

hipError_t launch_experts_input(const ExpertArgs &a, void *ws, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    if (!a.slots) return launch_rows_input(a, st);
    ExpertArgs r = a;
    r.out32 = static_cast<float *>(ws);
    const hipError_t e = launch_rows_input(r, st);
    if (e != hipSuccess) return e;
    auto sum = [&](auto *to) {
        using T = std::remove_pointer_t<decltype(to)>;
        const dim3 grid((unsigned)parts_of((int64_t)a.T * parts_of(a.K, 8), kThreads));
        hipLaunchKernelGGL((sk_experts_sum_slots<T>), grid, dim3(kThreads), 0, st, a, static_cast<const float *>(ws), to);
        return hipGetLastError();
    };
    if (a.out32) return sum(a.out32);
    return with_half(a.dtype, [&](auto type) { return sum(static_cast<decltype(type) *>(a.out)); });
}

hipError_t launch_experts_weight(const ExpertArgs &a, void *ws, hipStream_t st) {
    ExpertArgs r = a;
    const Cut c = cut_weight(a);
    r.parts = c.parts;
    r.out32 = c.parts > 1 ? static_cast<float *>(ws) : nullptr;
    const hipError_t e = launch_product<kWeight>(r, c, st);
    if (e != hipSuccess || c.parts == 1) return e;
    return with_half(a.dtype, [&](auto type) {
        using T = decltype(type);
        const int64_t n = (int64_t)a.E * a.N * a.K;
        hipLaunchKernelGGL((sk_experts_sum_parts<T>), dim3((unsigned)parts_of(n, 8 * kThreads)), dim3(kThreads), 0, st,
                           static_cast<const float *>(ws), static_cast<T *>(a.out), n, c.parts);
        return hipGetLastError();
    });
}

}  // namespace sk
