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

template <class T>
__device__ __forceinline__ f32x4 mfma16(const Frag8<T> &a, const Frag8<T> &b, f32x4 c) {
    if constexpr (std::is_same_v<T, __bf16>)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

// ---- tiles: columns in whole chunks of eight, every pointer aligned to 16 bytes ----
//
// A work-group computes BM x BN results; its wavefronts, WM x WN of them, a part of BM / WM x BN / WN each, held in
// registers.  The contraction goes in steps of 64 (128 bytes of a row, a whole cache line).  Operands are copied to LDS
// by the memory pipe itself, 16 bytes a lane, into one of two buffers, one step ahead of the products, with one barrier
// a step.  The copies are issued one by one among the products, since the pipe takes few at a time and a wavefront
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
// 65536 rows of 64 experts of 2048 x 2048, bf16: forward 509 us (1080 TFLOP/s), the input gradient's rows in 32 bits 561
// (981), weight gradient 647 (849); a library product of 65536 x 2048 x 2048 reaches 1410 TFLOP/s here.  Of a step's
// 1.55 us the products alone take 0.95 and the copies alone 1.28.  The LDS reads are not what bounds a step: 16-byte reads
// alone reach 248 bytes a cycle a CU, transposing ones 173, which for the weight gradient's 192 KB is a quarter of a step.
// Rows that are no whole 16 bytes take 2 times as long forward and 3 to 4 times in the gradients.

constexpr int kDeep = 64;

__device__ __attribute__((aligned(16))) uint32_t zero_page[4];

using LdsByte = __attribute__((address_space(3))) char;
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
using LdsShort4 = __attribute__((address_space(3))) s16x4;

// Copies 16 bytes a lane to LDS: from base + each lane's offset to `to` (one for the wavefront) + 16 lane.  WIDE: the
// offset is a whole address.  Written out, since the compiler puts a wait for every copy under way before each
// transposing read that follows it.  It has no result in registers, and the place is not read before all_copies.
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
// Every copy of the work-group has landed and every LDS read is done.
__device__ __forceinline__ void all_copies() {
    __builtin_amdgcn_sched_barrier(0);
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
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
template <class T, int MODE, int BM, int BN, int WM, int WN, bool GATHERED, bool WIDE, bool STAGED>
__global__ __launch_bounds__(WM *WN * 64) __attribute__((amdgpu_waves_per_eu(2))) void sk_experts_tile(ExpertArgs A) {
    constexpr int WAVES = WM * WN, FM = BM / WM / 16, FN = BN / WN / 16;
    using OpA = Operand<T, MODE == kWeight, BM, WAVES, FM>;
    using OpB = Operand<T, MODE != kForward, BN, WAVES, FN>;
    constexpr int kStep = OpA::kBytes + OpB::kBytes;
    constexpr bool kWideA = WIDE && MODE == kForward, kWideB = WIDE && MODE == kWeight;
    constexpr int kOut = BM * (BN * 2 + 32);  // the results, below
    static_assert(BM / WM * (BN * 4 + 32) <= kOut);
    __shared__ __attribute__((aligned(1024))) char lds[2 * kStep > kOut ? 2 * kStep : kOut];

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

    f32x4 acc[FM][FN] = {};
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
        auto step = [&](auto next, auto partial, int d0, const char *here, char *there) {
            constexpr int kTurns = kDeep / 32 * FM, kLead = 2, kEach = kCopies / (kTurns / 2);
            static_assert(kEach * (kTurns / 2) == kCopies && FM >= FN);
            all_copies();
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
                        for (int c = i * kEach; c < (i + 1) * kEach; ++c) copy(partial, c, d0 + kDeep, there);
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
        for (int c = 0; c < kCopies; ++c) copy(yes, c, 0, lds);
        put(lds);
        advance();
        look_up(kDeep);
        auto run = [&](auto one_step) {
            int d0 = 0, odd = 0;
            for (; d0 + 2 * kDeep <= deep; d0 += kDeep, odd ^= 1)
                one_step(yes, no, d0, lds + odd * kStep, lds + (odd ^ 1) * kStep);
            if (d0 + kDeep < deep) {
                one_step(yes, yes, d0, lds + odd * kStep, lds + (odd ^ 1) * kStep);
                d0 += kDeep, odd ^= 1;
            }
            one_step(no, no, d0, lds + odd * kStep, lds);
        };
        if (idle)
            run([&](auto next, auto partial, int d0, const char *, char *there) {
                all_copies();
                take_rows();
                look_up(d0 + 2 * kDeep);
                if constexpr (decltype(next)::value) {
#pragma unroll
                    for (int c = 0; c < kCopies; ++c) copy(partial, c, d0 + kDeep, there);
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
    __syncthreads();  // nobody reads the last step's operands any more
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
                    for (int v = 0; v < 4; ++v) o[v] = (O)acc[i][j][v];
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
            if constexpr (!STAGED) {
                *reinterpret_cast<Words4 *>(out) = v;
            } else if (cols - col >= kEach) {
                __builtin_memcpy(out, &v, 16);
            } else {
                for (int i = 0; i < cols - col; ++i)
                    reinterpret_cast<O *>(out)[i] = reinterpret_cast<const O *>(lds + r * kPitch + c % kChunks * 16)[i];
            }
        }
    };
    if (MODE != kForward && A.out32) {
#pragma unroll
        for (int q = 0; q < WM; ++q) {
            if (q) __syncthreads();
            pass(float{}, q * (BM / WM), BM / WM, wm == q * (BM / WM));
        }
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
// of 14 of 64 experts of 1024 x 2048: 59 MB in 13 us (4.5 TB/s); in tiles of 64 18 us.

constexpr int kFewRows = 16, kFewCols = 32, kFewChunk = 64, kFewAtOnce = 4;

template <class T, bool GATHERED>
__global__ __launch_bounds__(kThreads) void sk_experts_few(ExpertArgs A) {
    constexpr int NC = kFewCols / 16, kWaves = kThreads / 64, kPitch = kFewCols + 4;
    __shared__ __attribute__((aligned(16))) float part[kWaves][kFewRows][kPitch];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int K = A.K, N = A.N;
    const Tile t = find_tile(A, kFewRows, (N + kFewCols - 1) / kFewCols, blockIdx.x);
    if (t.expert < 0) return;
    const int c0 = t.column * kFewCols, row = min(t.begin + (lane & 15), t.end - 1);
    f32x4 acc[NC] = {};
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
        *reinterpret_cast<f32x4 *>(&part[wave][lane & 15][j * 16 + (lane >> 4) * 4]) = acc[j];
    __syncthreads();
    const int r = threadIdx.x / (kFewCols / 2), c = threadIdx.x % (kFewCols / 2) * 2;
    if (t.begin + r >= t.end || c0 + c >= N) return;
    float sum[2] = {};
#pragma unroll
    for (int q = 0; q < kWaves; ++q) sum[0] += part[q][r][c], sum[1] += part[q][r][c + 1];
    typedef T T2 __attribute__((ext_vector_type(2)));
    const T2 out = {(T)sum[0], (T)sum[1]};
    *reinterpret_cast<T2 *>(static_cast<T *>(A.out) + (int64_t)(t.begin + r) * N + c0 + c) = out;
}

// gx[t] = sum over the token's slots of the rows' gradients, kept in 32 bits until here; eight columns to a thread.
// Memory: 65536 rows of 2048 in 118 us (5.1 TB/s).
template <class T>
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

// How a product is cut: tiles of `tile` squared, the weight gradient's rows in `parts`.
struct Cut {
    int tile, parts;
};

// Rows' products.  The expected number of tiles (half a tile of each expert is empty) decides.  256: one work-group a
// CU; wherever its last round is filled it halves what the tiles read.  128: two a CU, which cover each other's first
// copies and last writes.  64: too few tiles of 128 to go round.  Measured, 256 / 128 / 64, in us: 65536 rows of 64
// experts of 2048 x 2048 (9.0 rounds) 527 / 609 / 914; 8192 rows of 8 of 4096 x 2048 (2.3 rounds) 147 / 143 / 205; 8000
// rows of 2 of 2048 x 1024 (1.0) 34 / 39 / 62; 2331 rows of 12 of 520 x 1000 25 / 12.5 / 11.6; 300 rows of 2 of
// 2048 x 2048 40 / 17 / 12.
Cut cut_rows(const ExpertArgs &a, int cols) {
    const int64_t rows = (int64_t)a.T * a.k;
    auto tiles = [&](int64_t tile) { return (rows / tile + (a.E + 1) / 2) * parts_of(cols, tile); };
    const int64_t large = tiles(256), rounds = parts_of(large, 256);
    if (large >= 256 && large * 20 >= rounds * 256 * 17) return {256, 1};
    return {tiles(128) >= 256 ? 128 : 64, 1};
}

// Weight gradients.  256 where there are two rounds of it and its edges waste no more than 128's would; else 128, or 64
// where that makes too few work-groups.  Few tiles over many rows are cut along the rows, into parts of eight steps or
// more, until there are two work-groups a CU.  Measured, in us: 256 / 128: 8192 rows of 8 of 4096 x 2048 197 / 231,
// 24000 rows of 32 of 2048 x 1024 147 / 174; 128 / 64: 9620 rows of 14 of 96 x 80 16.4 / 10.9; whole / in parts: 65536
// rows of 16 experts of 512 x 512 111 / 73, 32768 rows of 2 of 128 x 128 131 / 19, of 128 x 127 809 / 45.
Cut cut_weight(const ExpertArgs &a) {
    auto tiles = [&](int64_t tile) { return a.E * parts_of(a.N, tile) * parts_of(a.K, tile); };
    if (tiles(256) >= 512 && tiles(256) * 4 * 20 <= tiles(128) * 23) return {256, 1};
    const int64_t steps = parts_of((int64_t)a.T * a.k, (int64_t)a.E * kDeep);
    auto cut = [&](int tile) {
        int64_t parts = parts_of(512, tiles(tile));
        if (parts > steps / 8) parts = steps / 8;
        return Cut{tile, (int)(parts < 1 ? 1 : parts)};
    };
    const Cut c = cut(128);
    return tiles(128) * c.parts >= 256 ? c : cut(64);
}

// Whether rows can be copied in chunks of 16 bytes.
bool chunks(const ExpertArgs &a) {
    return a.K % 8 == 0 && a.N % 8 == 0 && (!a.x || aligned16(a.x)) && (!a.w || aligned16(a.w)) &&
           (!a.gy || aligned16(a.gy)) && aligned16(a.out) && aligned16(a.out32);
}

template <int MODE, int TILE, int WM, int WN, bool STAGED = false>
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
                           ? go(sk_experts_tile<T, MODE, TILE, TILE, WM, WN, kGathers, kGathers, false>)
                           : go(sk_experts_tile<T, MODE, TILE, TILE, WM, WN, kGathers, false, false>);
            return go(sk_experts_tile<T, MODE, TILE, TILE, WM, WN, false, false, false>);
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

template <int MODE>
hipError_t launch_product(const ExpertArgs &a, const Cut &c, hipStream_t st) {
    if (!chunks(a))
        return c.tile == 64 ? launch_tile<MODE, 64, 2, 2, true>(a, st) : launch_tile<MODE, 128, 2, 2, true>(a, st);
    if (c.tile == 256) return launch_tile<MODE, 256, 2, 4>(a, st);
    if (c.tile == 128) return launch_tile<MODE, 128, 2, 2>(a, st);
    return launch_tile<MODE, 64, 2, 2>(a, st);
}

hipError_t launch_rows_input(const ExpertArgs &a, hipStream_t st) {
    return launch_product<kInput>(a, cut_rows(a, a.K), st);
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
    // 95 / 115; 512 rows, 64 of 1024 x 1024 34 / 28.  Up to 64 rows of few experts, too, where tiles are too few: 64 rows
    // of one of 2048 x 2048 9.0 / 11.3, of 4096 x 4096 25 / 32, of 512 x 512 4.8 / 5.5; of four of 2048 x 2048 9.6 / 17.
    // Only large matrices have tiles enough then: 32 rows of 8192 x 8192 45 / 57, but 64 rows 87 / 61.
    const int64_t rows = (int64_t)a.T * a.k;
    if (chunks(a) && (rows <= 64 || rows <= 4 * a.E)) return launch_few(a, st);
    return launch_product<kForward>(a, cut_rows(a, a.N), st);
}

hipError_t launch_experts_input(const ExpertArgs &a, void *ws, hipStream_t st) {
    if (a.T == 0) return hipSuccess;
    if (!a.slots) return launch_rows_input(a, st);
    ExpertArgs r = a;
    r.out32 = static_cast<float *>(ws);
    const hipError_t e = launch_rows_input(r, st);
    if (e != hipSuccess) return e;
    return with_half(a.dtype, [&](auto type) {
        using T = decltype(type);
        const dim3 grid((unsigned)parts_of((int64_t)a.T * parts_of(a.K, 8), kThreads));
        hipLaunchKernelGGL((sk_experts_sum_slots<T>), grid, dim3(kThreads), 0, st, a, static_cast<const float *>(ws),
                           static_cast<T *>(a.out));
        return hipGetLastError();
    });
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
