// Products of the layers on block-scaled numbers (tern.h: tern_mx_linear, tern_mx_linear_grad) on the matrix cores.
//
// Every product is out[b][a] = sum over k of A[a][k] B[b][k] with both operands in records: 32 rows by one run of k,
// 4 KB, in the order in which the lanes of a wave take them (four matrix instructions, 16 bytes a lane each):
//   4-bit floats  256 k a record, 64 an instruction (32x32x64), a scale byte per row and 32 k: lane (row j, half h) holds
//                 32 k of one block, so its scale is its own, four instructions' in one dword;
//   bf16           64 k a record, 16 an instruction (32x32x16).
// Both take an instruction 32 cycles on a SIMD and 1 KB of each operand, so one loop serves both.
//
// Large products are bound by what the L2s give (a step of 256 x 256 outputs takes 68 KB, 1.05 us with half of the compute
// units at work on zeros, 0.85 of it multiplying, and 1.2 to 1.5 with all) and on random values by power, which holds the
// clock at 1.6 to 1.9 GHz: 4.2 PFLOP/s in 4 bits and 1.25 to 1.35 in bf16 at 8192^3 (5.3 and 1.55 on zeros).  Small ones are
// bound by launches and the way of their bytes; tern_mx_choice.h has the times that choose between the kernels.
//
// A's rows run along the output's rows in memory: lane l of an instruction's result holds column l % 32 (a row of B) and
// 16 rows (of A), four of them next to each other.
#include "tern_mx_product.h"

#include "tern_mx_sums.h"

namespace tern {
namespace {

typedef __attribute__((address_space(3))) void* LdsPointer;
typedef const __attribute__((address_space(1))) void* GlobalPointer;

// A workgroup's tile is WA x WB waves of UA x UB blocks of 32 x 32.  Half records of every row block (two instructions' k)
// come straight into LDS as one stage; four stages are there or on their way, scales with every other.
// PARTS operands for B meet a record of A together (or, with 1, one after the other, as if k were so many times as long:
// both gradients at 1537 x 1001 -> 775 in half 37 us, together 31).
template <bool F4, int UA, int UB, int WA, int WB, int PARTS>
struct Tile {
    static constexpr int kWaves = WA * WB, kThreads = 64 * kWaves;
    static constexpr int kA = UA * WA, kB = UB * WB, kBlocks = kA + PARTS * kB;
    static constexpr int kHalf = kMxRecord / 2, kStage = kBlocks * kHalf;
    static constexpr int kScales = F4 ? kBlocks * kMxScaleRecord : 0;
    // one wave's results on their way out: 32 rows of B by 32 UA of A, four bytes each at most
    static constexpr int kPitch = 32 * UA * 4 + 16, kOut = 32 * kPitch;
    static constexpr int kIn = 4 * kStage + 2 * kScales;
    static constexpr int kLds = kIn + kA * 32 * 4 > kWaves * kOut ? kIn + kA * 32 * 4 : kWaves * kOut;      // (and the bias)
    static_assert(kA % kWaves == 0 && kB % kWaves == 0, "whole records per wave");
};

// Until at most LEFT of this wave's loads are under way, every LDS read has returned, and all waves are here.
template <int LEFT>
__device__ __forceinline__ void arrive()
{
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(LEFT) : "memory");
}

// Which product, tile and share of k a workgroup has; false: none.  Workgroups go to the eight XCDs in turn: each takes a
// run of tiles, in bands of so many tiles of B by all of A, so that what neighbours read meets in its L2, and of one share of k
// before the next (against a run of every share's: gradients of 512 x 1024 -> 4096 in float 43.9 us for 47.5, of 23 x 1365 ->
// 3688 in half precision 25.6 for 30.3).  8192 x 4096 -> 16384 in 4 bits: bands of 2, 3, 5 and 6 are
// alike, one of 4 takes 3 % longer, of 8 or 16 8 %; the gradients of a layer of 8192 x 4096 -> 8192 are alike to 2 % with any of
// them up to 8 and take 2 % more with 16.  (Bands that are square in bytes, so narrower for a B in parts:
// between 5 % faster and 8 % slower.)
constexpr int kBand = 6;
struct Place {
    int tile_a, tile_b, split;
};
__device__ __forceinline__ bool place(const ProductJob& p, int index, Place& at)
{
    const int run = (index & 7) * p.per_xcd + (index >> 3), tiles = p.tiles_a * p.tiles_b;
    at.split = run / tiles;
    if (at.split >= p.splits) return false;
    const int tile = run - at.split * tiles;
    const int band = tile / (kBand * p.tiles_a), in_band = tile - band * kBand * p.tiles_a;
    const int wide = min(kBand, p.tiles_b - kBand * band);
    at.tile_a = in_band / wide;
    at.tile_b = kBand * band + in_band - at.tile_a * wide;
    return true;
}

// Workgroup `index` of a launch's columns: 32 of them, every eighth group to a thread of the first 256; through 1 KB of LDS.
__device__ __forceinline__ void sum_columns(const ColumnSums& c, int index, float* part)
{
    const int64_t col = (int64_t)index * 32 + (threadIdx.x & 31);
    const int slice = threadIdx.x >> 5;
    float s = 0.0f;
    if (slice < 8 && col < c.cols) {
#pragma unroll 4
        for (int64_t g = slice; g < c.groups; g += 8) s += c.sums[g * c.cols + col];
    }
    if (slice < 8) part[slice * 32 + (threadIdx.x & 31)] = s;
    __syncthreads();
    if (slice == 0 && col < c.cols) {
#pragma unroll
        for (int i = 1; i < 8; ++i) s += part[i * 32 + threadIdx.x];
        c.out[col] = s;
    }
}

template <bool F4, int UA, int UB, int WA, int WB, int PARTS>
__global__ __launch_bounds__(WA * WB * 64, UA * UB * PARTS > 4 ? 1 : 2) void tiled_kernel(ProductJobs jobs)
{
    typedef Tile<F4, UA, UB, WA, WB, PARTS> G;
    extern __shared__ __align__(16) uint8_t lds[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wa = wave % WA, wb = wave / WA;
    if ((int)blockIdx.x >= jobs.columns_first) {
        sum_columns(jobs.columns, (int)blockIdx.x - jobs.columns_first, reinterpret_cast<float*>(lds));
        return;
    }
    const bool second = (int)blockIdx.x >= jobs.first;
    const ProductJob& p = jobs.job[second];
    Place at;
    if (!place(p, (int)blockIdx.x - (second ? jobs.first : 0), at)) return;
    const int a0 = at.tile_a * G::kA, b0 = at.tile_b * G::kB;         // first row blocks
    const int from = at.split * p.split_steps;
    const int steps = min(p.groups * (PARTS > 1 ? 1 : p.parts) - from, p.split_steps);

    // A wave's share of a step's records.  Records past the operands' ends are read from their last row block; their
    // results are not stored.
    constexpr int kPerA = G::kA / G::kWaves, kPerB = G::kB / G::kWaves, kPer = kPerA + PARTS * kPerB;
    const uint8_t *source[kPer], *scale_source[kPer];
    const int part = from / p.groups;
    int group = from - part * p.groups;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const bool is_a = i < kPerA;
        const int64_t rec = (is_a ? (int64_t)min(a0 + i * G::kWaves + wave, p.a_blocks - 1)
                                  : (int64_t)min(b0 + (i - kPerA) % kPerB * G::kWaves + wave, p.b_blocks - 1)) * p.groups + group;
        source[i] = (is_a ? p.a : p.b + (part + (i - kPerA) / kPerB) * p.b_part) + rec * kMxRecord;
        if constexpr (F4) scale_source[i] = (is_a ? p.a_scales : p.b_scales) + rec * kMxScaleRecord;
    }
    // Stage `f` into its slot; `f` past the last one fetches that again (nobody reads it), so that counts stay the same.
    const int stages = 2 * steps;
    // (In two parts: a compute unit takes up 64 bytes of loads a cycle, and waves that have given it more than that stand
    // still, matrix instructions and all.)
    auto fetch = [&](int f, auto odd, auto second) {
        constexpr bool kOdd = decltype(odd)::value, kSecond = decltype(second)::value;
        uint8_t* to = lds + (f & 3) * G::kStage + wave * G::kHalf;
        uint8_t* to_scale = lds + 4 * G::kStage + ((f >> 1) & 1) * G::kScales + wave * kMxScaleRecord;
        const bool more = f + 1 < stages, more_scales = f + 2 < stages;
#pragma unroll
        for (int i = kSecond ? kPer / 2 : 0; i < (kSecond ? kPer : kPer / 2); ++i) {
            const GlobalPointer g = (GlobalPointer)(source[i] + lane * 16);
            const LdsPointer l = (LdsPointer)(to + i * G::kWaves * G::kHalf);
            __builtin_amdgcn_global_load_lds(g, l, 16, 0, 0);
            __builtin_amdgcn_global_load_lds(g, l, 16, 1024, 0);       // (the offset counts on both sides)
            source[i] += more ? G::kHalf : 0;
            if constexpr (F4 && !kOdd) {
                __builtin_amdgcn_global_load_lds((GlobalPointer)(scale_source[i] + lane * 4),
                                                 (LdsPointer)(to_scale + i * G::kWaves * kMxScaleRecord), 4, 0, 0);
                scale_source[i] += more_scales ? kMxScaleRecord : 0;
            }
        }
        // behind a part's last group: A from its beginning, B's next part
        if constexpr (!F4 && PARTS == 1 && kOdd && kSecond) {
            group += more ? 1 : 0;
            const bool wrap = group == p.groups;
            const int64_t back = wrap ? (int64_t)p.groups * kMxRecord : 0, on = wrap ? p.b_part : 0;
            group = wrap ? 0 : group;
#pragma unroll
            for (int i = 0; i < kPer; ++i) source[i] += (i < kPerA ? 0 : on) - back;
        }
    };

    // Operands of an instruction's k are read from LDS while the one before is multiplied.  A stage's second half is in
    // registers before it is multiplied: then the next stage has to be there, this one's slot is free, and what is loaded
    // into it has three stages' time.
    struct Operands {
        v4i a[UA], b[PARTS][UB];
    };
    struct Scales {
        int a[UA], b[UB];
    };
    v16f acc[UA][UB] = {};
    Operands even, odd;
    Scales scales = {}, next_scales = {};
    auto read = [&](Operands& o, int slot, int q) {
        const uint8_t *sa = lds + slot * G::kStage + wa * UA * G::kHalf + lane * 16, *sb = sa + (G::kA + wb * UB - wa * UA) * G::kHalf;
#pragma unroll
        for (int i = 0; i < UA; ++i) o.a[i] = *reinterpret_cast<const v4i*>(sa + i * G::kHalf + q * 1024);
#pragma unroll
        for (int e = 0; e < PARTS; ++e)
#pragma unroll
            for (int j = 0; j < UB; ++j) o.b[e][j] = *reinterpret_cast<const v4i*>(sb + (e * G::kB + j) * G::kHalf + q * 1024);
    };
    auto read_scales = [&](Scales& o, int record) {
        if constexpr (F4) {
            const uint8_t* sc = lds + 4 * G::kStage + (record & 1) * G::kScales + lane * 4;
#pragma unroll
            for (int i = 0; i < UA; ++i) o.a[i] = *reinterpret_cast<const int*>(sc + (wa * UA + i) * kMxScaleRecord);
#pragma unroll
            for (int j = 0; j < UB; ++j) o.b[j] = *reinterpret_cast<const int*>(sc + (G::kA + wb * UB + j) * kMxScaleRecord);
        }
    };
    auto multiply_all = [&](const Operands& o, auto q) {
#pragma unroll
        for (int e = 0; e < PARTS; ++e)
#pragma unroll
            for (int i = 0; i < UA; ++i)
#pragma unroll
                for (int j = 0; j < UB; ++j)
                    acc[i][j] = multiply_step<F4, decltype(q)::value>(o.a[i], o.b[e][j], acc[i][j], scales.a[i], scales.b[j]);
    };
    // Reads go between the first matrix instructions, loads between the others.
    const std::integral_constant<int, 0> k0;
    const std::integral_constant<int, 1> k1;
    const std::integral_constant<int, 2> k2;
    const std::integral_constant<int, 3> k3;
    const std::integral_constant<bool, false> in_even;
    const std::integral_constant<bool, true> in_odd;
    auto interleave = [&](auto reads, auto loads) {
#pragma unroll
        for (int i = 0; i < UA * UB * PARTS; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
            if (i < UA + PARTS * UB) __builtin_amdgcn_sched_group_barrier(0x100, decltype(reads)::value, 0);
            else if (decltype(loads)::value > 0) __builtin_amdgcn_sched_group_barrier(0x010, decltype(loads)::value, 0);
        }
        __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int kEven = (F4 ? 3 : 2) * kPer, kOddLoads = 2 * kPer;        // loads of a stage

    // The bias starts the sums (of the first split), by way of LDS.
    float* const start = reinterpret_cast<float*>(lds + G::kIn);
    const bool biased = p.bias && at.split == 0;
    float mine = 0.0f;
    static_assert(G::kA * 32 <= G::kThreads, "a thread to each row of A");
    if (biased && threadIdx.x < G::kA * 32 && (int64_t)a0 * 32 + threadIdx.x < p.na) mine = p.bias[(int64_t)a0 * 32 + threadIdx.x];
    fetch(0, in_even, in_even);
    fetch(0, in_even, in_odd);
    fetch(1, in_odd, in_even);
    fetch(1, in_odd, in_odd);
    fetch(2, in_even, in_even);
    fetch(2, in_even, in_odd);
    fetch(3, in_odd, in_even);
    if (biased && threadIdx.x < G::kA * 32) start[threadIdx.x] = mine;
    arrive<kOddLoads + kEven + 2 * (kPer / 2)>();     // (behind stage 0: 1, 2 and the first part of 3)
    read(even, 0, 0);
    read_scales(scales, 0);
    if (biased) {
#pragma unroll
        for (int i = 0; i < UA; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const float4 four = *reinterpret_cast<const float4*>(start + (wa * UA + i) * 32 + 8 * q + 4 * (lane >> 5));
#pragma unroll
                for (int j = 0; j < UB; ++j) {
                    acc[i][j][4 * q] = four.x; acc[i][j][4 * q + 1] = four.y;
                    acc[i][j][4 * q + 2] = four.z; acc[i][j][4 * q + 3] = four.w;
                }
            }
    }
    // (The last step reads operands of one more and drops them: stale bytes of the ring.)
    for (int r = 0; r < steps; ++r) {
        const int slot = 2 * (r & 1);
        read(odd, slot, 1);
        fetch(2 * r + 3, in_odd, in_odd);
        multiply_all(even, k0);
        interleave(k1, k1);
        arrive<kEven + kOddLoads>();
        read(even, slot + 1, 0);
        fetch(2 * r + 4, in_even, in_even);
        multiply_all(odd, k1);
        interleave(k1, k1);
        read(odd, slot + 1, 1);
        fetch(2 * r + 4, in_even, in_odd);
        multiply_all(even, k2);
        interleave(k1, k1);
        arrive<kEven + kOddLoads>();
        read(even, 2 - slot, 0);
        read_scales(next_scales, r + 1);
        fetch(2 * r + 5, in_odd, in_even);
        multiply_all(odd, k3);
        interleave(k2, k1);
        scales = next_scales;
    }
    arrive<0>();

    // Results leave by way of LDS, a region for each wave: 32 rows of B at a time, so that a store covers whole lines.
    // PAST: past the caches, for outputs that would not stay there anyhow (of 128 MB or more): their lines are then not in
    // the way of what comes next.  8192 x 4096 -> 16384 in bf16 (268 MB out), all of the call, 294 -> 284 us.
    auto leave = [&](auto* to, int64_t ld, auto past) {
        typedef std::remove_pointer_t<decltype(to)> T;
        constexpr int kVec = 16 / (int)sizeof(T), kRowLanes = 32 * UA / kVec, kRows = 64 / kRowLanes;
        uint8_t* mine = lds + wave * G::kOut;
        const int64_t a_at = (int64_t)(a0 + wa * UA) * 32 + (lane % kRowLanes) * kVec;
        const int left = (int)max((int64_t)0, min((int64_t)kVec, p.na - a_at));
#pragma unroll
        for (int j = 0; j < UB; ++j) {
#pragma unroll
            for (int i = 0; i < UA; ++i)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    Few<T, 4> four;
                    // (sums stay where they are until their turn: the compiler would fetch them all for every type at once)
                    if (q == 0) asm volatile("" : "+a"(acc[i][j]));
#pragma unroll
                    for (int r = 0; r < 4; ++r) four.v[r] = (T)acc[i][j][4 * q + r];
                    *reinterpret_cast<Few<T, 4>*>(mine + (lane & 31) * G::kPitch + (32 * i + 8 * q + 4 * (lane >> 5)) * sizeof(T)) = four;
                }
            asm volatile("" ::: "memory");      // (LDS serves a wave in its order; this keeps the compiler to it)
            const int64_t b_at = (int64_t)(b0 + wb * UB + j) * 32;
            const int rows = (int)max((int64_t)0, min((int64_t)32, p.nb - b_at));
#pragma unroll
            for (int r = 0; r < 32 / kRows; ++r) {
                const int row = r * kRows + lane / kRowLanes;
                const v4i w = *reinterpret_cast<const v4i*>(mine + row * G::kPitch + (lane % kRowLanes) * 16);
                typedef Few<T, kVec> Vec;
                typedef int Loose __attribute__((ext_vector_type(4), aligned(1)));
                if (row < rows && left > 0) {
                    T* const at = to + (b_at + row) * ld + a_at;
                    if (decltype(past)::value && left >= kVec) __builtin_nontemporal_store(w, (Loose*)at);
                    else store_few<kVec>(at, __builtin_bit_cast(Vec, w), left);
                }
            }
            asm volatile("" ::: "memory");
        }
    };
    auto leave_typed = [&](auto past) {
        if (p.type == TERN_F32) leave((float*)p.out, p.ld, past);
        else if (p.type == TERN_BF16) leave((__bf16*)p.out, p.ld, past);
        else leave((_Float16*)p.out, p.ld, past);
    };
    const std::integral_constant<bool, true> yes;
    const std::integral_constant<bool, false> no;
    if (p.splits > 1) {
        const int64_t ld = (p.na + 3) / 4 * 4;
        leave(p.partial + at.split * p.nb * ld, ld, no);
    } else if (UA * UB == 16 && p.na * p.nb >= ((int64_t)1 << (p.type == TERN_F32 ? 25 : 26))) {
        leave_typed(yes);
    } else {
        leave_typed(no);
    }
}

// Without a tile in LDS: a workgroup has UA x UB blocks, and each of its WAVES waves a share of k, whose records it
// takes from memory into registers, the next while one is multiplied.  Their sums are added through LDS, in order.  Bound by
// memory or the L2s: 16 rows of 4096 -> 16384 in 4 bits 8.0 us (35.7 MB, 4.5 TB/s), where a tile of 128 x 128 takes 12.
template <bool F4, int UA, int UB, int WAVES>
__global__ __launch_bounds__(WAVES * 64, 2) void direct_kernel(ProductJobs jobs)
{
    __shared__ __align__(16) float4 sums[WAVES * UA * UB * 4 * 64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if ((int)blockIdx.x >= jobs.columns_first) {
        sum_columns(jobs.columns, (int)blockIdx.x - jobs.columns_first, reinterpret_cast<float*>(sums));
        return;
    }
    const bool second = (int)blockIdx.x >= jobs.first;
    const ProductJob& p = jobs.job[second];
    Place at;
    if (!place(p, (int)blockIdx.x - (second ? jobs.first : 0), at)) return;
    const int a0 = at.tile_a * UA, b0 = at.tile_b * UB;
    const int first = at.split * p.split_steps, many = min(p.groups * p.parts - first, p.split_steps);
    const int each = (many + WAVES - 1) / WAVES;
    const int left = min(each, many - wave * each);     // this wave's records
    int ahead = left;

    const int start = first + wave * each;
    int part = start / p.groups, group = start - part * p.groups;
    const uint8_t *pa[UA], *pb[UB], *ps[UA + UB];
#pragma unroll
    for (int i = 0; i < UA; ++i) {
        const int64_t rec = (int64_t)min(a0 + i, p.a_blocks - 1) * p.groups + group;
        pa[i] = p.a + rec * kMxRecord;
        if constexpr (F4) ps[i] = p.a_scales + rec * kMxScaleRecord;
    }
    int at_b[UB];                                       // (rows that are not there: the first one's bytes once more)
#pragma unroll
    for (int j = 0; j < UB; ++j) {
        const int64_t rec = (int64_t)min(b0 + j, p.b_blocks - 1) * p.groups + group;
        pb[j] = p.b + part * p.b_part + rec * kMxRecord;
        if constexpr (F4) ps[UA + j] = p.b_scales + rec * kMxScaleRecord;
        at_b[j] = (int64_t)(b0 + j) * 32 + (lane & 31) < p.nb ? lane * 16 : (lane & 32) * 16;
    }
    struct Record {
        v4i a[UA][4], b[UB][4];
        int scale[UA + UB];
    };
    auto load = [&](Record& o) {
#pragma unroll
        for (int i = 0; i < UA; ++i) {
#pragma unroll
            for (int q = 0; q < 4; ++q) o.a[i][q] = *reinterpret_cast<const v4i*>(pa[i] + q * 1024 + lane * 16);
            if constexpr (F4) o.scale[i] = *reinterpret_cast<const int*>(ps[i] + lane * 4);
        }
#pragma unroll
        for (int j = 0; j < UB; ++j) {
#pragma unroll
            for (int q = 0; q < 4; ++q) o.b[j][q] = *reinterpret_cast<const v4i*>(pb[j] + q * 1024 + at_b[j]);
            if constexpr (F4) o.scale[UA + j] = *reinterpret_cast<const int*>(ps[UA + j] + lane * 4);
        }
        // (past the last one: that once more)
        const bool more = --ahead > 0;
        group += more ? 1 : 0;
        const bool wrap = !F4 && group == p.groups;
        const int64_t on = more ? kMxRecord - (wrap ? (int64_t)p.groups * kMxRecord : 0) : 0;
        group = wrap ? 0 : group;
#pragma unroll
        for (int i = 0; i < UA; ++i) pa[i] += on;
#pragma unroll
        for (int j = 0; j < UB; ++j) pb[j] += on + (wrap ? p.b_part : 0);
        if constexpr (F4) {
#pragma unroll
            for (int i = 0; i < UA + UB; ++i) ps[i] += more ? kMxScaleRecord : 0;
        }
    };
    v16f acc[UA][UB] = {};
    auto multiply = [&](const Record& o) {
        auto quarter = [&](auto q) {
            constexpr int Q = decltype(q)::value;
#pragma unroll
            for (int i = 0; i < UA; ++i)
#pragma unroll
                for (int j = 0; j < UB; ++j)
                    acc[i][j] = multiply_step<F4, Q>(o.a[i][Q], o.b[j][Q], acc[i][j], F4 ? o.scale[i] : 0, F4 ? o.scale[UA + j] : 0);
        };
        quarter(std::integral_constant<int, 0>());
        quarter(std::integral_constant<int, 1>());
        quarter(std::integral_constant<int, 2>());
        quarter(std::integral_constant<int, 3>());
    };
    if (left > 0) {
        Record even, odd;
        load(even);
        for (int i = left >> 1; i > 0; --i) {
            load(odd);
            multiply(even);
            __builtin_amdgcn_sched_barrier(0);
            load(even);
            multiply(odd);
            __builtin_amdgcn_sched_barrier(0);
        }
        if (left & 1) multiply(even);
    }

    add_up<UA, UB, WAVES>(p, acc, sums, a0, b0, at.split);
}

// A few rows straight from floats, in one launch: every workgroup has 32 rows of A and turns the rows of x into 4-bit
// numbers for itself, each wave the columns of its own share of k (two records, 512 columns, at a time, through LDS; the
// weights' loads are under way meanwhile).  One row of 4096 -> 4096: 3.9 us, with a launch that quantises in front 8.1; of
// 8192 -> 16384 13.0 us (71 MB, 5.5 TB/s).
template <typename T, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void few_rows_kernel(ProductJob p, const T* x, int64_t ldx, int64_t cols)
{
    __shared__ __align__(16) float4 sums[WAVES * 4 * 64];
    __shared__ __align__(16) uint8_t codes[WAVES][2][8][kMxFewRows][16];
    __shared__ __align__(16) uint8_t scales[WAVES][2][kMxFewRows][2][4];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int each = (p.groups + WAVES - 1) / WAVES, first = wave * each;
    const int left = min(each, p.groups - first);
    const int rows = (int)p.nb, row = (lane & 31) < rows ? lane & 31 : 0;
    const uint8_t* pa = p.a + ((int64_t)blockIdx.x * p.groups + first) * kMxRecord + lane * 16;
    const uint8_t* ps = p.a_scales + ((int64_t)blockIdx.x * p.groups + first) * kMxScaleRecord + lane * 4;
    struct Record {
        v4i a[4];
        int scale;
    };
    auto load = [&](Record& o, int i) {
        i = min(i, left - 1);
#pragma unroll
        for (int q = 0; q < 4; ++q) o.a[q] = *reinterpret_cast<const v4i*>(pa + (int64_t)i * kMxRecord + q * 1024);
        o.scale = *reinterpret_cast<const int*>(ps + (int64_t)i * kMxScaleRecord);
    };
    v16f acc[1][1] = {};
    if (left > 0) {
        Record even, odd;
        load(even, 0);
        load(odd, 1);
        for (int i = 0; i < left; i += 2) {
            const int64_t col = (int64_t)(first + i) * 256 + lane * 8;
            const int n = (int)max((int64_t)0, min((int64_t)8, cols - col));
            const int record = lane >> 5, block = (lane >> 2) & 7;
            for (int r0 = 0; r0 < rows; r0 += 4) {
                float v[4][8];                      // (four rows' loads under way together)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (r0 + r < rows) load_eight(v[r], x + (r0 + r) * ldx + col, n);
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (r0 + r < rows) {
                        const uint32_t byte = scale_byte<TERN_MX_F4>(block_most(v[r]));
                        *reinterpret_cast<uint32_t*>(&codes[wave][record][block][r0 + r][(lane & 3) * 4]) = f4_codes(v[r], byte);
                        if ((lane & 3) == 0) scales[wave][record][r0 + r][block & 1][block >> 1] = (uint8_t)byte;
                    }
            }
            auto multiply = [&](const Record& o, int rec) {
                const int scale = *reinterpret_cast<const int*>(&scales[wave][rec][row][lane >> 5][0]);
                auto quarter = [&](auto q) {
                    constexpr int Q = decltype(q)::value;
                    const v4i b = *reinterpret_cast<const v4i*>(&codes[wave][rec][2 * Q + (lane >> 5)][row][0]);
                    acc[0][0] = multiply_step<true, Q>(o.a[Q], b, acc[0][0], o.scale, scale);
                };
                quarter(std::integral_constant<int, 0>());
                quarter(std::integral_constant<int, 1>());
                quarter(std::integral_constant<int, 2>());
                quarter(std::integral_constant<int, 3>());
            };
            // (LDS serves a wave in its order; the fences keep the compiler to it)
            asm volatile("" ::: "memory");
            multiply(even, 0);
            load(even, i + 2);
            if (i + 1 < left) multiply(odd, 1);
            load(odd, i + 3);
            asm volatile("" ::: "memory");
        }
    }
    add_up<1, 1, WAVES>(p, acc, sums, blockIdx.x, 0, 0);
}

// Sums of the splits, in order, rounded once.
__global__ __launch_bounds__(256) void join_kernel(ProductJobs jobs)
{
    const bool second = (int)blockIdx.x >= jobs.first;
    const ProductJob& p = jobs.job[second];
    const int64_t quads = (p.na + 3) / 4;
    const int64_t e = (int64_t)((int)blockIdx.x - (second ? jobs.first : 0)) * 256 + threadIdx.x;
    if (e >= quads * p.nb) return;
    const int64_t b = e / quads, a = (e - b * quads) * 4;
    const float4* from = reinterpret_cast<const float4*>(p.partial) + e;
    float4 s = *from;
#pragma unroll 8
    for (int i = 1; i < p.splits; ++i) {
        const float4 t = from[i * quads * p.nb];
        s.x += t.x; s.y += t.y; s.z += t.z; s.w += t.w;
    }
    auto leave = [&](auto* to) {
        typedef std::remove_pointer_t<decltype(to)> T;
        const Few<T, 4> four = {{(T)s.x, (T)s.y, (T)s.z, (T)s.w}};
        store_few<4>(to + b * p.ld + a, four, (int)min((int64_t)4, p.na - a));
    };
    if (p.type == TERN_F32) leave((float*)p.out);
    else if (p.type == TERN_BF16) leave((__bf16*)p.out);
    else leave((_Float16*)p.out);
}

template <typename F>
int launch(F kern, int side, int threads, int lds, ProductJob* job, int n, const ColumnSums* columns, hipStream_t stream)
{
    if (lds > 64 * 1024)
        TERN_HIP_CHECK(hipFuncSetAttribute(reinterpret_cast<const void*>(kern), hipFuncAttributeMaxDynamicSharedMemorySize, lds));
    ProductJobs jobs = {};
    int64_t grid = 0;
    for (int i = 0; i < n; ++i) {
        ProductJob& p = jobs.job[i];
        p = job[i];
        p.tiles_a = (p.a_blocks + side - 1) / side;
        p.tiles_b = (p.b_blocks + side - 1) / side;
        const int64_t per_xcd = ((int64_t)p.tiles_a * p.tiles_b * p.splits + 7) / 8;
        if (i == 1) jobs.first = (int32_t)grid;
        grid += 8 * per_xcd;
        if (grid > INT32_MAX / 2) return TERN_ESHAPE;
        p.per_xcd = (int32_t)per_xcd;
    }
    if (n < 2) jobs.first = INT32_MAX;
    jobs.columns_first = INT32_MAX;
    if (columns) {
        jobs.columns = *columns;
        jobs.columns_first = (int32_t)grid;
        grid += ceil_div(columns->cols, 32);
        if (grid > INT32_MAX / 2) return TERN_ESHAPE;
    }
    kern<<<dim3((unsigned)grid), threads, lds, stream>>>(jobs);
    TERN_HIP_CHECK(hipGetLastError());
    return TERN_OK;
}
template <bool F4, int UA, int UB, int WA, int WB, int PARTS>
int launch_tiled(ProductJob* job, int n, const ColumnSums* columns, hipStream_t stream)
{
    typedef Tile<F4, UA, UB, WA, WB, PARTS> G;
    static_assert(G::kA == G::kB, "square tiles");
    return launch(tiled_kernel<F4, UA, UB, WA, WB, PARTS>, G::kA, G::kThreads, G::kLds, job, n, columns, stream);
}
template <bool F4>
int launch_form(int form, ProductJob* job, int n, const ColumnSums* columns, hipStream_t stream)
{
    switch (form) {
    case kDirect1: return launch(direct_kernel<F4, 1, 1, 8>, 1, 512, 0, job, n, columns, stream);
    case kDirect2: return launch(direct_kernel<F4, 2, 2, 4>, 2, 256, 0, job, n, columns, stream);
    case kTiled4:
        if constexpr (!F4) {
            if (job->parts == 2) return launch_tiled<F4, 2, 2, 2, 2, 2>(job, n, columns, stream);
            if (job->parts == 3) return launch_tiled<F4, 2, 2, 2, 2, 3>(job, n, columns, stream);
        }
        return launch_tiled<F4, 2, 2, 2, 2, 1>(job, n, columns, stream);
    default: return launch_tiled<F4, 4, 4, 2, 2, 1>(job, n, columns, stream);
    }
}

template <int WAVES>
int launch_few(const ProductJob& p, const void* x, int64_t ldx, int64_t cols, hipStream_t stream)
{
    const dim3 grid((unsigned)p.a_blocks);
    if (p.type == TERN_F32) few_rows_kernel<float, WAVES><<<grid, WAVES * 64, 0, stream>>>(p, (const float*)x, ldx, cols);
    else if (p.type == TERN_BF16) few_rows_kernel<__bf16, WAVES><<<grid, WAVES * 64, 0, stream>>>(p, (const __bf16*)x, ldx, cols);
    else few_rows_kernel<_Float16, WAVES><<<grid, WAVES * 64, 0, stream>>>(p, (const _Float16*)x, ldx, cols);
    TERN_HIP_CHECK(hipGetLastError());
    return TERN_OK;
}

}  // namespace

int launch_mx_few_rows(ProductJob p, const void* x, int64_t ldx, int64_t cols, hipStream_t stream)
{
    p.splits = 1;
    return launch_few<8>(p, x, ldx, cols, stream);
}

int launch_mx_product(bool f4, ProductJob* jobs, int n, const ProductPlan* plans, const ColumnSums* columns, hipStream_t stream,
                      const GradOperands* sources)
{
    ProductJobs join = {};
    int64_t grid = 0;
    int joined = 0;
    for (int i = 0; i < n; ++i) {
        ProductJob& p = jobs[i];
        p.splits = plans[i].splits;
        p.split_steps = (int32_t)ceil_div(steps_of(plans[i].form, {p.na, p.nb, p.groups, p.parts}), p.splits);
        if (p.splits > 1) {
            if (joined == 1) join.first = (int32_t)grid;
            join.job[joined++] = p;
            grid += ceil_div((p.na + 3) / 4 * p.nb, 256);
        }
    }
    if (joined < 2) join.first = INT32_MAX;
    if (grid > INT32_MAX / 2) return TERN_ESHAPE;
    for (int i = 0; i < n; ++i)
        if (plans[i].form == kNarrow) {
            const int rc = launch_mx_narrow(jobs[i], *sources, plans[i].wide, stream);
            if (rc != TERN_OK) return rc;
        }
    const int together = n == 2 && plans[0].form == plans[1].form ? 2 : 1;
    for (int i = 0; i < n; i += together) {
        if (plans[i].form == kNarrow) continue;
        const int rc = f4 ? launch_form<true>(plans[i].form, jobs + i, together, columns, stream)
                          : launch_form<false>(plans[i].form, jobs + i, together, columns, stream);
        if (rc != TERN_OK) return rc;
        columns = nullptr;
    }
    if (columns) {
        const int rc = launch_form<false>(kDirect1, nullptr, 0, columns, stream);
        if (rc != TERN_OK) return rc;
    }
    if (joined == 0) return TERN_OK;
    join_kernel<<<dim3((unsigned)grid), 256, 0, stream>>>(join);
    TERN_HIP_CHECK(hipGetLastError());
    return TERN_OK;
}

}  // namespace tern
