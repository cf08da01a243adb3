// Matrix product of 16-bit operands (float16 or bfloat16) on the 5th-generation tensor cores, float32
// accumulation, with the epilogues of the dense layer and of the orthogonalised update:
//
//   D[b][i, j] = epilogue( sum_r A[b][i, r] B[b][j, r] ),   i < m, j < n, b < batch
//
// Either operand may be stored with the reduction index r contiguous ("K-major") or with its own row index
// contiguous ("MN-major"): both are fetched by TMA in 64-element (128-byte) wide boxes with the 128-byte swizzle, and
// the instruction descriptor's major bits do the rest, so W x, W^T dy, dy x^T, X X^T, X^T X and B X all run without a
// transposed copy.
//
// One unit of work is a tile of D (or, with splits > 1, one slice of its reduction). Roles in a CTA:
//  * warp 0: TMA producer over a ring of 64-deep stages (full / empty mbarriers);
//  * warp 1: tcgen05.mma issue; the accumulator is double-buffered in tensor memory, so a tile's epilogue
//    overlaps the next tile's loads and products;
//  * warps 4..11: epilogue. Warp w reads TMEM lanes 32 (w & 3) .. + 31 and every other group of 32 columns, applies
//    the epilogue in float32, rounds once, and leaves through 64- or 128-byte swizzled staging and a TMA store
//    (where the output's rows are not 16-byte aligned, or its columns do not fill units of 16 bytes, which is what a TMA
//    store writes: by rows of 32 elements, a lane each). The accumulator goes back to the MMA warp by a relaxed arrival:
//    only tensor memory is handed over, whose reads are complete (tcgen05.wait::ld) and ordered before the arrival by
//    tcgen05.fence::before_thread_sync, as the next MMAs are after the wait by after_thread_sync; no write to shared or
//    global memory has to become visible with it.
// CG = 2 pairs two CTAs of a cluster on one tile of 2 x 128 rows: each holds its 128 rows of A and half the columns
// of B, and the leader issues the pair's MMAs.
//
// Long float32 sums: the tensor core adds each 16-deep block of products to the float32 accumulator with truncation,
// which drifts by about 4e-6 of the result over 4096 terms and 2.8e-5 where all terms have one sign (7e-9 a term,
// measured). Float32 outputs therefore take the accumulator out every kPromoteKb stages (512 terms) and add it, rounded
// to nearest, to float32 sums in the epilogue warps' registers (PROMOTE). 16-bit outputs take the PROMOTE kernel only where
// the drift of one accumulation would near their own rounding (kLongF16, kLongBf16; 300000 terms of one sign were 2e-3
// off in float16, half a step of which is 4.9e-4). The Newton-Schulz products, whose Gram matrix of 2 x 64 x 8000000 put
// the update 4% off, have instances of their own (LONG) that add every kLongKb stages to float32 sums in the workspace;
// the same code in the instances for ordinary lengths costs those 1%.
//
// Splits: where tiles are few, or where the tiles left over after whole waves are (GArgs::whole), a tile's reduction is
// shared. Each slice's warp leaves its float32 partial tile in the workspace and counts in; the last one adds the
// slices in slice order (one order whatever the timing, so results repeat bit for bit) and runs the epilogue.
//
// GEN = false is the kernel for aligned matrices (16-bit outputs, float32 ones with PROMOTE), without the code that
// turns unaligned rows: less to fetch for short products, whose one pass through the epilogue waits for instructions
// too (512 x 512 x 512: 5.4 against 6.6 us).
//
// Bounds and rates (GB300, measured): 4096 x 4096 x 8192 bfloat16 143 us, 1.91 PFLOP/s, which is the tensor cores' rate
// under load (the library's product takes 137 us); 8192 x 8192 x 4096 280 us, 1.96 PFLOP/s. dW in float32 takes 159
// instead of 149 us for the promoted sums. 256 x 256 tiles by pairs of SMs halve the operand traffic through L2 of 128 x
// 128 tiles, which bounds those at about 1.3 PFLOP/s; products too small for a wave of them take 256 x 128, 128 x 128 or
// 128 x 64 tiles and slices (gemm16_host.cuh). Short reductions are bound by the epilogue: a 128 x 256 share of a tile
// takes 5 us in it (4096 x 9216 from 256 columns, 151 MB of float32: 39 us, 22 at the measured copy rate; added to
// what is there 79, 45).
//
// An epilogue thread has 224 registers. Two of the 256-wide instances with promoted sums do not keep to them: the general
// backward one spills 1.7 KB a thread, the lean forward one 0.3 KB (4096 x 4096 x 8192 takes 168 us with a float32 y, 154
// with a bfloat16 one); all others less than 0.3 KB.
//
// Every wait is bounded: one that runs out sets the CTA's abort flag, the roles drain and meet, and the kernel ends
// with CSRT_DEV_TIMEOUT in the status word.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "tc_common.cuh"

namespace csrt {

constexpr int kGBK = 64;                 // reduction depth of a stage (128 bytes)
constexpr int kGThreads = 384;           // a warpgroup for TMA and MMA, two for the epilogue
constexpr int kGEpiWarps = 8;
constexpr int kPromoteKb = 8;            // stages per tensor-memory accumulation of a float32 output
constexpr int kLongF16 = 512;            // the most of a 16-bit one: 2.3e-4 after 32768 terms of one sign, half of half a step
constexpr int kLongBf16 = 2048;          // 9e-4 after 131072 terms, a quarter of half a step
constexpr int kLongKb = 256;             // and of a Newton-Schulz product: 1.2e-4 after 16384 terms
constexpr float kNsA = 3.4445f, kNsB = -4.7750f, kNsC = 2.0315f;
constexpr float kXScale = 32768.f, kInvXScale = 1.f / 32768.f;   // scale of X and A in float16; B's is half of it
enum { kEpiFwd = 0, kEpiBwd = 1, kEpiNs = 2 };
enum { kNsGram = 0, kNsPoly = 1, kNsApply = 2 };   // the products of a Newton-Schulz step (GArgs::kind)

// Staging bytes of an epilogue warp: 4 KB; kEpiNs has a float32 block and a float16 one, PROMOTE two float32 blocks
// (dW of 4096 x 9216 from 256 columns 45.7 -> 42.4 us; its operands then have one stage less, which costs nothing there).
template <int EPI, bool PROMOTE>
constexpr int stage_out() {
    return EPI == kEpiNs ? 6144 : PROMOTE ? 8192 : 4096;
}


// An epilogue operand or output: row-major m x n, batch matrices `stride` elements apart.
struct GMat {
    void *p;
    int64_t ld, stride;
    int32_t dtype;     // CSRT_DT_*
    int32_t vec;       // rows 16-byte aligned: vector access; outputs: TMA store (columns fill units of 16 bytes too)
    int32_t pad;       // rows may be read up to ld, whatever the matrix's columns
};

struct GArgs {
    int32_t m, n, kb, batch;          // output size, stages of the reduction, matrices
    int32_t tiles_m, tiles_n;
    int32_t units;                    // work units per launch: `whole` tiles, then the others in `splits` slices each
    int32_t whole, splits, kb_split;  // (splits == 1: whole is not used)
    int32_t a_mn, b_mn;               // operand stored MN-major
    int32_t slots;                    // 32-column groups that an epilogue warp can have in staging: 1 or (dense) 2
    int32_t f16;                      // operands and 16-bit epilogue tensors are float16 (else bfloat16)
    // epilogue
    const float *bias;
    const uint16_t *sum_src;          // kEpiBwd: matrix whose row sums the idle warps leave in sum_dst (NULL: none)
    int64_t sum_ld;
    int32_t sum_rows, sum_cols, sum_add;
    float *sum_dst;
    int32_t act;                      // activation (kEpiFwd), or act' of c0 as a factor (kEpiBwd)
    int32_t kind, sym, tall;          // kEpiNs: kNs*, tiles on and above the diagonal only, X has more rows than columns
    float alpha, gamma;               // kEpiNs: scale of the sum, of the result
    const float *diag_in;             // kEpiNs: diagonal of A (kNsPoly) or B (kNsApply), s_pad per matrix
    float *diag_out;                  // kEpiNs: diagonal of A (kNsGram) or B (kNsPoly)
    int32_t s_pad;
    GMat c0, c1;                      // z_below / A / X (float32); residual
    GMat out0, out1;                  // y, dx, dW, A, B, X (float16), o; z, X (float32)
    float *partial;                   // split slices; long sums (LONG): by slice, or by CTA where no tile is split
    int32_t *counters;
    WsHeader *hdr;
};

struct GMaps {
    CUtensorMap a, b, out0, out1;
};

// A launch: one product, or the products of all Newton-Schulz steps of all matrices (kNsSets different ones, see
// ns_set). In the latter the units of all phases form one sequence, phase by phase and matrix by matrix, dealt round to
// the CTAs of a cooperative grid; a unit waits until its own matrix's units of the phase before have finished, so
// matrices drift apart and fill each other's gaps. A CTA takes its units in order and all CTAs are resident, so the
// earliest unfinished unit can always run.
constexpr int kNsSets = 6;
constexpr int kGoRing = 16;   // more than the units that a CTA can have between its producer and its epilogue
template <int EPI>
struct GLaunch {
    static constexpr int kSets = EPI == kEpiNs ? kNsSets : 1;
    GMaps maps[kSets];
    GArgs args[kSets];
    int32_t phases;
    int32_t step_units[3];            // units per matrix of the three products of a step
    uint32_t *done;                   // per matrix: units finished, all phases together, by each CTA; zero at the start
};

// Sets of a Newton-Schulz launch: A of the even and odd steps' X, B, X' of the even and odd steps, the last X'.
__device__ __forceinline__ int ns_set(int phase, int phases) {
    const int step = phase / 3, k = phase - 3 * step;
    return k == 0 ? (step & 1) : k == 1 ? 2 : phase == phases - 1 ? 5 : 3 + (step & 1);
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}

__device__ __forceinline__ uint32_t mapa_u32(uint32_t addr, uint32_t rank) {
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}

__device__ __forceinline__ void cluster_sync_all() {
    asm volatile("barrier.cluster.arrive.aligned;" ::: "memory");
    asm volatile("barrier.cluster.wait.aligned;" ::: "memory");
}

// Bounded wait on an mbarrier phase: gives up after 4e9 cycles (about two seconds), or once the CTA aborts.
__device__ __forceinline__ bool gtry(uint32_t addr, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(done)
        : "r"(addr), "r"(parity)
        : "memory");
    return done != 0;
}
// One look that does not wait (try_wait may hold the warp for microseconds).
__device__ __forceinline__ bool glook(uint32_t addr, uint32_t parity) {
    uint32_t done;
    asm volatile(
        "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n"
        " selp.u32 %0, 1, 0, p;\n}\n"
        : "=r"(done)
        : "r"(addr), "r"(parity)
        : "memory");
    return done != 0;
}
__device__ __forceinline__ bool gwait(uint64_t *bar, uint32_t parity, volatile int *abort_flag) {
    const uint32_t addr = smem_u32(bar);
    long long t0 = 0;
#pragma unroll 1
    for (unsigned i = 1; i < (1u << 30); ++i) {
        if (gtry(addr, parity)) return true;
        if ((i & 255) == 0) {
            if (*abort_flag) return false;
            const long long t = clock64();
            if (t0 == 0) t0 = t;
            else if (t - t0 > 4000000000ll) break;
        }
    }
    *abort_flag = 1;
    return false;
}

// The same by a whole warp, which stays together whatever a lane saw.
__device__ __forceinline__ bool gwait_warp(uint64_t *bar, uint32_t parity, volatile int *abort_flag) {
    return __all_sync(0xffffffffu, gwait(bar, parity, abort_flag));
}

// As gwait_warp, where `seen` is the outcome of an earlier look at the barrier: looking at the next stage's barrier
// before the work of the present one hides the look's latency (about 100 cycles).
__device__ __forceinline__ bool gwait_seen(bool seen, uint64_t *bar, uint32_t parity, volatile int *abort_flag) {
    if (__all_sync(0xffffffffu, seen)) return true;
    return gwait_warp(bar, parity, abort_flag);
}

// Wait of a whole warp until a matrix's count reaches `target`; bounded like gwait.
__device__ __forceinline__ bool units_wait(const uint32_t *arrived, uint32_t target, volatile int *abort_flag) {
    bool ok = false;
    if ((threadIdx.x & 31) == 0) {
        const long long t0 = clock64();
        for (unsigned i = 1; i < (1u << 30); ++i) {
            uint32_t v;
            asm volatile("ld.acquire.gpu.global.u32 %0, [%1];" : "=r"(v) : "l"(arrived) : "memory");
            if (v >= target) {
                ok = true;
                break;
            }
            if (*abort_flag || ((i & 255) == 0 && clock64() - t0 > 4000000000ll)) break;
        }
        if (!ok) *abort_flag = 1;
    }
    ok = __all_sync(0xffffffffu, ok || (threadIdx.x & 31) != 0);
    __syncwarp();
    return ok;
}

// One lane of the (whole) warp, the same one every time.
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n .reg .pred e;\n elect.sync _|e, 0xffffffff;\n selp.u32 %0, 1, 0, e;\n}\n" : "=r"(p));
    return p != 0;
}

template <int CG>
__device__ __forceinline__ void tma_load_3d(void *dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar) {
    if constexpr (CG == 1)
        asm volatile(
            "cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
            ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.3d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
            "[%0], [%1, {%2, %3, %4}], [%5];"
            ::"r"(smem_u32(dst)), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(z), "r"(bar)
            : "memory");
}

__device__ __forceinline__ void tma_store_3d(const CUtensorMap *map, int x, int y, int z, const void *src) {
    asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(x), "r"(y), "r"(z), "r"(smem_u32(src))
                 : "memory");
}

// Shared-memory descriptor with the 128-byte swizzle. K-major: rows of 128 bytes, 8-row groups 1024 bytes apart.
// MN-major: 64 operand rows to a 128-byte line, a line per reduction index, 8-line groups 1024 bytes apart and the
// next 64 operand rows kGBK lines (8192 bytes) further on.
__device__ __forceinline__ uint64_t gdesc(uint32_t addr, bool mn) {
    uint64_t d = 0;
    d |= (uint64_t)((addr & 0x3FFFFu) >> 4);
    d |= (uint64_t)(mn ? (kGBK * 128) >> 4 : 1) << 16;
    d |= (uint64_t)(1024 >> 4) << 32;
    d |= (uint64_t)1 << 46;
    d |= (uint64_t)2 << 61;
    return d;
}

template <int CG>
__device__ __forceinline__ void mma_16(uint32_t d, uint64_t ad, uint64_t bd, uint32_t idesc, uint32_t acc) {
    if constexpr (CG == 1)
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
            "l"(ad), "l"(bd), "r"(idesc), "r"(acc)
            : "memory");
    else
        asm volatile(
            "{\n .reg .pred p;\n setp.ne.b32 p, %4, 0;\n"
            " tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n}\n" ::"r"(d),
            "l"(ad), "l"(bd), "r"(idesc), "r"(acc)
            : "memory");
}

// Arrive on a barrier (of both CTAs of a pair) once the MMAs issued so far are done.
template <int CG>
__device__ __forceinline__ void commit_to(uint64_t *bar) {
    if constexpr (CG == 1)
        mma_commit(bar);
    else
        asm volatile(
            "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
                smem_u32(bar)),
            "h"((uint16_t)3)
            : "memory");
}

// The same for a barrier of this CTA alone.
template <int CG>
__device__ __forceinline__ void commit_own(uint64_t *bar) {
    if constexpr (CG == 1)
        mma_commit(bar);
    else
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar))
                     : "memory");
}

__device__ __forceinline__ void tmem_st_32cols(uint32_t taddr, const float (&f)[32]) {
    uint32_t r[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) r[i] = __float_as_uint(f[i]);
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
        "{%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
        "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(taddr),
        "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
        "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
        "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
        "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

// ---------------------------------------------------------------------------
// Element types and activations
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t pack16(float lo, float hi, bool f16) {
    if (f16) {
        const __half2 h = __floats2half2_rn(lo, hi);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}

__device__ __forceinline__ void pack_all(uint32_t (&w)[16], const float (&v)[32], bool f16) {
    if (f16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = pack16(v[2 * i], v[2 * i + 1], true);
    } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) w[i] = pack16(v[2 * i], v[2 * i + 1], false);
    }
}

__device__ __forceinline__ float2 unpack16(uint32_t u, bool f16) {
    if (f16) return __half22float2(*reinterpret_cast<const __half2 *>(&u));
    return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
}

// 16 bytes through L2 into u where `yes`, u kept otherwise. One predicated instruction: a conditional assignment makes
// the compiler merge the two by a move, which waits for the load.
__device__ __forceinline__ void ld_cg_if(uint4 &u, const void *p, bool yes) {
    asm volatile(
        "{\n .reg .pred p;\n setp.ne.u32 p, %5, 0;\n @p ld.global.cg.v4.u32 {%0,%1,%2,%3}, [%4];\n}\n"
        : "+r"(u.x), "+r"(u.y), "+r"(u.z), "+r"(u.w)
        : "l"(p), "r"((uint32_t)yes));
}

// 16 bytes that are read once: not kept in L1.
__device__ __forceinline__ uint4 ld_stream_u4(const void *p) {
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p));
    return v;
}

__device__ __forceinline__ float load1(const void *p, int64_t i, int dtype) {
    if (dtype == CSRT_DT_F32) return static_cast<const float *>(p)[i];
    if (dtype == CSRT_DT_F16) return __half2float(static_cast<const __half *>(p)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16 *>(p)[i]);
}

__device__ __forceinline__ void store1(void *p, int64_t i, float v, int dtype) {
    if (dtype == CSRT_DT_F32) static_cast<float *>(p)[i] = v;
    else if (dtype == CSRT_DT_F16) static_cast<__half *>(p)[i] = __float2half_rn(v);
    else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}

// act(z) and act'(z) in float32. gelu is the tanh form, 0.5 z (1 + tanh u) = z / (1 + exp(-2u)) with
// u = sqrt(2/pi) (z + 0.044715 z^3); silu is z / (1 + exp(-z)). The fast exponential and quotient are off by a few
// 2^-22 of the sigmoid, far below the 16-bit rounding of the result.
constexpr float kGelu2 = 1.5957691216057308f;     // 2 sqrt(2/pi)
constexpr float kGelu3 = 0.044715f;

__device__ __forceinline__ float act_value(float z, int act) {
    if (act == CSRT_ACT_RELU) return z > 0.f ? z : (z != z ? z : 0.f);
    if (act == CSRT_ACT_GELU) return __fdividef(z, 1.f + __expf(-kGelu2 * (z + kGelu3 * z * z * z)));
    if (act == CSRT_ACT_SILU) return __fdividef(z, 1.f + __expf(-z));
    return z;
}

// gelu' and silu' are 0 or 1 to float32 from |z| = 104 on (exp(-104) is below its smallest step). z is held to 128, so that
// neither z^2 nor z (1 - p) overflows against a zero factor: a float16 z beyond 65504 is kept as an infinity and still has
// a derivative. A NaN stays.
__device__ __forceinline__ float act_deriv(float z, int act) {
    if (act == CSRT_ACT_RELU) return z > 0.f ? 1.f : 0.f;
    // min(|z|, 128) with z's sign: one instruction
    asm("min.NaN.xorsign.abs.f32 %0, %0, 0f43000000;" : "+f"(z));
    if (act == CSRT_ACT_GELU) {
        const float p = __fdividef(1.f, 1.f + __expf(-kGelu2 * (z + kGelu3 * z * z * z)));
        return p + z * p * (1.f - p) * kGelu2 * (1.f + 3.f * kGelu3 * z * z);
    }
    if (act == CSRT_ACT_SILU) {
        const float p = __fdividef(1.f, 1.f + __expf(-z));
        return p * (1.f + z * (1.f - p));
    }
    return 1.f;
}

// 32 consecutive elements of a row of a float32 epilogue operand in the general kernel (0 beyond the
// matrix). `row` is this lane's row, `col` the warp's first column. Aligned float32 rows are read in place. Rows that
// are not 16-byte aligned are read a row at a time, a lane per column, and turned in the warp's staging area `turn`
// (32 x 33 floats do not fit it, so 16 rows at a time).
__device__ __forceinline__ void load32(float (&v)[32], const GMat &c, int b, int row, int col, int m, int n,
                                       float *turn) {
    const int lane = threadIdx.x & 31;
    if (c.vec) {
        const float *p = static_cast<const float *>(c.p) + b * c.stride + (int64_t)row * c.ld + col;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
            if (row < m && 4 * i + 4 <= n - col) {
                f = *reinterpret_cast<const float4 *>(p + 4 * i);
            } else if (row < m) {
                if (col + 4 * i < n) f.x = p[4 * i];
                if (col + 4 * i + 1 < n) f.y = p[4 * i + 1];
                if (col + 4 * i + 2 < n) f.z = p[4 * i + 2];
            }
            v[4 * i] = f.x, v[4 * i + 1] = f.y, v[4 * i + 2] = f.z, v[4 * i + 3] = f.w;
        }
    } else {
        const int row0 = row - lane;
        const float *p = static_cast<const float *>(c.p) + b * c.stride;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            float f[16];
#pragma unroll
            for (int r = 0; r < 16; ++r) {
                const int rr = row0 + part * 16 + r;
                f[r] = rr < m && col + lane < n ? p[(int64_t)rr * c.ld + col + lane] : 0.f;
            }
            __syncwarp();
#pragma unroll
            for (int r = 0; r < 16; ++r) turn[r * 33 + lane] = f[r];
            __syncwarp();
            if ((lane >> 4) == part) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] = turn[(lane & 15) * 33 + i];
            }
            __syncwarp();
        }
    }
}

// Row `row` (of this lane) and columns col .. col + 31 of an output on their way out. Aligned outputs are staged at
// `slot` and leave with emit(): rows of 64 bytes (16-bit) take the 64-byte swizzle, rows of 128 bytes (float32) the
// 128-byte one. Others are turned there and stored at once, a row at a time, a lane per column.
template <bool GEN, bool WIDE>
__device__ __forceinline__ void put32(const float (&v)[32], const GMat &o, uint8_t *slot, int b, int row, int col, int m,
                                      int n) {
    const int lane = threadIdx.x & 31;
    const bool h = o.dtype == CSRT_DT_F16;
    if (!GEN || o.vec) {
        if (GEN ? o.dtype == CSRT_DT_F32 : WIDE) {
            __syncwarp();   // a row of 128 bytes lies over two rows of a 16-bit operand
#pragma unroll
            for (int i = 0; i < 8; ++i)
                *reinterpret_cast<float4 *>(slot + lane * 128 + ((i ^ (lane & 7)) << 4)) =
                    make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
        } else {
            uint32_t w[16];
            pack_all(w, v, h);
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<uint4 *>(slot + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4)) =
                    make_uint4(w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]);
        }
        return;
    }
    const int row0 = row - lane, rows = m - row0;
    const int64_t at = b * o.stride + (int64_t)row0 * o.ld + col + lane;
    if (o.dtype != CSRT_DT_F32) {
        uint32_t *turn = reinterpret_cast<uint32_t *>(slot);   // pairs of columns, 17 words to a row
        uint32_t w[16];
        pack_all(w, v, h);
        __syncwarp();
#pragma unroll
        for (int i = 0; i < 16; ++i) turn[lane * 17 + i] = w[i];
        __syncwarp();
        if (col + lane < n) {
            uint16_t *p = static_cast<uint16_t *>(o.p) + at;
            const uint16_t *t = reinterpret_cast<const uint16_t *>(slot) + lane;
#pragma unroll
            for (int r = 0; r < 32; ++r)
                if (r < rows) p[(int64_t)r * o.ld] = t[r * 34];
        }
    } else {
        float *turn = reinterpret_cast<float *>(slot);
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            __syncwarp();
            if ((lane >> 4) == part) {
#pragma unroll
                for (int i = 0; i < 32; ++i) turn[(lane & 15) * 33 + i] = v[i];
            }
            __syncwarp();
            if (col + lane < n) {
                float *p = static_cast<float *>(o.p) + at + part * 16 * o.ld;
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (part * 16 + r < rows) p[(int64_t)r * o.ld] = turn[r * 33 + lane];
            }
        }
    }
    __syncwarp();
}

// The 32 x 32 block turned about the diagonal, in the layout of put32 (float16).
__device__ __forceinline__ void put32_turned(const float (&v)[32], uint8_t *at) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 32; ++i)
        *reinterpret_cast<__half *>(at + i * 64 + (((lane >> 3) ^ ((i >> 1) & 3)) << 4) + (lane & 7) * 2) = __float2half_rn(v[i]);
}

// The staged outputs leave: out0 from at0, out1 - or the mirrored block of out0 - from at1.
template <bool GEN>
__device__ __forceinline__ void emit(const GArgs &a, const GMaps &maps, const uint8_t *at0, const uint8_t *at1, int b, int row,
                                     int col, bool mirror) {
    if (!GEN || a.out0.vec) {   // out1 likewise, if there is one
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        __syncwarp();
        if ((threadIdx.x & 31) == 0 && row < a.m && col < a.n) {   // lane 0's row is the block's first
            tma_store_3d(&maps.out0, col, row, b, at0);
            if (a.out1.p != nullptr) tma_store_3d(&maps.out1, col, row, b, at1);
            if (mirror) tma_store_3d(&maps.out0, row, col, b, at1);
        }
    }
}

// Sum of a 16-byte aligned row of 16-bit elements by a warp: four 16-byte loads a lane in flight, float32, lanes joined at the end.
template <bool F16>
__device__ __forceinline__ float warp_row_sum(const uint16_t *p, int cols) {
    const int lane = threadIdx.x & 31;
    float s0 = 0.f, s1 = 0.f, s2 = 0.f, s3 = 0.f;
    const uint32_t n = (uint32_t)cols, c = n & ~7u;   // unsigned: t may pass 2^31 on its last step
#pragma unroll 4
    for (uint32_t t = lane * 8; t < c; t += 256) {
        const uint4 u = __ldg(reinterpret_cast<const uint4 *>(p + t));
        const float2 x = unpack16(u.x, F16), y = unpack16(u.y, F16), z = unpack16(u.z, F16), w = unpack16(u.w, F16);
        s0 += x.x + x.y, s1 += y.x + y.y, s2 += z.x + z.y, s3 += w.x + w.y;
    }
    if (c + lane < n) s0 += load1(p, c + lane, F16 ? CSRT_DT_F16 : CSRT_DT_BF16);
    float s = (s0 + s1) + (s2 + s3);
#pragma unroll
    for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
    return s;
}

// ---------------------------------------------------------------------------
// Work units
// ---------------------------------------------------------------------------
struct GUnit {
    int b, tm, tn, kb0, kb1;
    int splits, split, tile;   // slices of its tile, its own one, and the tile's number among the split ones
};

// Unit u: batch matrix, tile and slice. Tiles run down bands of eight tile rows, so that the units in flight share
// operand tiles in L2. A symmetric product has the tiles that reach above the diagonal only: tile row i starts at
// tile column R i, R tile columns to a tile row.
template <int R>
__device__ __forceinline__ GUnit unit_of(const GArgs &a, int u) {
    GUnit r;
    const int tiles = a.sym ? a.tiles_m * a.tiles_n - R * (a.tiles_m * (a.tiles_m - 1) / 2) : a.tiles_m * a.tiles_n;
    int t = u;
    r.splits = 1;
    r.split = r.tile = 0;
    if (a.splits > 1 && u >= a.whole) {
        r.splits = a.splits;
        r.tile = (u - a.whole) / a.splits;
        r.split = u - a.whole - r.tile * a.splits;
        t = a.whole + r.tile;
    }
    r.b = a.batch > 1 ? t / tiles : 0;
    int q = t - r.b * tiles;
    if (a.sym) {
        int i = 0;
        while (q >= a.tiles_n - R * i) q -= a.tiles_n - R * i++;
        r.tm = i;
        r.tn = R * i + q;
    } else {
        constexpr int kBand = 8;
        const int band = a.tiles_m > kBand ? q / (kBand * a.tiles_n) : 0, first = band * kBand;
        const int rows = min(kBand, a.tiles_m - first);
        q -= first * a.tiles_n;
        r.tn = rows == kBand ? q / kBand : q / rows;
        r.tm = first + q - r.tn * rows;
    }
    r.kb0 = r.splits > 1 ? r.split * a.kb_split : 0;
    r.kb1 = r.splits > 1 ? min(a.kb, r.kb0 + a.kb_split) : a.kb;
    return r;
}

// The warp's 32 x 32 elements of a 16-bit epilogue operand, fetched ahead of their use: a load instruction
// takes eight whole rows of 64 bytes, four lanes to a row. Through L2 only: another SM may have written them earlier
// in this launch.
template <bool GEN, bool WIDE>
__device__ __forceinline__ bool ahead_ok(const GMat &c) {
    return c.p != nullptr && (GEN ? c.dtype != CSRT_DT_F32 : !WIDE);
}
// A unit's view of such an operand in the lean kernel, whose columns are a multiple of eight or padded to one.
struct GAhead {
    const char *p;     // this lane's place in the unit's first row and column (NULL: no operand)
    int64_t step;      // bytes to the lane's next row, eight further on
    int32_t lim;       // columns readable from the unit's first one
    uint32_t rows;     // bit i: row 8 i + lane / 4 exists
};
template <bool WIDE>
__device__ __forceinline__ GAhead ahead_of(const GMat &c, int b, int row0, int col0, int m, int n) {
    const int lane = threadIdx.x & 31, r = lane >> 2;
    GAhead g = {nullptr, 0, 0, 0};
    if (!ahead_ok<false, WIDE>(c)) return g;
    g.p = reinterpret_cast<const char *>(static_cast<const uint16_t *>(c.p) + b * c.stride + (int64_t)(row0 + r) * c.ld +
                                         col0 + 8 * (lane & 3));
    g.step = 16 * c.ld;
    g.lim = (c.pad ? (int)c.ld : n) - col0 - 8 * (lane & 3);
#pragma unroll
    for (int i = 0; i < 4; ++i) g.rows |= (row0 + r + 8 * i < m ? 1u : 0u) << i;
    return g;
}
// The same for an aligned float32 operand with `cols` readable columns, a multiple of four: eight lanes to a row of 128
// bytes, four rows to an instruction.
__device__ __forceinline__ GAhead ahead_of_f32(const GMat &c, int b, int row0, int col0, int m, int cols) {
    const int lane = threadIdx.x & 31, r = lane >> 3;
    GAhead g;
    g.p = reinterpret_cast<const char *>(static_cast<const float *>(c.p) + b * c.stride + (int64_t)(row0 + r) * c.ld + col0 +
                                         4 * (lane & 7));
    g.step = 16 * c.ld;
    g.lim = cols - col0 - 4 * (lane & 7);
    g.rows = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) g.rows |= (row0 + r + 4 * i < m ? 1u : 0u) << i;
    return g;
}
__device__ __forceinline__ void fetch_ahead_f32(uint4 (&u0)[4], uint4 (&u1)[4], const GAhead &g, int off) {
    const char *p = g.p + 4 * off;
    const uint32_t rows = off < g.lim ? g.rows : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) ld_cg_if(u0[i], p + i * g.step, (rows >> i) & 1);
#pragma unroll
    for (int i = 0; i < 4; ++i) ld_cg_if(u1[i], p + (i + 4) * g.step, (rows >> (i + 4)) & 1);
}
__device__ __forceinline__ void fetch_ahead(uint4 (&u)[4], const GAhead &g, int off) {
    if (g.p == nullptr) return;
    const char *p = g.p + 2 * off;
    const uint32_t rows = off < g.lim ? g.rows : 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) ld_cg_if(u[i], p + i * g.step, (rows >> i) & 1);
}

// Such a block through 4 KB of staging: this lane's row of it.
__device__ __forceinline__ void take32_f32(float (&v)[32], const uint4 (&u0)[4], const uint4 (&u1)[4], uint8_t *slot) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = 4 * i + (lane >> 3);
        *reinterpret_cast<uint4 *>(slot + r * 128 + (((lane & 7) ^ (r & 7)) << 4)) = i < 4 ? u0[i & 3] : u1[i & 3];
    }
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float4 f = *reinterpret_cast<const float4 *>(slot + lane * 128 + ((i ^ (lane & 7)) << 4));
        v[4 * i] = f.x, v[4 * i + 1] = f.y, v[4 * i + 2] = f.z, v[4 * i + 3] = f.w;
    }
}

// The eight 16-bit elements that start `off` bytes into the 32 of lo and hi.
__device__ __forceinline__ uint4 eight_at(const uint4 &lo, const uint4 &hi, uint32_t off) {
    uint32_t w[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
#pragma unroll
    for (int i = 0; i < 6; ++i) w[i] = off & 8 ? w[i + 2] : w[i];
#pragma unroll
    for (int i = 0; i < 5; ++i) w[i] = off & 4 ? w[i + 1] : w[i];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (off & 2) * 8);
    return make_uint4(w[0], w[1], w[2], w[3]);
}
// Up to eight elements from p on, one at a time.
__device__ __forceinline__ uint4 eight_singly(const uint16_t *p, int count) {
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 8; ++e)
        if (e < count) w[e >> 1] |= (uint32_t)p[e] << (16 * (e & 1));
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// The general kernel's fetch, rows at any alignment: the one or two aligned 16-byte words that hold a lane's eight
// elements, as long as they lie within the matrix (between its first and its last element; only its two ends may not),
// and the eight cut out of them. Reading them a row at a time, a lane per column, took
// dx of 4096 x 1777 from 1000 rows 68 us with z at odd rows, 43 this way
// on the same tiles (37 on those that it takes now).
template <bool GEN, bool WIDE>
__device__ __forceinline__ void fetch_ahead(uint4 (&u)[4], const GMat &c, int b, int row0, int col, int m, int n) {
    if (!ahead_ok<GEN, WIDE>(c)) return;
    const int lane = threadIdx.x & 31, r = row0 + (lane >> 2), c8 = col + 8 * (lane & 3), count = n - c8;
    const uint16_t *base = static_cast<const uint16_t *>(c.p) + b * c.stride;
    const uint16_t *p = base + (int64_t)r * c.ld + c8;
    if (c.vec && count >= 8) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
            if (r + 8 * i < m) u[i] = __ldcg(reinterpret_cast<const uint4 *>(p + (int64_t)(8 * i) * c.ld));
        return;
    }
    const uintptr_t first = reinterpret_cast<uintptr_t>(base);
    const uintptr_t end = reinterpret_cast<uintptr_t>(base + (int64_t)(m - 1) * c.ld + n);
    uint4 lo[4] = {}, hi[4] = {};
    uint32_t singly = 0;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uintptr_t at = reinterpret_cast<uintptr_t>(p + (int64_t)(8 * i) * c.ld), word = at & ~(uintptr_t)15;
        const bool there = r + 8 * i < m && count > 0, two = (at & 15) + 2 * imin(count, 8) > 16;
        const bool inside = word >= first && word + (two ? 32 : 16) <= end;
        ld_cg_if(lo[i], reinterpret_cast<const void *>(word), there && inside);
        ld_cg_if(hi[i], reinterpret_cast<const void *>(word + 16), there && inside && two);
        singly |= (there && !inside ? 1u : 0u) << i;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        u[i] = eight_at(lo[i], hi[i], (uint32_t)(reinterpret_cast<uintptr_t>(p + (int64_t)(8 * i) * c.ld) & 15));
        if (singly >> i & 1) u[i] = eight_singly(p + (int64_t)(8 * i) * c.ld, count);
    }
}
// This lane's row of it: stage_in() puts what the lanes fetched into 2 KB of staging, and after a __syncwarp() take32()
// reads the row; a lane may then write its own row's place. Operands that are not fetched ahead are read by take32().
template <bool GEN, bool WIDE>
__device__ __forceinline__ void stage_in(const uint4 (&u)[4], const GMat &c, uint8_t *at) {
    if (!ahead_ok<GEN, WIDE>(c)) return;
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = 8 * i + (lane >> 2);
        *reinterpret_cast<uint4 *>(at + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4)) = u[i];
    }
}
template <bool GEN, bool WIDE>
__device__ __forceinline__ void take32(float (&v)[32], const GMat &c, int b, int row, int col, int m, int n, uint8_t *at,
                                       float *turn) {
    const int lane = threadIdx.x & 31;
    if (!GEN || ahead_ok<GEN, WIDE>(c)) {
        uint32_t w[16];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint4 q = *reinterpret_cast<const uint4 *>(at + lane * 64 + ((i ^ ((lane >> 1) & 3)) << 4));
            w[4 * i] = q.x, w[4 * i + 1] = q.y, w[4 * i + 2] = q.z, w[4 * i + 3] = q.w;
        }
        if (c.dtype == CSRT_DT_F16) {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 f = unpack16(w[i], true);
                v[2 * i] = f.x, v[2 * i + 1] = f.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float2 f = unpack16(w[i], false);
                v[2 * i] = f.x, v[2 * i + 1] = f.y;
            }
        }
    } else {
        load32(v, c, b, row, col, m, n, turn);
    }
}
// The diagonal at this lane's row (once per unit) and at column col + lane.
__device__ __forceinline__ float diag_ahead(const GArgs &a, int b, int at, int limit) {
    float v = 0.f;   // one predicated load, see ld_cg_if
    asm volatile("{\n .reg .pred p;\n setp.ne.u32 p, %2, 0;\n @p ld.global.cg.f32 %0, [%1];\n}\n"
                 : "+f"(v)
                 : "l"(a.diag_in + (int64_t)b * a.s_pad + at), "r"((uint32_t)(a.diag_in != nullptr && at < limit)));
    return v;
}

// The epilogue of 32 columns of a row in float32, in one slot of staging (4 KB, or 2 KB where one operand and one
// 16-bit output are all): c0 and c1 come in at its halves, out0 and out1 leave from there. u0, u1: c0 and c1 fetched ahead; di, dj: the diagonal (GArgs::diag_in) at this lane's row
// and at column col + lane. An operand that has to be turned (unaligned) uses the slot after the fetched ones are out
// of it; so do unaligned outputs.
template <int EPI, bool GEN, bool WIDE>
__device__ __forceinline__ void epilogue32(float (&v)[32], const uint4 (&u0)[4], const uint4 (&u1)[4], float di, float dj,
                                           const GArgs &a, const GMaps &maps, uint8_t *slot, int b, int row, int col,
                                           bool mirror) {
    float *turn = reinterpret_cast<float *>(slot);
    const int lane = threadIdx.x & 31;
    if constexpr (EPI == kEpiFwd) {
        float r[32];
        if (a.c1.p != nullptr) {
            if constexpr (!GEN && WIDE) {
                take32_f32(r, u0, u1, slot);
            } else {
                stage_in<GEN, WIDE>(u1, a.c1, slot);
                __syncwarp();
                take32<GEN, WIDE>(r, a.c1, b, row, col, a.m, a.n, slot, turn);
            }
        }
        if (a.bias != nullptr) {
            const float bi = row < a.m ? __ldg(a.bias + row) : 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += bi;
        }
        // z and y are both aligned or both not (seen to on the host)
        if (a.out1.p != nullptr) put32<GEN, false>(v, a.out1, !GEN || a.out1.vec ? slot + 2048 : slot, b, row, col, a.m, a.n);
        if (a.act == CSRT_ACT_RELU) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = act_value(v[i], CSRT_ACT_RELU);
        } else if (a.act == CSRT_ACT_GELU) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = act_value(v[i], CSRT_ACT_GELU);
        } else if (a.act == CSRT_ACT_SILU) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = act_value(v[i], CSRT_ACT_SILU);
        }
        if (a.c1.p != nullptr) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += r[i];
        }
    } else if constexpr (EPI == kEpiBwd) {
        uint8_t *at1 = a.c0.p != nullptr ? slot + 2048 : slot;
        float r[32];
        if (GEN || !WIDE || a.c0.p != nullptr) {
            stage_in<GEN, false>(u0, a.c0, slot);
            stage_in<GEN, WIDE>(u1, a.c1, at1);
            __syncwarp();
        }
        // both leave the slot before either is turned in it
        if (a.c1.p != nullptr && ahead_ok<GEN, WIDE>(a.c1)) take32<GEN, WIDE>(r, a.c1, b, row, col, a.m, a.n, at1, turn);
        if (a.c0.p != nullptr) {
            float z[32];
            take32<GEN, false>(z, a.c0, b, row, col, a.m, a.n, slot, turn);
            if (a.act == CSRT_ACT_RELU) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] *= act_deriv(z[i], CSRT_ACT_RELU);
            } else if (a.act == CSRT_ACT_GELU) {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] *= act_deriv(z[i], CSRT_ACT_GELU);
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) v[i] *= act_deriv(z[i], CSRT_ACT_SILU);
            }
        }
        if (a.c1.p != nullptr) {
            if constexpr (!GEN && WIDE) {
                if (a.c0.p == nullptr) {
                    take32_f32(r, u0, u1, slot);
                } else {   // z had the place of what is fetched ahead
                    uint4 t0[4] = {}, t1[4] = {};
                    fetch_ahead_f32(t0, t1, ahead_of_f32(a.c1, b, row - lane, col, a.m, a.n), 0);
                    __syncwarp();
                    take32_f32(r, t0, t1, slot);
                }
            } else if (!ahead_ok<GEN, WIDE>(a.c1)) {
                __syncwarp();
                take32<GEN, WIDE>(r, a.c1, b, row, col, a.m, a.n, slot, turn);
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] += r[i];
        }
    } else if (a.kind != kNsApply) {
        // A or B: the diagonal goes to its own float32 vector and is left out of the float16 matrix. Warps' rows and
        // columns start at multiples of 32, so a diagonal element of this group, if any, is element `lane`.
        const bool on_diag = row - lane == col;
        float d = 0.f;
        if (a.kind == kNsGram) {
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] *= a.alpha;
            if (on_diag) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i == lane) d = v[i], v[i] = 0.f;
                d *= kInvXScale;
            }
        } else {
            // off the diagonal b R + c ((d_i + d_j) R + (R R)_ij), on it b d_i + c (d_i^2 + (R R)_ii)
            float r[32];
            stage_in<GEN, false>(u0, a.c0, slot);
            __syncwarp();
            take32<GEN, false>(r, a.c0, b, row, col, a.m, a.n, slot, turn);
#pragma unroll
            for (int i = 0; i < 32; ++i)
                v[i] = a.alpha * v[i] + 0.5f * (kNsB + kNsC * (di + __shfl_sync(0xffffffffu, dj, i))) * r[i];
            if (on_diag) {
#pragma unroll
                for (int i = 0; i < 32; ++i)
                    if (i == lane) d = v[i], v[i] = 0.f;
                d = kNsB * di + kNsC * di * di + d * (2.f * kInvXScale);
            }
        }
        if (on_diag && row < a.m) a.diag_out[(int64_t)b * a.s_pad + row] = d;
    } else {
        // (a + e) X + B X with the diagonal e of B by row (or by column where X has more rows than columns). X is
        // float32: it comes in at the slot's first 4 KB and leaves from there, the float16 operand of the next products
        // (or o) from the 2 KB behind.
        float c[32];
        take32_f32(c, u0, u1, slot);
        if (a.tall) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                v[i] = (a.alpha * v[i] + (kNsA + __shfl_sync(0xffffffffu, dj, i)) * c[i]) * a.gamma;
        } else {
            const float e = kNsA + di;
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = (a.alpha * v[i] + e * c[i]) * a.gamma;
        }
        if (a.out1.p != nullptr) put32<false, true>(v, a.out1, slot, b, row, col, a.m, a.n);
        put32<false, false>(v, a.out0, slot + 4096, b, row, col, a.m, a.n);
        emit<false>(a, maps, slot + 4096, slot, b, row, col, false);
        return;
    }
    put32<GEN, WIDE>(v, a.out0, slot, b, row, col, a.m, a.n);
    if (EPI == kEpiNs && mirror) put32_turned(v, slot + 2048);
    emit<GEN>(a, maps, slot, slot + 2048, b, row, col, EPI == kEpiNs && mirror);
}

// Units per matrix of the phases before `phase`, and this CTA's first unit of it.
__device__ __forceinline__ uint32_t units_before(const int32_t (&n)[3], int phase) {
    const int step = phase / 3, k = phase - 3 * step;
    return (uint32_t)(step * (n[0] + n[1] + n[2]) + (k > 0 ? n[0] : 0) + (k > 1 ? n[1] : 0));
}
template <int EPI>
__device__ __forceinline__ int first_unit(const GLaunch<EPI> &L, int phase, int batch, int unit0, int ustep) {
    if (EPI != kEpiNs || phase == 0) return unit0;
    const int r = (int)((uint64_t)units_before(L.step_units, phase) * (uint32_t)batch % (uint32_t)ustep);
    return unit0 >= r ? unit0 - r : unit0 - r + ustep;
}

template <int CG, int BN>
constexpr int gstage_bytes() {
    return 128 * 128 + (BN / CG) * 128;
}
template <int CG, int BN, int EPI, bool PROMOTE>
constexpr int gstages() {
    return (227 * 1024 - kGEpiWarps * stage_out<EPI, PROMOTE>() - 2048) / gstage_bytes<CG, BN>();
}
template <int CG, int BN, int EPI, bool PROMOTE>
constexpr int gsmem_bytes() {
    return gstages<CG, BN, EPI, PROMOTE>() * gstage_bytes<CG, BN>() + kGEpiWarps * stage_out<EPI, PROMOTE>() + 1024 + 512;
}

template <int CG, int BN, int EPI, bool PROMOTE, bool GEN, bool LONG>
__global__ void __cluster_dims__(CG, 1, 1) __launch_bounds__(kGThreads, 1)
    gemm16_kernel(const __grid_constant__ GLaunch<EPI> L) {
    static_assert(BN % 64 == 0 && BN / CG >= 64 && 2 * BN <= 512, "two accumulators in tensor memory");
    constexpr bool NS = EPI == kEpiNs;
    constexpr int R = 128 * CG / BN;                      // tile columns to a tile row (symmetric products)
    constexpr int kStages = gstages<CG, BN, EPI, PROMOTE>();
    constexpr int kStageBytes = gstage_bytes<CG, BN>();
    constexpr int kABytes = 128 * 128;
    constexpr int kBRows = BN / CG;                       // columns of D whose B rows this CTA holds
    constexpr int kChunks = BN / 32;
    constexpr uint32_t kCols = 2 * BN;
    constexpr int kAccKb = PROMOTE ? kPromoteKb : kLongKb;
    extern __shared__ uint8_t smem_raw[];
    uint8_t *smem = reinterpret_cast<uint8_t *>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    uint8_t *epi = smem + kStages * kStageBytes;
    uint64_t *full = reinterpret_cast<uint64_t *>(epi + kGEpiWarps * stage_out<EPI, PROMOTE>());
    uint64_t *empty = full + kStages;
    uint64_t *accf = empty + kStages;    // [2] accumulator ready
    uint64_t *acce = accf + 2;           // [2] accumulator drained
    uint64_t *fin = acce + 2;            // all MMAs complete
    uint64_t *go = fin + 1;              // [kGoRing] a unit's inputs are in place (kEpiNs)
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(go + kGoRing);
    __shared__ volatile int s_abort;
    __shared__ int s_done[kGoRing];      // epilogue warps through with a unit (kEpiNs)

    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = CG == 2 ? cluster_rank() : 0;
    const int unit0 = blockIdx.x / CG, ustep = gridDim.x / CG;

    if (threadIdx.x == 0) {
        s_abort = 0;
        for (int i = 0; i < kGoRing; ++i) s_done[i] = 0;
        for (int s = 0; s < kStages; ++s) {
            mbar_init(full + s, 1);
            mbar_init(empty + s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(accf + i, 1);
            mbar_init(acce + i, CG * kGEpiWarps);
        }
        mbar_init(fin, 1);
        for (int i = 0; i < kGoRing; ++i) mbar_init(go + i, 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&L.maps[0].a)) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&L.maps[0].b)) : "memory");
    }
    if (warp == 1) {
        if constexpr (CG == 1) {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                         "r"(kCols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                         "r"(kCols)
                         : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        }
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();   // the peer's barriers are initialised
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *tmem_slot;
    pdl_enter();

    // The epilogue (32 columns with two operands, or the sums of PROMOTE) takes the registers that the first warpgroup
    // does not need: 128 x 56 + 256 x 224 = 384 x 168, the launch's own total.
    if (warp == 0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        int s = 0, issued = 0;
        uint32_t ph = 1;
        bool seen = true;   // the ring starts empty
        int n_go = 0;
        for (int phase = 0; phase < L.phases && !s_abort; ++phase) {
        const GArgs &a = L.args[NS ? ns_set(phase, L.phases) : 0];
        const GMaps &maps = L.maps[NS ? ns_set(phase, L.phases) : 0];
        if constexpr (NS)
            if (elect_one()) {
                asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&maps.a)) : "memory");
                asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(&maps.b)) : "memory");
            }
        int known = -1;   // matrix whose inputs of this phase are known to be there
        for (int u = first_unit(L, phase, a.batch, unit0, ustep); u < a.units && !s_abort; u += ustep) {
            const GUnit w = unit_of<R>(a, u);
            if (NS) {
                if (phase > 0 && w.b != known) {
                    if (!units_wait(L.done + w.b, units_before(L.step_units, phase) * CG, &s_abort)) break;
                    known = w.b;
                }
                if (lane == 0)
                    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_u32(go + n_go % kGoRing)) : "memory");
                ++n_go;
                // the loads below go through the async proxy and follow what the wait ordered
                if (phase > 0) asm volatile("fence.proxy.async.global;" ::: "memory");
            }
            const int m0 = (w.tm * CG + (int)rank) * 128, n0 = w.tn * BN + (int)rank * kBRows;
            for (int kb = w.kb0; kb < w.kb1; ++kb) {
                if (!gwait_seen(seen, empty + s, ph, &s_abort)) break;
                const int s1 = s + 1 == kStages ? 0 : s + 1;
                seen = glook(smem_u32(empty + s1), s1 == 0 ? ph ^ 1 : ph);
                uint8_t *sa = smem + s * kStageBytes, *sb = sa + kABytes;
                uint32_t bar = smem_u32(full + s);
                if constexpr (CG == 2) bar = mapa_u32(bar, 0);
                if (elect_one()) {
                    if (rank == 0) mbar_expect_tx(full + s, CG * kStageBytes);
                    if (a.a_mn) {
#pragma unroll
                        for (int i = 0; i < 2; ++i)
                            tma_load_3d<CG>(sa + i * 8192, &maps.a, m0 + i * 64, kb * kGBK, w.b, bar);
                    } else {
                        tma_load_3d<CG>(sa, &maps.a, kb * kGBK, m0, w.b, bar);
                    }
                    if (a.b_mn) {
#pragma unroll
                        for (int i = 0; i < kBRows / 64; ++i)
                            tma_load_3d<CG>(sb + i * 8192, &maps.b, n0 + i * 64, kb * kGBK, w.b, bar);
                    } else {
                        tma_load_3d<CG>(sb, &maps.b, kb * kGBK, n0, w.b, bar);
                    }
                }
                issued = imin(issued + 1, kStages);
                if (++s == kStages) s = 0, ph ^= 1;
            }
        }
        }
        // an aborted CTA's loads in flight must land before it may exit (rank 0's barriers count the pair's bytes)
        if (s_abort && rank == 0 && lane == 0)
            for (int i = 0; i < issued; ++i) {
                if (--s < 0) s = kStages - 1, ph ^= 1;
                mbar_wait(full + s, ph ^ 1);
            }
    } else if (warp == 1) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (rank == 0) {
            // The whole warp walks the stages and one lane issues: descriptors and addresses stay uniform, which
            // keeps the issue of a stage's four MMAs short (a lone lane took about 290 cycles for them, more than a
            // 128-column tile's MMAs themselves).
            int s = 0, j = 0;
            uint32_t ph = 0;
            bool seen = false;
            for (int phase = 0; phase < L.phases && !s_abort; ++phase) {
            const GArgs &a = L.args[NS ? ns_set(phase, L.phases) : 0];
            const uint32_t idesc = (1u << 4) | ((a.f16 ? 0u : 1u) << 7) | ((a.f16 ? 0u : 1u) << 10) |
                                   ((uint32_t)a.a_mn << 15) | ((uint32_t)a.b_mn << 16) | ((uint32_t)(BN >> 3) << 17) |
                                   ((uint32_t)((128 * CG) >> 4) << 24);
            const uint32_t a_step = (a.a_mn ? 2048 : 32) >> 4, b_step = (a.b_mn ? 2048 : 32) >> 4;
            const uint64_t a0 = gdesc(smem_u32(smem), a.a_mn), b0 = gdesc(smem_u32(smem) + kABytes, a.b_mn);
            for (int u = first_unit(L, phase, a.batch, unit0, ustep); u < a.units && !s_abort; u += ustep) {
                const GUnit w = unit_of<R>(a, u);
                int kb = w.kb0;
                do {   // one accumulation: the whole unit, or kAccKb stages of it
                    const int stop = PROMOTE || LONG ? min(w.kb1, kb + kAccKb) : w.kb1;
                    const int acc = j & 1;
                    if (!gwait_warp(acce + acc, ((j >> 1) & 1) ^ 1, &s_abort)) break;
                    ++j;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint32_t d = tmem + (uint32_t)(acc * BN);
                    uint32_t more = 0;   // the first product overwrites the accumulator
                    for (; kb < stop; ++kb) {
                        if (!gwait_seen(seen, full + s, ph, &s_abort)) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        const int s1 = s + 1 == kStages ? 0 : s + 1;
                        seen = glook(smem_u32(full + s1), s1 == 0 ? ph ^ 1 : ph);
                        const uint64_t ad = a0 + (uint32_t)(s * (kStageBytes >> 4)), bd = b0 + (uint32_t)(s * (kStageBytes >> 4));
                        if (elect_one()) {
                            mma_16<CG>(d, ad, bd, idesc, more);
#pragma unroll
                            for (uint32_t k = 1; k < kGBK / 16; ++k)
                                mma_16<CG>(d, ad + k * a_step, bd + k * b_step, idesc, 1);
                            commit_to<CG>(empty + s);
                        }
                        more = 1;
                        if (++s == kStages) s = 0, ph ^= 1;
                    }
                    if (elect_one()) commit_to<CG>(accf + acc);
                } while (kb < w.kb1 && !s_abort);
                __syncwarp();
            }
            }
            __syncwarp();
            if (elect_one()) commit_own<CG>(fin);
            mbar_wait(fin, 0);   // nothing of ours still runs on the tensor cores
            __syncwarp();
        }
    } else if (warp < 4) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if constexpr (EPI == kEpiBwd) {   // the bias gradient beside the product: two rows of dy at a time
            const GArgs &a = L.args[0];
            if (a.sum_dst != nullptr)
                for (uint32_t r = blockIdx.x * 2 + warp - 2; r < (uint32_t)a.sum_rows; r += gridDim.x * 2) {
                    const uint16_t *p = a.sum_src + (int64_t)r * a.sum_ld;
                    const float t = a.f16 ? warp_row_sum<true>(p, a.sum_cols) : warp_row_sum<false>(p, a.sum_cols);
                    if (lane == 0) a.sum_dst[r] = a.sum_add ? a.sum_dst[r] + t : t;
                }
        }
    } else {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        const int q = warp & 3, half = (warp - 4) >> 2;
        uint8_t *stage0 = epi + (warp - 4) * stage_out<EPI, PROMOTE>();
        uint32_t acce_bar[2] = {smem_u32(acce), smem_u32(acce + 1)};
        if constexpr (CG == 2) {
            acce_bar[0] = mapa_u32(acce_bar[0], 0);
            acce_bar[1] = mapa_u32(acce_bar[1], 0);
        }
        int j = 0;
        int n_go = 0;
        GUnit ahead = {};
        uint4 u0[4] = {}, u1[4] = {};
        float di = 0.f, dj = 0.f;
        for (int phase = 0; phase < L.phases; ++phase) {
        // the next phase may use the staging in other portions
        if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
        int slot = 0;
        const GArgs &a = L.args[NS ? ns_set(phase, L.phases) : 0];
        const GMaps &maps = L.maps[NS ? ns_set(phase, L.phases) : 0];
        for (int u = first_unit(L, phase, a.batch, unit0, ustep); u < a.units; u += ustep) {
            if (NS) {
                if (!gwait_warp(go + n_go % kGoRing, (n_go / kGoRing) & 1, &s_abort)) break;
                ++n_go;
            }
            // float32 results, whose units are bound by this warp: decoded while the unit before was on its way out (the
            // divisions take 500 cycles)
            const GUnit w = !PROMOTE || u == unit0 ? unit_of<R>(a, u) : ahead;
            const int row = (w.tm * CG + (int)rank) * 128 + q * 32 + lane, n0 = w.tn * BN;
            const bool empty_sum = w.kb1 <= w.kb0;
            GAhead g0 = {}, g1 = {};
            const bool in32 = !GEN && PROMOTE && a.c1.p != nullptr && a.c0.p == nullptr;   // its place is u0 and u1
            if constexpr (!GEN) {
                if (NS && a.kind == kNsApply) {
                    g0 = ahead_of_f32(a.c0, w.b, row - lane, n0, a.m, (int)imin<int64_t>(a.c0.ld, INT32_MAX));
                } else if (in32) {
                    g0 = ahead_of_f32(a.c1, w.b, row - lane, n0, a.m, a.n);
                } else {
                    g0 = ahead_of<false>(a.c0, w.b, row - lane, n0, a.m, a.n);
                    g1 = ahead_of<PROMOTE>(a.c1, w.b, row - lane, n0, a.m, a.n);
                }
            }
            const bool by_col = NS && (a.kind == kNsPoly || a.tall);
            auto fetch = [&](int ci) {   // the operands of the 32 columns n0 + 32 ci ..
                if constexpr (GEN) {
                    fetch_ahead<GEN, false>(u0, a.c0, w.b, row - lane, n0 + ci * 32, a.m, a.n);
                    fetch_ahead<GEN, PROMOTE>(u1, a.c1, w.b, row - lane, n0 + ci * 32, a.m, a.n);
                } else if ((NS && a.kind == kNsApply) || in32) {
                    fetch_ahead_f32(u0, u1, g0, ci * 32);
                } else {
                    fetch_ahead(u0, g0, ci * 32);
                    if (!NS) fetch_ahead(u1, g1, ci * 32);
                }
                if (by_col) dj = diag_ahead(a, w.b, n0 + ci * 32 + lane, imin(a.n, a.s_pad));
            };
            if (NS) di = diag_ahead(a, w.b, row, imin(a.m, a.s_pad));
            if (w.splits == 1) fetch(half);
            bool ok = true;
            uint32_t d = 0;
            const int64_t slab = 128 * BN;
            [[maybe_unused]] float *sums_at = nullptr;
            if constexpr (LONG) {
                // a long sum: all but its last part go to the workspace, a lane's own elements each
                if (w.kb1 - w.kb0 > kLongKb) {
                    const int64_t own = w.splits > 1 ? ((int64_t)w.tile * w.splits + w.split) * CG + rank : blockIdx.x;
                    sums_at = a.partial + own * slab + (q * 32 + lane) * 4;
                    for (int kb = w.kb0; kb + kLongKb < w.kb1; kb += kLongKb) {
                        const int acc = j & 1;
                        ok = gwait_warp(accf + acc, (j >> 1) & 1, &s_abort);
                        if (!ok) break;
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                        d = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN);
#pragma unroll 1
                        for (int ci = half; ci < kChunks; ci += 2) {
                            uint32_t r[32];
                            tmem_ld_32cols(d + (uint32_t)(ci * 32), r);
                            float4 *p = reinterpret_cast<float4 *>(sums_at + (int64_t)ci * 32 * 128);
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                float4 f = kb == w.kb0 ? make_float4(0.f, 0.f, 0.f, 0.f) : p[e * 128];
                                f.x += __uint_as_float(r[4 * e]), f.y += __uint_as_float(r[4 * e + 1]);
                                f.z += __uint_as_float(r[4 * e + 2]), f.w += __uint_as_float(r[4 * e + 3]);
                                p[e * 128] = f;
                            }
                        }
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0)
                            asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(acce_bar[acc])
                                         : "memory");
                        ++j;
                    }
                    if (!ok) break;   // the abort flag is set
                }
            }
            if (!PROMOTE || w.kb1 - w.kb0 <= kPromoteKb) {
                ok = gwait_warp(accf + (j & 1), (j >> 1) & 1, &s_abort);
                if (!ok) break;
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                d = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)((j & 1) * BN);
            } else {
                // a long float32 sum: taken out every kPromoteKb stages, the whole sums put back for the epilogue
                float sums[PROMOTE ? kChunks / 2 : 1][32];
#pragma unroll
                for (int i = 0; i < (PROMOTE ? kChunks / 2 : 1); ++i)
#pragma unroll
                    for (int e = 0; e < 32; ++e) sums[i][e] = 0.f;
                int kb = w.kb0;
                do {
                    const int acc = j & 1;
                    ok = gwait_warp(accf + acc, (j >> 1) & 1, &s_abort);
                    if (!ok) break;
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    d = tmem + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * BN);
                    kb += kPromoteKb;
#pragma unroll
                    for (int i = 0; i < (PROMOTE ? kChunks / 2 : 1); ++i) {
                        uint32_t r[32];
                        tmem_ld_32cols(d + (uint32_t)((2 * i + half) * 32), r);
#pragma unroll
                        for (int e = 0; e < 32; ++e) sums[i][e] += __uint_as_float(r[e]);
                    }
                    if (kb < w.kb1) {
                        asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                        __syncwarp();
                        if (lane == 0)
                            asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(acce_bar[acc])
                                         : "memory");
                        ++j;
                    } else {
#pragma unroll
                        for (int i = 0; i < (PROMOTE ? kChunks / 2 : 1); ++i)
                            tmem_st_32cols(d + (uint32_t)((2 * i + half) * 32), sums[i]);
                        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                    }
                } while (kb < w.kb1);
            }
            if (!ok) break;   // the abort flag is set

            if (PROMOTE && u + ustep < a.units) ahead = unit_of<R>(a, u + ustep);
            bool last = true;
            float *part = nullptr;
            if (w.splits > 1) part = a.partial + ((int64_t)w.tile * w.splits * CG + rank) * slab + (q * 32 + lane) * 4;
#pragma unroll 1
            for (int pass = 0; pass < 2; ++pass) {
                // pass 0: this unit's sums (to the epilogue, or to its slab); pass 1: the slices joined
                if (pass == 1) {
                    if (w.splits == 1) break;
                    __threadfence();
                    __syncwarp();
                    int n_in = 0;
                    int32_t *cnt = a.counters + ((int64_t)w.tile * CG + rank) * kGEpiWarps + (warp - 4);
                    if (lane == 0) n_in = atomicAdd(cnt, 1);
                    n_in = __shfl_sync(0xffffffffu, n_in, 0);
                    last = n_in == w.splits - 1;
                    if (!last) break;
                    if (lane == 0) *cnt = 0;
                    __threadfence();
                }
#pragma unroll 1
                for (int i = 0; i < kChunks / 2; ++i) {
                    const int ci = 2 * i + half;
                    float v[32];
                    if (pass == 0) {
                        uint32_t r[32];
                        tmem_ld_32cols(d + (uint32_t)(ci * 32), r);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = empty_sum ? 0.f : __uint_as_float(r[e]);
                        if constexpr (LONG)
                            if (sums_at != nullptr) {
                                const float4 *p = reinterpret_cast<const float4 *>(sums_at + (int64_t)ci * 32 * 128);
#pragma unroll
                                for (int e = 0; e < 8; ++e) {
                                    const float4 f = p[e * 128];
                                    v[4 * e] += f.x, v[4 * e + 1] += f.y, v[4 * e + 2] += f.z, v[4 * e + 3] += f.w;
                                }
                            }
                        if (i == kChunks / 2 - 1) {
                            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                            __syncwarp();
                            if (lane == 0)
                                asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(
                                                 acce_bar[j & 1])
                                             : "memory");
                            ++j;
                        }
                        if (n0 + ci * 32 >= a.n) continue;
                        if (w.splits > 1) {
                            float *p = part + (int64_t)w.split * CG * slab + (int64_t)ci * 32 * 128;
#pragma unroll
                            for (int e = 0; e < 8; ++e)
                                *reinterpret_cast<float4 *>(p + e * 512) =
                                    make_float4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
                            continue;
                        }
                    } else {
                        if (n0 + ci * 32 >= a.n) continue;
                        fetch(ci);
#pragma unroll
                        for (int e = 0; e < 32; ++e) v[e] = 0.f;
                        for (int sl = 0; sl < w.splits; sl += 2) {   // two slices' loads in flight
                            const float *p = part + (int64_t)sl * CG * slab + (int64_t)ci * 32 * 128;
                            const bool two = sl + 1 < w.splits;
                            float4 f[8], g[8];
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                f[e] = __ldcg(reinterpret_cast<const float4 *>(p + e * 512));
                                g[e] = two ? __ldcg(reinterpret_cast<const float4 *>(p + CG * slab + e * 512))
                                           : make_float4(0.f, 0.f, 0.f, 0.f);
                            }
#pragma unroll
                            for (int e = 0; e < 8; ++e) {
                                v[4 * e] = (v[4 * e] + f[e].x) + g[e].x;
                                v[4 * e + 1] = (v[4 * e + 1] + f[e].y) + g[e].y;
                                v[4 * e + 2] = (v[4 * e + 2] + f[e].z) + g[e].z;
                                v[4 * e + 3] = (v[4 * e + 3] + f[e].w) + g[e].w;
                            }
                        }
                    }
                    const int col = n0 + ci * 32;
                    if (lane == 0) {
                        if (a.slots == 2) asm volatile("cp.async.bulk.wait_group.read 1;" ::: "memory");
                        else asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
                    }
                    __syncwarp();
                    epilogue32<EPI, GEN, PROMOTE>(v, u0, u1, di, dj, a, maps, stage0 + slot * (stage_out<EPI, PROMOTE>() / 2), w.b, row, col,
                                                  NS && a.sym && w.tn >= R * (w.tm + 1));
                    if (lane == 0) asm volatile("cp.async.bulk.commit_group;" ::: "memory");
                    slot = a.slots == 2 ? slot ^ 1 : 0;
                    if (pass == 0 && i + 1 < kChunks / 2) fetch(ci + 2);   // the next group's, while this one leaves
                }
            }
            if (NS) {
                // This warp's share of the unit is in place: its TMA stores are complete, its lanes' own stores are
                // ordered before the count by the block-scope fences. The unit's last warp says so for its matrix.
                if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
                __threadfence_block();
                __syncwarp();
                int *count = &s_done[(n_go - 1) % kGoRing];
                if (lane == 0 && atomicAdd(count, 1) == kGEpiWarps - 1) {
                    *count = 0;
                    __threadfence_block();
                    asm volatile("red.release.gpu.global.add.u32 [%0], 1;" ::"l"(L.done + w.b) : "memory");
                }
                __syncwarp();
            }
        }
        }
        if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
        __syncwarp();
    }
    if (s_abort)   // copies that nothing waits for any more land before the shared memory goes
        for (int i = 0; i < 64; ++i) __nanosleep(1000);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    if constexpr (CG == 2) cluster_sync_all();
    if (threadIdx.x == 0 && s_abort) {
        dev_flag(L.args[0].hdr, CSRT_DEV_TIMEOUT);
        L.args[0].hdr->timeout_site = 6;
    }
    if (warp == 1) {
        __syncwarp();
        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
        if constexpr (CG == 1)
            asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
        else
            asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
    }
}

}  // namespace csrt
