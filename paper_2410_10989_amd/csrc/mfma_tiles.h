// Building blocks of the matrix products on 16-bit operands (gemm_bf16_nt.h describes them): the tiles of an operand
// in memory and in LDS, and the fragments that 32 x 32 x 16 MFMAs take.  The 16 bits are bf16 or fp16 alike.
#pragma once
#include <type_traits>

#include "flce_device.h"
#include "scheduler.h"

namespace flce {

constexpr int FG_BM = 256, FG_BN = 256, FG_BK = 64, FG_THREADS = 256;
constexpr int FG_XCDS = 8;
constexpr int FG_SLOTS = 5;                         // ring of operand-tile slots
constexpr int fg_slot_bytes(int tile) { return tile * FG_BK * 2; }   // one operand tile of one K step: 32 or 16 KB
constexpr int fg_lds_bytes(int tile) { return FG_SLOTS * fg_slot_bytes(tile); }   // 160 KB, the whole LDS of a CU, or half of it

// How a row-form operand's K loop runs (kernel variants: one more scalar instruction per step of the
// plain loop costs the logits product 0.6 %): plain, for K % 64 == 0 or rows padded with zeros;
// rotated (see gemm_bf16); with a last K step that K cuts; over the products of operands held in two planes
// (FgOperand::plane_steps).
enum { FG_PLAIN = 0, FG_ROTATED = 1, FG_K_TAIL = 2, FG_PLANES = 3 };

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) void* fg_lds_ptr;

__device__ __forceinline__ __amdgpu_buffer_rsrc_t fg_make_rsrc(const void* base, uint32_t bytes) {
    // raw buffer, no stride: offsets >= bytes read as zero / are not written
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00020000);
}

// 16 bytes per lane from the buffer to LDS (lane l to dst + 16 l).  A free function: inside a
// class template the host pass cannot type-check the builtin and silently drops the launch stubs
// of the kernels that use it.
__device__ __forceinline__ void fg_load_lds(__amdgpu_buffer_rsrc_t rsrc, unsigned char* dst, int voff, int soff) {
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (fg_lds_ptr)dst, 16, voff, soff, 0, 0);
}

// One GEMM operand: where its tiles come from in global memory, where they land
// in LDS, and how MFMA fragments (32 rows x 16 K, lane l = row l%32, K values
// 8*(l/32) .. +7) are read back.  KM = false: row form, KM = true: column form.
template <bool KM, int TILE, int ORDER = FG_PLAIN>
struct FgOperand {
    static constexpr int NL = TILE / 32;   // loads a wavefront issues per tile
    static constexpr int W = TILE / 64;    // fragments per wavefront
    // The buffer descriptor covers the operand from K step kt_base on; the loads of K
    // step kt add (kt - kt_base) * kstep as scalar offset.  All offsets are 32-bit, so
    // the descriptor is moved forward every seg_steps K steps (a rarely taken uniform
    // branch; for most operands never), which lets operands be of any size.
    const unsigned char* base0;   // first byte of K step kt_base of this workgroup's tiles
    int64_t bytes;                // bytes from base0 to the end of the operand's valid range
    __amdgpu_buffer_rsrc_t rsrc;
    int kt_base, seg_steps;
    int kt_tail;  // FG_K_TAIL: the K step that holds the last, partial group of 64 K values, if any
    int off[NL];  // per-lane byte offset of each of the loads a wavefront issues per tile
    int kstep;    // bytes between consecutive K steps
    int rot, wrap;   // FG_ROTATED: the K steps are taken in the order rot, rot + 1, ..., wrap - 1, 0, 1, ...
    // FG_PLANES: an operand of two planes, plane_bytes apart, whose product with another is taken as hi lo, lo hi,
    // hi hi one after the other; this one's lo plane is the one of part lo_part.
    int plane_steps, plane_bytes, lo_part;
    int rd[4];    // per-lane LDS byte offsets of the fragment reads

    // base/ld: the matrix; r0: first row (row form) or column (column form) of this
    // tile; extent: number of rows / columns of the matrix; sub: which half of the tile
    // this wavefront multiplies.
    // rows (row form, not null): LDS, the tile's rows are rows[0], rows[1], ... of the matrix instead, which has
    // `all` rows (below 2^30 bytes); the caller keeps them there until every thread has returned.
    __device__ __forceinline__ void init(const bf16_t* base, int64_t ld, int r0, int extent, int K,
                                         int tid, int sub, const int* rows_at = nullptr, int all = 0) {
        const int lane = tid & 63, wave = tid >> 6;
        const int ildb = (int)ld * 2;   // leading dimension in bytes
        if constexpr (!KM) {
            // a wavefront-wide load = 8 consecutive tile rows of 128 B; lane l owns the
            // physical position (row l/8, piece l%8) and fetches the logical piece
            // (l%8) ^ swizzle(row); wavefront w fills rows 8w..8w+7 of every 32-row group
            const int rows = min(TILE, extent - r0);
            base0 = reinterpret_cast<const unsigned char*>(base + (int64_t)r0 * ld);
            bytes = (int64_t)rows * ildb;
            const int ld_row = tid >> 3;
            const int piece = (tid & 7) ^ ((ld_row >> 1) & 7);
#pragma unroll
            for (int r = 0; r < NL; ++r) off[r] = (ld_row + 32 * r) * ildb + piece * 16;
            if (rows_at) {
                base0 = reinterpret_cast<const unsigned char*>(base);
                bytes = (int64_t)all * ildb;
#pragma unroll
                for (int r = 0; r < NL; ++r)
                    off[r] = ld_row + 32 * r < rows ? rows_at[ld_row + 32 * r] * ildb + piece * 16 : 0x7fffffff;
            }
            kstep = FG_BK * 2;
            const int frow = lane & 31, fhalf = lane >> 5, fsw = (frow >> 1) & 7;
#pragma unroll
            for (int kk = 0; kk < 4; ++kk)
                rd[kk] = (sub * (TILE / 2) + frow) * 128 + ((((kk << 1) | fhalf) ^ fsw) << 4);
        } else {
            // a wavefront-wide load = 2 (TILE 256) or 4 (TILE 128) consecutive K rows of 512 or
            // 256 B; load r of wavefront w covers the K rows from (4 r + w) * 2 or * 4 on; the
            // lane owns one physical 16-byte piece of one row and fetches the logical 64-byte
            // chunk (piece / 4) ^ f(k), f(k) = k%4 + 4 * ((k/8) % 2), for TILE 128 (4 chunks) k%4
            constexpr int LPR = TILE / 8, RPL = 64 / LPR;   // lanes per K row, K rows per load
            base0 = reinterpret_cast<const unsigned char*>(base + r0);
            bytes = ((int64_t)K * ld - r0) * 2;
#pragma unroll
            for (int r = 0; r < NL; ++r) {
                const int k = (4 * r + wave) * RPL + lane / LPR;
                const int chunk = ((lane % LPR) >> 2) ^ fold(k & 3, (k >> 3) & 1);
                off[r] = k * ildb + chunk * 64 + (lane & 3) * 16;
            }
            kstep = FG_BK * ildb;
            // transposing read: group g = l/16 of the wavefront reads K rows
            // 8*(g/2) + {0..3} (+4 for the second read), columns 16*(g%2) + 0..15 of the
            // 32-wide fragment; source lane s = l%16 supplies row s/4, columns 4*(s%4)..+3
            const int g = lane >> 4, s = lane & 15;
            const int f = fold(s >> 2, g >> 1);
#pragma unroll
            for (int i = 0; i < W; ++i)
                rd[i] = (8 * (g >> 1) + (s >> 2)) * (2 * TILE) + (((sub * W + i) ^ f) * 64) + 32 * (g & 1) +
                        8 * (s & 3);
        }
        // FG_K_TAIL, a row-form operand whose K is not a multiple of 64: in the last K step, the lanes whose
        // 16-byte piece lies past K fetch from beyond the descriptor, i.e. zero (a piece that K
        // cuts has to hold zeros past it: none when K % 8 == 0).
        kt_tail = (!KM && (K & (FG_BK - 1))) ? K / FG_BK : 0x7fffffff;
        piece_past = !KM && ((tid & 7) ^ (((tid >> 3) >> 1) & 7)) * 8 >= (K & (FG_BK - 1));
    }
    bool piece_past;
    static __device__ __forceinline__ int fold(int k4, int k8) { return TILE == 256 ? k4 | (k8 << 2) : k4; }

    __device__ __forceinline__ void make_rsrc() {
        const int64_t left = bytes < 0 ? 0 : (bytes > 0xFFFFFFFFll ? 0xFFFFFFFFll : bytes);
        rsrc = fg_make_rsrc(base0, (uint32_t)left);
    }
    // K step 0 of the loads below is K step k_begin of the matrix
    __device__ __forceinline__ void start_at(int k_begin) {
        base0 += (int64_t)k_begin * kstep;
        bytes -= (int64_t)k_begin * kstep;
        kt_base = 0;
        seg_steps = max(1, (1 << 30) / kstep);
        if (kt_tail != 0x7fffffff) kt_tail -= k_begin;
        make_rsrc();
    }
    // call before the first load of K step kt (kt never decreases)
    __device__ __forceinline__ void before_step(int kt) {
        if constexpr (ORDER == FG_PLANES) return;   // (its users keep operands below 2^30 bytes)
        if (kt - kt_base >= seg_steps) {
            base0 += (int64_t)seg_steps * kstep;
            bytes -= (int64_t)seg_steps * kstep;
            kt_base += seg_steps;
            make_rsrc();
        }
        if constexpr (!KM && ORDER == FG_K_TAIL) {
            if (kt >= kt_tail) {   // uniform, once (a row-form tile's extent is below 2^30 bytes)
#pragma unroll
                for (int r = 0; r < NL; ++r) off[r] = piece_past ? 0x7fffffff : off[r];
                kt_tail = 0x7fffffff;
            }
        }
    }

    __device__ __forceinline__ int step_offset(int kt) const {
        if constexpr (ORDER == FG_ROTATED) kt = rotated_step(kt, rot, wrap);
        if constexpr (ORDER == FG_PLANES) {
            const int part = kt >= 2 * plane_steps ? 2 : kt >= plane_steps ? 1 : 0;
            return (kt - part * plane_steps) * kstep + (part == lo_part ? plane_bytes : 0);
        }
        return (kt - kt_base) * kstep;
    }

    // start the loads of this wavefront for K step kt into ring slot `slot`
    __device__ __forceinline__ void load(unsigned char* smem, int slot, int kt, int uwave) {
        before_step(kt);
        const int soff = step_offset(kt);
        unsigned char* dst = smem + slot * fg_slot_bytes(TILE) + uwave * 1024;
#pragma unroll
        for (int r = 0; r < NL; ++r)
            fg_load_lds(rsrc, dst + r * 4096, off[r], soff);
    }

    // start one of the loads of this wavefront for K step kt into ring slot `slot`
    __device__ __forceinline__ void load_one(unsigned char* smem, int slot, int kt, int uwave, int r) const {
        unsigned char* dst = smem + slot * fg_slot_bytes(TILE) + uwave * 1024 + r * 4096;
        fg_load_lds(rsrc, dst, off[r], step_offset(kt));
    }
};

// Registers an in-flight fragment lands in.  The reads are asynchronous inline
// assembly: nothing may touch these registers until fg_wait has run.
template <bool KM> struct FgRaw;
template <> struct FgRaw<false> { bf16x8 v; };
template <> struct FgRaw<true> { s16x4 lo, hi; };

// Issue the LDS read(s) of fragment I (32-row block) of K sub-step KK; `slot_addr`
// is the LDS byte address of the ring slot.
template <int KK, int I, int TILE, int ORDER>
__device__ __forceinline__ void fg_issue(FgRaw<false>& r, const FgOperand<false, TILE, ORDER>& op, unsigned slot_addr) {
    const unsigned addr = slot_addr + (unsigned)op.rd[KK];
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(r.v) : "v"(addr), "n"(I * 4096));
}
template <int KK, int I, int TILE, int ORDER>
__device__ __forceinline__ void fg_issue(FgRaw<true>& r, const FgOperand<true, TILE, ORDER>& op, unsigned slot_addr) {
    const unsigned addr = slot_addr + (unsigned)op.rd[I];
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r.lo) : "v"(addr), "n"(KK * 32 * TILE));
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(r.hi) : "v"(addr), "n"(KK * 32 * TILE + 8 * TILE));
}

// Wait until every LDS read issued so far has returned.  The registers are tied
// to the asm statements so that nothing that uses them is moved above the wait.
__device__ __forceinline__ void fg_tie(FgRaw<false> (&r)[4]) {
    asm volatile("" : "+v"(r[0].v), "+v"(r[1].v), "+v"(r[2].v), "+v"(r[3].v));
}
__device__ __forceinline__ void fg_tie(FgRaw<true> (&r)[4]) {
    asm volatile("" : "+v"(r[0].lo), "+v"(r[0].hi), "+v"(r[1].lo), "+v"(r[1].hi), "+v"(r[2].lo),
                 "+v"(r[2].hi), "+v"(r[3].lo), "+v"(r[3].hi));
}
__device__ __forceinline__ void fg_tie(FgRaw<false> (&r)[2]) { asm volatile("" : "+v"(r[0].v), "+v"(r[1].v)); }
__device__ __forceinline__ void fg_tie(FgRaw<true> (&r)[2]) {
    asm volatile("" : "+v"(r[0].lo), "+v"(r[0].hi), "+v"(r[1].lo), "+v"(r[1].hi));
}
template <bool AKM, bool BKM, int W>
__device__ __forceinline__ void fg_wait(FgRaw<AKM> (&ra)[W], FgRaw<BKM> (&rb)[W]) {
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    fg_tie(ra);
    fg_tie(rb);
}
__device__ __forceinline__ bf16x8 fg_value(const FgRaw<false>& r) { return r.v; }
__device__ __forceinline__ bf16x8 fg_value(const FgRaw<true>& r) {
    const s16x8 both = __builtin_shufflevector(r.lo, r.hi, 0, 1, 2, 3, 4, 5, 6, 7);
    return __builtin_bit_cast(bf16x8, both);
}
__device__ __forceinline__ void fg_zero(FgRaw<false>& r) {
#pragma unroll
    for (int e = 0; e < 8; ++e) r.v[e] = (bf16_t)0.f;
}
__device__ __forceinline__ void fg_zero(FgRaw<true>& r) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        r.lo[e] = 0;
        r.hi[e] = 0;
    }
}

}  // namespace flce
