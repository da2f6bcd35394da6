// C = A B^T of two matrices whose rows lie along the contraction: the pipeline that the 4-bit product and the
// orthogonalisation share (not installed).
//
// A workgroup owns a BM x BN tile of C.  The contraction runs in steps of 128 bytes of every row of A and B.  A step's
// rows go from memory to LDS without passing through registers (16 bytes a lane) into one of several buffers, while the
// matrix instructions read another.  A row of a step is 8 chunks of 16 bytes; chunk c of row r lies at
// place c ^ (r / 2 & 7), so that the sixteen lanes that one cycle serves (16 rows, the same chunk) touch all 64 banks once (with
// c ^ (r & 7) every read took 8 cycles and not 4).
//
// A step falls into parts; the fragments of the next part are read from LDS while the matrix instructions of this one run.  The
// barrier stands before the last part's instructions, whose fragments are in registers by then: behind it the next buffer
// is complete and this one free, so the next step's first fragments and the loads of a later step are on their way while the last
// part still keeps the matrix units busy.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace qesgd {

typedef float acc16 __attribute__((ext_vector_type(16)));
typedef int int4v __attribute__((ext_vector_type(4)));
typedef int int8v __attribute__((ext_vector_type(8)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));

constexpr uint32_t kStepBytes = 128;

// WM x WN waves, each of FM x FN fragments of 32 x 32, and the number of buffers: two where a step's instructions take longer than
// memory, four where a small tile, or a CU with one workgroup, would wait for it.
template <int WM_, int WN_, int FM_, int FN_, int BUFFERS_>
struct TileShape {
    static constexpr int WM = WM_, WN = WN_, FM = FM_, FN = FN_;
    static constexpr int BM = WM * FM * 32, BN = WN * FN * 32;
    static constexpr int threads = WM * WN * 64;
    static constexpr int BUFFERS = BUFFERS_;
};

// 16 (4) bytes a lane from base + offset to LDS, the wave's lanes one behind the other from `to` on.  In assembly, because the
// compiler, which does not know which buffer a load goes to, waits for all loads before it reads any buffer once there are more than two.  The
// waiting is wait_and_meet's; no register is written but M0, which needs one wait state before the load takes it.
// The compiler warns that M0 is a register it gives no value to keep; it is named all the same, for the instructions before which the compiler sets M0 itself.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void load_to_lds_16(const unsigned char* base, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(to), "v"(offset), "s"(base) : "m0", "memory");
}
__device__ __forceinline__ void load_to_lds_4(const unsigned char* base, uint32_t offset, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" : : "s"(to), "v"(offset), "s"(base) : "m0", "memory");
}
#pragma clang diagnostic pop
// Number of an LDS byte, as M0 takes it.
__device__ __forceinline__ uint32_t lds_number(const unsigned char* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) unsigned char*)p;
}

// One step of ROWS rows to LDS.  `off` holds the lane's byte offsets from the tile's first row.
template <int ROWS, int THREADS>
struct TileLoader {
    static constexpr int N = ROWS * 8 / THREADS;
    static_assert(N >= 1 && ROWS * 8 % THREADS == 0 && THREADS % 128 == 0, "every thread moves the same number of chunks, of rows with the same r / 2 & 7");
    uint32_t off[N];
    uint32_t wave_at;

    // Row r of the tile is row min(r, rows - 1) of what is there: no row beyond the end is read.
    __device__ __forceinline__ void init(uint32_t pitch, uint32_t rows) {
        wave_at = __builtin_amdgcn_readfirstlane((threadIdx.x >> 6) * 1024u);
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const uint32_t at = i * THREADS + threadIdx.x, r = at >> 3, c = (at & 7u) ^ ((r >> 1) & 7u);
            off[i] = min(r, rows - 1u) * pitch + c * 16u;
        }
    }
    // From the byte of the rows that `base` points at.  half: only 64 bytes are left, the chunks of the second half repeat the first.
    __device__ __forceinline__ void load(const unsigned char* base, unsigned char* lds, bool half) const {
        const uint32_t c4 = half ? (((threadIdx.x & 7u) ^ ((threadIdx.x >> 4) & 7u)) & 4u) * 16u : 0u;
        const uint32_t to = lds_number(lds) + wave_at;
#pragma unroll
        for (int i = 0; i < N; ++i) load_to_lds_16(base, off[i] - c4, to + i * (THREADS * 16));
    }
};

// Where a lane finds its chunk of row lane & 31 of a fragment: chunk 2 s + h of part s (h: the half of the wave) at place
// (2 s + h) ^ (row / 2 & 7), so part s is at the place of part 0 with s * 32 flipped.
__device__ __forceinline__ uint32_t lane_place(uint32_t lane) { return (lane & 31u) * kStepBytes + (((lane >> 5) ^ ((lane >> 1) & 7u)) * 16u); }

// Waits until at most LEFT of the wave's loads are on their way and all LDS reads are done, then for the other waves.
template <int LEFT>
__device__ __forceinline__ void wait_and_meet() {
    static_assert(LEFT < 64, "the counter has six bits");
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4 << 14) | 0x70);       // vmcnt(LEFT) lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// The contraction.  Ops: PARTS (even), LOADS (of a wave, for a step), Frag, fetch(step, buffer), read(frag, buffer, part),
// multiply(frag, part), fetch_pair(step) (PAIR_LOADS loads for two steps at once, step even), arrive(step) (its data is there), next()
// (between two steps), at_a and at_b (places of part 0 of the lane's first fragments).  What the reads behind the last
// step find, nothing uses.
template <int N, class Ops>
__device__ __forceinline__ void run_steps(Ops& ops, uint32_t steps, unsigned char* const (&lds)[N]) {
    static_assert(N == 2 || N == 4, "steps come in pairs");
    typename Ops::Frag f[2];
    auto step = [&](auto even, uint32_t t, unsigned char* here, unsigned char* there) {
        asm volatile("" : "+v"(ops.at_a), "+v"(ops.at_b));      // the parts' places are worked out where they are used, not kept in 16 registers
#pragma unroll
        for (int p = 0; p + 1 < Ops::PARTS; ++p) {
            ops.read(f[(p + 1) & 1], here, p + 1);
            ops.multiply(f[p & 1], p);
            __builtin_amdgcn_sched_barrier(0);       // otherwise all reads go to the front and the instructions behind the barrier
        }
        // of the later steps' loads as many may be left as were issued behind the next step's
        wait_and_meet<(N - 2) * Ops::LOADS + (N > 2 ? Ops::PAIR_LOADS : 0)>();
        ops.arrive(t + 1);
        // Without a branch, which the compiler would move the matrix instructions above past: behind the end the last step comes once more.
        ops.fetch(min(t + N, steps - 1), here);
        if (decltype(even)::value) ops.fetch_pair(t + N);
        ops.read(f[0], there, 0);
        __builtin_amdgcn_sched_barrier(0);
        ops.multiply(f[1], Ops::PARTS - 1);
        ops.next();
    };
    ops.fetch(0, lds[0]);
    ops.fetch_pair(0);
#pragma unroll
    for (int i = 1; i < N; ++i) {
        ops.fetch(min((uint32_t)i, steps - 1), lds[i]);
        if (i == 2) ops.fetch_pair(2);
    }
    wait_and_meet<(N - 1) * Ops::LOADS + (N > 2 ? Ops::PAIR_LOADS : 0)>();
    ops.arrive(0);
    ops.next();
    ops.read(f[0], lds[0], 0);
    for (uint32_t t = 0; t < steps; t += N) {
        step(std::true_type{}, t, lds[0], lds[1]);
        if (t + 1 < steps) step(std::false_type{}, t + 1, lds[1], lds[2 % N]);
        if constexpr (N > 2) {
            if (t + 2 < steps) step(std::true_type{}, t + 2, lds[2], lds[3]);
            if (t + 3 < steps) step(std::false_type{}, t + 3, lds[3], lds[0]);
        }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);             // vmcnt(0): nothing is on its way to LDS when the workgroup ends
}

// Number of the tile that workgroup b of n takes: ids go round-robin over the 8 XCDs, so each XCD gets one run of tiles, whose rows
// of A and B its own L2 then holds.
__device__ __forceinline__ uint32_t tile_of_workgroup(uint32_t b, uint32_t n) {
    const uint32_t per = n >> 3, left = n & 7u, x = b & 7u;
    return (b >> 3) + x * per + (x < left ? x : left);
}
// Tile t of tiles_m x tiles_n in bands of kBand rows of tiles, column by column within a band: what an XCD has in work at a time
// is a block about as high as it is wide, which reads the fewest rows of A and B.  Five steps of orthogonalising 4096 x 25088 in bands of 1 / 2 /
// 4 / 8 / 16: 14.47 / 14.04 / 13.91 / 13.90 / 14.07 ms, 3000 x 3000 2487 / 2228 / 2184 / 2175 / 2225 us; 4-bit 8192 x 4096 x 4096 in 1 to 8 79.0 / 78.6 / 77.2 / 78.6.
constexpr uint32_t kBand = 4;
__device__ __forceinline__ void banded_tile(uint32_t t, uint32_t tiles_m, uint32_t tiles_n, uint32_t& tm, uint32_t& tn) {
    const uint32_t width = kBand * tiles_n, band = t / width, first = band * kBand, in = t - band * width;
    const uint32_t high = min(tiles_m - first, kBand);
    tn = in / high;
    tm = first + in - tn * high;
}

}  // namespace qesgd
