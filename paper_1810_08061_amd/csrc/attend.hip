// attend.hip -- linear attention with a decay for each head: S_t = a S_{t-1} + k_t v_t^T,
// y_t = S_t^T q_t, over whole sequences, its backward pass, and single steps.
//
// All four products over a sequence have one form (a "pass"), with a state M [P][R]:
//     out_i = sum_j a^|i-j| (x_i . y_j) z_j + a^e(i) M^T x_i
// over j <= i going forward, j >= i going back:
//            x   y   z   M      direction
//     y      q   k   v   S      forward
//     dq     dy  v   k   S^T    forward
//     dk     v   dy  q   R^T    back        (R_t = q_t dy_t^T + a R_{t+1})
//     dv     k   q   dy  R      back, leaves dS0
// so the backward forms S and R again and needs nothing kept.
//
// A workgroup goes through a sequence (or a share of it) of one head in chunks, M in its
// registers in fp32: inside a chunk the products are those of attention under a mask of decays,
// between chunks they go through M.  A wave owns columns of M and of out.  The
// layout in which a product leaves M (four rows of one column a lane) is the one in which
// the next product takes it as an operand, if the other operand's rows are fetched in the
// same order, so M never leaves the registers.
//
// bf16 data: operands of the matrix units are bf16.  x, y and z are that already; the
// masked products and M are given as two parts (16 bits; 2^-17 of them is left, below the rounding of
// out where a sum does not cancel to less than 2^-8 of its terms: one bf16 value in 400 to 900 of out is another
// than with all bits, and the error against 64 bits, 1.7e-3, is the same), what is added to M, a^. z, as three (24
// bits: the state is fp32).
// fp32 data: the matrix units' fp32 products.
//
// Where rows and heads are fewer than workgroups should be, the time axis is cut into shares:
// a launch forms what each share adds to the state, one joins them in their order, and
// the pass's shares start from the joined states.
//
// Measured, bf16, heads of 128: 1 x 32768 x 16, forward, 74 us for the shares' states (3.6 TB/s), 15 to join them, 144 to 147
// for the pass (3.7 TB/s; 223 to 229 us together, 2.4 TB/s of what the call cannot do without); 8 x 4096 x 16, ragged, forward
// and backward 530 to 560 us, the three passes back 264.  What bounds a pass: for 64 steps a wave issues 208
// products for the matrix unit (3300 clocks), 870 vector instructions (3500: splitting into parts, decays,
// addresses) and LDS reads, in phases between barriers; two workgroups a CU, which its registers allow, take 14800
// clocks for a chunk each.  Tried and not kept: eight waves of 16 columns (199 us: spills, and every wave reads all rows);
// operands fetched from LDS a phase ahead by scheduling barriers (no gain); vector and matrix instructions interleaved by
// scheduling groups (no gain); workgroups of half the columns for the states (no gain: they wait for memory);
// workgroups that are behind issued first (no gain over outputs first).
// fp32, heads of 128: a training step of 4 x 1024 x 8 takes 194 us, its bytes 40.  For 32 steps a wave issues 176 fp32 products in
// a pass (144 in the half of the waves that form no masked ones) and 64 for a share's state, of 32 clocks each: 89 us of the
// matrix unit, which stands while the one workgroup of a CU is at its LDS reads and barriers.
// A step of 16 x 8 heads of 64: 4.0 us, 4.2 TB/s of states.
#include "ops.h"
#include "../../include/lstm_dyn_layer.h"
#include "attend_shares.h"

#include <cmath>
#include <type_traits>
#include <vector>

namespace ldyn {
namespace {

constexpr int MAX_D = 128;
constexpr int MAX_HEADS = 16384; // a chunk of 64 rows of heads 3 x 128 elements stays below NOWHERE
constexpr int TABLE = 65;        // powers of a head's decay

typedef __bf16 bf16x4_t __attribute__((ext_vector_type(4)));

// One pass: addresses of its operands in [B][T][ld], their widths, its state.
struct Pass {
    const void *x, *y, *z;
    void* out;
    long long ldx, ldy, ldz, ldo;   // elements from one step to the next
    int P, R;
    int back;                       // direction
    int transposed;                 // M [P][R] is the transpose of the state as it is kept
    const float* start;             // [B][heads][Dk][Dv], or NULL: zeros
    float* end;                     // the same (written), or NULL
    float* share;                   // [B heads][shares][Dk][Dv]
};

struct AttendParams {
    Pass pass[3];
    const int32_t* lengths; // [B], or one for all rows
    int32_t* status;
    const float* powers;    // [heads][TABLE]
    const double* log2a;    // [heads]
    int passes, T, heads, rows, shares, span, Dv, mode, length_step;   // rows = B heads; span: steps of a share
};

template <class E>
struct Chunk;
template <>
struct Chunk<__bf16> {
    static constexpr int C = 64;
    static constexpr int waves(int DP) { return DP == 32 ? 2 : 4; }
    static constexpr int per_unit(int DP) { return DP == 128 ? 2 : 3; }   // waves a SIMD unit holds: registers and LDS
};
template <>
struct Chunk<float> {
    static constexpr int C = 32;
    static constexpr int waves(int DP) { return DP / 16; }
    static constexpr int per_unit(int) { return 4; }
};

__device__ inline double power(const double* log2a, int head, int n) { return n ? exp2(log2a[head] * n) : 1.0; }

template <int N>
using Part = std::integral_constant<int, N>;

// The thread's number as one that the compiler does not know: what is formed from it inside the loop
// over chunks is not kept in registers across it.
__device__ inline int here() {
    int t = threadIdx.x;
    asm volatile("" : "+v"(t));
    return t;
}

// Pairs of numbers as sums of bf16 parts, each pair of parts in one register.
typedef float f32x2_t __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
__device__ inline uint32_t pack(f32x2_t x) { return __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2_t)); }
__device__ inline f32x2_t unpack(uint32_t x) { return f32x2_t{__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u)}; }
__device__ inline void parts(f32x2_t x, uint32_t& hi, uint32_t& lo) {
    hi = pack(x);
    lo = pack(x - unpack(hi));
}
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));

// How rows lie in memory.  PIECES: every head's row is whole pieces of 16 bytes at multiples of 16.
// SHIFTED: it starts at any element and has at least 16 bytes; its last piece is fetched from where the row
// ends 16 bytes later, and moved.  ELEMENTS: any row.
enum { PIECES, SHIFTED, ELEMENTS };

// A chunk's x, y and z: fetched into registers while the chunk before is worked on, then put into LDS.  The
// fetches are under no condition: where ways meet, the compiler waits for what is on its way.
// PIECES go through a descriptor of the chunk's rows, which gives zeros past them and in
// columns that are not there (set beyond it); the others fetch rows and columns that
// are there in place of ones that are not.
constexpr uint32_t NOWHERE = 1u << 30;   // a chunk's rows have fewer bytes
template <class E, int DP, bool STATE, int MODE>
struct Stage {
    static constexpr int C = Chunk<E>::C, THREADS = 64 * Chunk<E>::waves(DP), N = 16 / (int)sizeof(E);
    static constexpr int COLS = DP / N, ROWS = C * COLS / THREADS;  // a thread's rows, one after another
    typedef typename Vec<E, N>::type piece_t;
    struct __attribute__((packed, aligned(sizeof(E)))) Loose { piece_t v; };
    piece_t x[ROWS], y[ROWS], z[ROWS];
    int n;   // steps of the chunk

    __device__ void fetch(piece_t (&v)[ROWS], const E* p, long long ld, int r0, int c, int width) const {
        if constexpr (MODE == PIECES) {
            const uint32_t row = (uint32_t)ld * (uint32_t)sizeof(E);
            const auto rows = __builtin_amdgcn_make_buffer_rsrc(const_cast<E*>(p), 0, (int)(n * row), 0x00027000);
            const uint32_t at = c < width ? (uint32_t)r0 * row + (uint32_t)c * (uint32_t)sizeof(E) : NOWHERE;
#pragma unroll
            for (int q = 0; q < ROWS; ++q)
                v[q] = __builtin_bit_cast(piece_t, __builtin_amdgcn_raw_buffer_load_b128(rows, at + q * row, 0, 0));
            return;
        }
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
            const E* r = p + min(r0 + q, n - 1) * ld;
            if constexpr (MODE == SHIFTED) {
                v[q] = reinterpret_cast<const Loose*>(r + min(c, width - N))->v;
            } else {
#pragma unroll
                for (int i = 0; i < N; ++i) v[q][i] = r[min(c + i, width - 1)];
            }
        }
    }
    // Zeros where nothing is.
    __device__ void settle(piece_t (&v)[ROWS], int r0, int c, int width) const {
        const int by = (int)sizeof(E) * max(0, min(c, width) - (width - N));   // bytes; 16: none of them is there
#pragma unroll
        for (int q = 0; q < ROWS; ++q) {
            const bool on = r0 + q < n;
            if constexpr (MODE == ELEMENTS) {
#pragma unroll
                for (int i = 0; i < N; ++i) v[q][i] = on && c + i < width ? v[q][i] : (E)0.0f;
            } else {
                const unsigned __int128 w = __builtin_bit_cast(unsigned __int128, v[q]);
                v[q] = __builtin_bit_cast(piece_t, on && by < 16 ? w >> (8 * by) : (unsigned __int128)0);
            }
        }
    }
    // PART of a chunk: 0 x, 1 y, 2 z.
    template <int PART>
    __device__ void get(const E* px, const E* py, const E* pz, const Pass& a, int steps) {
        const unsigned id = here();
        const int c = (int)(id % COLS) * N, r0 = (int)(id / COLS) * ROWS;
        n = steps;
        if constexpr (!STATE && PART == 0) fetch(x, px, a.ldx, r0, c, a.P);
        if constexpr (PART == 1) fetch(y, py, a.ldy, r0, c, a.P);
        if constexpr (PART == 2) fetch(z, pz, a.ldz, r0, c, a.R);
    }
    __device__ void settle(const Pass& a) {
        if constexpr (MODE == PIECES) return;
        const unsigned id = here();
        const int c = (int)(id % COLS) * N, r0 = (int)(id / COLS) * ROWS;
        if constexpr (!STATE) settle(x, r0, c, a.P);
        settle(y, r0, c, a.P);
        settle(z, r0, c, a.R);
    }
};

// out's rows 16 it + l from tiles whose lanes hold four columns of a row, from column c on.  WHOLE (fp32; bf16 has its own
// way through LDS): through a descriptor, as Stage fetches.
template <class E, int TI, int RT, bool WHOLE>
__device__ inline void put_rows(E* out, const Pass& a, int n, int c, int l, const f32x4_t (&O)[TI][RT]) {
    static_assert(!WHOLE || sizeof(E) == 4, "a tile's four columns are the 16 bytes of a store");
    const uint32_t row = (uint32_t)a.ldo * (uint32_t)sizeof(E);
    const auto rows = __builtin_amdgcn_make_buffer_rsrc(out, 0, (int)(n * row), 0x00027000);
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
        const int cc = c + 16 * rt;
        const uint32_t to = WHOLE && cc >= a.R ? NOWHERE : (uint32_t)l * row + (uint32_t)cc * (uint32_t)sizeof(E);
#pragma unroll
        for (int it = 0; it < TI; ++it) {
            if constexpr (WHOLE) {
                __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u32x4_t, O[it][rt]), rows, to + it * 16 * row, 0, 0);
            } else if (16 * it + l < n) {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (cc + i < a.R) out[(16 * it + l) * a.ldo + cc + i] = (E)O[it][rt][i];
            }
        }
    }
}

// A lane's decays under the mask, of its wave's tiles of the masked products (one column i a lane,
// four rows j in a register each): a^|i-j| where j is not later than i in the pass's direction, else 0.
template <class E, int DP>
struct Mask {
    static constexpr int W = Chunk<E>::waves(DP), C = Chunk<E>::C;
    static constexpr int IT = C == 64 ? 4 / W : (4 + W - 1) / W, JT = C == 64 ? 4 : 1;
    f32x4_t f[IT][JT];
    __device__ void init(const float* powers, bool back, int w, int l, int g) {
#pragma unroll
        for (int q = 0; q < IT; ++q)
#pragma unroll
            for (int j = 0; j < JT; ++j) {
                // fp32: tile (pair / 2, pair % 2) of pairs w, w + W, ...
                const int pair = (w + q * W) & 3, it = C == 64 ? w * IT + q : pair >> 1, jt = C == 64 ? j : pair & 1;
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int d = (16 * it + l) - (16 * jt + 4 * g + r), dist = back ? -d : d;
                    const float x = powers[max(dist, 0)];
                    f[q][j][r] = dist >= 0 ? x : 0.0f;
                }
            }
    }
};

// A tile under the mask: what it leaves out is zero even where the product was no finite number.
__device__ inline f32x4_t masked(f32x4_t A, f32x4_t f) {
#pragma unroll
    for (int r = 0; r < 4; ++r) A[r] = f[r] != 0.0f ? A[r] * f[r] : 0.0f;
    return A;
}

// --- bf16 ------------------------------------------------------------------

// LDS holds the chunk's rows by steps, each in 16-byte pieces whose places are exchanged within the row: piece k
// of row r lies at k ^ swap_of(r), so that neither a column of pieces over eight rows nor one of pairs of
// pieces over four rows (what the transposing read takes) lies in few banks.  The parts of a row's number
// may be exchanged one by one (swap_of(a ^ b) = swap_of(a) ^ swap_of(b)).  What a lane's numbers
// give (row, exchange and piece together) is formed once and the rest are constants, so that few addresses are kept.
template <int COLS>
__device__ constexpr int swap_of(int row) {
    return COLS >= 8 ? (row & 3) << 1 | (row >> 2 & 1) : (row >> 3 & 1) << 1 | (row >> 2 & 1);
}
template <int COLS>
__device__ inline __bf16* at(__bf16* base, int row, int piece, int lane_swap) {
    return base + row * COLS * 8 + (piece & ~7) * 8 + ((piece & 7) ^ lane_swap) * 8;
}

template <int DP, bool STATE>
struct LdsBf16 {
    // x makes room for the masked products, two parts of 64 x 64, once it has been read
    __bf16 x[STATE ? 8 : (DP > 64 ? 64 * DP : 64 * 128)];
    __bf16 y[64 * DP];
    __bf16 z[64 * DP];
    __bf16 out[STATE ? 8 : 64 * DP];
    float of_x[64], of_z[64], of_state[4];   // what a step's product with the state, what it adds to the state, and the state decay by
};

template <int DP, bool STATE, int MODE>
__device__ inline void put_chunk(LdsBf16<DP, STATE>& s, const Stage<__bf16, DP, STATE, MODE>& g) {
    typedef Stage<__bf16, DP, STATE, MODE> G;
    constexpr int ROWS = G::ROWS, COLS = G::COLS;
    const unsigned id = here();
    const int o = (int)(id % COLS), r0 = (int)(id / COLS) * ROWS, swap = (o & 7) ^ swap_of<COLS>(r0), o8 = (o & ~7) * 8;
#pragma unroll
    for (int q = 0; q < ROWS; ++q) {
        if constexpr (!STATE) *reinterpret_cast<bf16x8_t*>(at<COLS>(s.x + o8, r0 + q, swap_of<COLS>(q), swap)) = g.x[q];
        *reinterpret_cast<bf16x8_t*>(at<COLS>(s.y + o8, r0 + q, swap_of<COLS>(q), swap)) = g.y[q];
        *reinterpret_cast<bf16x8_t*>(at<COLS>(s.z + o8, r0 + q, swap_of<COLS>(q), swap)) = g.z[q];
    }
}

__device__ inline f32x4_t mfma(bf16x8_t a, bf16x8_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
__device__ inline bf16x8_t join(bf16x4_t a, bf16x4_t b) { return __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7); }

// Where a lane reads columns: sixteen lanes read four rows of sixteen columns, and each is given the four
// elements of its column (an LDS read that transposes).  Rows 8 g to 8 g + 7 in two such reads.
// A piece of the masked products [64][64]: piece k of row r at k ^ (r & 7).
__device__ inline __bf16* in_square(__bf16* base, int row, int piece, int lane_swap) {
    return base + row * 64 + (piece ^ lane_swap) * 8;
}
struct Columns {
    int row, swap, half;
    template <int COLS>
    __device__ void init(int l, int g) {
        row = 8 * g + (l >> 2);
        swap = ((l & 3) >> 1) ^ swap_of<COLS>(row);
        half = 4 * (l & 1);
    }
};
// Column l of tile ct (16 columns), rows 32 kb + 8 g + 0 .. 7: an operand's part of a lane.
template <int COLS>
__device__ inline bf16x8_t columns(__bf16* base, const Columns& c, int ct, int kb) {
    typedef short s16x4_t __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4_t* lds_t;
    __bf16* lo = at<COLS>(base + c.half, 32 * kb + c.row, 2 * ct, c.swap);
    __bf16* hi = at<COLS>(base + c.half, 32 * kb + 4 + c.row, (2 * ct) ^ swap_of<COLS>(4), c.swap);
    return join(__builtin_bit_cast(bf16x4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)lo)),
                __builtin_bit_cast(bf16x4_t, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_t)hi)));
}

// One chunk of n steps, out at its first step: what it gives.
template <int DP, bool WHOLE>
__device__ inline void give(LdsBf16<DP, false>& s, const Pass& a, const f32x4_t (&M)[DP / 16][DP / 16 / Chunk<__bf16>::waves(DP)],
                            const Mask<__bf16, DP>& mask, int n, __bf16* out) {
    constexpr int W = Chunk<__bf16>::waves(DP), RT = DP / 16 / W, KB = DP / 32, COLS = DP / 8;
    constexpr int IT = 4 / W;   // a wave's rows of tiles of the masked products
    const int lane = here() & 63, l = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int by_step = g ^ swap_of<COLS>(l), by_half = (g >> 1) ^ swap_of<COLS>(l);
    const int in_a = g ^ (l & 7), half_in_a = (g >> 1) ^ (l & 7);
    // the products under the mask: this wave's steps i against all j, one column i a lane
    f32x4_t A[IT][4];
    const int it0 = w * IT;
#pragma unroll
    for (int q = 0; q < IT; ++q) {
        const int it = it0 + q;
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) A[q][jt] = f32x4_t{0, 0, 0, 0};
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const bf16x8_t b = *reinterpret_cast<const bf16x8_t*>(at<COLS>(s.x, 16 * it + l, 4 * kb, by_step));
#pragma unroll
            for (int jt = 0; jt < 4; ++jt)   // all of them: branches would cost more than the masked tiles
                A[q][jt] = mfma(*reinterpret_cast<const bf16x8_t*>(at<COLS>(s.y, 16 * jt + l, 4 * kb, by_step)), b, A[q][jt]);
        }
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) A[q][jt] = masked(A[q][jt], mask.f[q][jt]);
    }
    __builtin_amdgcn_sched_barrier(0);
    // through the state
    f32x4_t O[4][RT];
#pragma unroll
    for (int it = 0; it < 4; ++it)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) O[it][rt] = f32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int kb = 0; kb < KB; ++kb) {
        bf16x8_t hi[RT], lo[RT];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            u32x4_t h4, l4;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                uint32_t h, o;
                parts(f32x2_t{M[2 * kb + e / 2][rt][2 * e % 4], M[2 * kb + e / 2][rt][2 * e % 4 + 1]}, h, o);
                h4[e] = h;
                l4[e] = o;
            }
            hi[rt] = __builtin_bit_cast(bf16x8_t, h4);
            lo[rt] = __builtin_bit_cast(bf16x8_t, l4);
        }
        bf16x8_t x[4];
#pragma unroll
        for (int it = 0; it < 4; ++it) {
            // rows of M in the order in which a lane holds them
            x[it] = join(*reinterpret_cast<const bf16x4_t*>(at<COLS>(s.x + 4 * (g & 1), 16 * it + l, 4 * kb, by_half)),
                                    *reinterpret_cast<const bf16x4_t*>(at<COLS>(s.x + 4 * (g & 1), 16 * it + l, 4 * kb + 2, by_half)));
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) O[it][rt] = mfma(lo[rt], x[it], O[it][rt]);
        }
#pragma unroll
        for (int it = 0; it < 4; ++it)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) O[it][rt] = mfma(hi[rt], x[it], O[it][rt]);
        __builtin_amdgcn_sched_barrier(0);   // (what is fetched early takes registers that are short)
    }
    __syncthreads();   // x has been read
#pragma unroll
    for (int q = 0; q < IT; ++q)
#pragma unroll
        for (int jt = 0; jt < 4; ++jt) {
            u32x2_t hi, lo;
#pragma unroll
            for (int r = 0; r < 2; ++r) {
                uint32_t h, o;
                parts(f32x2_t{A[q][jt][2 * r], A[q][jt][2 * r + 1]}, h, o);
                hi[r] = h;
                lo[r] = o;
            }
            __bf16* to = in_square(s.x + 4 * (g & 1), 16 * (it0 + q) + l, 2 * jt, half_in_a);
            *reinterpret_cast<u32x2_t*>(to) = hi;
            *reinterpret_cast<u32x2_t*>(to + 64 * 64) = lo;
        }
    __syncthreads();
    Columns c;
    c.init<COLS>(l, g);
    bf16x8_t z[2][RT];
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) z[kb][rt] = columns<COLS>(s.z, c, w * RT + rt, kb);
#pragma unroll
    for (int it = 0; it < 4; ++it) {
        const float f = s.of_x[16 * it + l];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) O[it][rt] *= f;
    }
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int part = 1; part >= 0; --part)
#pragma unroll
            for (int it = 0; it < 4; ++it) {
                const bf16x8_t A8 = *reinterpret_cast<const bf16x8_t*>(in_square(s.x + part * 64 * 64, 16 * it + l, 4 * kb, in_a));
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) O[it][rt] = mfma(z[kb][rt], A8, O[it][rt]);
            }
    if constexpr (!WHOLE) {
        put_rows<__bf16, 4, RT, false>(out, a, n, 16 * w * RT + 4 * g, l, O);
        return;
    }
    // a wave's columns go through LDS into pieces of 16 bytes: stores of 8 bytes, 32 of a row, made a pass
    // over 1 x 32768 x 16 heads of 128 take 180 us instead of 173
    __bf16* mine = s.out + w * 64 * 16 * RT;
#pragma unroll
    for (int it = 0; it < 4; ++it)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const f32x4_t v = O[it][rt];
            const u32x2_t e = {pack(f32x2_t{v[0], v[1]}), pack(f32x2_t{v[2], v[3]})};
            const int row = 16 * it + l, piece = (2 * rt + (g >> 1)) ^ ((l >> 2) & (2 * RT - 1));
            *reinterpret_cast<u32x2_t*>(mine + (row * 2 * RT + piece) * 8 + 4 * (g & 1)) = e;
        }
    constexpr int PER = 2 * RT;   // pieces of a row
    const uint32_t row_bytes = (uint32_t)a.ldo * 2u;
    const auto rows = __builtin_amdgcn_make_buffer_rsrc(out, 0, (int)(n * row_bytes), 0x00027000);
    const int k = lane & (PER - 1), r0 = lane / PER, cc = 16 * w * RT + 8 * k;
    const uint32_t to = cc < a.R ? (uint32_t)r0 * row_bytes + (uint32_t)cc * 2u : NOWHERE;
#pragma unroll
    for (int j = 0; j < PER; ++j) {
        const int row = r0 + j * (64 / PER);
        const u32x4_t v = *reinterpret_cast<const u32x4_t*>(mine + (row * PER + (k ^ ((row >> 2) & (PER - 1)))) * 8);
        __builtin_amdgcn_raw_buffer_store_b128(v, rows, to + (uint32_t)(j * (64 / PER)) * row_bytes, 0, 0);
    }
}

// The same chunk: the state after it. fetch(Part): asks for an operand of the next chunk.
template <int DP, bool STATE, class F>
__device__ inline void carry(LdsBf16<DP, STATE>& s, const Pass& a, f32x4_t (&M)[DP / 16][DP / 16 / Chunk<__bf16>::waves(DP)], F fetch) {
    constexpr int W = Chunk<__bf16>::waves(DP), RT = DP / 16 / W, PT = DP / 16, COLS = DP / 8;
    const int lane = here() & 63, l = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    Columns c;
    c.init<COLS>(l, g);
    const float keep = s.of_state[0];
#pragma unroll
    for (int pt = 0; pt < PT; ++pt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) M[pt][rt] *= keep;
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
        bf16x8_t z1[RT], z2[RT], z3[RT];
        const f32x4_t f0 = *reinterpret_cast<const f32x4_t*>(s.of_z + 32 * kb + 8 * g);
        const f32x4_t f1 = *reinterpret_cast<const f32x4_t*>(s.of_z + 32 * kb + 8 * g + 4);
        const float f[8] = {f0[0], f0[1], f0[2], f0[3], f1[0], f1[1], f1[2], f1[3]};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
            const u32x4_t zz = __builtin_bit_cast(u32x4_t, columns<COLS>(s.z, c, w * RT + rt, kb));
            u32x4_t p1, p2, p3;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const f32x2_t v = unpack(zz[e]) * f32x2_t{f[2 * e], f[2 * e + 1]};
                const uint32_t hi = pack(v);
                uint32_t mid, lo;
                parts(v - unpack(hi), mid, lo);
                p1[e] = hi;
                p2[e] = mid;
                p3[e] = lo;
            }
            z1[rt] = __builtin_bit_cast(bf16x8_t, p1);
            z2[rt] = __builtin_bit_cast(bf16x8_t, p2);
            z3[rt] = __builtin_bit_cast(bf16x8_t, p3);
        }
        // the three parts one after another: a product waits for the one before in its sum
        bf16x8_t y[PT];
        // the next chunk's operands are asked for in between: all at once they would fill the way to memory, and the
        // wave would wait for room
        __builtin_amdgcn_sched_barrier(0);
        if (kb == 0) fetch(Part<0>());
        else fetch(Part<2>());
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int pt = 0; pt < PT; ++pt) {
            y[pt] = columns<COLS>(s.y, c, pt, kb);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) M[pt][rt] = mfma(y[pt], z3[rt], M[pt][rt]);
        }
#pragma unroll
        for (int pt = 0; pt < PT; ++pt)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) M[pt][rt] = mfma(y[pt], z2[rt], M[pt][rt]);
        if (kb == 0) {
            __builtin_amdgcn_sched_barrier(0);
            fetch(Part<1>());
            __builtin_amdgcn_sched_barrier(0);
        }
#pragma unroll
        for (int pt = 0; pt < PT; ++pt)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) M[pt][rt] = mfma(y[pt], z1[rt], M[pt][rt]);
    }
}

// --- fp32 ------------------------------------------------------------------

template <int DP, bool STATE>
struct LdsF32 {
    static constexpr int LD = DP + 4;
    float x[STATE ? 4 : 32 * LD];
    float y[32 * LD];
    float z[32 * LD];
    float a[STATE ? 4 : 32 * 36];
    float of_x[32], of_z[32], of_state[4];
};

template <int DP, bool STATE, int MODE>
__device__ inline void put_chunk(LdsF32<DP, STATE>& s, const Stage<float, DP, STATE, MODE>& g) {
    typedef Stage<float, DP, STATE, MODE> G;
    constexpr int LD = LdsF32<DP, STATE>::LD;
    const int c = ((int)threadIdx.x % G::COLS) * 4, r0 = ((int)threadIdx.x / G::COLS) * G::ROWS;
#pragma unroll
    for (int q = 0; q < G::ROWS; ++q) {
        if constexpr (!STATE) *reinterpret_cast<f32x4_t*>(s.x + (r0 + q) * LD + c) = g.x[q];
        *reinterpret_cast<f32x4_t*>(s.y + (r0 + q) * LD + c) = g.y[q];
        *reinterpret_cast<f32x4_t*>(s.z + (r0 + q) * LD + c) = g.z[q];
    }
}

__device__ inline f32x4_t mfma(float a, float b, f32x4_t c) { return __builtin_amdgcn_mfma_f32_16x16x4f32(a, b, c, 0, 0, 0); }

template <int DP, bool WHOLE>
__device__ inline void give(LdsF32<DP, false>& s, const Pass& a, const f32x4_t (&M)[DP / 16][DP / 16 / Chunk<float>::waves(DP)],
                            const Mask<float, DP>& mask, int n, float* out) {
    constexpr int W = Chunk<float>::waves(DP), RT = DP / 16 / W, PT = DP / 16, LD = LdsF32<DP, false>::LD;
    const int lane = here() & 63, l = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
#pragma unroll
    for (int pair = 0; pair < 4; ++pair) {
        if (pair % W != w) continue;
        const int it = pair >> 1, jt = pair & 1;
        f32x4_t A = {0, 0, 0, 0}, A2 = {0, 0, 0, 0};   // two, since a product waits for the one before in its sum
#pragma unroll
        for (int pt = 0; pt < PT; ++pt) {
            const f32x4_t y = *reinterpret_cast<const f32x4_t*>(s.y + (16 * jt + l) * LD + 16 * pt + 4 * g);
            const f32x4_t x = *reinterpret_cast<const f32x4_t*>(s.x + (16 * it + l) * LD + 16 * pt + 4 * g);
#pragma unroll
            for (int r = 0; r < 4; r += 2) {
                A = mfma(y[r], x[r], A);
                A2 = mfma(y[r + 1], x[r + 1], A2);
            }
        }
        A += A2;
        A = masked(A, mask.f[pair / W][0]);
        *reinterpret_cast<f32x4_t*>(s.a + (16 * it + l) * 36 + 16 * jt + 4 * g) = A;
    }
    __syncthreads();
    float z[2][RT][4];
#pragma unroll
    for (int jt = 0; jt < 2; ++jt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) z[jt][rt][r] = s.z[(16 * jt + 4 * g + r) * LD + 16 * (w * RT + rt) + l];
    f32x4_t O[2][RT];
#pragma unroll
    for (int it = 0; it < 2; ++it)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) O[it][rt] = f32x4_t{0, 0, 0, 0};
#pragma unroll
    for (int pt = 0; pt < PT; ++pt) {
        f32x4_t x[2];
#pragma unroll
        for (int it = 0; it < 2; ++it) x[it] = *reinterpret_cast<const f32x4_t*>(s.x + (16 * it + l) * LD + 16 * pt + 4 * g);
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) O[it][rt] = mfma(M[pt][rt][r], x[it][r], O[it][rt]);
    }
    f32x4_t A[2][2];
#pragma unroll
    for (int it = 0; it < 2; ++it) {
        const int i = 16 * it + l;
        const float f = s.of_x[i];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) O[it][rt] *= f;
#pragma unroll
        for (int jt = 0; jt < 2; ++jt) A[it][jt] = *reinterpret_cast<const f32x4_t*>(s.a + i * 36 + 16 * jt + 4 * g);
    }
#pragma unroll
    for (int jt = 0; jt < 2; ++jt)
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int it = 0; it < 2; ++it)
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) O[it][rt] = mfma(z[jt][rt][r], A[it][jt][r], O[it][rt]);
    put_rows<float, 2, RT, WHOLE>(out, a, n, 16 * w * RT + 4 * g, l, O);
}

template <int DP, bool STATE>
__device__ inline void carry(LdsF32<DP, STATE>& s, const Pass& a, f32x4_t (&M)[DP / 16][DP / 16 / Chunk<float>::waves(DP)]) {
    constexpr int W = Chunk<float>::waves(DP), RT = DP / 16 / W, PT = DP / 16, LD = LdsF32<DP, STATE>::LD;
    const int lane = here() & 63, l = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    float z[2][RT][4];
#pragma unroll
    for (int jt = 0; jt < 2; ++jt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r) z[jt][rt][r] = s.z[(16 * jt + 4 * g + r) * LD + 16 * (w * RT + rt) + l];
    const float keep = s.of_state[0];
#pragma unroll
    for (int pt = 0; pt < PT; ++pt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) M[pt][rt] *= keep;
#pragma unroll
    for (int jt = 0; jt < 2; ++jt)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            const int j = 16 * jt + 4 * g + r;
            const float f = s.of_z[j];
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) z[jt][rt][r] *= f;
#pragma unroll
            for (int pt = 0; pt < PT; ++pt) {
                const float y = s.y[j * LD + 16 * pt + l];
#pragma unroll
                for (int rt = 0; rt < RT; ++rt) M[pt][rt] = mfma(y, z[jt][rt][r], M[pt][rt]);
            }
        }
}

template <class E, int DP, bool STATE>
struct LdsOf { typedef LdsBf16<DP, STATE> type; };
template <int DP, bool STATE>
struct LdsOf<float, DP, STATE> { typedef LdsF32<DP, STATE> type; };

// --- the passes ----------------------------------------------------------------

// STATE: what each share adds to the state, alone.
template <class E, int DP, bool STATE, int MODE>
__global__ void __launch_bounds__(64 * Chunk<E>::waves(DP), Chunk<E>::per_unit(DP)) attend_kernel(AttendParams p) {
    constexpr int C = Chunk<E>::C, W = Chunk<E>::waves(DP), RT = DP / 16 / W, PT = DP / 16;
    __shared__ typename LdsOf<E, DP, STATE>::type s;
    // the passes of one share, which read the same rows, go to one chiplet (eight in turn) one after another
    // (quotients are formed by the vector unit: made scalar again, so that what follows from them is)
    auto scalar = [](unsigned x) { return (unsigned)__builtin_amdgcn_readfirstlane((int)x); };
    const unsigned eight = blockIdx.x / 8u, turn = scalar(eight / (unsigned)p.passes);
    const unsigned item = turn * 8u + blockIdx.x % 8u;
    if (item >= (unsigned)p.rows * (unsigned)p.shares) return;
    const Pass& a = p.pass[eight - turn * (unsigned)p.passes];
    // (first shares first: of sequences of different lengths the later ones are empty, and a CU's groups, far
    // apart in this order, are not all early ones)
    const int share = (int)scalar(item / (unsigned)p.rows), row = (int)(item - (unsigned)share * (unsigned)p.rows);
    const int b = (int)scalar((unsigned)row / (unsigned)p.heads), head = row - b * p.heads;
    const int lane = threadIdx.x & 63, l = lane & 15, g = lane >> 4;
    const int w = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int given = p.lengths[b * p.length_step], L = max(0, min(given, p.T));
    const int t0 = share * p.span, span = min(p.span, p.T - t0);
    const int len = max(0, min(L - t0, span));
    const int used = shares_used(L, p.span);
    if (STATE && !adds(share, used, a.back)) return;

    const float* powers = p.powers + head * TABLE;
    // (a chunk of n steps: rows that are not there are zeros, whatever they decay by)
    auto decays = [&](int n) {
        for (int i = threadIdx.x; i < C; i += 64 * W) {
            s.of_x[i] = powers[a.back ? max(n - 1 - i, 0) : i + 1];
            s.of_z[i] = powers[a.back ? i + 1 : max(n - 1 - i, 0)];
        }
        if (threadIdx.x == 0) s.of_state[0] = powers[n];
    };
    const long long step0 = (long long)b * p.T + t0;
    const E* px = static_cast<const E*>(a.x) + step0 * a.ldx + head * a.P;
    const E* py = static_cast<const E*>(a.y) + step0 * a.ldy + head * a.P;
    const E* pz = static_cast<const E*>(a.z) + step0 * a.ldz + head * a.R;
    E* out = STATE ? nullptr : static_cast<E*>(a.out) + step0 * a.ldo + head * a.R;

    // All that comes before the first chunk is on its way before any of it is looked at: a share may be a chunk alone.
    const int chunks = (len + C - 1) / C;
    Stage<E, DP, STATE, MODE> stage;
    auto chunk_of = [&](int c) { return a.back ? chunks - 1 - c : c; };
    auto fetch = [&](int c, auto part) {
        // (behind the last chunk: through descriptors of no rows, otherwise the last one again)
        const int k = chunk_of(min(c, chunks - 1)) * C;
        stage.template get<decltype(part)::value>(px + k * a.ldx, py + k * a.ldy, pz + k * a.ldz, a,
                                                  MODE == PIECES && c == chunks ? 0 : min(C, len - k));
    };
    auto fetch_all = [&](int c) {
        fetch(c, Part<0>());
        fetch(c, Part<1>());
        fetch(c, Part<2>());
    };
    if (chunks) fetch_all(0);
    f32x4_t M[PT][RT];
    const int PR = a.P * a.R;
    const Start from = start_of(share, used);
    const float* start = from == Start::SLOT            ? a.share + ((long long)row * p.shares + share) * PR
                         : from == Start::GIVEN && a.start ? a.start + (long long)row * PR
                                                           : nullptr;
    const int step_i = a.transposed ? 1 : p.Dv, step_c = a.transposed ? p.Dv : 1;
#pragma unroll
    for (int pt = 0; pt < PT; ++pt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) M[pt][rt] = f32x4_t{0, 0, 0, 0};
    if (!STATE && start) {
#pragma unroll
        for (int pt = 0; pt < PT; ++pt)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = min(16 * pt + 4 * g + r, a.P - 1), c = min(16 * (w * RT + rt) + l, a.R - 1);
                    M[pt][rt][r] = start[i * step_i + c * step_c];
                }
    }
    Mask<E, DP> mask;
    if constexpr (!STATE) mask.init(powers, a.back, w, l, g);
    decays(C);
#pragma unroll
    for (int pt = 0; pt < PT; ++pt)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
            for (int r = 0; r < 4; ++r)
                if (16 * pt + 4 * g + r >= a.P || 16 * (w * RT + rt) + l >= a.R) M[pt][rt][r] = 0.0f;
    float* end = STATE ? a.share + ((long long)row * p.shares + share) * PR : a.end ? a.end + (long long)row * PR : nullptr;
    if (!STATE && !ends_row(share, used, a.back)) end = nullptr;

    for (int c = 0; c < chunks; ++c) {
        const int k = chunk_of(c) * C;
        const int n = min(C, len - k);
        // only the last chunk of a row may be shorter: the first that is gone through, or the last
        if (n < C || (a.back && c == 1)) decays(n);
        stage.settle(a);
        put_chunk(s, stage);
        __syncthreads();
        // A state that is neither read again nor kept is not formed. (carry fetches nothing else from memory: it would
        // wait for all of the next chunk.)
        const bool carried = c + 1 < chunks || end;
        if constexpr (C == 64) {
            // (a wave at its outputs comes before one at its state; so they alternate better, 3 to 4%)
            if constexpr (!STATE) {
                __builtin_amdgcn_s_setprio(1);
                give<DP, MODE == PIECES>(s, a, M, mask, n, out + k * a.ldo);
                __builtin_amdgcn_s_setprio(0);
            }
            if (carried) carry<DP, STATE>(s, a, M, [&](auto part) { fetch(c + 1, part); });
        } else {
            if constexpr (!STATE) give<DP, MODE == PIECES>(s, a, M, mask, n, out + k * a.ldo);
            if (c + 1 < chunks) fetch_all(c + 1);   // (here, where few registers are in use)
            if (carried) carry<DP, STATE>(s, a, M);
        }
        __syncthreads();
    }

    if (end) {
#pragma unroll
        for (int pt = 0; pt < PT; ++pt)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int i = 16 * pt + 4 * g + r, c = 16 * (w * RT + rt) + l;
                    if (i < a.P && c < a.R) end[i * step_i + c * step_c] = M[pt][rt][r];
                }
    }
    if constexpr (!STATE) {
        // (here and not above: in a branch of some lanes, what follows it would be taken for lanes' own)
        if (given != L && head == 0 && share == 0 && threadIdx.x == 0) atomicOr(p.status, STATUS_BAD_LENGTHS);
        // rows past the length: zeros
        const int c = threadIdx.x % DP;
        if (c < a.R)
            for (int i = len + (int)threadIdx.x / DP; i < span; i += 64 * W / DP) out[i * a.ldo + c] = (E)0.0f;
    }
}

// The states that a row's shares start from: what share k adds to the state lies in its slot until it has been read, and
// its start takes that place.
__global__ void __launch_bounds__(256) attend_join_kernel(AttendParams p) {
    const Pass& a = p.pass[blockIdx.z];
    const int row = blockIdx.y, PR = a.P * a.R, e = blockIdx.x * 256 + threadIdx.x;
    if (e >= PR) return;
    const int b = row / p.heads, head = row % p.heads;
    const int L = clamp_length(p.lengths[b * p.length_step], p.T, p.status, false);
    const int used = shares_used(L, p.span);
    if (used < 2) return;
    float* share = a.share + (long long)row * p.shares * PR + e;
    float state = a.start ? a.start[(long long)row * PR + e] : 0.0f;
    // all shares are whole but for the last of the row
    const float whole = (float)power(p.log2a, head, p.span);
    const float part = a.back ? (float)power(p.log2a, head, L - (used - 1) * p.span) : whole;
    constexpr int AT_ONCE = 8;   // fetched before the first is used
    auto place = [&](int i) { return share + (long long)(a.back ? used - 1 - i : i) * PR; };
    float add = *place(0);
    *place(0) = state;
    for (int i0 = 1; i0 < used; i0 += AT_ONCE) {
        float next[AT_ONCE];   // (of the last share, whatever lies there: it is not used)
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) next[j] = *place(min(i0 + j, used - 1));
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            if (i0 + j >= used) break;
            state = (i0 + j == 1 ? part : whole) * state + add;
            *place(i0 + j) = state;
            add = next[j];
        }
    }
}

// --- one step --------------------------------------------------------------------

struct StepParams {
    const void* z;
    const float* S;
    float* out_S;
    void* out_y;
    const float* powers;
    int heads, Dk, Dv;
};

// A workgroup holds one head of one row; V columns of the state a lane.
template <class E, int V>
__global__ void __launch_bounds__(256) attend_step_kernel(StepParams a) {
    __shared__ float kq[2][MAX_D], y[256 * V];
    const long long n = blockIdx.x, row = n / a.heads;
    const int head = (int)(n % a.heads), Dk = a.Dk, Dv = a.Dv;
    const E* z = static_cast<const E*>(a.z) + row * a.heads * (2 * Dk + Dv);
    for (int i = threadIdx.x; i < 2 * Dk; i += 256)
        kq[i >= Dk][i >= Dk ? i - Dk : i] = (float)z[(i >= Dk ? a.heads * Dk + i - Dk : i) + head * Dk];
    __syncthreads();
    const float decay = a.powers[head * TABLE + 1];
    const int cols = (Dv + V - 1) / V, groups = 256 / cols;
    const int col = threadIdx.x % cols, group = threadIdx.x / cols, c = col * V;
    float sum[V];
#pragma unroll
    for (int j = 0; j < V; ++j) sum[j] = 0.0f;
    if (group < groups) {
        float v[V];
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (float)z[2 * a.heads * Dk + head * Dv + c + j];
        const float* S = a.S + n * Dk * Dv + c;
        float* O = a.out_S + n * Dk * Dv + c;
#pragma unroll 4
        for (int i = group; i < Dk; i += groups) {
            float s[V];
            load_vec<float, V>(S + i * Dv, s);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                s[j] = decay * s[j] + kq[1][i] * v[j];
                sum[j] += kq[0][i] * s[j];
            }
            store_vec<float, V>(O + i * Dv, s);
        }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) y[threadIdx.x * V + j] = sum[j];
    __syncthreads();
    E* out = static_cast<E*>(a.out_y) + n * Dv;
    for (int e = threadIdx.x; e < Dv; e += 256) {
        float t = 0.0f;
        for (int k = 0; k < groups; ++k) t += y[(k * cols) * V + e];
        out[e] = (E)t;
    }
}

// --- host ----------------------------------------------------------------------

int check_sizes(int B, int heads, int Dk, int Dv, int T, int dtype, const float* decay) {
    if (B < 1 || heads < 1 || Dk < 1 || Dv < 1 || T < 1 || !valid_dtype(dtype) || !decay) return LSTM_DYN_ERR_INVALID;
    if (Dk > MAX_D || Dv > MAX_D || heads > MAX_HEADS || (long long)B * heads >= 1 << 20 || (long long)B * T >= 1LL << 31 || T >= 1 << 30)
        return LSTM_DYN_ERR_UNSUPPORTED;
    for (int i = 0; i < heads; ++i)
        if (!(decay[i] >= 0.0f && decay[i] <= 1.0f)) return LSTM_DYN_ERR_INVALID;
    return LSTM_DYN_OK;
}

int check_buffers(int B, int heads, int Dk, int Dv, int T, int dtype, const void* z, const int32_t* lengths,
                  const float* S0, const float* out_S, const void* out_y, const void* dy, const float* d_out_S,
                  const void* dz, const float* dS0) {
    const int e = dtype_bytes(dtype);
    const long long nz = (long long)B * T * heads * (2 * Dk + Dv) * e, ny = (long long)B * T * heads * Dv * e;
    const long long ns = 4LL * B * heads * Dk * Dv;
    Span s[8];
    int k = 0;
    s[k++] = Span{z, nz, e, false};
    s[k++] = Span{S0, ns, 4, false};
    if (lengths) s[k++] = Span{lengths, 4LL * B, 4, false};
    if (!dy && !dz && !dS0) {
        s[k++] = Span{out_S, ns, 4, true, S0};
        s[k++] = Span{out_y, ny, e, true};
    } else {
        s[k++] = Span{dy, ny, e, false};
        if (d_out_S) s[k++] = Span{d_out_S, ns, 4, false};
        s[k++] = Span{dz, nz, e, true};
        s[k++] = Span{dS0, ns, 4, true};
    }
    return check_spans(s, k);
}

}  // namespace
}  // namespace ldyn

using namespace ldyn;

struct lstm_dyn_attend : OpsHandle {
    int B = 0, heads = 0, Dk = 0, Dv = 0, T = 0, dtype = 0;
    int shares = 1, span = 0;
    const int32_t* whole = nullptr;   // T
    const float* powers = nullptr;
    const double* log2a = nullptr;
    float* share = nullptr;   // [2][B heads][shares][Dk][Dv]: going forward, going back
    long long share_floats() const { return (long long)B * heads * shares * Dk * Dv; }
};

extern "C" int lstm_dyn_check_attend_args(int B, int heads, int Dk, int Dv, int T, int dtype, const float* decay,
                                          const void* z, const int32_t* lengths, const float* S0, const float* out_S,
                                          const void* out_y, const void* dy, const float* d_out_S, const void* dz,
                                          const float* dS0) {
    const int rc = check_sizes(B, heads, Dk, Dv, T, dtype, decay);
    if (rc != LSTM_DYN_OK || !z) return rc;
    return check_buffers(B, heads, Dk, Dv, T, dtype, z, lengths, S0, out_S, out_y, dy, d_out_S, dz, dS0);
}

static int attend_make(lstm_dyn_attend* h, const float* decay) {
    // As many shares as bring the workgroups that bf16 calls have on the device at once (two a CU of 128 columns, four of
    // 64), since a share costs a second reading of two operands and its states; with fp32 data, where two workgroups
    // of 128 columns would fit, 256 by measurement at all widths.  From 256
    // rows and heads on, which fill the device by themselves, a share has to be 16 chunks: below, the
    // states cost more than the even load gains.  us, calls one after another in a graph, by the number of workgroups:
    //                                                      256    512   1024   2048
    //   bf16   1 x 32768 x 16 heads of 128, forward        276    235    255    306   (512 taken)
    //          8 x 4096 x 16 of 128, ragged, training      766    674    738    848   (512)
    //          16 x 4096 x 16 of 64, forward               208    190    214    212   (1024, as the next four)
    //          the same, ragged                            204    182    172
    //          the same, ragged, training                  485    511    525
    //          2 x 4096 x 8 of 64, forward                  31     31     37
    //          2 x 4096 x 8 of 32, training                 58     59     65
    //   fp32   4 x 1024 x 8 of 128, training               194    219    286    286   (256, as the others)
    //          4 x 1024 x 8 of 64, training                 82     86    101    102
    //          4 x 1024 x 8 of 32, training                 53     50     54     54
    //          1 x 4096 x 4 of 64, training                 67     79     80     80
    //          16 x 1024 x 8 of 64, training               234    221    223    255
    // (Heads of 64 and less take 512 better, by 3 to 18%, but for the ragged forward.)  The last rule: training steps of 32 x 512 x 8 heads of 64, 72 and 130 without it.  Four chunks and more a share: 5 x 301 x 3 heads in
    // fp32, 110 and 53 without.
    const int C = h->dtype == LSTM_DYN_BF16 ? Chunk<__bf16>::C : Chunk<float>::C;
    const int groups = h->dtype != LSTM_DYN_BF16 ? 256 : h->Dk > 64 || h->Dv > 64 ? 512 : 1024;
    const int rows = h->B * h->heads, chunks = (h->T + C - 1) / C;
    const int want = rows >= groups ? 1 : (groups + rows - 1) / rows;
    int each = (chunks + want - 1) / want;
    if (rows >= 256 && each < 16) each = 16;
    h->shares = (chunks + each - 1) / each;
    h->span = each * C;
    std::vector<float> powers((size_t)h->heads * TABLE);
    std::vector<double> logs((size_t)h->heads);
    for (int i = 0; i < h->heads; ++i) {
        const double a = (double)decay[i];
        for (int n = 0; n < TABLE; ++n) powers[(size_t)i * TABLE + n] = (float)std::pow(a, n);
        logs[(size_t)i] = a > 0.0 ? std::log2(a) : -1e9;
    }
    const long long np = (4LL * (long long)powers.size() + 255) / 256 * 256, nl = (8LL * h->heads + 255) / 256 * 256;
    const long long ns = h->shares > 1 ? 8 * h->share_floats() : 0;
    int rc = ops_device(h);
    if (rc != LSTM_DYN_OK || (rc = ops_init(h, 256 + np + nl + ns)) != LSTM_DYN_OK) return rc;
    h->whole = reinterpret_cast<const int32_t*>(h->block + 64);
    h->powers = reinterpret_cast<const float*>(h->block + 256);
    h->log2a = reinterpret_cast<const double*>(h->block + 256 + np);
    h->share = reinterpret_cast<float*>(h->block + 256 + np + nl);
    if (hipMemcpy(h->block + 64, &h->T, 4, hipMemcpyHostToDevice) != hipSuccess ||
        hipMemcpy(h->block + 256, powers.data(), 4 * powers.size(), hipMemcpyHostToDevice) != hipSuccess ||
        hipMemcpy(h->block + 256 + np, logs.data(), 8 * logs.size(), hipMemcpyHostToDevice) != hipSuccess) {
        (void)hipGetLastError();
        (void)ops_free(h);
        return LSTM_DYN_ERR_HIP;
    }
    return LSTM_DYN_OK;
}

extern "C" int lstm_dyn_attend_create(lstm_dyn_attend_t** out, int B, int heads, int Dk, int Dv, int T, int dtype,
                                      const float* decay) {
    if (!out) return LSTM_DYN_ERR_INVALID;
    *out = nullptr;
    const int ok = check_sizes(B, heads, Dk, Dv, T, dtype, decay);
    if (ok != LSTM_DYN_OK) return ok;
    lstm_dyn_attend* h = nullptr;
    try {
        h = new lstm_dyn_attend();
        h->B = B;
        h->heads = heads;
        h->Dk = Dk;
        h->Dv = Dv;
        h->T = T;
        h->dtype = dtype;
        const int rc = attend_make(h, decay);
        if (rc != LSTM_DYN_OK) {
            delete h;
            return rc;
        }
    } catch (...) {
        delete h;
        return LSTM_DYN_ERR_NOMEM;
    }
    *out = h;
    return LSTM_DYN_OK;
}

template <class E, bool STATE, int MODE>
static int launch_mode(lstm_dyn_attend* h, const AttendParams& p) {
    const int d = h->Dk > h->Dv ? h->Dk : h->Dv;
    const long long items = (long long)p.rows * p.shares, grid = (items + 7) / 8 * 8 * p.passes;
    if (d <= 32)
        hipLaunchKernelGGL((attend_kernel<E, 32, STATE, MODE>), dim3((unsigned)grid), dim3(64 * Chunk<E>::waves(32)), 0, h->last_stream, p);
    else if (d <= 64)
        hipLaunchKernelGGL((attend_kernel<E, 64, STATE, MODE>), dim3((unsigned)grid), dim3(64 * Chunk<E>::waves(64)), 0, h->last_stream, p);
    else
        hipLaunchKernelGGL((attend_kernel<E, 128, STATE, MODE>), dim3((unsigned)grid), dim3(64 * Chunk<E>::waves(128)), 0, h->last_stream, p);
    return ops_launched(h);
}
template <class E, bool STATE>
static int launch_pass(lstm_dyn_attend* h, const AttendParams& p) {
    return p.mode == PIECES    ? launch_mode<E, STATE, PIECES>(h, p)
           : p.mode == SHIFTED ? launch_mode<E, STATE, SHIFTED>(h, p)
                               : launch_mode<E, STATE, ELEMENTS>(h, p);
}

// The shares' starts for passes `state`, then passes `p`.
static int run_passes(lstm_dyn_attend* h, const AttendParams& state, const AttendParams& p) {
    int rc;
    const bool bf16 = h->dtype == LSTM_DYN_BF16;
    if (h->shares > 1) {
        if ((rc = bf16 ? launch_pass<__bf16, true>(h, state) : launch_pass<float, true>(h, state)) != LSTM_DYN_OK) return rc;
        hipLaunchKernelGGL(attend_join_kernel, dim3((unsigned)((h->Dk * h->Dv + 255) / 256), (unsigned)p.rows, (unsigned)state.passes),
                           dim3(256), 0, h->last_stream, state);
        if ((rc = ops_launched(h)) != LSTM_DYN_OK) return rc;
    }
    return bf16 ? launch_pass<__bf16, false>(h, p) : launch_pass<float, false>(h, p);
}

// Addresses of q, k and v (or their gradients) in z.
struct Parts {
    char *q, *k, *v;
    long long ld;
    Parts(const lstm_dyn_attend* h, const void* z) {
        const long long e = dtype_bytes(h->dtype);
        q = static_cast<char*>(const_cast<void*>(z));
        k = q + e * h->heads * h->Dk;
        v = k + e * h->heads * h->Dk;
        ld = (long long)h->heads * (2 * h->Dk + h->Dv);
    }
};

static AttendParams attend_params(const lstm_dyn_attend* h, const int32_t* lengths) {
    AttendParams p{};
    p.lengths = lengths ? lengths : h->whole;
    p.length_step = lengths ? 1 : 0;
    p.status = h->status();
    p.powers = h->powers;
    p.log2a = h->log2a;
    p.T = h->T;
    p.heads = h->heads;
    p.rows = h->B * h->heads;
    p.shares = h->shares;
    p.span = h->span;
    p.Dv = h->Dv;
    return p;
}

// How every head's rows of these buffers lie.
static int mode_of(const lstm_dyn_attend* h, const void* a, const void* b, const void* c) {
    const int n = 16 / dtype_bytes(h->dtype);
    const uintptr_t low = reinterpret_cast<uintptr_t>(a) | reinterpret_cast<uintptr_t>(b) | reinterpret_cast<uintptr_t>(c);
    if (h->Dk % n == 0 && h->Dv % n == 0 && (low & 15) == 0) return PIECES;
    return h->Dk >= n && h->Dv >= n ? SHIFTED : ELEMENTS;
}

extern "C" int lstm_dyn_attend_forward(lstm_dyn_attend_t* h, const void* z, const int32_t* lengths, const float* S0,
                                       float* out_S, void* out_y, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc = check_buffers(h->B, h->heads, h->Dk, h->Dv, h->T, h->dtype, z, lengths, S0, out_S, out_y, nullptr, nullptr,
                           nullptr, nullptr);
    if (rc != LSTM_DYN_OK || (rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const Parts in(h, z);
    AttendParams p = attend_params(h, lengths);
    p.passes = 1;
    p.mode = mode_of(h, z, out_y, nullptr);
    p.pass[0] = Pass{in.q, in.k, in.v, out_y, in.ld, in.ld, in.ld, (long long)h->heads * h->Dv, h->Dk, h->Dv, 0, 0, S0,
                     out_S, h->share};
    return run_passes(h, p, p);
}

extern "C" int lstm_dyn_attend_backward(lstm_dyn_attend_t* h, const void* z, const int32_t* lengths, const float* S0,
                                        const void* dy, const float* d_out_S, void* dz, float* dS0, void* stream) {
    if (!h || !dz) return LSTM_DYN_ERR_INVALID;
    int rc = check_buffers(h->B, h->heads, h->Dk, h->Dv, h->T, h->dtype, z, lengths, S0, nullptr, nullptr, dy, d_out_S,
                           dz, dS0);
    if (rc != LSTM_DYN_OK || (rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const Parts in(h, z), out(h, dz);
    const long long ld = in.ld, ly = (long long)h->heads * h->Dv;
    float *fw = h->share, *bw = h->share + (h->shares > 1 ? h->share_floats() : 0);
    AttendParams p = attend_params(h, lengths);
    p.mode = mode_of(h, z, dy, dz);
    AttendParams state = p;
    state.passes = 2;
    state.pass[0] = Pass{nullptr, in.k, in.v, nullptr, 0, ld, ld, 0, h->Dk, h->Dv, 0, 0, S0, nullptr, fw};
    state.pass[1] = Pass{nullptr, in.q, dy, nullptr, 0, ld, ly, 0, h->Dk, h->Dv, 1, 0, d_out_S, nullptr, bw};
    p.passes = 3;
    p.pass[0] = Pass{dy, in.v, in.k, out.q, ly, ld, ld, ld, h->Dv, h->Dk, 0, 1, S0, nullptr, fw};
    p.pass[1] = Pass{in.v, dy, in.q, out.k, ld, ly, ld, ld, h->Dv, h->Dk, 1, 1, d_out_S, nullptr, bw};
    p.pass[2] = Pass{in.k, in.q, dy, out.v, ld, ld, ly, ld, h->Dk, h->Dv, 1, 0, d_out_S, dS0, bw};
    return run_passes(h, state, p);
}

extern "C" int lstm_dyn_attend_step(lstm_dyn_attend_t* h, int rows, const void* z, const float* S, float* out_S,
                                    void* out_y, void* stream) {
    if (!h || rows < 1) return LSTM_DYN_ERR_INVALID;
    const long long n = (long long)rows * h->heads;
    if (n >= 1LL << 24) return LSTM_DYN_ERR_UNSUPPORTED;
    const int e = dtype_bytes(h->dtype);
    const long long ns = 4 * n * h->Dk * h->Dv;
    const Span s[4] = {{z, n * (2 * h->Dk + h->Dv) * e, e, false}, {S, ns, 4, false}, {out_S, ns, 4, true, S},
                       {out_y, n * h->Dv * e, e, true}};
    int rc = check_spans(s, 4);
    if (rc != LSTM_DYN_OK || (rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const StepParams a{z, S, out_S, out_y, h->powers, h->heads, h->Dk, h->Dv};
    const bool four = h->Dv % 4 == 0 && ((reinterpret_cast<uintptr_t>(S) | reinterpret_cast<uintptr_t>(out_S)) & 15) == 0;
    auto* k = h->dtype == LSTM_DYN_BF16 ? (four ? attend_step_kernel<__bf16, 4> : attend_step_kernel<__bf16, 1>)
                                        : (four ? attend_step_kernel<float, 4> : attend_step_kernel<float, 1>);
    hipLaunchKernelGGL(k, dim3((unsigned)n), dim3(256), 0, h->last_stream, a);
    return ops_launched(h);
}

extern "C" int lstm_dyn_attend_query(lstm_dyn_attend_t* h, int what, long long* value) {
    return ops_query(h, what, value);
}

extern "C" int lstm_dyn_attend_destroy(lstm_dyn_attend_t* h) {
    if (!h) return LSTM_DYN_OK;
    const int rc = ops_free(h);
    delete h;
    return rc;
}
