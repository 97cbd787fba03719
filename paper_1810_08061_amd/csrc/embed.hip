// embed.hip -- rows of a token table as the loop's input, and the gradient of
// the table by sorted tokens.
//
//   x[b][t] = scale table[tok[b][t]] (t < L[b], else 0)
//   d_table[v] = scale sum_{(b, t): tok = v} dx[b][t]
//
// The gradient: a stable radix sort of the places n = b T + t by token (places
// past a length or with a bad token sort last, as token V), then sums over
// pieces of R sorted places.  A token whose places lie inside one piece is
// written at once; of the others each piece leaves a partial sum, joined
// afterwards in the pieces' order.  No atomics on the sums, so the same sizes
// give the same bits.  Rows of tokens that do not occur are found by a stamp
// per token and written with zeros.
//
// Bound by memory: the lookup by the rows it writes (256 x 1000 x 1024 in bf16, half of it
// past lengths: 138 us, 4.8 TB/s), the sums by dx and d_table (65536 x 1024 from fp32:
// 164 us, 4.8 TB/s; a wave holds 256 columns of eight places at a time).  The sort
// (256000 places, two digits of nine bits: 49 us) and the join (20 us) come on top; a
// small batch (945 places) is four launches, 19 us, of which the sort is 7.
#include "ops.h"

namespace ldyn {
namespace {

constexpr int SORT_THREADS = 512, SORT_WAVES = SORT_THREADS / 64, SORT_ITEMS = 8;
constexpr int SORT_TILE = SORT_THREADS * SORT_ITEMS;  // places ranked at once
constexpr int SORT_BITS = 9, SORT_BINS = 1 << SORT_BITS;
constexpr int SORT_BLOCKS = 256;  // at most; each reads the counts of all
static_assert(SORT_BINS == SORT_THREADS, "a thread per digit");

constexpr long long FAR_BYTES = 256LL << 20;  // of x; see the launch

struct EmbedParams {
    const int32_t* tokens;
    const int32_t* lengths;
    int32_t* status;
    uint32_t* epoch;   // bumped once per gradient
    uint32_t* stamp;   // [V] the epoch of the last gradient that saw the token
    uint32_t* hist;    // [blocks][bins]
    float* part;       // [pieces][2][D]
    int N, T, V, D;
    float scale;
};

// The sort key of place n: its token, or V.  Length and token are loaded side
// by side: the token of a place past the length lies in the array all the same.
__device__ inline uint32_t key_of(const EmbedParams& p, int n, bool report) {
    const int b = n / p.T, t = n - b * p.T;
    const int tok = p.tokens[n];
    const int L = row_length(p.lengths, b, p.T, p.status, report && t == 0);
    if (t >= L) return (uint32_t)p.V;
    if ((unsigned)tok < (unsigned)p.V) return (uint32_t)tok;
    if (report) atomicOr(p.status, STATUS_BAD_TOKENS);
    return (uint32_t)p.V;
}

// --- lookup: one wave per row ---------------------------------------------------

template <bool NT, class E, int W>
__global__ void __launch_bounds__(256)
embed_forward_kernel(EmbedParams p, const E* __restrict__ table, E* __restrict__ x) {
    const int lane = threadIdx.x & 63;
    for (long n = blockIdx.x * 4L + (threadIdx.x >> 6); n < p.N; n += gridDim.x * 4L) {
        const uint32_t v = (uint32_t)__builtin_amdgcn_readfirstlane((int)key_of(p, (int)n, lane == 0));
        E* dst = x + n * p.D;
        const E* src = table + (long)v * p.D;
        for (int c = lane * W; c < p.D; c += 64 * W) {
            float q[W];
            if (v < (uint32_t)p.V) {
                load_vec<E, W>(src + c, q);
#pragma unroll
                for (int i = 0; i < W; ++i) q[i] *= p.scale;
            } else {
#pragma unroll
                for (int i = 0; i < W; ++i) q[i] = 0.0f;
            }
            put<NT, E, W>(dst + c, q);
        }
    }
}

// --- sort -------------------------------------------------------------------------

struct SortPass {
    const uint32_t* key_in;  // null in the first pass: key_of
    const uint32_t* pos_in;
    uint32_t* key_out;
    uint32_t* pos_out;
    int shift, bits, blocks;
    int span;                // places of a block, a multiple of SORT_TILE
};

__device__ inline uint32_t sort_key(const EmbedParams& p, const SortPass& s, int n, bool report) {
    return s.key_in ? s.key_in[n] : key_of(p, n, report);
}

// Ranks a wave's items among equal digits: 64 at a time, the lanes of a digit
// told apart by one ballot per bit, the wave's count of the digit in LDS.
template <int ITEMS>
__device__ inline void rank_items(const uint32_t* key, const bool* on, int items, int shift, int bits, uint32_t* cnt,
                                  uint32_t* rank) {
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int j = 0; j < ITEMS; ++j) {
        if (j >= items) break;
        const uint32_t d = (key[j] >> shift) & ((1u << bits) - 1);
        unsigned long long peers = __ballot(on[j]);
        for (int bit = 0; bit < bits; ++bit) {
            const unsigned long long m = __ballot((d >> bit) & 1);
            peers &= (d >> bit) & 1 ? m : ~m;
        }
        const int before = __popcll(peers & ((1ull << lane) - 1));
        uint32_t old = 0;
        if (on[j] && before == 0) old = atomicAdd(&cnt[d], (uint32_t)__popcll(peers));
        old = __shfl(old, on[j] ? __ffsll(peers) - 1 : lane);
        rank[j] = old + before;
    }
}

// The sum of x over the workgroup's threads before this one.
__device__ inline uint32_t sum_before(uint32_t x, uint32_t* wsum) {
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    uint32_t incl = x;
    for (int o = 1; o < 64; o <<= 1) {
        const uint32_t u = __shfl_up(incl, o);
        if (lane >= o) incl += u;
    }
    if (lane == 63) wsum[w] = incl;
    __syncthreads();
    uint32_t run = incl - x;
    for (int i = 0; i < w; ++i) run += wsum[i];
    return run;
}

__global__ void __launch_bounds__(SORT_THREADS) sort_hist_kernel(EmbedParams p, SortPass s) {
    __shared__ uint32_t cnt[SORT_BINS];
    const int bins = 1 << s.bits;
    cnt[threadIdx.x] = 0;
    __syncthreads();
    const uint32_t now = *p.epoch + 1;
    const int first = blockIdx.x * s.span, end = min(p.N, first + s.span);
    for (int tile = first; tile < end; tile += SORT_TILE) {
        uint32_t key[SORT_ITEMS];
#pragma unroll
        for (int j = 0; j < SORT_ITEMS; ++j) {
            const int n = tile + j * SORT_THREADS + (int)threadIdx.x;
            key[j] = n < end ? sort_key(p, s, n, true) : ~0u;
        }
#pragma unroll
        for (int j = 0; j < SORT_ITEMS; ++j) {
            if (key[j] == ~0u) continue;
            if (!s.key_in && key[j] < (uint32_t)p.V) p.stamp[key[j]] = now;
            atomicAdd(&cnt[(key[j] >> s.shift) & (bins - 1)], 1u);
        }
    }
    __syncthreads();
    if ((int)threadIdx.x < bins) p.hist[(long)blockIdx.x * bins + threadIdx.x] = cnt[threadIdx.x];
}

// Places of a block go behind those of smaller digits and of earlier blocks;
// within the block in order (each wave holds a run of places).  Every block
// adds up all blocks' counts itself: 64 blocks at 256 K places, 128 KB.
__global__ void __launch_bounds__(SORT_THREADS) sort_scatter_kernel(EmbedParams p, SortPass s) {
    __shared__ uint32_t cnt[SORT_WAVES][SORT_BINS];
    __shared__ uint32_t wsum[SORT_WAVES];
    const int bins = 1 << s.bits, lane = threadIdx.x & 63, w = threadIdx.x >> 6, d = threadIdx.x;
    if (!s.key_in && blockIdx.x == 0 && threadIdx.x == 0) *p.epoch += 1;  // the stamps' reader comes later
    uint32_t total = 0, earlier = 0;
    if (d < bins) {
#pragma unroll 16
        for (int b = 0; b < s.blocks; ++b) {
            const uint32_t c = p.hist[(long)b * bins + d];
            total += c;
            earlier += b < (int)blockIdx.x ? c : 0;
        }
    }
    uint32_t base = sum_before(total, wsum) + earlier;  // where this block's next place of digit d goes
    const int end = min(p.N, (int)(blockIdx.x + 1) * s.span);
    for (int tile = blockIdx.x * s.span; tile < end; tile += SORT_TILE) {
        for (int i = threadIdx.x; i < SORT_WAVES * SORT_BINS; i += SORT_THREADS) (&cnt[0][0])[i] = 0;
        __syncthreads();
        uint32_t key[SORT_ITEMS], rank[SORT_ITEMS];
        bool on[SORT_ITEMS];
        const int first = tile + w * 64 * SORT_ITEMS + lane;
#pragma unroll
        for (int j = 0; j < SORT_ITEMS; ++j) {
            on[j] = first + j * 64 < end;
            key[j] = on[j] ? sort_key(p, s, first + j * 64, false) : 0;
        }
        rank_items<SORT_ITEMS>(key, on, SORT_ITEMS, s.shift, s.bits, cnt[w], rank);
        __syncthreads();
        if (d < bins)
            for (int i = 0; i < SORT_WAVES; ++i) {
                const uint32_t c = cnt[i][d];
                cnt[i][d] = base;
                base += c;
            }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < SORT_ITEMS; ++j) {
            if (!on[j]) continue;
            const int n = first + j * 64;
            const uint32_t at = cnt[w][(key[j] >> s.shift) & (bins - 1)] + rank[j];
            s.key_out[at] = key[j];
            s.pos_out[at] = s.pos_in ? s.pos_in[n] : (uint32_t)n;
        }
        __syncthreads();
    }
}

// All passes in one workgroup, for at most SORT_TILE places: the order is
// exchanged through LDS between the passes.
__global__ void __launch_bounds__(SORT_THREADS)
sort_small_kernel(EmbedParams p, uint32_t* key_out, uint32_t* pos_out, int passes, int bits) {
    __shared__ uint32_t cnt[SORT_WAVES][SORT_BINS];
    __shared__ uint32_t wsum[SORT_WAVES];
    __shared__ uint32_t skey[SORT_TILE];
    __shared__ uint16_t spos[SORT_TILE];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, bins = 1 << bits, d = threadIdx.x;
    const int items = (p.N + SORT_THREADS - 1) / SORT_THREADS;  // of a thread
    const int first = w * 64 * items + lane;
    const uint32_t now = *p.epoch + 1;
    uint32_t key[SORT_ITEMS], pos[SORT_ITEMS], rank[SORT_ITEMS];
    bool on[SORT_ITEMS];
#pragma unroll
    for (int j = 0; j < SORT_ITEMS; ++j) {
        const int n = first + j * 64;
        on[j] = j < items && n < p.N;
        key[j] = 0;
        pos[j] = (uint32_t)n;
        if (!on[j]) continue;
        key[j] = key_of(p, n, true);
        if (key[j] < (uint32_t)p.V) p.stamp[key[j]] = now;
    }
    for (int pass = 0; pass < passes; ++pass) {
        for (int i = threadIdx.x; i < SORT_WAVES * SORT_BINS; i += SORT_THREADS) (&cnt[0][0])[i] = 0;
        __syncthreads();
        rank_items<SORT_ITEMS>(key, on, items, pass * bits, bits, cnt[w], rank);
        __syncthreads();
        uint32_t total = 0;
        for (int i = 0; i < SORT_WAVES; ++i) total += cnt[i][d];
        uint32_t base = sum_before(total, wsum);
        for (int i = 0; i < SORT_WAVES; ++i) {
            const uint32_t c = cnt[i][d];
            cnt[i][d] = base;
            base += c;
        }
        __syncthreads();
        const bool last = pass == passes - 1;
#pragma unroll
        for (int j = 0; j < SORT_ITEMS; ++j) {
            if (!on[j]) continue;
            const uint32_t at = cnt[w][(key[j] >> (pass * bits)) & (bins - 1)] + rank[j];
            if (last) {
                key_out[at] = key[j];
                pos_out[at] = pos[j];
            } else {
                skey[at] = key[j];
                spos[at] = (uint16_t)pos[j];
            }
        }
        __syncthreads();
        if (last) break;
#pragma unroll
        for (int j = 0; j < SORT_ITEMS; ++j) {
            if (!on[j]) continue;
            key[j] = skey[first + j * 64];
            pos[j] = spos[first + j * 64];
        }
    }
    if (threadIdx.x == 0) *p.epoch = now;
}

// --- sums over sorted places --------------------------------------------------------

// The first `zero_waves` waves write the zeros; beside them the others sum: piece
// w / tiles, columns of tile w % tiles (64 W of them).
template <class E, int W>
__global__ void __launch_bounds__(256)
embed_sum_kernel(EmbedParams p, const uint32_t* __restrict__ key, const uint32_t* __restrict__ pos,
                 const E* __restrict__ dx, float* __restrict__ dt, int R, int pieces, int tiles,
                 int zero_waves) {
    const int lane = threadIdx.x & 63;
    const long w = blockIdx.x * 4L + (threadIdx.x >> 6) - zero_waves;
    if (w >= (long)pieces * tiles) return;
    if (w < 0) {
        const uint32_t now = *p.epoch;
        float zero[W] = {};
        for (long v = w + zero_waves; v < p.V; v += zero_waves) {
            if (p.stamp[v] == now) continue;
            for (int c = lane * W; c < p.D; c += 64 * W) store_vec<float, W>(dt + v * p.D + c, zero);
        }
        return;
    }
    const int piece = (int)(w / tiles), c = (int)(w - (long)piece * tiles) * 64 * W + lane * W;
    const int first = piece * R, n = min(R, p.N - first);
    const bool on = c < p.D;
    const uint32_t V = (uint32_t)p.V;
    uint32_t k = V, q = 0;
    if (lane < n) {
        k = key[first + lane];
        q = pos[first + lane];
    }
    const uint32_t before = piece > 0 ? key[first - 1] : V, after = first + n < p.N ? key[first + n] : V;
    float acc[W] = {};
    uint32_t cur = (uint32_t)__builtin_amdgcn_readlane((int)k, 0);
    bool opened = before == cur;  // the token's places begin in an earlier piece

    auto close = [&](bool goes_on) {
        if (!on) return;
        if (opened || goes_on) {
            store_vec<float, W>(p.part + ((long)piece * 2 + (opened ? 0 : 1)) * p.D + c, acc);
        } else {
            float o[W];
#pragma unroll
            for (int i = 0; i < W; ++i) o[i] = acc[i] * p.scale;
            store_vec<float, W>(dt + (long)cur * p.D + c, o);
        }
    };
    constexpr int U = 8;  // rows in flight
    for (int i0 = 0; i0 < n && cur != V; i0 += U) {
        float row[U][W];
#pragma unroll
        for (int j = 0; j < U; ++j) {
            const int i = min(i0 + j, n - 1);
            const uint32_t r = (uint32_t)__builtin_amdgcn_readlane((int)q, i);
            if (on) load_vec<E, W>(dx + (long)r * p.D + c, row[j]);
        }
#pragma unroll
        for (int j = 0; j < U; ++j) {
            if (i0 + j >= n || cur == V) break;
            const uint32_t kj = (uint32_t)__builtin_amdgcn_readlane((int)k, i0 + j);
            if (kj != cur) {
                close(false);
                cur = kj;
                opened = false;
#pragma unroll
                for (int i = 0; i < W; ++i) acc[i] = 0.0f;
                if (cur == V) break;
            }
#pragma unroll
            for (int i = 0; i < W; ++i) acc[i] += row[j][i];
        }
    }
    if (cur != V) close(after == cur);
}

// acc += the slots 0 of pieces [lo, hi), in order.
template <int W>
__device__ inline void add_parts(const EmbedParams& p, int lo, int hi, int c, float* acc) {
    constexpr int U = 16;  // in flight, also the last few
    for (int i0 = lo; i0 < hi; i0 += U) {
        float q[U][W];
#pragma unroll
        for (int u = 0; u < U; ++u) load_vec<float, W>(p.part + (long)min(i0 + u, hi - 1) * 2 * p.D + c, q[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int j = 0; j < W; ++j) acc[j] += i0 + u < hi ? q[u][j] : 0.0f;
    }
}

// The tokens whose places span pieces, one column tile: a wave takes the token
// that begins in its piece and goes on, if there is one.  One with more than LONG parts
// is shared out over the workgroup's waves.
template <int W>
__global__ void __launch_bounds__(256)
embed_join_kernel(EmbedParams p, const uint32_t* __restrict__ key, float* __restrict__ dt, int R,
                  int pieces) {
    constexpr int LONG = 32;
    __shared__ float sum[4][64 * W];
    __shared__ int parts_of[4];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, piece = blockIdx.x * 4 + w;
    const int c = blockIdx.y * 64 * W + lane * W;
    const bool on = c < p.D;
    int parts = 0;  // in slot 0 of the pieces after this one
    const long end = (long)(piece + 1) * R;
    // four keys at once: the waves that find nothing to do are most of them
    const long far = p.N - 1;
    const uint32_t next = key[min(end, far)], mine = key[min(end - 1, far)], begin = key[min(end - R, far)],
                   before = key[min(max(end - R - 1, 0L), far)];
    const uint32_t V = (uint32_t)p.V, v = piece < pieces && end < p.N ? next : V;
    if (v != V && mine == v && !(piece > 0 && begin == v && before == v)) {
        // whole pieces 64 at a time
        parts = 1;
        for (;;) {
            const long at = end + (long)(parts + lane) * R;  // the place after piece + parts + lane
            const unsigned long long goes = __ballot(at < p.N && key[min(at, (long)p.N - 1)] == v);
            const int whole = goes == ~0ull ? 64 : __ffsll(~goes) - 1;
            parts += whole;
            if (whole < 64) break;
        }
    }
    auto write = [&](const float* acc) {
        float o[W];
#pragma unroll
        for (int j = 0; j < W; ++j) o[j] = acc[j] * p.scale;
        store_vec<float, W>(dt + (long)v * p.D + c, o);
    };
    if (parts > 0 && parts <= LONG && on) {
        float acc[W];
        load_vec<float, W>(p.part + ((long)piece * 2 + 1) * p.D + c, acc);
        add_parts<W>(p, piece + 1, piece + 1 + parts, c, acc);
        write(acc);
    }
    if (lane == 0) parts_of[w] = parts;
    __syncthreads();
    for (int i = 0; i < 4; ++i) {
        const int n = parts_of[i], from = blockIdx.x * 4 + i;
        if (n <= LONG) continue;
        const int per = (n + 3) / 4, lo = min(n, w * per), hi = min(n, lo + per);
        float acc[W] = {};
        if (on) {
            if (w == 0) load_vec<float, W>(p.part + ((long)from * 2 + 1) * p.D + c, acc);
            add_parts<W>(p, from + 1 + lo, from + 1 + hi, c, acc);
        }
#pragma unroll
        for (int j = 0; j < W; ++j) sum[w][lane * W + j] = acc[j];
        __syncthreads();
        if (w == i && on) {
#pragma unroll
            for (int j = 0; j < W; ++j) {
                acc[j] = sum[0][lane * W + j];
                for (int q = 1; q < 4; ++q) acc[j] += sum[q][lane * W + j];
            }
            write(acc);
        }
        __syncthreads();
    }
}

constexpr int PIECE = 32;  // places of a piece, where there are many
int columns_of(int D) { return D % 4 == 0 ? 4 : D % 2 == 0 ? 2 : 1; }  // of a lane
int column_tiles(int D) { return (D + 64 * columns_of(D) - 1) / (64 * columns_of(D)); }

int check_embed_sizes(int B, int T, int V, int D, int dtype) {
    if (B < 1 || T < 1 || V < 1 || D < 1 || !valid_dtype(dtype)) return LSTM_DYN_ERR_INVALID;
    if ((long long)B * T >= 1LL << 30 || V >= 1 << 27 || D >= 1 << 21) return LSTM_DYN_ERR_UNSUPPORTED;
    return LSTM_DYN_OK;
}

int check_embed_forward(int B, int T, int V, int D, int dtype, const int32_t* tokens,
                        const int32_t* lengths, const void* table, const void* x) {
    const long long e = dtype_bytes(dtype), N = (long long)B * T;
    const Span s[] = {{tokens, 4 * N, 4, false}, {table, e * V * D, 16, false}, {x, e * N * D, 16, true},
                      {lengths, 4LL * B, 4, false}};
    return check_spans(s, lengths ? 4 : 3);
}

int check_embed_backward(int B, int T, int V, int D, const int32_t* tokens, const int32_t* lengths,
                         const void* dx, int dx_dtype, const float* dt) {
    if (!valid_dtype(dx_dtype)) return LSTM_DYN_ERR_INVALID;
    const long long N = (long long)B * T;
    // the sums' threads: a wave for 32 places and a tile of columns, and those that write the zeros
    if ((N + PIECE - 1) / PIECE * column_tiles(D) + (1 << 16) >= 1LL << 26) return LSTM_DYN_ERR_UNSUPPORTED;
    const Span s[] = {{tokens, 4 * N, 4, false}, {dx, dtype_bytes(dx_dtype) * N * D, 16, false},
                      {dt, 4LL * V * D, 16, true}, {lengths, 4LL * B, 4, false}};
    return check_spans(s, lengths ? 4 : 3);
}

inline long long up256(long long n) { return (n + 255) / 256 * 256; }

}  // namespace
}  // namespace ldyn

using namespace ldyn;

struct lstm_dyn_embed : OpsHandle {
    int B, T, V, D, dtype;
    int N, passes, bits, blocks, span;
    int W, tiles, R, pieces;  // columns of a lane, column tiles of a row; places of a piece
    uint32_t *epoch, *stamp, *hist, *key[2], *pos[2];
    float* part;
};

// Pieces of up to 32 places, shorter where they would leave fewer than eight
// waves a CU on the gradient (945 places of 333 columns: 16 us with 64, 5.6 with 8).
static void embed_shape(lstm_dyn_embed* h) {
    h->W = columns_of(h->D);
    h->tiles = column_tiles(h->D);
    h->R = PIECE;
    while (h->R > 8 && (long long)h->N / h->R * h->tiles < 8LL * h->num_cus) h->R /= 2;
}

extern "C" int lstm_dyn_check_embed_args(int B, int T, int V, int D, int dtype,
                                         const int32_t* tokens, const int32_t* lengths,
                                         const void* table, const void* out_x, const void* dx,
                                         int dx_dtype, const float* d_table) {
    const int rc = check_embed_sizes(B, T, V, D, dtype);
    if (rc != LSTM_DYN_OK) return rc;
    if (!dx && !d_table) return check_embed_forward(B, T, V, D, dtype, tokens, lengths, table, out_x);
    return check_embed_backward(B, T, V, D, tokens, lengths, dx, dx_dtype, d_table);
}

extern "C" int lstm_dyn_embed_create(lstm_dyn_embed_t** out, int B, int T, int V, int D, int dtype) {
    if (!out) return LSTM_DYN_ERR_INVALID;
    *out = nullptr;
    int rc = check_embed_sizes(B, T, V, D, dtype);
    if (rc != LSTM_DYN_OK) return rc;
    lstm_dyn_embed* h = new (std::nothrow) lstm_dyn_embed();
    if (!h) return LSTM_DYN_ERR_NOMEM;
    h->B = B; h->T = T; h->V = V; h->D = D; h->dtype = dtype;
    if ((rc = ops_device(h)) != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    const long long N = (long long)B * T;
    h->N = (int)N;
    int bits = 1;
    while ((1LL << bits) < (long long)V + 1) ++bits;
    h->passes = (bits + SORT_BITS - 1) / SORT_BITS;
    h->bits = (bits + h->passes - 1) / h->passes;
    // tiles of places, shared out over at most SORT_BLOCKS blocks
    const long long tiles = (N + SORT_TILE - 1) / SORT_TILE, each = (tiles + SORT_BLOCKS - 1) / SORT_BLOCKS;
    h->span = (int)(each * SORT_TILE);
    h->blocks = (int)((N + h->span - 1) / h->span);
    embed_shape(h);
    h->pieces = (int)((N + h->R - 1) / h->R);
    long long at = 256;
    auto take = [&](long long n) {
        const long long o = at;
        at += up256(n);
        return o;
    };
    const long long o_epoch = take(4), o_stamp = take(4LL * V), o_hist = take(4LL * h->blocks << h->bits);
    long long o_key[2], o_pos[2];
    for (int i = 0; i < 2; ++i) o_key[i] = take(4 * N), o_pos[i] = take(4 * N);
    const long long o_part = take(8LL * h->pieces * D);
    if ((rc = ops_init(h, at)) != LSTM_DYN_OK) {
        delete h;
        return rc;
    }
    auto u32 = [&](long long o) { return reinterpret_cast<uint32_t*>(h->block + o); };
    h->epoch = u32(o_epoch); h->stamp = u32(o_stamp); h->hist = u32(o_hist);
    for (int i = 0; i < 2; ++i) h->key[i] = u32(o_key[i]), h->pos[i] = u32(o_pos[i]);
    h->part = reinterpret_cast<float*>(h->block + o_part);
    *out = h;
    return LSTM_DYN_OK;
}

static EmbedParams embed_params(const lstm_dyn_embed* h, const int32_t* tokens,
                                const int32_t* lengths, float scale) {
    return EmbedParams{tokens, lengths, h->status(), h->epoch, h->stamp, h->hist, h->part,
                       h->N, h->T, h->V, h->D, scale};
}

extern "C" int lstm_dyn_embed_forward(lstm_dyn_embed_t* h, const int32_t* tokens,
                                      const int32_t* lengths, const void* table, float scale,
                                      void* out_x, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc = check_embed_forward(h->B, h->T, h->V, h->D, h->dtype, tokens, lengths, table, out_x);
    if (rc != LSTM_DYN_OK) return rc;
    if ((rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const EmbedParams p = embed_params(h, tokens, lengths, scale);
    long grid = ((long)h->N + 3) / 4;
    if (grid > 64L * h->num_cus) grid = 64L * h->num_cus;
    // An x about as large as the last cache is read from memory by whoever comes next: its stores
    // bypass the caches, which then keep what else there is.  The lookup alone takes the same
    // time; with a product that reads x behind it 128 MB take 75 us so and 78 past the caches, 192 MB
    // 122 and 119, 256 MB 161 and 157, 512 MB 318 and 299; with a plain reading pass 192 MB 98
    // and 116, 256 MB 164 and 151.
    const bool far = (long long)h->N * h->D * dtype_bytes(h->dtype) >= FAR_BYTES;
#define LDYN_EMB(E, W)                                                                               \
    hipLaunchKernelGGL((far ? embed_forward_kernel<true, E, W> : embed_forward_kernel<false, E, W>), \
                       dim3((unsigned)grid), dim3(256), 0, h->last_stream, p,                        \
                       static_cast<const E*>(table), static_cast<E*>(out_x))
    if (h->dtype == LSTM_DYN_BF16) {
        if (h->D % 8 == 0) LDYN_EMB(__bf16, 8);
        else if (h->D % 2 == 0) LDYN_EMB(__bf16, 2);
        else LDYN_EMB(__bf16, 1);
    } else {
        if (h->D % 4 == 0) LDYN_EMB(float, 4);
        else if (h->D % 2 == 0) LDYN_EMB(float, 2);
        else LDYN_EMB(float, 1);
    }
#undef LDYN_EMB
    return ops_launched(h);
}

extern "C" int lstm_dyn_embed_backward(lstm_dyn_embed_t* h, const int32_t* tokens,
                                       const int32_t* lengths, const void* dx, int dx_dtype,
                                       float scale, float* d_table, void* stream) {
    if (!h) return LSTM_DYN_ERR_INVALID;
    int rc = check_embed_backward(h->B, h->T, h->V, h->D, tokens, lengths, dx, dx_dtype, d_table);
    if (rc != LSTM_DYN_OK) return rc;
    if ((rc = ops_begin(h, stream)) != LSTM_DYN_OK) return rc;
    const EmbedParams p = embed_params(h, tokens, lengths, scale);
    int in = 0;
    if (h->blocks == 1) {  // 4000 places: 31 us for lookup and gradient so, 41 in passes of two launches
        hipLaunchKernelGGL(sort_small_kernel, dim3(1), dim3(SORT_THREADS), 0, h->last_stream, p, h->key[0],
                           h->pos[0], h->passes, h->bits);
        if ((rc = ops_launched(h)) != LSTM_DYN_OK) return rc;
    } else {
        for (int i = 0; i < h->passes; ++i, in ^= 1) {
            const SortPass s{i ? h->key[in] : nullptr, i ? h->pos[in] : nullptr, h->key[in ^ 1],
                             h->pos[in ^ 1], i * h->bits, h->bits, h->blocks, h->span};
            hipLaunchKernelGGL(sort_hist_kernel, dim3(h->blocks), dim3(SORT_THREADS), 0, h->last_stream, p, s);
            if ((rc = ops_launched(h)) != LSTM_DYN_OK) return rc;
            hipLaunchKernelGGL(sort_scatter_kernel, dim3(h->blocks), dim3(SORT_THREADS), 0, h->last_stream, p, s);
            if ((rc = ops_launched(h)) != LSTM_DYN_OK) return rc;
        }
    }
    const int W = h->W, tiles = h->tiles;
    const int zero_waves = h->V < 8 * h->num_cus ? h->V : 8 * h->num_cus;
    const long waves = (long)h->pieces * tiles + zero_waves;
    const unsigned grid = (unsigned)((waves + 3) / 4);
#define LDYN_SUM(E, W)                                                                              \
    hipLaunchKernelGGL((embed_sum_kernel<E, W>), dim3(grid), dim3(256), 0, h->last_stream, p,       \
                       h->key[in], h->pos[in], static_cast<const E*>(dx), d_table, h->R, h->pieces, \
                       tiles, zero_waves)
    if (dx_dtype == LSTM_DYN_BF16) {
        if (W == 4) LDYN_SUM(__bf16, 4);
        else if (W == 2) LDYN_SUM(__bf16, 2);
        else LDYN_SUM(__bf16, 1);
    } else {
        if (W == 4) LDYN_SUM(float, 4);
        else if (W == 2) LDYN_SUM(float, 2);
        else LDYN_SUM(float, 1);
    }
#undef LDYN_SUM
    if ((rc = ops_launched(h)) != LSTM_DYN_OK || h->pieces < 2) return rc;
    auto* join = W == 4 ? embed_join_kernel<4> : W == 2 ? embed_join_kernel<2> : embed_join_kernel<1>;
    hipLaunchKernelGGL(join, dim3((h->pieces + 3) / 4, tiles), dim3(256), 0, h->last_stream, p, h->key[in],
                       d_table, h->R, h->pieces);
    return ops_launched(h);
}

extern "C" int lstm_dyn_embed_query(lstm_dyn_embed_t* h, int what, long long* value) {
    return ops_query(h, what, value);
}

extern "C" int lstm_dyn_embed_destroy(lstm_dyn_embed_t* h) {
    if (!h) return LSTM_DYN_OK;
    const int rc = ops_free(h);
    delete h;
    return rc;
}
