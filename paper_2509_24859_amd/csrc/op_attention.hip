// Softmax attention over packed or padded sequences, its gradients, and their C entry points.
//
// Heads that share keys are rows of one matrix: packed row r of a kv head is query r / group of head kv * group + r % group, so that
// a tile of rows meets each key once whatever the group, and one new token of a large group fills a tile.
//
// Products are taken transposed where that spares a way through LDS.  S^T = K Q^T leaves a lane with 16 keys of one query (column
// l % 32, keys 8 (i / 4) + 4 (l / 32) + i % 4 of 32): maxima and sums of a row are then within a lane and its partner 32 lanes
// on, and P^T is the second operand of O^T = V^T P^T as it lies in the registers, the keys of a step of 16 in the order
// 4 h .. 4 h + 3, 8 + 4 h .. 11 + 4 h for lane half h, in which V^T is read too.
#include <math.h>

#include <type_traits>
#include <utility>

#include "harp_ctx.h"
#include "op_attention_plan.h"
#include "ops_common.h"

using namespace harp;
using namespace harp::attention;
using namespace harp::ops;

namespace {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));

template <typename T> struct Mfma32;
template <> struct Mfma32<__bf16> {
    typedef bf16x8 Frag;
    static __device__ __forceinline__ f32x16 run(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};
template <> struct Mfma32<_Float16> {
    typedef f16x8 Frag;
    static __device__ __forceinline__ f32x16 run(Frag a, Frag b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// What the kernels know of a call.
struct Call {
    int64_t tokens_q, tokens_k;
    int batch, heads, kv_heads, head, group, causal;
    uint32_t group_magic;            // floor(2^32 / group)
    float c;                         // scale * log2(e)
    const int32_t *q_begin, *k_begin, *k_count;
    int64_t q_token, q_step, k_token, k_step, v_token, v_step, o_token, o_step;
    const void *q, *k, *v;
    void *o;
    float *lse;
};

// r / group for 0 <= r < 2^31: the estimate is the quotient or one less.
__device__ __forceinline__ int query_of(const Call &a, int r) {
    uint32_t q = __umulhi(uint32_t(r), a.group_magic);
    if (a.group == 1) return r;
    if (r - int(q) * a.group >= a.group) ++q;
    return int(q);
}

struct Sequence {
    int64_t q0, k0;                  // first tokens
    int nq, nk, used;                // queries, keys, keys used
};
__device__ __forceinline__ int64_t kept(int64_t x, int64_t lo, int64_t hi) { return x < lo ? lo : x > hi ? hi : x; }
__device__ __forceinline__ void span(const int32_t *begin, int64_t tokens, int batch, int b, int64_t &first, int &count) {
    if (begin) {
        first = kept(begin[b], 0, tokens);
        count = int(kept(begin[b + 1], first, tokens) - first);
    } else {
        count = int(tokens / batch);
        first = int64_t(b) * count;
    }
}
__device__ __forceinline__ Sequence sequence(const Call &a, int b) {
    Sequence s;
    span(a.q_begin, a.tokens_q, a.batch, b, s.q0, s.nq);
    span(a.k_begin, a.tokens_k, a.batch, b, s.k0, s.nk);
    s.used = a.k_count ? int(kept(a.k_count[b], 0, s.nk)) : s.nk;
    return s;
}

// Sum over the lanes up to and with this one.  Sums of tiles stop at 2^31 - 1: spans that lie over each other (begins that do not
// rise) may have more, and a sum that turned negative would find a sequence that is none.
__device__ __forceinline__ int up_to(int x) {
#pragma unroll
    for (int d = 1; d < kWave; d *= 2) {
        const int below = __shfl_up(x, d);
        if (int(threadIdx.x % kWave) >= d) x = __builtin_elementwise_add_sat(x, below);
    }
    return x;
}
// The sequence that tile `id` of `side` rows belongs to, rows being `times` the tokens of `begin`'s spans, and its place there;
// false behind the last.  Every wavefront looks for itself: runs of up to 16 sequences a lane, then the sequences of one run.
__device__ __forceinline__ bool locate(const int32_t *begin, int64_t tokens, int batch, int times, int side, int id, int &b, int &tile) {
    if (!begin) {
        const int each = int((tokens / batch * times + side - 1) / side);
        if (each == 0) return false;
        b = id / each;
        tile = id - b * each;
        return b < batch;
    }
    const int lane = threadIdx.x % kWave, run = batch <= kWave ? 1 : 16;
    auto tiles_of_one = [&](int i) {
        if (i >= batch) return 0;
        int64_t at;
        int count;
        span(begin, tokens, batch, i, at, count);
        return int((int64_t(count) * times + side - 1) / side);
    };
    auto before = [](int upto, int lane) { return lane > 0 ? __builtin_amdgcn_readlane(upto, lane - 1) : 0; };
    for (int first = 0; first < batch; first += kWave * run) {
        int tiles = 0;
        for (int i = 0; i < run; ++i) tiles = __builtin_elementwise_add_sat(tiles, tiles_of_one(first + lane * run + i));
        int upto = up_to(tiles);
        uint64_t past = __ballot(id < upto);
        if (!past) {
            id -= __builtin_amdgcn_readlane(upto, kWave - 1);
            continue;
        }
        int at = __builtin_ctzll(past);
        id -= before(upto, at);
        b = first + at * run;
        if (run > 1) {
            tiles = lane < run ? tiles_of_one(b + lane) : 0;
            upto = up_to(tiles);
            past = __ballot(id < upto);
            at = __builtin_ctzll(past);
            id -= before(upto, at);
            b += at;
        }
        tile = id;
        return true;
    }
    return false;
}

// What a workgroup takes of `places` tiles, the heaviest first, of every kv head, shared out.  Workgroups go to the 8 dies in turn, each
// with an L2 of its own: a die takes neighbours, which share keys.  Within a die they go to its shader engines in turn, and wait
// for room in that one: under the causal order, where tiles differ in their work, the same place of each head comes first, then the
// next, so that every engine has tiles of all weights and those that follow find room where the lightest end (gradients of
// 4,096 keys, 32 heads, when this was made: 332 us, heads one after the other 448; 4 heads of 96, 2 sequences: 307 and 491).
// A die takes whole heads where they can be dealt out.
struct Work { int share, kv, place; };
__device__ __forceinline__ Work work_of(int id, int places, int kv_heads, int shares, bool causal) {
    Work w;
    if (causal && kv_heads % kDies == 0) {
        const int heads = kv_heads / kDies, i = id / kDies, each = heads * shares;
        w.place = i / each;
        w.share = i % each % shares;
        w.kv = id % kDies * heads + i % each / shares;
    } else if (causal) {
        w.share = id % shares;
        w.kv = id / shares % kv_heads;
        w.place = id / shares / kv_heads;
    } else {
        const int n = places * kv_heads * shares, die = id % kDies, each = n / kDies, more = n % kDies;
        id = id / kDies + die * each + (die < more ? die : more);
        w.share = id % shares;
        w.place = id / shares % places;
        w.kv = id / shares / places;
    }
    return w;
}

// LDS holds rows of D elements in pieces of 16 bytes.  It gives 256 bytes a cycle: to 16 lanes that read a piece each, or to 32
// that read half of one across (ds_read_tr: 4 rows of 4 neighbouring pieces).  Pieces are moved within a row so that neither 16
// neighbouring rows, one piece of each, nor 4 rows, 4 pieces of each, meet at the same place of 256 bytes.
template <int D> __device__ __forceinline__ int moved(int row, int piece) {
    if (D == 128) return piece ^ ((row & 3) << 2 | (row >> 2 & 3));
    if (D == 64) return piece ^ ((row >> 1 & 1) << 2 | (row >> 2 & 3));
    return piece ^ (row >> 2 & 3);
}
template <typename T> __device__ __forceinline__ uint32_t lds_address(const T *p) {
    return uint32_t(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const void *)p));
}
// Fragments of 32 rows by 16 columns: lane l has row l % 32 and columns 16 k + 8 (l / 32) .. + 7.  `at` is the lane's place in LDS, rows
// aligned to 256 bytes.  Only low bits of a place in the row are moved: another k is another place by those bits, and what else is
// known when compiled is in the instruction.  refresh(): the places are not kept in registers over it.
template <typename T, int D> struct Along {
    static constexpr int N = D == 96 ? 2 : D / 16;
    uint32_t at;
    __device__ __forceinline__ explicit Along(const T *lds) {
        const int lane = threadIdx.x % kWave, row = lane % 32;
        at = lds_address(lds) + uint32_t(row * D + moved<D>(row, lane / 32) * 8) * 2;
    }
    __device__ __forceinline__ void refresh() { asm volatile("" : "+v"(at)); }
    // row0 a multiple of 32
    __device__ __forceinline__ typename Mfma32<T>::Frag read(int row0, int k) const {
        typedef __attribute__((address_space(3))) const char *Bytes;
        typedef __attribute__((address_space(3))) const typename Mfma32<T>::Frag *Lds;
        return *(Lds)((Bytes)(uintptr_t)(at ^ uint32_t(k % N * 32)) + (row0 * D + k / N * (N * 16)) * 2);
    }
};
// Fragments of 32 columns by 16 rows, transposed: lane l has column 32 m + l % 32 and, h = l / 32, rows row0 + 4 h .. + 3 and
// row0 + 8 + 4 h .. + 3.
template <typename T, int D> struct Across {
    static constexpr int N = D == 96 ? 1 : D / 32;
    uint32_t at;
    __device__ __forceinline__ explicit Across(const T *lds) {
        const int lane = threadIdx.x % kWave, i = lane % 16, row = lane / 32 * 4 + i / 4;
        at = lds_address(lds) + uint32_t(row * D + moved<D>(row, lane / 16 % 2 * 2 + i % 4 / 2) * 8 + i % 2 * 4) * 2;
    }
    __device__ __forceinline__ void refresh() { asm volatile("" : "+v"(at)); }
    // row0 a multiple of 16; a row 8 further on has its pieces moved by 2 more
    __device__ __forceinline__ typename Mfma32<T>::Frag read(int row0, int m) const {
        typedef __attribute__((address_space(3))) char *Bytes;
        typedef __attribute__((address_space(3))) s16x4 *Lds;
        const int more = (row0 * D + m / N * (N * 32)) * 2;
        const uint32_t lo = at ^ uint32_t(m % N * 64), hi = lo ^ 32;
        const s16x4 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)((Bytes)(uintptr_t)lo + more));
        const s16x4 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)((Bytes)(uintptr_t)hi + more + 16 * D));
        const s16x8 v = __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7);
        return __builtin_bit_cast(typename Mfma32<T>::Frag, v);
    }
};

// 8 elements wherever they lie, or zeros.
template <typename T> __device__ __forceinline__ typename Mfma32<T>::Frag eight(const T *p, bool there) {
    typedef typename Mfma32<T>::Frag Loose __attribute__((aligned(sizeof(T))));
    typename Mfma32<T>::Frag v = {};
    if (there) v = *reinterpret_cast<const Loose *>(p);
    return v;
}

// A tile of ROWS rows on its way from memory through registers into LDS.  Rows from `limit` on, and channels from `head` on, are zeros:
// what memory holds there is not looked at.
template <typename T, int D, int ROWS, int THREADS> struct Stage {
    static constexpr int kAll = ROWS * (D / 8), kEach = (kAll + THREADS - 1) / THREADS;
    typename Mfma32<T>::Frag piece[kEach];
    __device__ __forceinline__ static int row(int i) { return (i * THREADS + int(threadIdx.x)) / (D / 8); }
    __device__ __forceinline__ static int part(int i) { return (i * THREADS + int(threadIdx.x)) % (D / 8); }
    template <typename At> __device__ __forceinline__ void ask(At at, int limit, int head) {
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const bool there = row(i) < limit && part(i) * 8 < head && (kAll % THREADS == 0 || i * THREADS + int(threadIdx.x) < kAll);
            piece[i] = eight<T>(at(there ? row(i) : 0) + (there ? part(i) * 8 : 0), there);
        }
    }
    __device__ __forceinline__ void put(T *lds) const {
#pragma unroll
        for (int i = 0; i < kEach; ++i)
            if (kAll % THREADS == 0 || i * THREADS + int(threadIdx.x) < kAll)
                *reinterpret_cast<typename Mfma32<T>::Frag *>(lds + row(i) * D + moved<D>(row(i), part(i)) * 8) = piece[i];
    }
};
// The same of rows `token` apart, tile after tile.
template <typename T, int D, int ROWS, int THREADS> struct Stream : Stage<T, D, ROWS, THREADS> {
    typedef Stage<T, D, ROWS, THREADS> Base;
    const T *at;                     // of this thread's first piece
    __device__ __forceinline__ void begin(const T *from, int64_t token) { at = from + Base::row(0) * token + Base::part(0) * 8; }
    // `limit` rows are there, of this tile and those after it
    __device__ __forceinline__ void ask(int64_t token, int limit, int head) {
#pragma unroll
        for (int i = 0; i < Base::kEach; ++i) {
            const bool there = Base::row(i) < limit && Base::part(i) * 8 < head && (Base::kAll % THREADS == 0 || i * THREADS + int(threadIdx.x) < Base::kAll);
            const T *p = THREADS % (D / 8) == 0 ? at + i * (THREADS / (D / 8)) * token
                                                : at + (Base::row(i) - Base::row(0)) * token + (Base::part(i) - Base::part(0)) * 8;
            Base::piece[i] = eight<T>(p, there);
        }
        at += ROWS * token;
    }
};

// call(0) .. call(N - 1) written out, the number known to the compiler.
template <typename F, int... I> __device__ __forceinline__ void written_out(F call, std::integer_sequence<int, I...>) { (call(std::integral_constant<int, I>()), ...); }
template <int N, typename F> __device__ __forceinline__ void written_out(F call) { written_out(call, std::make_integer_sequence<int, N>()); }

__device__ __forceinline__ float other_half(float x) { return __shfl_xor(x, 32); }

// A wavefront's 32 packed rows, one to a lane and its partner.
struct Row {
    int64_t token;
    int head, limit;                 // keys before `limit` are seen; -1: no such row
};
__device__ __forceinline__ int limit_of(const Call &a, const Sequence &s, int query) {
    if (!a.causal) return s.used;
    const int seen = query + 1 + s.used - s.nq;
    return seen < 0 ? 0 : seen;
}
__device__ __forceinline__ Row row_of(const Call &a, const Sequence &s, int kv, int r) {
    if (r >= int64_t(s.nq) * a.group) return Row{0, 0, -1};
    const int query = query_of(a, r);
    return Row{s.q0 + query, kv * a.group + r - query * a.group, limit_of(a, s, query)};
}

// Weights go into the matrix instructions rounded to T.  bfloat16 has the range of 32 bits.  float16 loses what is below 2^-25, so there
// they are taken times 2^kShift: they are normal numbers from 2^-26 of the row's largest on and lost below 2^-37 of it, 2^-17 of a
// result over 2^20 keys at most.  In the forward pass the reference may be 2^kBehind less than the largest: together they stay below 2^16.
template <typename T> struct Weights {
    static constexpr bool kNarrow = __is_same(T, _Float16);
    static constexpr float kShift = kNarrow ? 12.0f : 0.0f, kBehind = kNarrow ? 3.0f : 8.0f;
};

// Partial results of a share of the keys: unscaled sums [share][token][head][channel], what exponents were taken against and the sum of
// weights [share][token][head].
struct Shares {
    int count, paired;
    float *sums, *stats;
    int first_kv, kv_heads;          // of this launch
};

// One pass over the keys with the running reference and sum of a softmax: o = sum of 2^(c s - top) v, sum likewise, both times
// 2^(top before - top) when the reference grows.  WAVES wavefronts of 32 rows; keys go through LDS 64 at a time, two tiles of them, in
// steps of 32.  8 wavefronts read a key from L2 once for 256 rows; 4 where rows are few.
// 4,096 queries and keys, 32 heads of 128, bfloat16: 255 to 268 us by the card, 1,025 to 1,078 TFLOP/s, matrix units busy 56% of the
// cycles; causal 146 to 162.  What bounds it: a tile's 32 matrix instructions of a wavefront take 1,024 cycles, its 179 vector
// instructions some 800, and 56% is what one after the other gives: a SIMD's two wavefronts hardly have the one's beside the other's.
// LDS, 256 bytes a cycle, is busy a third.  One token of 16 sequences, 174,103 keys in all, 8 heads of 128: 151 us, 4.7 TB/s, where
// reading reaches 6.1: shares are as many for each sequence, the longest's are the last.  With 4 wavefronts and 128 channels 11
// registers are spilled, outside the loop of whole tiles.
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, 2) void forward(Call a, int tiles, Shares shares) {
    constexpr int kThreads = WAVES * kWave, kRows = WAVES * 32;
    typedef typename Mfma32<T>::Frag Frag;
    __shared__ __align__(1024) T lds[4][kKeys * D];               // two tiles of K, two of V
    T(*const lk)[kKeys * D] = lds, (*const lv)[kKeys * D] = lds + 2;
    auto one = [&](int share, int kv, int id) {
        int b, tile;
        if (!locate(a.q_begin, a.tokens_q, a.batch, a.group, kRows, id, b, tile)) return;
        const Sequence s = sequence(a, b);
        const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, h = lane / 32;
        const int r0 = tile * kRows, rows = int(int64_t(s.nq) * a.group);
        const Row mine = row_of(a, s, kv, r0 + wave * 32 + lane % 32);
        // keys that some row of the workgroup sees: its last row sees most
        const int last = r0 + kRows < rows ? r0 + kRows - 1 : rows - 1, most = limit_of(a, s, query_of(a, last));
        const int all = (most + kKeys - 1) / kKeys, first = int(int64_t(all) * share / shares.count), end = int(int64_t(all) * (share + 1) / shares.count);
        // limits within the wavefront
        int wave_most = mine.limit, wave_least = mine.limit < 0 ? 1 << 30 : mine.limit;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            wave_most = max(wave_most, __shfl_xor(wave_most, d));
            wave_least = min(wave_least, __shfl_xor(wave_least, d));
        }
        wave_most = __builtin_amdgcn_readfirstlane(wave_most);
        wave_least = __builtin_amdgcn_readfirstlane(wave_least);

        const Along<T, D> along(lds[0]);
        const Across<T, D> across(lds[0]);
        f32x16 o[D / 32] = {}, p = {}, n = {};
        Frag w[2] = {};
        float top = -INFINITY, against = 0, sum = 0, shrink = 1;

        const T *keys = static_cast<const T *>(a.k) + (s.k0 + first * kKeys) * a.k_token + kv * a.k_step;
        const T *values = static_cast<const T *>(a.v) + (s.k0 + first * kKeys) * a.v_token + kv * a.v_step;
        Stream<T, D, kKeys, kThreads> sk, sv;
        sk.begin(keys, a.k_token);
        sv.begin(values, a.v_token);
        auto ask_k = [&](int t) {
            if (t < end) sk.ask(a.k_token, s.used - t * kKeys, a.head);
        };
        auto ask_v = [&](int t) {
            if (t < end) sv.ask(a.v_token, s.used - t * kKeys, a.head);
        };
        ask_k(first);
        ask_v(first);
        Frag q[D / 16];
        const T *from = static_cast<const T *>(a.q) + mine.token * a.q_token + mine.head * a.q_step;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) q[k] = eight<T>(from + 16 * k + 8 * h, mine.limit >= 0 && 16 * k + 8 * h < a.head);
        __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0): or the loop would wait for these, and with them for its own
        // Scores of half a tile of keys; weighted values of one.
        auto scores = [&](int buffer, int half) {
            f32x16 x = {};
#pragma unroll
            for (int k = 0; k < D / 16; ++k) x = Mfma32<T>::run(along.read(buffer * kKeys + half * 32, k), q[k], x);
            return x;
        };
        auto weigh = [&](int buffer, int half) {
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
                for (int m = 0; m < D / 32; ++m) o[m] = Mfma32<T>::run(across.read((2 + buffer) * kKeys + half * 32 + 16 * k, m), w[k], o[m]);
        };
        // Of step i's scores p: hides what a row does not see; the reference that exponents are taken against follows the maximum only
        // when that has grown by 2^kBehind over it (sums in 32 bits and weights of 16 have room for the factor), and o has then to
        // be shrunk once the weights of the step before are in it.
        auto hide = [&](int i, f32x16 &p) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
                if (i * 32 + 8 * (j / 4) + 4 * h + j % 4 >= mine.limit) p[j] = -INFINITY;
        };
        auto refer = [&](const f32x16 &p) -> bool {
            float high = p[0];
#pragma unroll
            for (int j = 1; j < 16; ++j) high = fmaxf(high, p[j]);
            high *= a.c;
            if (!__any(high > top + Weights<T>::kBehind)) return false;
            high = fmaxf(fmaxf(high, other_half(high)), top);
            shrink = top == high ? 1.0f : __builtin_amdgcn_exp2f(top - high);
            top = high;
            against = top == -INFINITY ? 0.0f : top - Weights<T>::kShift;
            sum *= shrink;
            return true;
        };
        // A step's weights are summed apart before they meet the sum of all: one rounding of that for 16 of them, or those that are less
        // than 2^-24 of it would be lost one by one, however many (2^16 of them beside a first key of weight 1: 6e-4 of the sum).
        auto weights = [&](f32x16 &p, Frag (&x)[2]) {
            float part[2] = {0, 0};
#pragma unroll
            for (int j = 0; j < 16; ++j) {
                p[j] = __builtin_amdgcn_exp2f(fmaf(p[j], a.c, -against));
                part[j % 2] += p[j];
                x[j / 8][j % 8] = T(p[j]);
            }
            sum += part[0] + part[1];
        };
        auto shrink_o = [&] {
#pragma unroll
            for (int m = 0; m < D / 32; ++m) o[m] *= shrink;
        };
        // A step's weights, while the matrix instructions make the next step's scores and the sum of the last one's weighted values.
        // Tile t's scores are made a step ahead, its weighted values a step behind, so K of a tile is in LDS a barrier before V.
        const int steps = min(2 * end, (wave_most + 31) / 32);       // of this wavefront
        // Written in the order in which it is to be issued: two matrix instructions, arithmetic that takes about as long, reads for the
        // pair after the next; the fences keep the compiler from sorting by kind (943 TFLOP/s at 4,096 x 4,096, not causal).
        auto step = [&](int k_buffer, int v_buffer, int half, f32x16 &now, f32x16 &next) {
            constexpr int kPairs = D / 16, kAhead = 2;
            Frag kf[kAhead + 1], vf[kAhead + 1], x[2];
            auto read = [&](int j) {
                kf[j % (kAhead + 1)] = along.read(k_buffer * kKeys + half * 32, j);
                vf[j % (kAhead + 1)] = across.read((2 + v_buffer) * kKeys + half * 32 + j / (D / 32) * 16, j % (D / 32));
            };
            auto fence = [] { __builtin_amdgcn_sched_barrier(0); };
#pragma unroll
            for (int j = 0; j < kAhead; ++j) read(j);
            fence();
            int grown = __builtin_amdgcn_readfirstlane(refer(now));
            asm volatile("" : "+s"(grown));                          // so that there is one copy of what follows, not one for either case
            float part[2] = {0, 0};
            auto summed = [&](int e) {                               // of exponentials
                part[e % 2] += now[e];
                x[e / 8][e % 8] = T(now[e]);
            };
            fence();
#pragma unroll
            for (int j = 0; j < kPairs; ++j) {
                const int from = 16 * j / kPairs, to = 16 * (j + 1) / kPairs, before = 16 * (j - 1) / kPairs;
                next = Mfma32<T>::run(kf[j % (kAhead + 1)], q[j], j ? next : f32x16{});
#pragma unroll
                for (int e = from; e < to; ++e) now[e] = __builtin_amdgcn_exp2f(fmaf(now[e], a.c, -against));
                fence();
                o[j % (D / 32)] = Mfma32<T>::run(vf[j % (kAhead + 1)], w[j / (D / 32)], o[j % (D / 32)]);
                if (j + kAhead < kPairs) read(j + kAhead);
                if (j > 0) {
#pragma unroll
                    for (int e = before; e < from; ++e) summed(e);
                }
                fence();
            }
#pragma unroll
            for (int e = 16 * (kPairs - 1) / kPairs; e < 16; ++e) summed(e);
            sum += part[0] + part[1];
            w[0] = x[0], w[1] = x[1];
            asm volatile("" : "+v"(w[0]), "+v"(w[1]), "+v"(sum));    // here, not where they are used
            if (grown) shrink_o();
        };
        auto edge = [&](int i, f32x16 &now, f32x16 &next) {          // a step that lacks one of these, or hides keys
            if (i > steps) return;
            if (i + 1 < steps) next = scores((i + 1) / 2 - first & 1, i + 1 & 1);
            if (i > 2 * first) weigh((i - 1) / 2 - first & 1, i - 1 & 1);
            if (i == steps) return;
            if (32 * i + 32 > wave_least) hide(i, now);
            if (refer(now)) shrink_o();
            weights(now, w);
        };
        if (first < end) {
            sk.put(lk[0]);
            sv.put(lv[0]);
        }
        ask_k(first + 1);
        ask_v(first + 1);
        __syncthreads();
        if (2 * first < steps) p = scores(0, 0);
        // A tile that lies in `buffer`; the next one's K is put behind its first step, V behind the barrier.
        auto whole = [&](int t, int buffer) {
            step(buffer, 1 - buffer, 1, p, n);
            sk.put(lk[1 - buffer]);
            ask_k(t + 2);
            __syncthreads();
            sv.put(lv[1 - buffer]);
            ask_v(t + 2);
            step(1 - buffer, buffer, 0, n, p);
        };
        auto partial = [&](int t) {
            const int next = t + 1 - first & 1;
            edge(2 * t, p, n);
            if (t + 1 < end) sk.put(lk[next]);
            ask_k(t + 2);
            __syncthreads();
            if (t + 1 < end) sv.put(lv[next]);
            ask_v(t + 2);
            edge(2 * t + 1, n, p);
        };
        // Loops of their own: the compiler merges what two branches of one have in common, and then nothing goes on meanwhile.  A whole
        // tile has another behind it and hides nothing.
        const int whole_end = min(end - 1, min((steps - 1) / 2, wave_least / kKeys));
        int t = first;
        if (t < end) partial(t++);
#pragma unroll 1
        for (; t + 1 < whole_end; t += 2) {
            whole(t, 1);
            whole(t + 1, 0);
        }
#pragma unroll 1
        for (; t < end; ++t) partial(t);
        if (first < end) edge(2 * end, p, n);                        // the last weighted values
        if (mine.limit < 0) return;
        sum += other_half(sum);
        if (sum == 0) {                                              // no key seen, or none of any weight: zeros whatever the values
#pragma unroll
            for (int m = 0; m < D / 32; ++m) o[m] = f32x16{};
        }
        if (shares.count > 1) {
            const int64_t at = (int64_t(share) * a.tokens_q + mine.token) * a.heads + mine.head;
            if (h == 0) {
                shares.stats[2 * at] = against;
                shares.stats[2 * at + 1] = sum;
            }
#pragma unroll
            for (int m = 0; m < D / 32; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int col = 32 * m + 8 * i + 4 * h;
                    if (col < a.head) *reinterpret_cast<f32x4 *>(shares.sums + at * a.head + col) = f32x4{o[m][4 * i], o[m][4 * i + 1], o[m][4 * i + 2], o[m][4 * i + 3]};
                }
            return;
        }
        const float scale = sum == 0 ? 0.0f : 1.0f / sum;    // no key: zeros; scores that are NaN: NaN
        if (a.lse && h == 0) a.lse[mine.head * a.tokens_q + mine.token] = sum == 0 ? -INFINITY : (against + __log2f(sum)) * kLn2;
        T *to = static_cast<T *>(a.o) + mine.token * a.o_token + mine.head * a.o_step;
#pragma unroll
        for (int m = 0; m < D / 32; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = 32 * m + 8 * i + 4 * h;
                if (col < a.head) store4(to + col, f32x4{o[m][4 * i] * scale, o[m][4 * i + 1] * scale, o[m][4 * i + 2] * scale, o[m][4 * i + 3] * scale});
            }
    };
    // Tiles of rows that see most keys first; with shares.paired a workgroup takes one of them and one of the least in turn.
    const Work work = work_of(blockIdx.x, shares.paired ? (tiles + 1) / 2 : tiles, shares.kv_heads, shares.count, a.causal);
#pragma unroll 1
    for (int turn = 0; turn < (shares.paired && work.place != tiles - 1 - work.place ? 2 : 1); ++turn) {
        if (turn) __syncthreads();               // all have read what lies in LDS
        one(work.share, shares.first_kv + work.kv, turn ? work.place : tiles - 1 - work.place);
    }
}

// Shares of the keys, joined: 32 lanes a row of four channels each, rows of sequences only.
template <typename T> __global__ __launch_bounds__(kJoinRows * 32) void forward_join(Call a, int tiles, Shares shares) {
    int b, tile;
    if (!locate(a.q_begin, a.tokens_q, a.batch, a.group, kJoinRows, blockIdx.x % tiles, b, tile)) return;
    const Sequence s = sequence(a, b);
    const Row mine = row_of(a, s, blockIdx.x / tiles, tile * kJoinRows + threadIdx.x / 32);
    if (mine.limit < 0) return;
    const int64_t each = a.tokens_q * a.heads, at = mine.token * a.heads + mine.head;
    // a lane looks at two shares' reference and sum
    const int lane = threadIdx.x % 32, col = lane * 4;
    float refer[2], part[2], top = -INFINITY, sum = 0;
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int i = lane + 32 * k;
        const float *stats = shares.stats + 2 * (i * each + at);
        part[k] = i < shares.count ? stats[1] : 0;
        refer[k] = part[k] == 0 ? -INFINITY : stats[0];
        top = fmaxf(top, refer[k]);
    }
#pragma unroll
    for (int d = 1; d < 32; d *= 2) top = fmaxf(top, __shfl_xor(top, d));
    float weight[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        weight[k] = part[k] == 0 ? 0.0f : refer[k] == top ? 1.0f : __builtin_amdgcn_exp2f(refer[k] - top);
        sum += weight[k] * part[k];
    }
#pragma unroll
    for (int d = 1; d < 32; d *= 2) sum += __shfl_xor(sum, d);
    f32x4 o = {0, 0, 0, 0};
    const float *sums = shares.sums + at * a.head + (col < a.head ? col : 0);
    int i = 0;
    for (; i + 8 <= shares.count; i += 8) {
        f32x4 x[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) x[k] = load4(sums + (i + k) * each * a.head);
#pragma unroll
        for (int k = 0; k < 8; ++k) o += __shfl(i < 32 ? weight[0] : weight[1], (i + k) % 32, 32) * x[k];
    }
    for (; i < shares.count; ++i) o += __shfl(i < 32 ? weight[0] : weight[1], i % 32, 32) * load4(sums + i * each * a.head);
    const float scale = sum == 0 ? 0.0f : 1.0f / sum;    // no key: zeros; scores that are NaN: NaN
    if (col < a.head) store4(static_cast<T *>(a.o) + mine.token * a.o_token + mine.head * a.o_step + col, o * scale);
    if (a.lse && col == 0) a.lse[mine.head * a.tokens_q + mine.token] = sum == 0 ? -INFINITY : (top + __log2f(sum)) * kLn2;
}

// ---------------------------------------------------------------------------------------------- gradients
struct Grads {
    const void *d_o;
    int64_t do_token, do_step, dq_token, dq_step, dk_token, dk_step, dv_token, dv_step;
    void *dq, *dk, *dv;
    float *delta;                    // [heads][tokens_q]: sum over channels of dO O, and one 0 behind
    float *against;                  // the same: what exponents of 2 are taken against, infinity behind and where no key is seen
    float *peaks;                    // HARP_F16: [2][kPeaks] largest finite squared norms of rows of dO and of V, one from each workgroup
    float scale;
};

// Weights and their gradients on their way into the matrix instructions.  In float16 weights go in times 2^12 as in the forward pass
// (10^5 equal ones of a row are still rounded to 2^-11 of themselves), and gradients times a power of two taken from the largest
// norms: |P (dP - D)| <= 2 |dO_i| |v_j|, which is brought to 2^14 at most.
constexpr int kPeaks = 512;
template <typename T> struct Range {
    static constexpr bool kNarrow = Weights<T>::kNarrow;
    static constexpr float kShift = Weights<T>::kShift, kWeight = kNarrow ? 0.000244140625f : 1.0f;
    float factor = 1;                // of dP - D where a weight carries 2^kShift
    __device__ __forceinline__ explicit Range(const float *peaks) {
        if constexpr (kNarrow) {
            uint32_t high[2] = {0, 0};                           // of floats that are not negative: as their bits
#pragma unroll
            for (int i = 0; i < kPeaks; i += kWave)
#pragma unroll
                for (int j = 0; j < 2; ++j) high[j] = larger(high[j], __float_as_uint(peaks[j * kPeaks + i + threadIdx.x % kWave]));
            const float bound = 4 * __uint_as_float(wave_max(high[0])) * __uint_as_float(wave_max(high[1]));
            int e = 0;
            if (bound > 0) {
                (void)frexpf(bound, &e);
                factor = ldexpf(1.0f, 14 - ((e + 1) >> 1) - int(kShift));
            }
        }
    }
    __device__ __forceinline__ float less(float dp, float delta) const { return kNarrow ? fmaf(dp, factor, -delta) : dp - delta; }     // delta times factor
    __device__ __forceinline__ float scaled(float ds) const { return kNarrow ? ds * factor : ds; }
    __device__ __forceinline__ float back() const { return kNarrow ? kWeight / factor : 1.0f; }       // of what gradients are summed into
};

// Sums over channels of dO O of every row of a sequence, 16 lanes a row; in HARP_F16 the largest norms of dO's rows too, and, by as many
// workgroups more (kPeaks), of V's.  A workgroup takes a tile of 128 rows in `groups`.
constexpr int kMeasured = 128;
template <typename T>
__global__ __launch_bounds__(256) void measure(Call a, Grads g, int of_q, int of_k, int groups) {
    __shared__ uint32_t highest[4];
    const bool q = int(blockIdx.x) < groups;
    if (blockIdx.x == 0 && threadIdx.x == 0) g.delta[a.heads * a.tokens_q] = 0, g.against[a.heads * a.tokens_q] = INFINITY;
    const int times = q ? a.heads : a.kv_heads, col = threadIdx.x % 16 * 8;
    uint32_t high = 0;
    for (int id = blockIdx.x % groups; id < (q ? of_q : of_k); id += groups) {
        int b, tile;
        if (!locate(q ? a.q_begin : a.k_begin, q ? a.tokens_q : a.tokens_k, a.batch, times, kMeasured, id, b, tile)) break;
        const Sequence s = sequence(a, b);
        const int64_t rows = int64_t(q ? s.nq : s.used) * times, first = int64_t(tile) * kMeasured;
#pragma unroll
        for (int i = 0; i < kMeasured / 16; ++i) {
            const int64_t r = first + i * 16 + threadIdx.x / 16, token = r / times, head = r % times;
            const bool there = r < rows && col < a.head;
            const T *from = q ? static_cast<const T *>(g.d_o) + (s.q0 + token) * g.do_token + head * g.do_step
                              : static_cast<const T *>(a.v) + (s.k0 + token) * a.v_token + head * a.v_step;
            const auto x = eight<T>(from + col, there);
            bool counts = true;
            if (q) {
                const auto y = eight<T>(static_cast<const T *>(a.o) + (s.q0 + token) * a.o_token + head * a.o_step + col, there);
                float d = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) d += to_f32(T(x[k])) * to_f32(T(y[k]));
                d = sum16(d);
                const int64_t at = head * a.tokens_q + s.q0 + token;
                float lse = 0;
                if (r < rows && (Range<T>::kNarrow || threadIdx.x % 16 == 0)) lse = a.lse[at];
                counts = lse != -INFINITY;
                if (r < rows && threadIdx.x % 16 == 0) {
                    g.delta[at] = d;
                    g.against[at] = lse == -INFINITY ? INFINITY : lse * kLog2e - Range<T>::kShift;
                }
            }
            if (Range<T>::kNarrow) {
                float d = 0;
#pragma unroll
                for (int k = 0; k < 8; ++k) d += to_f32(T(x[k])) * to_f32(T(x[k]));
                // not of rows that see nothing, nor of those that are not finite, whose results scaling does not save
                const uint32_t norm = __float_as_uint(sum16(d));
                if (counts && norm < 0x7f800000) high = larger(high, norm);
            }
        }
    }
    if (!Range<T>::kNarrow) return;
    high = wave_max(high);
    if (threadIdx.x % kWave == 0) highest[threadIdx.x / kWave] = high;
    __syncthreads();
    if (threadIdx.x == 0) g.peaks[blockIdx.x] = __uint_as_float(larger(larger(highest[0], highest[1]), larger(highest[2], highest[3])));
}

// dQ, as the forward pass goes: dQ^T = K^T dS^T, dS^T = P^T (V dO^T - delta).  4,096 queries and keys, 32 heads of 128, not causal: 350 us
// (1,180 TFLOP/s of its three products), causal 205 to 215.  Bound as the forward pass.  With 128 channels 3 and 7 registers (bfloat16,
// float16) are spilled by 8 wavefronts, 16 and 23 by 4.
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, 2) void grad_queries(Call a, Grads g, int tiles, Shares shares) {
    constexpr int kThreads = WAVES * kWave, kRows = WAVES * 32;
    typedef typename Mfma32<T>::Frag Frag;
    __shared__ __align__(1024) T lds[4][kKeys * D];               // two tiles of K, two of V
    T(*const lk)[kKeys * D] = lds, (*const lv)[kKeys * D] = lds + 2;
    auto one = [&](int share, int kv, int id) {
        int b, tile;
        if (!locate(a.q_begin, a.tokens_q, a.batch, a.group, kRows, id, b, tile)) return;
        const Sequence s = sequence(a, b);
        const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, h = lane / 32;
        const int r0 = tile * kRows, rows = int(int64_t(s.nq) * a.group);
        const Row mine = row_of(a, s, kv, r0 + wave * 32 + lane % 32);
        const int last = r0 + kRows < rows ? r0 + kRows - 1 : rows - 1, most = limit_of(a, s, query_of(a, last));
        const int all = (most + kKeys - 1) / kKeys, first = int(int64_t(all) * share / shares.count), end = int(int64_t(all) * (share + 1) / shares.count);
        const bool here = mine.limit >= 0;
        float lse = here ? a.lse[mine.head * a.tokens_q + mine.token] * kLog2e : 0;
        const Range<T> range(g.peaks);
        const float delta = here ? g.delta[mine.head * a.tokens_q + mine.token] * range.factor : 0;
        const int limit = lse == -INFINITY ? 0 : mine.limit;
        lse = lse == -INFINITY ? 0 : lse - Range<T>::kShift;
        int wave_most = limit, wave_least = limit < 0 ? 1 << 30 : limit;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            wave_most = max(wave_most, __shfl_xor(wave_most, d));
            wave_least = min(wave_least, __shfl_xor(wave_least, d));
        }
        wave_most = __builtin_amdgcn_readfirstlane(wave_most);
        wave_least = __builtin_amdgcn_readfirstlane(wave_least);
        Along<T, D> along(lds[0]);
        Across<T, D> across(lds[0]);
        f32x16 dq[D / 32] = {};
        const T *keys = static_cast<const T *>(a.k) + (s.k0 + first * kKeys) * a.k_token + kv * a.k_step;
        const T *values = static_cast<const T *>(a.v) + (s.k0 + first * kKeys) * a.v_token + kv * a.v_step;
        Stream<T, D, kKeys, kThreads> sk, sv;
        sk.begin(keys, a.k_token);
        sv.begin(values, a.v_token);
        auto ask = [&](int t) {
            if (t >= end) return;
            sk.ask(a.k_token, s.used - t * kKeys, a.head);
            sv.ask(a.v_token, s.used - t * kKeys, a.head);
        };
        ask(first);
        Frag q[D / 16], d_o[D / 16];
        const T *from = static_cast<const T *>(a.q) + mine.token * a.q_token + mine.head * a.q_step;
        const T *from_do = static_cast<const T *>(g.d_o) + mine.token * g.do_token + mine.head * g.do_step;
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
            q[k] = eight<T>(from + 16 * k + 8 * h, here && 16 * k + 8 * h < a.head);
            d_o[k] = eight<T>(from_do + 16 * k + 8 * h, here && 16 * k + 8 * h < a.head);
        }
        __builtin_amdgcn_s_waitcnt(0x0f70);          // vmcnt(0): or the loop would wait for these, and with them for its own
        // A tile's matrix instructions, one operand of each from LDS, and what goes on under them:
        //   S of the first 32 keys;  their dP, exponentials;  S of the others, dS of the first;  dP, exponentials;  dQ of the first,
        //   dS of the others;  dQ of those.
        constexpr int kPart = D / 16, kAhead = 2;
        auto tile_of_keys = [&](int t, int buffer, auto masked) {
            f32x16 p[2], dp[2];
            Frag f[kAhead + 1], w[2][2];
            auto read = [&](auto n) {
                constexpr int part = n / kPart, j = n % kPart;
                Frag &to = f[n % (kAhead + 1)];
                if (part < 4) to = along.read((part % 2 * 2 + buffer) * kKeys + part / 2 * 32, j);
                else to = across.read(buffer * kKeys + (part - 4) * 32 + j / (D / 32) * 16, j % (D / 32));
            };
            auto exponential = [&](int u, int e) { p[u][e] = __builtin_amdgcn_exp2f(fmaf(p[u][e], a.c, -lse)); };
            auto gradient = [&](int u, int e) {
                float ds = p[u][e] * range.less(dp[u][e], delta);
                if (masked.value && t * kKeys + 32 * u + 8 * (e / 4) + 4 * h + e % 4 >= limit) ds = 0;
                w[u][e / 8][e % 8] = T(ds);
            };
            written_out<kAhead>(read);
            written_out<6 * kPart>([&](auto n) {
                constexpr int part = n / kPart, j = n % kPart, from = 16 * j / kPart, to = 16 * (j + 1) / kPart;
                const Frag &x = f[n % (kAhead + 1)];
                if constexpr (part == 0 || part == 2) p[part / 2] = Mfma32<T>::run(x, q[j], j ? p[part / 2] : f32x16{});
                else if constexpr (part == 1 || part == 3) dp[part / 2] = Mfma32<T>::run(x, d_o[j], j ? dp[part / 2] : f32x16{});
                else dq[j % (D / 32)] = Mfma32<T>::run(x, w[part - 4][j / (D / 32)], dq[j % (D / 32)]);
                if constexpr (n + kAhead < 6 * kPart) read(std::integral_constant<int, n + kAhead>());
#pragma unroll
                for (int e = from; e < to; ++e) {
                    if (part == 1 || part == 3) exponential(part / 2, e);
                    if (part == 2) gradient(0, e);
                    if (part == 4) gradient(1, e);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        if (first < end) {
            sk.put(lk[0]);
            sv.put(lv[0]);
        }
        ask(first + 1);
        __syncthreads();
        const int whole = min(end, wave_least / kKeys);              // tiles of which nothing is hidden
        auto turn = [&](int t, int buffer, auto masked) {
            along.refresh();
            across.refresh();
            if (t * kKeys < wave_most) tile_of_keys(t, buffer, masked);
            if (t + 1 < end) {
                sk.put(lk[1 - buffer]);
                sv.put(lv[1 - buffer]);
            }
            ask(t + 2);
            __syncthreads();
        };
        int t = first;
#pragma unroll 1
        for (; t + 1 < whole; t += 2) {
            turn(t, 0, std::false_type());
            turn(t + 1, 1, std::false_type());
        }
#pragma unroll 1
        for (; t < end; ++t) turn(t, t - first & 1, std::true_type());
        if (!here) return;
        if (limit == 0) {                                            // nothing seen: zeros whatever the keys
#pragma unroll
            for (int m = 0; m < D / 32; ++m) dq[m] = f32x16{};
        }
        const float scale = g.scale * range.back();
        float *sums = shares.sums + ((int64_t(share) * a.tokens_q + mine.token) * a.heads + mine.head) * a.head;
        T *to = static_cast<T *>(g.dq) + mine.token * g.dq_token + mine.head * g.dq_step;
#pragma unroll
        for (int m = 0; m < D / 32; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int col = 32 * m + 8 * i + 4 * h;
                if (col >= a.head) continue;
                const f32x4 v = f32x4{dq[m][4 * i], dq[m][4 * i + 1], dq[m][4 * i + 2], dq[m][4 * i + 3]} * scale;
                if (shares.count > 1) *reinterpret_cast<f32x4 *>(sums + col) = v;
                else store4(to + col, v);
            }
    };
    // Tiles of rows that see most keys first; with shares.paired a workgroup takes one of them and one of the least in turn.
    const Work work = work_of(blockIdx.x, shares.paired ? (tiles + 1) / 2 : tiles, shares.kv_heads, shares.count, a.causal);
#pragma unroll 1
    for (int turn = 0; turn < (shares.paired && work.place != tiles - 1 - work.place ? 2 : 1); ++turn) {
        if (turn) __syncthreads();               // all have read what lies in LDS
        one(work.share, shares.first_kv + work.kv, turn ? work.place : tiles - 1 - work.place);
    }
}

// A value of which the compiler keeps nothing that it has made of it before: in registers that are wanted otherwise.
__device__ __forceinline__ int anew(int x) {
    asm volatile("" : "+v"(x));
    return x;
}

// 4 bytes a lane from `from` to LDS, lane after lane from `to` on (the same for the wavefront): without a register for them on their way.
// m0 is named so that the compiler keeps no value of its own there; that it hands m0 out to nobody is what its warning, turned off
// here, is about.  What waits for it is written out too: the compiler does not count it.
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
__device__ __forceinline__ void word_to_lds(const float *from, uint32_t to) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(to), "v"(from) : "memory", "m0");
}
#pragma clang diagnostic pop

// dK and dV of 32 keys a wavefront, whose rows come through LDS kBack at a time.  dV^T = dO^T P, dK^T = Q^T dS, where a lane has
// 16 rows of one key: both sums of a wavefront stay in registers over all rows and heads of the group, 128 of 256 with 128 channels, so
// that nothing is added up in memory but shares.  4,096 queries and keys, 32 heads of 128, bfloat16, not causal: 530 us (1,040 TFLOP/s of
// its four products), matrix units busy 51%; causal 310 to 330.  Bound as the forward pass, and by registers: with five of them spilled,
// whose reloads wait for the rows on their way, it took 590.  8 wavefronts spill none; 4, which take few keys, spill 9 and 10 with 128
// channels (bfloat16, float16), one or two of them reloaded every step.
template <typename T, int D, int WAVES>
__global__ __launch_bounds__(WAVES * kWave, 2) void grad_keys(Call a, Grads g, int tiles, Shares shares) {
    constexpr int kThreads = WAVES * kWave, kCols = WAVES * 32;
    typedef typename Mfma32<T>::Frag Frag;
    __shared__ __align__(1024) T lds[4][kBack * D];               // two steps of Q, two of dO
    __shared__ __align__(1024) T lv[kCols * D];
    __shared__ __align__(16) float l_stat[2][2 * kBack];          // against and delta of a step's rows
    __shared__ __align__(16) int l_limit[2][kBack];
    const Work work = work_of(blockIdx.x, tiles, shares.kv_heads, shares.count, a.causal);
    const int share = work.share, kv = shares.first_kv + work.kv;
    int b, tile;
    if (!locate(a.k_begin, a.tokens_k, a.batch, 1, kCols, work.place, b, tile)) return;
    const Sequence s = sequence(a, b);
    const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, h = lane / 32;
    const int key0 = tile * kCols, key = key0 + wave * 32 + lane % 32, rows = int(int64_t(s.nq) * a.group);
    const bool used = key < s.used;
    // rows that see none of the workgroup's keys come first, if any
    int skip = a.causal ? key0 - (s.used - s.nq) : 0;
    skip = skip < 0 ? 0 : skip;
    const int64_t begin_row = int64_t(skip) * a.group;
    const int all = key0 < s.used && begin_row < rows ? int((rows - begin_row + kBack - 1) / kBack) : 0, row_first = int(begin_row);
    const int first = int(int64_t(all) * share / shares.count), end = int(int64_t(all) * (share + 1) / shares.count);
    Frag k[D / 16];
    const T *from_k = static_cast<const T *>(a.k) + (s.k0 + (used ? key : 0)) * a.k_token + kv * a.k_step;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) k[i] = eight<T>(from_k + 16 * i + 8 * h, used && 16 * i + 8 * h < a.head);
    // V stays in LDS: dK and dV leave no room for it in registers
    Stage<T, D, kCols, kThreads> sv;
    const T *values = static_cast<const T *>(a.v) + (s.k0 + key0) * a.v_token + kv * a.v_step;
    sv.ask([&](int row) { return values + row * a.v_token; }, s.used - key0, a.head);
    // of rows in the buffer of the step, by turns one and the other; of V
    Along<T, D> along(lds[0]), along_v(lv + wave * 32 * D);
    Across<T, D> across(lds[0]);
    f32x16 dk[D / 32] = {}, dv[D / 32] = {};
    Stage<T, D, kBack, kThreads> sq, sd;
    const Range<T> range(g.peaks);
    const int wave_id = __builtin_amdgcn_readfirstlane(int(threadIdx.x)) / kWave;
    auto ask = [&](int t) {
        const int r0 = row_first + t * kBack;
        auto place = [&](int row, int64_t token, int64_t step) {
            const int query = query_of(a, r0 + row);
            return (s.q0 + query) * token + (kv * a.group + r0 + row - query * a.group) * step;
        };
        sq.ask([&](int row) { return static_cast<const T *>(a.q) + place(row, a.q_token, a.q_step); }, rows - r0, a.head);
        sd.ask([&](int row) { return static_cast<const T *>(g.d_o) + place(row, g.do_token, g.do_step); }, rows - r0, a.head);
        // of no row: what makes every weight 0
        if (wave_id == 0) {
            const int id = anew(int(threadIdx.x)), row = id % 32;
            word_to_lds((id < 32 ? g.against : g.delta) + (r0 + row < rows ? place(row, 1, a.tokens_q) : a.heads * a.tokens_q), lds_address(l_stat[t - first & 1]));
        }
    };
    auto put = [&](int t) {
        const int at = t - first & 1;
        sq.put(lds[at]);
        sd.put(lds[2 + at]);
        if (a.causal && threadIdx.x < kBack) {
            const int row = anew(int(threadIdx.x));
            l_limit[at][row] = limit_of(a, s, query_of(a, row_first + t * kBack + row));
        }
        asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    };
    if (first < end) ask(first);
    sv.put(lv);
    if (first < end) put(first);
    __syncthreads();
    // A step's matrix instructions and what goes on under them:  S;  dP, weights;  dV, their gradients;  dK.
    constexpr int kPart = D / 16, kAhead = 2;
    auto rows_step = [&](int at, bool masked) {
        const float *stats = l_stat[at] + 4 * h;
        f32x16 p, dp;
        Frag f[kAhead + 1], v[2], w[2], ds[2];
        auto read = [&](auto n) {
            constexpr int part = n / kPart, j = n % kPart;
            Frag &to = f[n % (kAhead + 1)];
            if (part < 2) to = along.read(part * 2 * kBack, j);
            else to = across.read((part == 2 ? 2 * kBack : 0) + j / (D / 32) * 16, j % (D / 32));
        };
        written_out<kAhead>(read);
        f32x4 against = {}, less = {};
        written_out<4 * kPart>([&](auto n) {
            constexpr int part = n / kPart, j = n % kPart, from = 16 * j / kPart, to = 16 * (j + 1) / kPart;
            const Frag &x = f[n % (kAhead + 1)];
            if constexpr (part == 2 && j == 0) {
                if (masked) {
#pragma unroll
                    for (int e = 0; e < 16; ++e)
                        if (key >= l_limit[at][8 * (e / 4) + 4 * h + e % 4]) p[e] = 0;
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e / 8][e % 8] = T(p[e]);
            }
            if constexpr (part == 0) p = Mfma32<T>::run(x, k[j], j ? p : f32x16{});
            else if constexpr (part == 1) dp = Mfma32<T>::run(x, v[n % 2], j ? dp : f32x16{});
            else if constexpr (part == 2) dv[j % (D / 32)] = Mfma32<T>::run(x, w[j / (D / 32)], dv[j % (D / 32)]);
            else dk[j % (D / 32)] = Mfma32<T>::run(x, ds[j / (D / 32)], dk[j % (D / 32)]);
            if constexpr (n + kAhead < 4 * kPart) read(std::integral_constant<int, n + kAhead>());
            if constexpr (n + 1 >= kPart && n + 1 < 2 * kPart) v[(n + 1) % 2] = along_v.read(0, n + 1 - kPart);
#pragma unroll
            for (int e = from; e < to; ++e) {
                if (part == 1) {
                    if (e % 4 == 0) against = *reinterpret_cast<const f32x4 *>(stats + 8 * (e / 4));
                    p[e] = __builtin_amdgcn_exp2f(fmaf(p[e], a.c, -against[e % 4]));
                }
                if (part == 2) {
                    if (e % 4 == 0) less = *reinterpret_cast<const f32x4 *>(stats + kBack + 8 * (e / 4));
                    ds[e / 8][e % 8] = T(range.scaled(p[e] * (dp[e] - less[e % 4])));
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        });
    };
    // Under the causal order the first rows may see none or not all of the wavefront's keys.
    const int64_t none = a.causal ? int64_t(key0 + wave * 32 - s.used + s.nq) * a.group : 0, some = a.causal ? none + 31 * a.group : 0;
#pragma unroll 1
    for (int t = first; t < end; ++t) {
        const int at = t - first & 1;
        if (t + 1 < end) ask(t + 1);
        along.refresh();
        along_v.refresh();
        across.refresh();
        const int r0 = row_first + t * kBack;
        if (r0 + kBack > none) rows_step(at, r0 < some);
        const uint32_t other = at ? -uint32_t(kBack * D * 2) : kBack * D * 2;
        along.at += other;
        across.at += other;
        if (t + 1 < end) put(t + 1);
        __syncthreads();
    }
    // what keys that are not used were given has stayed in their own columns
    if (!used) {
#pragma unroll
        for (int m = 0; m < D / 32; ++m) dk[m] = dv[m] = f32x16{};
    }
    if (key >= s.nk) return;
    const float scale = g.scale * range.back();
    const int64_t token = s.k0 + key, each = a.tokens_k * a.kv_heads * a.head;
    float *sums = shares.sums + 2 * share * each + (token * a.kv_heads + kv) * a.head;
    T *to_k = static_cast<T *>(g.dk) + token * g.dk_token + kv * g.dk_step, *to_v = static_cast<T *>(g.dv) + token * g.dv_token + kv * g.dv_step;
#pragma unroll
    for (int m = 0; m < D / 32; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int col = 32 * m + 8 * i + 4 * h;
            if (col >= a.head) continue;
            const f32x4 x = f32x4{dk[m][4 * i], dk[m][4 * i + 1], dk[m][4 * i + 2], dk[m][4 * i + 3]} * scale;
            const f32x4 y = f32x4{dv[m][4 * i], dv[m][4 * i + 1], dv[m][4 * i + 2], dv[m][4 * i + 3]} * Range<T>::kWeight;
            if (shares.count > 1) {
                *reinterpret_cast<f32x4 *>(sums + col) = x;
                *reinterpret_cast<f32x4 *>(sums + each + col) = y;
            } else {
                if (g.dk) store4(to_k + col, x);
                if (g.dv) store4(to_v + col, y);
            }
        }
}

// Sums of shares, in their order, for the rows of sequences: `rows` of them per token of begin's spans, share i's of element (token, row)
// at first + i * stride + .., to p.  Two results that lie alike in one launch.
template <typename T> struct Joined {
    T *p;
    int64_t token, step, first;
};
template <typename T>
__global__ __launch_bounds__(kJoinRows * 32) void join_sums(const int32_t *begin, int64_t tokens, int batch, int rows, int head, const float *sums, int count,
                                                            int64_t stride, Joined<T> one, Joined<T> two) {
    const Joined<T> to = blockIdx.y ? two : one;
    int b, tile;
    if (!to.p) return;
    if (!locate(begin, tokens, batch, rows, kJoinRows, blockIdx.x, b, tile)) return;
    int64_t first;
    int n;
    span(begin, tokens, batch, b, first, n);
    const int64_t r = int64_t(tile) * kJoinRows + threadIdx.x / 32;
    const int col = threadIdx.x % 32 * 4;
    if (r >= int64_t(n) * rows || col >= head) return;
    const int64_t token = first + r / rows, row = r % rows;
    const float *at = sums + to.first + (token * rows + row) * head + col;
    f32x4 x = {0, 0, 0, 0};
#pragma unroll 4
    for (int i = 0; i < count; ++i) x += load4(at + i * stride);
    store4(to.p + token * to.token + row * to.step + col, x);
}

// ---------------------------------------------------------------------------------------------- on the host
// Where parts of the workspace begin; what the passes need of these plans.
struct Space { size_t peaks, stats, sums, all; };
Space space_for(const harp_attention *g, const Plan *q, const Plan *k) {
    const size_t rows = size_t(g->tokens_q) * g->heads, kv = size_t(g->tokens_k) * g->kv_heads;
    Space s = {};
    s.peaks = 2 * round_up((rows + 1) * 4, 256);         // behind delta and against
    s.stats = s.peaks + 2 * kPeaks * 4;
    s.sums = s.stats + (q && q->shares > 1 ? round_up(rows * q->shares * 8, 256) : 0);
    const size_t of_q = q && q->shares > 1 ? rows * q->shares * g->head * 4 : 0, of_k = k && k->shares > 1 ? kv * k->shares * g->head * 8 : 0;
    s.all = s.sums + round_up(of_q > of_k ? of_q : of_k, 256) + 256;
    return s;
}

int attention_sizes(harp_ctx *ctx, const harp_attention *g) {
    if (!sizes_fit(g))
        return fail(ctx, HARP_ERR_SHAPE, "tokens, batch, heads, kv_heads or head out of range: %lld and %lld tokens, batch %d, %d heads, %d of keys, head %d",
                    (long long)g->tokens_q, (long long)g->tokens_k, g->batch, g->heads, g->kv_heads, g->head);
    return HARP_OK;
}

struct Tensor { const char *name; const void *p; int64_t tokens, heads, token, step; bool needed, written; };

// q, k: how the call is launched; k is null in the forward pass.
int check(harp_ctx *ctx, const harp_attention *g, const Tensor *t, int count, const void *workspace, size_t workspace_bytes, Plan *q, Plan *k,
          Space *space) {
    const int rc = attention_sizes(ctx, g);
    if (rc != HARP_OK) return rc;
    if (g->type != HARP_BF16 && g->type != HARP_F16) return fail(ctx, HARP_ERR_INVALID_ARG, "type must be HARP_BF16 or HARP_F16");
    if (!(g->scale > 0) || !isfinite(g->scale * kLog2e)) return fail(ctx, HARP_ERR_INVALID_ARG, "scale must be positive and below 2^127");
    if ((!g->q_begin && g->tokens_q % g->batch) || (!g->k_begin && g->tokens_k % g->batch))
        return fail(ctx, HARP_ERR_SHAPE, "tokens are no multiple of the batch, and begins are missing");
    if (!aligned(g->q_begin, 4) || !aligned(g->k_begin, 4) || !aligned(g->k_count, 4) || !aligned(g->lse, 4))
        return fail(ctx, HARP_ERR_INVALID_ARG, "begins, counts or lse are not aligned to their elements");
    const int64_t far = int64_t(1) << 40;
    for (int i = 0; i < count; ++i) {
        if (!t[i].p && t[i].needed && t[i].tokens > 0) return fail(ctx, HARP_ERR_INVALID_ARG, "null %s", t[i].name);
        if (!t[i].p) continue;
        if (!aligned(t[i].p, 2)) return fail(ctx, HARP_ERR_INVALID_ARG, "%s is not aligned to its elements", t[i].name);
        if (t[i].token < 0 || t[i].step < 0 || t[i].token > far || t[i].step > far)
            return fail(ctx, HARP_ERR_SHAPE, "%s: distances must be in 0 .. 2^40", t[i].name);
        if (t[i].written && !clear_of_each_other(t[i].tokens, t[i].heads, g->head, t[i].token, t[i].step))
            return fail(ctx, HARP_ERR_SHAPE, "%s: elements lie over each other", t[i].name);
        for (int j = 0; t[i].written && j < count; ++j)
            if (j != i && t[j].p == t[i].p && t[i].tokens > 0 && t[j].tokens > 0)
                return fail(ctx, HARP_ERR_INVALID_ARG, "%s is %s", t[i].name, t[j].name);
    }
    *q = plan_queries(ctx->n_cu, g, g->causal);
    if (k) *k = plan_keys(ctx->n_cu, g, g->causal);
    *space = space_for(g, q, k);
    const size_t need = space->all;
    if (!workspace || !aligned(workspace, 256) || workspace_bytes < need)
        return fail(ctx, HARP_ERR_WORKSPACE, "the workspace needs %zu bytes, aligned to 256", need);
    const int64_t half = int64_t(1) << 31;
    const bool fits = tiles_of(g->tokens_q, g->heads, g->batch, kMeasured) < half && tiles_of(g->tokens_k, g->kv_heads, g->batch, kMeasured) < half;
    if (!fits)
        return fail(ctx, HARP_ERR_SHAPE, "too many rows for one launch");
    const hipError_t e = hipSetDevice(ctx->device);
    return e == hipSuccess ? HARP_OK : hip_fail(ctx, e, "hipSetDevice");
}

Call call_of(const harp_attention *g) {
    Call a = {};
    a.tokens_q = g->tokens_q, a.tokens_k = g->tokens_k;
    a.batch = g->batch, a.heads = g->heads, a.kv_heads = g->kv_heads, a.head = g->head, a.group = g->heads / g->kv_heads, a.causal = g->causal;
    a.group_magic = uint32_t((uint64_t(1) << 32) / uint32_t(a.group));
    a.c = g->scale * kLog2e;
    a.q_begin = g->q_begin, a.k_begin = g->k_begin, a.k_count = g->k_count;
    a.q_token = g->q_token, a.q_step = g->q_step, a.k_token = g->k_token, a.k_step = g->k_step, a.v_token = g->v_token, a.v_step = g->v_step;
    a.o_token = g->o_token, a.o_step = g->o_step;
    a.q = g->Q, a.k = g->K, a.v = g->V, a.o = g->O, a.lse = g->lse;
    return a;
}

int launched(harp_ctx *ctx) {
    const hipError_t e = hipGetLastError();
    return e == hipSuccess ? HARP_OK : hip_fail(ctx, e, "launching the attention's kernels");
}

// A pass in as many launches as its kv heads take: one, but for a great many short sequences.
template <typename L> void over_heads(const Plan &p, int kv_heads, Shares shares, L launch) {
    const int most = int(p.heads_of_a_launch(kv_heads));
    for (int first = 0; first < kv_heads; first += most) {
        shares.first_kv = first;
        shares.kv_heads = kv_heads - first < most ? kv_heads - first : most;
        launch(dim3(uint32_t(p.places() * p.shares * shares.kv_heads)), shares);
    }
}
template <typename T, int D> void launch_forward(const Plan &p, const Call &a, const Shares &all, hipStream_t st) {
    over_heads(p, a.kv_heads, all, [&](dim3 grid, const Shares &shares) {
        if (p.waves == 8) forward<T, D, 8><<<grid, dim3(512), 0, st>>>(a, int(p.tiles), shares);
        else forward<T, D, 4><<<grid, dim3(256), 0, st>>>(a, int(p.tiles), shares);
    });
}
template <typename T, int D> void launch_queries(const Plan &p, const Call &a, const Grads &g, const Shares &all, hipStream_t st) {
    over_heads(p, a.kv_heads, all, [&](dim3 grid, const Shares &shares) {
        if (p.waves == 8) grad_queries<T, D, 8><<<grid, dim3(512), 0, st>>>(a, g, int(p.tiles), shares);
        else grad_queries<T, D, 4><<<grid, dim3(256), 0, st>>>(a, g, int(p.tiles), shares);
    });
}
template <typename T, int D> void launch_keys(const Plan &p, const Call &a, const Grads &g, const Shares &all, hipStream_t st) {
    over_heads(p, a.kv_heads, all, [&](dim3 grid, const Shares &shares) {
        if (p.waves == 8) grad_keys<T, D, 8><<<grid, dim3(512), 0, st>>>(a, g, int(p.tiles), shares);
        else grad_keys<T, D, 4><<<grid, dim3(256), 0, st>>>(a, g, int(p.tiles), shares);
    });
}

template <typename T> void run_forward(const harp_attention *g, const Plan &p, const Space &space, unsigned char *ws, hipStream_t st) {
    const Call a = call_of(g);
    const Shares shares = {p.shares, p.paired, reinterpret_cast<float *>(ws + space.sums), reinterpret_cast<float *>(ws + space.stats), 0, 0};
    if (g->head <= 64) launch_forward<T, 64>(p, a, shares, st);
    else if (g->head <= 96) launch_forward<T, 96>(p, a, shares, st);
    else launch_forward<T, 128>(p, a, shares, st);
    if (p.shares > 1) {
        const int64_t tiles = tiles_of(g->tokens_q, a.group, g->batch, kJoinRows);
        forward_join<T><<<dim3(uint32_t(query_joins(g))), dim3(kJoinRows * 32), 0, st>>>(a, int(tiles), shares);
    }
}

template <typename T>
void run_backward(const harp_attention *g, const harp_attention_grads *d, const Plan &of_queries, const Plan &of_keys, const Space &space,
                  unsigned char *ws, hipStream_t st) {
    const Call a = call_of(g);
    const Grads grads = {d->dO, d->do_token, d->do_step, d->dq_token, d->dq_step, d->dk_token, d->dk_step, d->dv_token, d->dv_step,
                         d->dQ, d->dK, d->dV, reinterpret_cast<float *>(ws), reinterpret_cast<float *>(ws + space.peaks / 2), reinterpret_cast<float *>(ws + space.peaks), g->scale};
    const int64_t rows = g->tokens_q * g->heads;
    float *sums = reinterpret_cast<float *>(ws + space.sums);
    const int of_q = int(tiles_of(g->tokens_q, g->heads, g->batch, kMeasured)), of_k = int(tiles_of(g->tokens_k, g->kv_heads, g->batch, kMeasured));
    const int groups = Range<T>::kNarrow ? kPeaks : of_q < 1 ? 1 : of_q < 8192 ? of_q : 8192;
    measure<T><<<dim3(Range<T>::kNarrow ? 2 * kPeaks : groups), dim3(256), 0, st>>>(a, grads, of_q, of_k, groups);
    if (d->dQ && rows) {
        const Plan &p = of_queries;
        const Shares shares = {p.shares, p.paired, sums, nullptr, 0, 0};
        if (g->head <= 64) launch_queries<T, 64>(p, a, grads, shares, st);
        else if (g->head <= 96) launch_queries<T, 96>(p, a, grads, shares, st);
        else launch_queries<T, 128>(p, a, grads, shares, st);
        if (p.shares > 1)
            join_sums<T><<<dim3(uint32_t(tiles_of(g->tokens_q, g->heads, g->batch, kJoinRows))), dim3(kJoinRows * 32), 0, st>>>(
                a.q_begin, a.tokens_q, a.batch, a.heads, a.head, sums, p.shares, rows * a.head, Joined<T>{static_cast<T *>(d->dQ), d->dq_token, d->dq_step, 0}, Joined<T>());
    }
    if ((d->dK || d->dV) && g->tokens_k) {
        const Plan &p = of_keys;
        const Shares shares = {p.shares, p.paired, sums, nullptr, 0, 0};
        if (g->head <= 64) launch_keys<T, 64>(p, a, grads, shares, st);
        else if (g->head <= 96) launch_keys<T, 96>(p, a, grads, shares, st);
        else launch_keys<T, 128>(p, a, grads, shares, st);
        if (p.shares > 1) {
            const int64_t each = a.tokens_k * a.kv_heads * a.head;
            join_sums<T><<<dim3(uint32_t(tiles_of(g->tokens_k, g->kv_heads, g->batch, kJoinRows)), 2), dim3(kJoinRows * 32), 0, st>>>(
                a.k_begin, a.tokens_k, a.batch, a.kv_heads, a.head, sums, p.shares, 2 * each,
                Joined<T>{static_cast<T *>(d->dK), d->dk_token, d->dk_step, 0}, Joined<T>{static_cast<T *>(d->dV), d->dv_token, d->dv_step, each});
        }
    }
}

}  // namespace

extern "C" {

size_t harp_attention_workspace_bytes(harp_ctx *ctx, const harp_attention *g) {
    if (!ctx || !g || attention_sizes(ctx, g) != HARP_OK) return 0;
    size_t most = 0;
    for (int causal = 0; causal < 2; ++causal) {
        const Plan q = plan_queries(ctx->n_cu, g, causal), k = plan_keys(ctx->n_cu, g, causal);
        const size_t all = space_for(g, &q, &k).all;
        most = all > most ? all : most;
    }
    return most;
}

int harp_attention_forward(harp_ctx *ctx, const harp_attention *g, void *workspace, size_t workspace_bytes, void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!g) return fail(ctx, HARP_ERR_INVALID_ARG, "null args");
    const bool some = g->tokens_q > 0;
    const Tensor t[] = {{"Q", g->Q, g->tokens_q, g->heads, g->q_token, g->q_step, true, false},
                        {"K", g->K, some ? g->tokens_k : 0, g->kv_heads, g->k_token, g->k_step, true, false},
                        {"V", g->V, some ? g->tokens_k : 0, g->kv_heads, g->v_token, g->v_step, true, false},
                        {"O", g->O, g->tokens_q, g->heads, g->o_token, g->o_step, true, true}};
    Plan p;
    Space space;
    const int rc = check(ctx, g, t, 4, workspace, workspace_bytes, &p, nullptr, &space);
    if (rc != HARP_OK || !some) return rc;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) run_forward<__bf16>(g, p, space, static_cast<unsigned char *>(workspace), st);
    else run_forward<_Float16>(g, p, space, static_cast<unsigned char *>(workspace), st);
    return launched(ctx);
}

int harp_attention_backward(harp_ctx *ctx, const harp_attention *g, const harp_attention_grads *d, void *workspace, size_t workspace_bytes,
                            void *hip_stream) {
    if (!ctx) return HARP_ERR_INVALID_ARG;
    if (!g || !d) return fail(ctx, HARP_ERR_INVALID_ARG, "null args");
    if (!g->lse && g->tokens_q > 0) return fail(ctx, HARP_ERR_INVALID_ARG, "null lse");
    const Tensor t[] = {{"Q", g->Q, g->tokens_q, g->heads, g->q_token, g->q_step, true, false},
                        {"K", g->K, g->tokens_k, g->kv_heads, g->k_token, g->k_step, true, false},
                        {"V", g->V, g->tokens_k, g->kv_heads, g->v_token, g->v_step, true, false},
                        {"O", g->O, g->tokens_q, g->heads, g->o_token, g->o_step, true, false},
                        {"dO", d->dO, g->tokens_q, g->heads, d->do_token, d->do_step, true, false},
                        {"dQ", d->dQ, g->tokens_q, g->heads, d->dq_token, d->dq_step, false, true},
                        {"dK", d->dK, g->tokens_k, g->kv_heads, d->dk_token, d->dk_step, false, true},
                        {"dV", d->dV, g->tokens_k, g->kv_heads, d->dv_token, d->dv_step, false, true}};
    Plan q, k;
    Space space;
    const int rc = check(ctx, g, t, 8, workspace, workspace_bytes, &q, &k, &space);
    if (rc != HARP_OK) return rc;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (g->type == HARP_BF16) run_backward<__bf16>(g, d, q, k, space, static_cast<unsigned char *>(workspace), st);
    else run_backward<_Float16>(g, d, q, k, space, static_cast<unsigned char *>(workspace), st);
    return launched(ctx);
}

}  // extern "C"
