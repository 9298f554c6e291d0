// Attention of several new tokens of a sequence: query row (token i, head h) attends to the n cached tokens, as the cache holds
// them, and to the new tokens 0 .. i.
//
// Rows of one kv head (its query heads x the new tokens) share every key and value, so keys and values are brought to fp16 once a
// work-group, in LDS, and the products are matrix products:
//   S^T = K Q^T   (32 x 32 x 16 instructions: rows are tokens, columns query rows)
//   O^T = V^T P^T (rows are channels)
// With the transposed products a lane holds sixteen scores of ONE query row, so the softmax statistics are the lane's own but for one
// exchange of the two halves of a wavefront, and its weights are, rounded to fp16, the operand of the second product where they stand: the order of
// the tokens inside a product does not matter as long as both operands agree, so V^T is laid out in LDS in the order in which the first
// product leaves the tokens (16 tokens: 0 8 1 9 2 10 3 11 4 12 ...), which is also the order in which fields come out of packed words
// two at a time.  Keys use the same order for channels, queries are brought into it once.
//
// Stored fields become fp16 exactly: masked in place under the exponent that gives their bits weight one (1024 + u, 256 + u, ..), that
// constant subtracted (exact), then one fused |S| u + Z rounded to fp16 (relative 2^-12 rms, as the weights; scores, statistics and sums are fp32).
//
// The softmax reference level is put 2^9 below the score that raises it, and raised again only when a score passes it by 2^15: the outputs are
// scaled rarely, and weights keep fp16's full precision down to 2^-23 of the largest one and some of it down to 2^-34.  (With the level at the
// largest score, tokens 17 nats below it were off by 14 % and those 18 below it lost, which a long flat tail of them is not.)
//
// Many rows are bound by the matrix and the vector pipes, which hardly overlap: 2048 new tokens over 32k cached ones (32 / 8 heads, 4 bits)
// take 1160 to 1230 us by session, 980 to 920 TFLOP/s, the matrix pipes 49 % and the vector pipes 54 % busy (a large library product: 1270 to
// 1320 TFLOP/s).  Few rows are bound by the decoding: 5 new tokens over 8 x 32k at 2 bits 77 to 82 us, 2.7 to 2.5 TB/s, vector pipes 69 %
// busy; without the decoding 63 us of 87 remained.
#include "attention_chunk.h"

#ifndef INNERQ_CHUNK_G
#define INNERQ_CHUNK_G 32
#endif

namespace innerq {
namespace {

typedef _Float16 half2_t __attribute__((ext_vector_type(2)));
typedef _Float16 half8_t __attribute__((ext_vector_type(8)));
typedef float float16_t __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

constexpr int D = kHeadDim;
constexpr int kKeyPitch = 2 * D + 16;                    // bytes of a key row in LDS (16 apart in the banks)
// log2 of the weight that the largest score has when it raises the level, and of the largest weight before the level is raised: as high in fp16 as
// rare raises allow, because weights are rounded coarser below 2^-14 and vanish below 2^-25 (2^-34 of the largest weight then).
constexpr float kTop = 9.0f, kRaise = 15.0f;
constexpr float kFar = 0x1p19f;                          // levels beyond: neighbours in fp32 are 2^-4 apart and more
constexpr float kFarShare = 0x1p-16f;                    // of its own size, by which a level is raised the sooner

__device__ __forceinline__ half2_t as_half2(uint32_t w) { return __builtin_bit_cast(half2_t, w); }
__device__ __forceinline__ uint32_t as_u32(half2_t h) { return __builtin_bit_cast(uint32_t, h); }
__device__ __forceinline__ uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100u); }
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302u); }
__device__ __forceinline__ float other_half(float x) {   // lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32u) ? r[0] : r[1]);
}

// ---- packed fields

// 32 fields of one group (a quarter of a key row, 32 tokens of a value channel) as they are loaded.
template <int BITS>
struct Piece {
  static constexpr int BYTES = 32 * (BITS == 3 ? 2 : BITS) / 8;       // of the (low) plane
  uint32_t w[BITS];
  uint32_t scale, zero;
  // low: the fields (3-bit: their low two bits), high: the plane of high bits
  __device__ __forceinline__ void load(const uint8_t* low, const uint8_t* high, const __half* s, const __half* z) {
    if constexpr (BITS == 4) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(low);
      w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
    } else {
      const u32x2 x = *reinterpret_cast<const u32x2*>(low);
      w[0] = x.x; w[1] = x.y;
      if constexpr (BITS == 3) w[2] = *reinterpret_cast<const uint32_t*>(high);
    }
    scale = *reinterpret_cast<const unsigned short*>(s);
    zero = *reinterpret_cast<const unsigned short*>(z);
  }
};

// Masks of fields at bits 0, 2, .. of both halves of a word, in registers: an instruction that ANDs and ORs takes no literals.
template <int BITS>
struct Masks {
  uint32_t at[BITS == 2 ? 5 : BITS == 3 ? 4 : 2], high[BITS == 3 ? 4 : 1];
  __device__ __forceinline__ void start() {
#pragma unroll
    for (int i = 0; i < (BITS == 2 ? 5 : BITS == 3 ? 4 : 2); ++i) {
      at[i] = (BITS == 4 ? 0x000f000fu << (4 * i) : 0x00030003u << (2 * i));
      asm("" : "+v"(at[i]));
    }
    if constexpr (BITS == 3) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        high[i] = 0x00040004u << (2 * i);
        asm("" : "+v"(high[i]));
      }
    }
  }
};

template <int BITS>
struct Decoder {
  half2_t s, z;                                          // (the low half, which an operand's selection brings to both)
  half2_t off[5];                                        // -(1024 + o), -(256 + o), -(64 + o), -(16 + o), -(4 + o), o = 2^(b-1) if symmetric
  __device__ __forceinline__ void start(uint32_t scale, uint32_t zero) {
    const bool asym = (scale & 0x8000u) != 0u;
    uint32_t a = scale & 0x7fffu, b = asym ? zero : 0u;
    asm("" : "+v"(a), "+v"(b));                          // (whole words: their halves taken apart, the loads they come from go through memory)
    s = as_half2(a);
    z = as_half2(b);
    constexpr float H = (float)(1 << (BITS - 1));
#pragma unroll
    for (int i = 0; i < 5; ++i) {
      const float base = (float)(1024 >> (2 * i));
      const half2_t c0 = {(_Float16)-base, (_Float16)-base}, c1 = {(_Float16)(-base - H), (_Float16)(-base - H)};
      off[i] = asym ? c0 : c1;
    }
  }
  // the field at bit AT of each half (AT even, up to 8); three bits: its high bit, in the place above the low ones, in `high`
  template <int AT>
  __device__ __forceinline__ uint32_t value(const Masks<BITS>& m, uint32_t x, uint32_t high = 0u) const {
    constexpr uint32_t base = ((25u - AT) << 10) * 0x10001u;
    uint32_t raw = (x & m.at[BITS == 4 ? AT / 4 : AT / 2]) | base;
    if constexpr (BITS == 3) raw = (high & m.high[AT / 2]) | raw;
    return as_u32(__builtin_elementwise_fma(as_half2(raw) + off[AT / 2], half2_t{s.x, s.x}, half2_t{z.x, z.x}));
  }
};

// Fields 16 B .. of a piece as fp16, in the order of the products; PART 0, 1: the first and the last four words, those of one half
// of a wavefront.
template <int BITS, int B, int PART>
__device__ __forceinline__ u32x4 decode_part(const Masks<BITS>& m, const Decoder<BITS>& d, const uint32_t (&w)[BITS]) {
  if constexpr (BITS == 4) {
    const uint32_t x = PART ? high_halves(w[2 * B], w[2 * B + 1]) : low_halves(w[2 * B], w[2 * B + 1]);
    return u32x4{d.template value<0>(m, x), d.template value<4>(m, x), d.template value<0>(m, x >> 8), d.template value<4>(m, x >> 8)};
  } else if constexpr (BITS == 2) {
    const uint32_t x = w[B], y = x >> 10;
    if constexpr (PART == 0) return u32x4{d.template value<0>(m, x), d.template value<2>(m, x), d.template value<4>(m, x), d.template value<6>(m, x)};
    else return u32x4{d.template value<8>(m, x), d.template value<0>(m, y), d.template value<2>(m, y), d.template value<4>(m, y)};
  } else {
    // low bits of fields k and 8 + k at bits 2 k of the halves, their high bits at bit k of h
    const uint32_t n = w[2] >> (16 * B), h = (n & 0xffu) | (n & 0xff00u) << 8;
    const uint32_t x = PART ? w[B] >> 8 : w[B];
    if constexpr (PART == 0)
      return u32x4{d.template value<0>(m, x, h << 2), d.template value<2>(m, x, h << 3), d.template value<4>(m, x, h << 4), d.template value<6>(m, x, h << 5)};
    else
      return u32x4{d.template value<0>(m, x, h >> 2), d.template value<2>(m, x, h >> 1), d.template value<4>(m, x, h), d.template value<6>(m, x, h << 1)};
  }
}

// The piece's 32 values: 16 words.
template <int BITS>
__device__ __forceinline__ void decode(const Masks<BITS>& m, const Piece<BITS>& p, uint32_t (&out)[16]) {
  Decoder<BITS> d;
  d.start(p.scale, p.zero);
  const u32x4 w[4] = {decode_part<BITS, 0, 0>(m, d, p.w), decode_part<BITS, 0, 1>(m, d, p.w),
                      decode_part<BITS, 1, 0>(m, d, p.w), decode_part<BITS, 1, 1>(m, d, p.w)};
#pragma unroll
  for (int i = 0; i < 16; ++i) out[i] = w[i / 4][i % 4];
}

__device__ __forceinline__ void put_words(char* dst, const uint32_t (&w)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4*>(dst + 16 * i) = u32x4{w[4 * i], w[4 * i + 1], w[4 * i + 2], w[4 * i + 3]};
}

// Matrix instructions and LDS reads stay in the order in which they are written; arithmetic, global loads and LDS writes may move.
__device__ __forceinline__ void keep_order() { __builtin_amdgcn_sched_barrier(0x616); }

// ---- a sequence

// Cached and new tokens; sink tokens; packed rows of keys and of values; cached tokens beside the packed_v rows of the store (number w of
// them is token w of the sink, else token w + packed_v).
struct ChunkSeq { int n, t, sink, packed_k, packed_v, beside; };
__device__ __forceinline__ ChunkSeq chunk_seq(const ChunkArgs& a, int b, int group) {
  const int cap = (int)a.capacity;
  ChunkSeq s;
  s.n = a.n_tokens;
  s.t = a.t_new;
  if (a.n_dev) {
    s.n = a.n_dev[b];
    s.n = s.n < 0 ? 0 : s.n > cap ? cap : s.n;
    s.t = a.t_dev[b];
    s.t = s.t < 0 ? 0 : s.t > a.t_new ? a.t_new : s.t;
  }
  s.sink = s.n < a.w_sink ? s.n : a.w_sink;
  s.packed_k = (int)quantised_rows(a.w_sink, a.w_recent, group, kPerToken, s.n);
  s.packed_v = (int)quantised_rows(a.w_sink, a.w_recent, group, kPerChannel, s.n);
  s.beside = s.n - s.packed_v;
  return s;
}

// Where a thread finds its piece of a tile of packed rows: offsets from the tile's first row (a row takes 16 BITS bytes of codes
// and 128 / G scales in either tensor).
template <int BITS, int G>
struct PieceAt {
  uint32_t low, high, scale;
  // quarter of a key row
  __device__ __forceinline__ void key(int token, int quarter) {
    low = (uint32_t)(token * 16 * BITS + quarter * Piece<BITS>::BYTES);
    high = (uint32_t)(token * 16 * BITS + D * 2 / 8 + quarter * 4);
    scale = (uint32_t)(token * (D / G) + quarter * 32 / G);
  }
  // 32 tokens of a value channel
  __device__ __forceinline__ void value(int channel, int block) {
    const int group = G == 64 ? 0 : block, part = G == 64 ? block : 0;
    const uint32_t run = (uint32_t)((group * D + channel) * (G * BITS / 8));
    low = run + (uint32_t)(part * Piece<BITS>::BYTES);
    high = run + (uint32_t)(G * 2 / 8 + part * 4);
    scale = (uint32_t)(group * D + channel);
  }
};

// First store row of a tile (uniform: row0, and so the page, are the same for a wavefront).
__device__ __forceinline__ long long tile_row(const ChunkArgs& a, int b, int h, int row0) {
  if (!a.pages.table) return ((long long)b * a.n_kv_heads + h) * a.capacity + row0;
  int page = __builtin_amdgcn_readfirstlane(a.pages.table[(long long)b * a.pages.tiles_per_seq + (row0 >> 6)]);
  page = page < 0 ? 0 : page >= a.pages.pool_pages ? a.pages.pool_pages - 1 : page;
  return ((long long)page * a.n_kv_heads + h) * kPageTokens + (row0 & 63);
}

template <int KB, int VB, int G, int RW, int TW>
struct ChunkKernel {
  static constexpr int KT = RW == 1 ? 32 : 64;           // tokens of a tile
  static constexpr int NB = KT / 32;                     // blocks of 32 of them
  static constexpr int NT = 64 * RW;                     // threads that bring a tile
  static constexpr bool APART = RW == 8;                 // half of the wavefronts bring keys, half values
  static constexpr int P = APART ? 1 : KT * 4 / NT;      // pieces of each tensor a thread brings
  static constexpr int VPITCH = 2 * KT + 16;             // bytes of a channel of V^T
  static constexpr int VALUES = KT * kKeyPitch;          // where they begin
  static constexpr int BUF = VALUES + D * VPITCH;
  static constexpr int NBUF = RW == 1 ? 1 : RW == 4 ? 2 : 4;          // buffers (a wavefront by itself takes its LDS operations in order)
  static constexpr int JOIN = TW > 1 ? TW * (64 * 64 + 128) * 4 : 0;
  static constexpr int LDS = BUF * NBUF * TW > JOIN ? BUF * NBUF * TW : JOIN;

  static constexpr bool ONE = APART && KB == VB;         // a thread's piece is a key's or a value's, decoded alike
  struct Packed { Piece<KB> k[P]; Piece<VB> v[ONE ? 1 : P]; };
  struct Plain { u32x4 k[P][4]; u32x4 v[P][4]; };
  enum Which { kBoth, kKeys, kValues };                  // of a thread's pieces

  // Store rows row0 .. (a multiple of the tile of 64, so one page holds them): pieces in registers.  Behind the last packed row: the
  // same rows again, whose scores are masked.
  static __device__ __forceinline__ void load_packed(const ChunkArgs& a, const ChunkSeq& s, int b, int h, int row0, int tid, bool values, Packed& x) {
    const long long lin = tile_row(a, b, h, row0);
    static_assert(KT == 64);
    const bool whole = s.packed_v - row0 >= KT;
    if constexpr (ONE) {
      const int p = tid % (NT / 2);
      PieceAt<KB, G> k, v;
      k.key(whole ? p >> 2 : (p >> 2) & 31, p & 3);
      v.value(p % D, whole ? p / D : 0);
      const ChunkTensor& t = values ? a.v : a.k;
      const uint8_t* codes = t.codes + lin * (16 * KB);
      const uint32_t scale = values ? v.scale : k.scale;
      x.k[0].load(codes + (values ? v.low : k.low), codes + (values ? v.high : k.high), t.scales + lin * (D / G) + scale, t.zeros + lin * (D / G) + scale);
      return;
    }
#pragma unroll
    for (int m = 0; m < P; ++m) {
      const int p = (APART ? tid % (NT / 2) : tid) + m * NT;
      if (!APART || !values) {
        PieceAt<KB, G> at;
        at.key(whole ? p >> 2 : (p >> 2) & 31, p & 3);
        const uint8_t* codes = a.k.codes + lin * (16 * KB);
        x.k[m].load(codes + at.low, codes + at.high, a.k.scales + lin * (D / G) + at.scale, a.k.zeros + lin * (D / G) + at.scale);
      }
      if (!APART || values) {
        PieceAt<VB, G> at;
        at.value(p % D, whole ? p / D : 0);
        const uint8_t* codes = a.v.codes + lin * (16 * VB);
        x.v[m].load(codes + at.low, codes + at.high, a.v.scales + lin * (D / G) + at.scale, a.v.zeros + lin * (D / G) + at.scale);
      }
    }
  }
  struct FieldMasks { Masks<KB> k; Masks<VB> v; };
  static __device__ __forceinline__ void put_packed(const FieldMasks& f, char* buf, int tid, bool values, const Packed& x) {
#pragma unroll
    for (int m = 0; m < P; ++m) {
      const int p = (APART ? tid % (NT / 2) : tid) + m * NT;
      uint32_t w[16];
      char* k = buf + (p >> 2) * kKeyPitch + (p & 3) * 64;
      char* v = buf + VALUES + (p % D) * VPITCH + (p / D) * 64;
      if constexpr (!APART) {
        decode<KB>(f.k, x.k[m], w);
        put_words(k, w);
        decode<VB>(f.v, x.v[m], w);
        put_words(v, w);
      } else if constexpr (KB == VB) {
        decode<KB>(f.k, x.k[0], w);
        put_words(values ? v : k, w);
      } else if (values) {
        decode<VB>(f.v, x.v[m], w);
        put_words(v, w);
      } else {
        decode<KB>(f.k, x.k[m], w);
        put_words(k, w);
      }
    }
  }

  // Number w of the cached tokens beside the packed rows: its fp16 row; null for a key that is packed.
  static __device__ __forceinline__ const __half* cached_row(const ChunkArgs& a, const ChunkSeq& s, const ChunkTensor& x, int packed, long long bh, int w) {
    if (w < s.sink) return x.sink + (bh * a.w_sink + w) * D;
    const int token = w + s.packed_v;
    if (token - a.w_sink < packed) return nullptr;
    return x.ring + (bh * x.slots + (uint32_t)token % (uint32_t)x.slots) * D;
  }
  // Tile of numbers w0 .. (behind the last one: the last one again, whose scores are masked).
  template <Which WHICH = kBoth>
  static __device__ __forceinline__ void load_cached(const ChunkArgs& a, const ChunkSeq& s, long long bh, int w0, int tid, bool values, Plain& x) {
#pragma unroll
    for (int m = 0; m < P; ++m) {
      const int p = (APART ? tid % (NT / 2) : tid) + m * NT;
      if (WHICH != kValues && (!APART || !values)) {
        const int w = w0 + (p >> 2) < s.beside ? w0 + (p >> 2) : s.beside - 1, quarter = p & 3;
        const __half* row = cached_row(a, s, a.k, s.packed_k, bh, w);
        if (row) {
#pragma unroll
          for (int i = 0; i < 4; ++i) x.k[m][i] = *reinterpret_cast<const u32x4*>(row + quarter * 32 + 8 * i);
        } else {
          // (a key that has left its window before the values of its group have left theirs)
          const long long lin = store_row(a.pages, a.n_kv_heads, a.capacity, bh, w + s.packed_v - a.w_sink);
          const uint8_t* codes = a.k.codes + lin * (D * KB / 8);
          const long long at = lin * (D / G) + quarter * 32 / G;
          Piece<KB> piece;
          piece.load(codes + quarter * Piece<KB>::BYTES, codes + D * 2 / 8 + quarter * 4, a.k.scales + at, a.k.zeros + at);
          uint32_t o[16];
          Masks<KB> masks;
          masks.start();
          decode<KB>(masks, piece, o);
#pragma unroll
          for (int i = 0; i < 2; ++i) {                    // (back into the order of the channels, as the other rows are)
            const uint32_t* q = o + 8 * i;
            x.k[m][2 * i] = u32x4{low_halves(q[0], q[1]), low_halves(q[2], q[3]), low_halves(q[4], q[5]), low_halves(q[6], q[7])};
            x.k[m][2 * i + 1] = u32x4{high_halves(q[0], q[1]), high_halves(q[2], q[3]), high_halves(q[4], q[5]), high_halves(q[6], q[7])};
          }
        }
      }
      if (WHICH == kKeys || (APART && !values)) continue;
      const int set = p % (KT / 4), chunk = p / (KT / 4);
      const int first = w0 + 16 * (set >> 2) + 2 * (set & 3);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int w = first + (i & 1) * 8 + (i >> 1);
        x.v[m][i] = *reinterpret_cast<const u32x4*>(cached_row(a, s, a.v, s.packed_v, bh, w < s.beside ? w : s.beside - 1) + 8 * chunk);
      }
    }
  }
  // Tile of new tokens i0 .. (behind the last one, `last`: that one again, whose scores are masked).
  template <Which WHICH = kBoth>
  static __device__ __forceinline__ void load_fresh(const ChunkArgs& a, int b, int h, int i0, int last, int tid, bool values, Plain& x) {
    const RowView &k = a.k.fresh, &v = a.v.fresh;
#pragma unroll
    for (int m = 0; m < P; ++m) {
      const int p = (APART ? tid % (NT / 2) : tid) + m * NT;
      if (WHICH != kValues && (!APART || !values)) {
        const int i = i0 + (p >> 2) < last ? i0 + (p >> 2) : last;
        const __half* src = k.p + b * k.batch + h * k.head + i * k.token + (p & 3) * 32;
#pragma unroll
        for (int e = 0; e < 4; ++e) x.k[m][e] = *reinterpret_cast<const u32x4*>(src + 8 * e);
      }
      if (WHICH == kKeys || (APART && !values)) continue;
      const int set = p % (KT / 4), chunk = p / (KT / 4);
      const int first = i0 + 16 * (set >> 2) + 2 * (set & 3);
      const __half* src = v.p + b * v.batch + h * v.head + 8 * chunk;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int i = first + (e & 1) * 8 + (e >> 1);
        x.v[m][e] = *reinterpret_cast<const u32x4*>(src + (i < last ? i : last) * v.token);
      }
    }
  }
  template <Which WHICH = kBoth>
  static __device__ __forceinline__ void put_plain(char* buf, int tid, bool values, const Plain& x) {
#pragma unroll
    for (int m = 0; m < P; ++m) {
      const int p = (APART ? tid % (NT / 2) : tid) + m * NT;
      if (WHICH != kValues && (!APART || !values)) {
        char* k = buf + (p >> 2) * kKeyPitch + (p & 3) * 64;
#pragma unroll
        for (int i = 0; i < 4; i += 2) {
          const u32x4 f = x.k[m][i], g = x.k[m][i + 1];
          *reinterpret_cast<u32x4*>(k + 16 * i) = u32x4{low_halves(f.x, g.x), high_halves(f.x, g.x), low_halves(f.y, g.y), high_halves(f.y, g.y)};
          *reinterpret_cast<u32x4*>(k + 16 * i + 16) = u32x4{low_halves(f.z, g.z), high_halves(f.z, g.z), low_halves(f.w, g.w), high_halves(f.w, g.w)};
        }
      }
      if (WHICH == kKeys || (APART && !values)) continue;
      const int set = p % (KT / 4), chunk = p / (KT / 4);
      char* v = buf + VALUES + 8 * chunk * VPITCH + 8 * set;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const uint32_t r0 = x.v[m][0][c], r1 = x.v[m][1][c], r2 = x.v[m][2][c], r3 = x.v[m][3][c];
        *reinterpret_cast<u32x2*>(v + 2 * c * VPITCH) = u32x2{low_halves(r0, r1), low_halves(r2, r3)};
        *reinterpret_cast<u32x2*>(v + (2 * c + 1) * VPITCH) = u32x2{high_halves(r0, r1), high_halves(r2, r3)};
      }
    }
  }

  // A wavefront's 32 query rows: operand, outputs (lane: row lane % 32; channels 32 x + 8 (i / 4) + 4 (lane / 32) + i % 4), level, sum.
  struct Rows {
    half8_t q[8];
    float16_t o[4];
    float m, l;
  };

  static __device__ __forceinline__ void scores(const char* buf, const Rows& r, int lane, float16_t (&s)[NB]) {
    const char* keys = buf + (lane & 31) * kKeyPitch + 128 * (lane >> 5);
    // operands eight ahead of their instructions; what decodes the next tile may stand between these
    half8_t k[8];
#pragma unroll
    for (int st = 0; st < 8; ++st) k[st] = *reinterpret_cast<const half8_t*>(keys + 16 * st);
    keep_order();
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      s[n] = float16_t{};
#pragma unroll
      for (int st = 0; st < 8; ++st) {
        s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[st], r.q[st], s[n], 0, 0, 0);
        if (n + 1 < NB) k[st] = *reinterpret_cast<const half8_t*>(keys + 32 * (n + 1) * kKeyPitch + 16 * st);
        keep_order();
      }
    }
  }
  // masked: some row does not attend to every token of the tile; limit: the last one that the lane's row attends to, counted from the tile's first.
  static __device__ __forceinline__ void finish(const char* buf, Rows& r, float16_t (&s)[NB], int lane, bool masked, int limit, float scale) {
    const char* values = buf + VALUES + (lane & 31) * VPITCH + 16 * (lane >> 5);
    half8_t v[8];                                        // (the first values are on their way under the softmax)
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = *reinterpret_cast<const half8_t*>(values + 32 * (x & 3) * VPITCH + 32 * (x >> 2));
    half8_t p[2 * NB];
    weights(r, s, lane >> 5, masked, limit, scale, p);
#pragma unroll
    for (int st = 0; st < 2 * NB; ++st)
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const int at = 4 * st + x;
        r.o[x] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[at & 7], p[st], r.o[x], 0, 0, 0);
        if (at + 8 < 8 * NB) v[at & 7] = *reinterpret_cast<const half8_t*>(values + 32 * x * VPITCH + 32 * (st + 2));
        keep_order();
      }
  }
  // The softmax weights of a tile's scores, as operands; level and sum move on.
  static __device__ __forceinline__ void weights(Rows& r, float16_t (&s)[NB], int half, bool masked, int limit, float scale, half8_t (&p)[2 * NB]) {
    if (masked) {
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (32 * n + 8 * (i / 4) + 4 * half + i % 4 > limit) s[n][i] = -INFINITY;
    }
    float top = s[0][0];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, s[n][i]);
    top = fmaxf(top, other_half(top)) * scale;
    // (from the empty state: if there is a token at all; the larger the level, the sooner, and beyond kFar always)
    const bool raise = top > __builtin_fmaf(-kFarShare, __builtin_fabsf(r.m), r.m) + kRaise;
    if (__builtin_amdgcn_ballot_w64(raise)) {
      const float level = raise ? fmaxf(r.m, __builtin_fabsf(top) > kFar ? top : top - kTop) : r.m;
      const float f = raise ? __builtin_amdgcn_exp2f(r.m - level) : 1.f;       // (0 from the empty state)
      r.l *= f;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int i = 0; i < 16; ++i) r.o[x][i] *= f;
      r.m = level;
    }
    const float level = r.m == -INFINITY ? 0.f : r.m;    // (a row that has met no token yet)
    if (__builtin_amdgcn_ballot_w64(__builtin_fabsf(level) > kFar)) {
      // The fused form below takes the level, which is rounded, from the exact product: at 2^28 the largest score would be up to 16 above its own
      // level and its weight beyond fp16.  Scores of such tiles are rounded as the level is.
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[n][i] *= scale;
          asm volatile("" : "+v"(s[n][i]));              // (one rounding here and one below)
        }
      scale = 1.f;
    }
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        p[2 * n + i / 8][2 * (i % 4) + (i / 4) % 2] = (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[n][i], scale, -level));
    // (the sum is that of the weights as they are rounded; of the tile first: two at a time they would vanish in a row's sum of 2^25 times as much)
    float sum = 0.f;
#pragma unroll
    for (int st = 0; st < 2 * NB; ++st)
#pragma unroll
      for (int e = 0; e < 8; e += 2)
        sum = __builtin_amdgcn_fdot2(half2_t{p[st][e], p[st][e + 1]}, half2_t{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
    r.l += sum;
  }

  // ---- a wavefront by itself takes packed tiles of 32 tokens straight from memory to its operands.  Keys: a lane has half a row of one
  // token, 64 channels.  Values: a lane has four channels, of which it needs the sixteen tokens of its half (the other half of the
  // wavefront loads the same words).
  struct Direct {
    uint32_t k[2][KB], kscale, kzero;
    uint32_t v[4][VB], vscale[4], vzero[4];
  };
  // (addresses: a uniform one and 32 bits of a lane's own)
  static __device__ __forceinline__ void load_direct_keys(const ChunkArgs& a, long long lin, int lane, Direct& x) {
    const uint32_t tok = (uint32_t)lane & 31u, half = (uint32_t)lane >> 5;
    const uint8_t* codes = a.k.codes + lin * (16 * KB);
    const uint32_t low = tok * (16 * KB) + half * (2 * Piece<KB>::BYTES);
    constexpr int N = KB == 3 ? 2 : KB;                  // words of a piece's (low) plane
    uint32_t w[2 * N];
#pragma unroll
    for (int i = 0; i < 2 * N; i += 4) {
      const u32x4 q = *reinterpret_cast<const u32x4*>(codes + (low + 4 * i));
      w[i] = q.x; w[i + 1] = q.y; w[i + 2] = q.z; w[i + 3] = q.w;
    }
#pragma unroll
    for (int p = 0; p < 2; ++p)
#pragma unroll
      for (int i = 0; i < N; ++i) x.k[p][i] = w[p * N + i];
    if constexpr (KB == 3) {
      const u32x2 q = *reinterpret_cast<const u32x2*>(codes + (tok * (16 * KB) + D * 2 / 8 + half * 8));
      x.k[0][2] = q.x; x.k[1][2] = q.y;
    }
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(a.k.scales + lin * (D / G));
    const uint8_t* zeros = reinterpret_cast<const uint8_t*>(a.k.zeros + lin * (D / G));
    const uint32_t at = tok * (2 * D / G) + half * (128 / G);
    if constexpr (G == 32) {                             // (both groups' in one word)
      x.kscale = *reinterpret_cast<const uint32_t*>(scales + at);
      x.kzero = *reinterpret_cast<const uint32_t*>(zeros + at);
    } else {
      x.kscale = *reinterpret_cast<const unsigned short*>(scales + at);
      x.kzero = *reinterpret_cast<const unsigned short*>(zeros + at);
    }
  }
  static __device__ __forceinline__ void load_direct_values(const ChunkArgs& a, long long lin, int row0, int lane, Direct& x) {
    const int part = G == 64 ? (row0 & 63) / 32 : 0;     // (half a group of 64)
    const long long first = G == 64 ? lin - (row0 & 63) : lin;
    constexpr uint32_t RUN = G * VB / 8;                 // bytes of a channel
    const uint32_t c = (uint32_t)lane & 31u;
    const uint8_t* codes = a.v.codes + first * (16 * VB) + part * Piece<VB>::BYTES;
    const uint8_t* high = a.v.codes + first * (16 * VB) + G * 2 / 8 + part * 4;
    const uint8_t* scales = reinterpret_cast<const uint8_t*>(a.v.scales + first * (D / G));
    const uint8_t* zeros = reinterpret_cast<const uint8_t*>(a.v.zeros + first * (D / G));
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      const uint32_t run = c * RUN + 32 * n * RUN, at = 2 * c + 64 * n;
      Piece<VB> p;
      p.load(codes + run, high + run, reinterpret_cast<const __half*>(scales + at), reinterpret_cast<const __half*>(zeros + at));
#pragma unroll
      for (int i = 0; i < VB; ++i) x.v[n][i] = p.w[i];
      x.vscale[n] = p.scale;
      x.vzero[n] = p.zero;
    }
  }
  template <int P>
  static __device__ __forceinline__ void direct_scores(const FieldMasks& f, const Direct& x, const Rows& r, Decoder<KB>& d, float16_t& s) {
    if (P == 0) d.start(x.kscale & 0xffffu, x.kzero & 0xffffu);
    else if (G == 32) d.start(x.kscale >> 16, x.kzero >> 16);
    s = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, decode_part<KB, 0, 0>(f.k, d, x.k[P])), r.q[4 * P], s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, decode_part<KB, 0, 1>(f.k, d, x.k[P])), r.q[4 * P + 1], s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, decode_part<KB, 1, 0>(f.k, d, x.k[P])), r.q[4 * P + 2], s, 0, 0, 0);
    s = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, decode_part<KB, 1, 1>(f.k, d, x.k[P])), r.q[4 * P + 3], s, 0, 0, 0);
  }
  // Words of the fields that the lane's half needs, brought to the places of half 0, so that one code serves both.
  static __device__ __forceinline__ void own_half(const uint32_t (&w)[VB], int half, uint32_t (&out)[VB]) {
    constexpr int N = VB == 3 ? 2 : VB;
    uint32_t by = half ? (VB == 4 ? 16u : 8u) : 0u;
    asm("" : "+v"(by));                                  // (known, it becomes a load at another byte of what is put into memory first)
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = w[i] >> by;
    if constexpr (VB == 3) out[2] = w[2] >> (by / 2);
  }
  static __device__ __forceinline__ void direct_keys(const FieldMasks& f, const Direct& x, const Rows& r, float16_t (&s)[NB]) {
    s[0] = float16_t{};
    Decoder<KB> d;
    direct_scores<0>(f, x, r, d, s[0]);
    direct_scores<1>(f, x, r, d, s[0]);
  }
  static __device__ __forceinline__ void direct_values(const FieldMasks& f, const Direct& x, Rows& r, float16_t (&s)[NB], int lane, float scale) {
    half8_t p[2 * NB];
    weights(r, s, lane >> 5, false, 0, scale, p);
#pragma unroll
    for (int n = 0; n < 4; ++n) {
      Decoder<VB> d;
      d.start(x.vscale[n], x.vzero[n]);
      uint32_t w[VB];
      own_half(x.v[n], lane >> 5, w);
      r.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, decode_part<VB, 0, 0>(f.v, d, w)), p[0], r.o[n], 0, 0, 0);
      r.o[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8_t, decode_part<VB, 1, 0>(f.v, d, w)), p[1], r.o[n], 0, 0, 0);
    }
  }

  static __device__ __forceinline__ void load_queries(const ChunkArgs& a, int b, int h, int row, bool live, int half, Rows& r) {
    const int i = row / a.heads_per_kv;
    const __half* src = a.q.p + b * a.q.batch + (h * a.heads_per_kv + row - i * a.heads_per_kv) * a.q.head + i * a.q.token;
#pragma unroll
    for (int st = 0; st < 8; ++st) {
      u32x2 x = {0u, 0u}, y = {0u, 0u};
      if (live) {
        const int c = 64 * half + 16 * (st / 2) + 4 * (st % 2);
        x = *reinterpret_cast<const u32x2*>(src + c);
        y = *reinterpret_cast<const u32x2*>(src + c + 8);
        if (a.q_scale) {
          const float* f = a.q_scale + h * D + c;
          __half* hx = reinterpret_cast<__half*>(&x);
          __half* hy = reinterpret_cast<__half*>(&y);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            hx[e] = scaled_half(__half2float(hx[e]), f[e]);
            hy[e] = scaled_half(__half2float(hy[e]), f[8 + e]);
          }
        }
      }
      r.q[st] = __builtin_bit_cast(half8_t, u32x4{low_halves(x.x, y.x), high_halves(x.x, y.x), low_halves(x.y, y.y), high_halves(x.y, y.y)});
    }
  }

  // Channels 32 x .. of a row: the output itself, or (split) the partial result of a slot.
  static __device__ __forceinline__ void store_channels(const ChunkArgs& a, int b, int h, int row, long long slot_row, bool split, int x, int half,
                                                        const float16_t& o, float l) {
    const int c0 = 32 * x + 4 * half;
    if (split) {
      float* dst = a.ws + a.slots * (32 * RW * 2) + slot_row * D + c0;
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<float4*>(dst + 8 * i) = float4{o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]};
      return;
    }
    const float f = 1.0f / l;
    const int i = row / a.heads_per_kv;
    const long long at = b * a.out_batch + (h * a.heads_per_kv + row - i * a.heads_per_kv) * a.out_head + i * a.out_token + c0;
    if (a.out_is_fp32) {
      float* dst = static_cast<float*>(a.out) + at;
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4)
        *reinterpret_cast<float4*>(dst + 8 * i4) = float4{o[4 * i4] * f, o[4 * i4 + 1] * f, o[4 * i4 + 2] * f, o[4 * i4 + 3] * f};
    } else {
      __half* dst = static_cast<__half*>(a.out) + at;
#pragma unroll
      for (int i4 = 0; i4 < 4; ++i4) {
        const half2_t lo = {(_Float16)(o[4 * i4] * f), (_Float16)(o[4 * i4 + 1] * f)}, hi = {(_Float16)(o[4 * i4 + 2] * f), (_Float16)(o[4 * i4 + 3] * f)};
        *reinterpret_cast<u32x2*>(dst + 8 * i4) = u32x2{as_u32(lo), as_u32(hi)};
      }
    }
  }
  static __device__ __forceinline__ void store_state(const ChunkArgs& a, long long slot_row, float m, float l) {
    *reinterpret_cast<float2*>(a.ws + slot_row * 2) = float2{m, l};
  }
};

// ---- a ragged batch: what a work-group does, from the counts of all sequences (four a lane; the arithmetic is the plan's).  Every wavefront
// finds the same.
struct ChunkWork { int b, h, row_block, split, n_splits, slot; };

__device__ __forceinline__ int wave_sum(int x) {
#pragma unroll
  for (int i = 1; i < 64; i *= 2) x += __shfl_xor(x, i);
  return x;
}
template <int ROWS, int TILE>                            // TILE: tokens that the work-group takes a turn
__device__ __forceinline__ bool find_work(const ChunkArgs& a, int group, int item, ChunkWork& w) {
  constexpr int N = kChunkListMost / 64;
  const int lane = (int)threadIdx.x & 63;
  int units[N], tiles[N];                                // of the lane's sequences
  int most = 1;
  float work = 0.f;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int b = N * lane + j;
    units[j] = tiles[j] = 0;
    if (b < a.batch) {
      const ChunkSeq s = chunk_seq(a, b, group);
      const ChunkShare share = chunk_share(s.n, s.t, a.heads_per_kv, a.n_kv_heads, a.rows_from, a.rows_to, ROWS, TILE);
      units[j] = share.units;
      tiles[j] = share.tiles;
    }
    most = tiles[j] > most ? tiles[j] : most;
    work += (float)units[j] * (float)tiles[j];
  }
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    const int x = __shfl_xor(most, i);
    most = x > most ? x : most;
    work += __shfl_xor(work, i);
  }
  most = __builtin_amdgcn_readfirstlane(most);
  int length = __builtin_amdgcn_readfirstlane(chunk_first_length(work));
  int mine;
  for (;; length = chunk_next_length(length)) {
    mine = 0;
#pragma unroll
    for (int j = 0; j < N; ++j) mine += units[j] * chunk_ranges(tiles[j], length);
    if (chunk_length_fits(length, most, __builtin_amdgcn_readfirstlane(wave_sum(mine)))) break;
  }
  // the sequence whose items hold this one
  int before = mine;
#pragma unroll
  for (int i = 1; i < 64; i *= 2) {
    const int x = __shfl_up(before, i);
    if (lane >= i) before += x;
  }
  const unsigned long long reach = __builtin_amdgcn_ballot_w64(before > item);
  if (reach == 0) return false;                          // (uniform)
  const int owner = __builtin_ctzll(reach);
  int first = __builtin_amdgcn_readlane(before - mine, owner);
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const int u = __builtin_amdgcn_readlane(units[j], owner), splits = chunk_ranges(__builtin_amdgcn_readlane(tiles[j], owner), length), all = u * splits;
    if (item >= first && item < first + all) {
      const ChunkPlace at = chunk_place(item - first, u, a.n_kv_heads, splits);
      w.b = N * owner + j;
      w.h = at.h;
      w.row_block = at.row_block;
      w.split = at.split;
      w.n_splits = splits;
      w.slot = item;
      if (item == first && threadIdx.x == 0) {
        a.table[2 * w.b] = item;
        a.table[2 * w.b + 1] = splits;
      }
      return true;
    }
    first += all;
  }
  return false;
}

// Tiles u0 .. u1 of one kind: load(u, registers), put(buffer, registers), masks(u) -> {masked, limit} as for finish.  This wavefront's rows
// attend to those before `mine`.  One buffer (a wavefront by itself): load also puts.  Else the next tile is put into LDS, and the one after
// it loaded, between the two products (behind the last tile: the same again).
struct TileMask { bool masked; int limit; };
template <typename C, typename Regs, typename Load, typename Put, typename Mask>
__device__ __forceinline__ void pass_tiles(int u0, int u1, int mine, char* lds, typename C::Rows& r, int lane, float scale, Load load, Put put, Mask mask) {
  if (u0 >= u1) return;
  Regs x;
  float16_t sc[C::NB];
  if constexpr (C::NBUF == 1) {
    for (int u = u0; u < u1; ++u) {
      load(u, x);                                        // (brings them into LDS, too)
      asm volatile("" ::: "memory");                     // (a wavefront's LDS operations are performed in order)
      __builtin_amdgcn_wave_barrier();
      if (u < mine) {
        C::scores(lds, r, lane, sc);
        const TileMask m = mask(u);
        C::finish(lds, r, sc, lane, m.masked, m.limit, scale);
      }
      asm volatile("" ::: "memory");
      __builtin_amdgcn_wave_barrier();
    }
  } else {
    constexpr int STEP = C::NBUF / 2;                      // tiles that the work-group takes between two barriers
    auto at = [&](int u) { return lds + ((u - u0) % C::NBUF) * C::BUF; };
    auto bound = [&](int u) { return u < u1 ? u : u1 - 1; };
    load(u0, x);
#pragma unroll
    for (int i = 0; i < STEP; ++i) {
      put(at(u0 + i), x);
      load(bound(u0 + i + 1), x);
    }
    int u = u0;
    for (; u < mine && u < u1; ++u) {
      if (STEP == 1 || (u - u0) % STEP == 0) __syncthreads();
      C::scores(at(u), r, lane, sc);
      put(at(u + STEP), x);
      load(bound(u + STEP + 1), x);
      const TileMask m = mask(u);
      C::finish(at(u), r, sc, lane, m.masked, m.limit, scale);
    }
    for (; u < u1; ++u) {
      if (STEP == 1 || (u - u0) % STEP == 0) __syncthreads();
      put(at(u + STEP), x);
      load(bound(u + STEP + 1), x);
    }
    __syncthreads();
  }
}

// Work-groups: the last rows, which have the most keys, first; where the sequence-heads can be shared out evenly, those of one stay on one XCD (its L2
// then brings every tile from memory once).
template <int KB, int VB, int G, int RW, int TW>
__global__ void __launch_bounds__(64 * RW * TW) __attribute__((amdgpu_waves_per_eu(2, 2))) attention_chunk_kernel(ChunkArgs a) {
  using C = ChunkKernel<KB, VB, G, RW, TW>;
  __shared__ __align__(16) char lds[C::LDS];
  ChunkWork work;
  bool listed = false;
  if constexpr (RW != 8) listed = a.table != nullptr;
  if (listed) {
    if (!find_work<32 * RW, C::KT * TW>(a, G, (int)blockIdx.x, work)) return;      // (uniform)
  } else {
    const unsigned heads = (unsigned)(a.batch * a.n_kv_heads);
    const bool pinned = heads % 8u == 0u;
    const unsigned slot = pinned ? blockIdx.x / 8u : blockIdx.x, mine_heads = pinned ? heads / 8u : heads;
    const unsigned rank = slot / (mine_heads * (unsigned)a.n_splits), rest = slot % (mine_heads * (unsigned)a.n_splits);
    const unsigned bh = rest / (unsigned)a.n_splits + (pinned ? blockIdx.x % 8u * mine_heads : 0u);
    work.split = (int)(rest % (unsigned)a.n_splits);
    work.n_splits = a.n_splits;
    work.b = (int)(bh / (unsigned)a.n_kv_heads);
    work.h = (int)(bh % (unsigned)a.n_kv_heads);
    work.row_block = a.row_blocks - 1 - (int)rank;
    work.slot = ((int)bh * a.row_blocks + work.row_block) * a.n_splits + work.split;
  }
  const int b = work.b, h = work.h, split = work.split, n_splits = work.n_splits;
  const long long bh = (long long)b * a.n_kv_heads + h;
  const ChunkSeq s = chunk_seq(a, b, G);
  const int rows = s.t * a.heads_per_kv, row_base = work.row_block * 32 * RW;
  if (row_base >= rows) return;                          // (uniform)
  const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6), lane = (int)threadIdx.x & 63, half = lane >> 5;
  const int group = wave / RW, tid = (int)threadIdx.x % C::NT;
  const int first = row_base + (wave % RW) * 32, row = first + (lane & 31);
  const bool live = row < rows;
  typename C::Rows r;
  C::load_queries(a, b, h, live ? row : 0, live, half, r);
#pragma unroll
  for (int x = 0; x < 4; ++x) r.o[x] = float16_t{};
  r.m = -INFINITY;
  r.l = 0.f;
  const float scale = 0.08838834764831845f * 1.4426950408889634f;

  // new tokens that the rows of the work-group, of the wavefront and of the lane attend to
  const int last_row = row_base + 32 * RW < rows ? row_base + 32 * RW : rows;
  const int last = (last_row - 1) / a.heads_per_kv;
  const int wave_last = first + 32 < rows ? first + 32 : rows;
  const int newest = (live ? row : rows - 1) / a.heads_per_kv, oldest = first / a.heads_per_kv;
  const bool has_rows = first < rows;

  // tiles: packed rows, cached tokens beside them, new tokens; this wavefront's share of them.  A wavefront by itself brings fp16 tiles through
  // LDS, one after the other: three times a packed tile.  Counted so where there are eight tiles a wavefront: of the time with all tiles alike
  // 0.89 to 0.97 at 8 to 16 tiles a wavefront, 0.95 to 1.05 at 60 and more; not below: 0.96 to 1.04 at 1 to 4 (1, 4 and 32 sequences, 32 / 8
  // heads, 1k to 32k tokens, 1 to 8 new, 2 and 4 bits).
  const int tiles1 = (s.packed_v + C::KT - 1) / C::KT, tiles2 = tiles1 + (s.beside + C::KT - 1) / C::KT, tiles = tiles2 + last / C::KT + 1;
  const int parts = n_splits * TW, part = split * TW + group, plain = RW == 1 && tiles >= 8 * parts ? 3 : 1;
  const int cost = tiles1 + (tiles - tiles1) * plain, per = cost / parts, more = cost % parts;
  auto tile_at = [&](int c) { return c <= tiles1 ? c : tiles1 + (c - tiles1 + plain - 1) / plain; };
  const int c0 = part * per + (part < more ? part : more);
  const int t0 = tile_at(c0), t1 = tile_at(c0 + per + (part < more ? 1 : 0));
  auto from = [&](int t) { return t0 > t ? t0 - t : 0; };
  auto to = [&](int t, int end) { return (t1 < end ? t1 : end) - t; };
  const bool values = wave >= RW / 2;
  char* mine = lds + group * C::BUF * C::NBUF;
  typename C::FieldMasks masks;
  masks.k.start();
  masks.v.start();
  auto put_plain = [&](char* at, const typename C::Plain& x) { C::put_plain(at, tid, values, x); };
  if constexpr (RW == 1) {
    const int u0 = from(0), u1 = to(0, tiles1);
    auto row = [&](int u) { return (u < u1 ? u : u1 - 1) * C::KT; };
    auto place = [&](int row0) { return tile_row(a, b, h, row0); };
    if (u0 < u1) {
      // Two tiles under way, their registers loaded again as soon as they have been used; the scores of the next tile are formed in front of
      // the present one's weights, so that nothing waits for a product (behind the last tile: its own once more).
      typename C::Direct x, y;
      float16_t sx[C::NB], sy[C::NB];
      C::load_direct_keys(a, place(row(u0)), lane, x);
      C::load_direct_values(a, place(row(u0)), row(u0), lane, x);
      C::load_direct_keys(a, place(row(u0 + 1)), lane, y);
      C::load_direct_values(a, place(row(u0 + 1)), row(u0 + 1), lane, y);
      C::direct_keys(masks, x, r, sx);
      C::load_direct_keys(a, place(row(u0 + 2)), lane, x);
      for (int u = u0;;) {
        C::direct_keys(masks, y, r, sy);
        C::load_direct_keys(a, place(row(u + 3)), lane, y);
        C::direct_values(masks, x, r, sx, lane, scale);
        C::load_direct_values(a, place(row(u + 2)), row(u + 2), lane, x);
        if (++u == u1) break;
        C::direct_keys(masks, x, r, sx);
        C::load_direct_keys(a, place(row(u + 3)), lane, x);
        C::direct_values(masks, y, r, sy, lane, scale);
        C::load_direct_values(a, place(row(u + 2)), row(u + 2), lane, y);
        if (++u == u1) break;
      }
    }
  } else {
    pass_tiles<C, typename C::Packed>(from(0), to(0, tiles1), has_rows ? tiles1 : 0, mine, r, lane, scale,
        [&](int u, typename C::Packed& x) { C::load_packed(a, s, b, h, u * C::KT, tid, values, x); },
        [&](char* at, const typename C::Packed& x) { C::put_packed(masks, at, tid, values, x); },
        [&](int u) { return TileMask{s.packed_v - u * C::KT < C::KT, s.packed_v - u * C::KT - 1}; });
  }
  pass_tiles<C, typename C::Plain>(from(tiles1), to(tiles1, tiles2), has_rows ? tiles2 : 0, mine, r, lane, scale,
      [&](int u, typename C::Plain& x) {
        if constexpr (RW > 1) {
          C::load_cached(a, s, bh, u * C::KT, tid, values, x);
        } else {                                           // (one tensor after the other: all registers are not there for both)
          C::template load_cached<C::kKeys>(a, s, bh, u * C::KT, tid, values, x);
          C::template put_plain<C::kKeys>(mine, tid, values, x);
          C::template load_cached<C::kValues>(a, s, bh, u * C::KT, tid, values, x);
          C::template put_plain<C::kValues>(mine, tid, values, x);
        }
      }, put_plain,
      [&](int u) { return TileMask{s.beside - u * C::KT < C::KT, s.beside - u * C::KT - 1}; });
  pass_tiles<C, typename C::Plain>(from(tiles2), to(tiles2, tiles), has_rows ? (wave_last - 1) / a.heads_per_kv / C::KT + 1 : 0, mine, r, lane, scale,
      [&](int u, typename C::Plain& x) {
        if constexpr (RW > 1) {
          C::load_fresh(a, b, h, u * C::KT, last, tid, values, x);
        } else {
          C::template load_fresh<C::kKeys>(a, b, h, u * C::KT, last, tid, values, x);
          C::template put_plain<C::kKeys>(mine, tid, values, x);
          C::template load_fresh<C::kValues>(a, b, h, u * C::KT, last, tid, values, x);
          C::template put_plain<C::kValues>(mine, tid, values, x);
        }
      }, put_plain,
      [&](int u) { return TileMask{u * C::KT + C::KT - 1 > oldest, newest - u * C::KT}; });
  r.l += other_half(r.l);

  const long long slot_row = (long long)work.slot * (32 * RW) + row - row_base;
  if constexpr (TW == 1) {
    if (!live) return;
    if (n_splits > 1 && half == 0) C::store_state(a, slot_row, r.m, r.l);
#pragma unroll
    for (int x = 0; x < 4; ++x) C::store_channels(a, b, h, row, slot_row, n_splits > 1, x, half, r.o[x], r.l);
  } else {
    // the wavefronts' results meet in LDS, each joins the channels of its own number
    static_assert(TW == 4 && RW == 1);
    __syncthreads();
    float* o = reinterpret_cast<float*>(lds);
    float* ml = o + TW * 64 * 64;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[(wave * 64 + x * 16 + i) * 64 + lane] = r.o[x][i];
    ml[wave * 128 + lane] = r.m;
    ml[wave * 128 + 64 + lane] = r.l;
    __syncthreads();
    float top = ml[lane];
#pragma unroll
    for (int n = 1; n < TW; ++n) top = fmaxf(top, ml[n * 128 + lane]);
    float l = 0.f;
    float16_t sum = {};
#pragma unroll
    for (int n = 0; n < TW; ++n) {
      const float m = ml[n * 128 + lane];
      const float f = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - top);
      l = __builtin_fmaf(f, ml[n * 128 + 64 + lane], l);
#pragma unroll
      for (int i = 0; i < 16; ++i) sum[i] = __builtin_fmaf(f, o[(n * 64 + wave * 16 + i) * 64 + lane], sum[i]);
    }
    if (!live) return;
    if (n_splits > 1 && half == 0 && wave == 0) C::store_state(a, slot_row, top, l);
    C::store_channels(a, b, h, row, slot_row, n_splits > 1, wave, half, sum, l);
  }
}

template <int KB, int VB, int G, int RW, int TW>
hipError_t launch_form(const ChunkArgs& a, hipStream_t stream) {
  const long long items = a.table ? a.list_groups : (long long)a.batch * a.n_kv_heads * a.n_splits * a.row_blocks;
  if (items >= (1LL << 30)) return hipErrorInvalidValue;
  attention_chunk_kernel<KB, VB, G, RW, TW><<<(unsigned)items, 64 * RW * TW, 0, stream>>>(a);
  return hipGetLastError();
}
template <int KB, int VB, int G>
hipError_t launch_bits(const ChunkArgs& a, const ChunkForm& form, hipStream_t stream) {
  return form.row_waves == 1   ? launch_form<KB, VB, G, 1, 4>(a, stream)
         : form.row_waves == 4 ? launch_form<KB, VB, G, 4, 1>(a, stream)
                               : launch_form<KB, VB, G, 8, 1>(a, stream);
}
template <int G>
hipError_t launch_group(const ChunkArgs& a, int kb, int vb, const ChunkForm& form, hipStream_t stream) {
  switch (kb * 10 + vb) {
    case 22: return launch_bits<2, 2, G>(a, form, stream);
    case 23: return launch_bits<2, 3, G>(a, form, stream);
    case 24: return launch_bits<2, 4, G>(a, form, stream);
    case 32: return launch_bits<3, 2, G>(a, form, stream);
    case 33: return launch_bits<3, 3, G>(a, form, stream);
    case 34: return launch_bits<3, 4, G>(a, form, stream);
    case 42: return launch_bits<4, 2, G>(a, form, stream);
    case 43: return launch_bits<4, 3, G>(a, form, stream);
    case 44: return launch_bits<4, 4, G>(a, form, stream);
    default: return hipErrorInvalidValue;
  }
}

#if INNERQ_CHUNK_G == 32
// The splits of a row joined: a wavefront takes four rows of a head, a lane two channels of each; levels and sums come sixteen splits of the
// four rows a load.  slot_rows: rows of a slot.
constexpr int kMergeRows = 4;
__global__ void __launch_bounds__(256) chunk_merge_kernel(ChunkArgs a, int blocks, int slot_rows) {
  const int lane = (int)threadIdx.x & 63;
  const int rows = a.t_new * a.heads_per_kv;
  const long long bh = blockIdx.x / (unsigned)blocks;
  const int row0 = ((int)(blockIdx.x % (unsigned)blocks) * 4 + __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6)) * kMergeRows;
  const int b = (int)(bh / a.n_kv_heads), h = (int)(bh - (long long)b * a.n_kv_heads);
  const int own = a.t_dev ? chunk_seq(a, b, 32).t * a.heads_per_kv : rows;       // (the group does not matter)
  if (row0 >= own) return;
  int n_splits = a.n_splits;
  const float* ws = a.ws;
  long long slots = a.slots, slot;
  if (a.table) {
    n_splits = a.table[2 * b + 1];
    if (n_splits == 1) return;                           // (written already)
    const bool few = own <= kChunkWaveRows;
    slot_rows = few ? kFewRows.row_waves * kChunkWaveRows : kSomeRows.row_waves * kChunkWaveRows;
    if (few) ws = a.ws_few;
    slots = kChunkListItems;
    slot = a.table[2 * b] + (long long)(h * ((own + slot_rows - 1) / slot_rows) + row0 / slot_rows) * n_splits;
  } else {
    slot = (bh * a.row_blocks + row0 / slot_rows) * n_splits;
  }
  // (slots have a multiple of four rows, those behind the last one as well: what stands there goes nowhere)
  const long long slot_row = slot * slot_rows + row0 % slot_rows;
  const float* ml = ws + slot_row * 2;
  const float* po = ws + slots * slot_rows * 2 + slot_row * D + 2 * lane;
  const long long step_ml = slot_rows * 2, step_o = (long long)slot_rows * D;
  const int r = lane >> 4, p16 = lane & 15;              // the lane's row and split of what is loaded sixteen at a time
  auto state = [&](int p) {
    float2 s = {-INFINITY, 0.f};
    if (p < n_splits && row0 + r < own) s = *reinterpret_cast<const float2*>(ml + p * step_ml + r * 2);
    return s;
  };
  const float2 first = state(p16);
  float top = first.x;
  for (int p = p16 + 16; p < n_splits; p += 16) top = fmaxf(top, state(p).x);
#pragma unroll
  for (int x = 8; x > 0; x /= 2) top = fmaxf(top, __shfl_xor(top, x));
  float den = 0.f;
  float2 n[kMergeRows] = {};
  for (int p0 = 0; p0 < n_splits; p0 += 16) {
    const float2 s = p0 == 0 ? first : state(p0 + p16);
    const float f = s.x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.x - top);
    den = __builtin_fmaf(f, s.y, den);
    const int count = n_splits - p0 < 16 ? n_splits - p0 : 16;
    for (int p = 0; p < count; p += 4) {                 // (sixteen partial results under way)
      float2 o[4][kMergeRows];
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < kMergeRows; ++i) o[e][i] = *reinterpret_cast<const float2*>(po + (p0 + (p + e < count ? p + e : count - 1)) * step_o + i * D);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < kMergeRows; ++i) {
          const float w = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(f), 16 * i + ((p + e) & 15)));
          if (p + e < count && row0 + i < own) {
            n[i].x = __builtin_fmaf(w, o[e][i].x, n[i].x);
            n[i].y = __builtin_fmaf(w, o[e][i].y, n[i].y);
          }
        }
    }
  }
#pragma unroll
  for (int x = 8; x > 0; x /= 2) den += __shfl_xor(den, x);
#pragma unroll
  for (int i = 0; i < kMergeRows; ++i) {
    const int row = row0 + i;
    if (row >= own) return;
    const float inv = 1.0f / __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(den), 16 * i));
    const int token = row / a.heads_per_kv;
    const long long dst = b * a.out_batch + (h * a.heads_per_kv + row - token * a.heads_per_kv) * a.out_head + token * a.out_token + 2 * lane;
    if (a.out_is_fp32) *reinterpret_cast<float2*>(static_cast<float*>(a.out) + dst) = float2{n[i].x * inv, n[i].y * inv};
    else *reinterpret_cast<half2_t*>(static_cast<_Float16*>(a.out) + dst) = half2_t{(_Float16)(n[i].x * inv), (_Float16)(n[i].y * inv)};
  }
}
#endif

}  // namespace

#if INNERQ_CHUNK_G == 32
hipError_t launch_chunk_g32(const ChunkArgs& a, int kb, int vb, const ChunkForm& form, hipStream_t stream) { return launch_group<32>(a, kb, vb, form, stream); }
hipError_t launch_chunk_merge(const ChunkArgs& a, const ChunkForm& form, hipStream_t stream) {
  const long long blocks = ceil_div((long long)a.t_new * a.heads_per_kv, 4 * kMergeRows), all = (long long)a.batch * a.n_kv_heads * blocks;
  if (all >= (1LL << 31)) return hipErrorInvalidValue;
  chunk_merge_kernel<<<(unsigned)all, 256, 0, stream>>>(a, (int)blocks, form.rows());
  return hipGetLastError();
}
#else
hipError_t launch_chunk_g64(const ChunkArgs& a, int kb, int vb, const ChunkForm& form, hipStream_t stream) { return launch_group<64>(a, kb, vb, form, stream); }
#endif

}  // namespace innerq
