// Attention over the cache in 8 bits with block scales, many rows of a kv head (chunks of a prompt, a decoder's prompt).
//
// A work-group of eight wavefronts (or four) has 32 rows of a kv head a wavefront and walks over the tokens in units of 32:
//   S^T = K Q^T   (32 x 32 x 16 instructions: rows are tokens, columns query rows)
//   O^T = V^T P^T (rows are channels)
// Every unit is brought to fp16 once, in LDS, in the order of the operands (a wavefront's reads are whole kilobytes), an equal part of it by every
// wavefront.  A lane's scores are those of 16 tokens of one query row, which, as weights rounded to fp16, are the second product's operand where
// they stand.
//
// Matrix and vector instructions run side by side: the scores of the next unit are formed while the weights of this one are, and what
// is left of the vector work, the next unit's level and the decoding of the one after, stands between the matrix instructions of the
// second product, with the keys of the unit after the next on their way to registers.
//
// Codes are exact in fp16 and scales are taken as block_math.h says.
//
// What bounds it is the matrix cores with the vector work beside them, and the power that both take: 2048 new tokens of 32 heads (8 of keys) over 32k,
// 1134 GFLOP, take 1140 to 1180 us, 1000 to 960 TFLOP/s (a library product of two fp16 matrices 1330), matrix pipes 46 % and vector pipes 52 % busy; a
// form with 8 % fewer cycles took the same time at a lower clock.  Without one part at a time, in copies (of 1178 us): the first product 924, the second
// 934, decoding and LDS writes 1037, exponentials 1118, barriers 1147, loads 1080.  Every wavefront with units of its own, decoded for itself: 2770;
// units decoded once, in LDS, 64 rows a wavefront: 1534; the two products interleaved with what stands between them: 1196; keys read ahead of the barrier:
// 1153; 32 rows and eight wavefronts leave registers (no spills) and are as fast here, and faster for ragged batches (474 us, 441).
#include "block.h"
#include "block_few.h"
#include "block_math.h"

namespace innerq {
namespace {

constexpr int D = kHeadDim;
constexpr int kUnitBytes = 2 * kBlockTile * D * 2;       // keys, then values, in fp16
constexpr int kUnitValues = kUnitBytes / 2;
constexpr int kUnits = 4;                                // that LDS holds

typedef float float16_t __attribute__((ext_vector_type(16)));

__device__ __forceinline__ float other_half(float x) {   // lane ^ 32
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float((threadIdx.x & 32u) ? r[0] : r[1]);
}

struct State {
  half8_t q[8];
  float16_t o[4];
  float m, l;                  // level, the lane's part of the sum
  float zero, raise;           // the level (0: none yet), and what raises it
  bool far;                            // some row's level is
};

// ---- a unit on its way into LDS
//
// Keys: [channel octet 16][row 32] of 16 bytes; values: [channels 32 x][tokens, two parts][half][channel 16 m + c] of 16 bytes.  The row of a token
// is its number with bits 3 and 4 exchanged: then a lane's scores 8 e .. 8 e + 7 are those of tokens 4 g + j and 16 + 4 g + j, g = 2 e + half, which
// is how values lie in the store.
__device__ __forceinline__ int row_of(int token) { return (token & 7) | (token & 8) << 1 | (token & 16) >> 1; }
__device__ __forceinline__ int token_of(int i, int half) { return (i & 4) << 2 | (i >> 3) << 3 | half << 2 | (i & 3); }

struct Staged { u32x4 a, b, c, d; };                     // packed: keys, values; fp16: two pieces of a key row, four of values

// Sixteen codes: number `lane` of the kilobyte `part` (0 .. 3) of a tensor's tile.
__device__ __forceinline__ int put_at(bool keys, int part, int lane) {
  const int g = lane >> 4, c = lane & 15;
  if (keys) return (2 * g + (part & 1)) * 1024 + row_of(16 * (part >> 1) + c) * 16;        // channels 32 g + 16 h + ..
  return kUnitValues + part * 2048 + (g >> 1) * 1024 + (g & 1) * 512 + c * 16;
}
template <bool E4M3>
__device__ __forceinline__ void put_codes(char* dst, int apart, const u32x4& w, uint32_t by) {
  *reinterpret_cast<half8_t*>(dst) = expand<E4M3>(w.x, w.y, by);
  *reinterpret_cast<half8_t*>(dst + apart) = expand<E4M3>(w.z, w.w, by);
}

// fp16 rows.  Keys: a thread has 64 / WAVES channels of a token, pairs of lanes next to each other and 32 / WAVES tokens of a wavefront in turn (a token's
// channels in a row of lanes would all go to the same banks); values: four tokens of 8 / WAVES pairs of channels, with eight wavefronts the same
// four for a wavefront, so that where the rows are is worked out once for all lanes.  (First prompt of 16384 tokens of 32 heads: 2770 us with neither, 2540
// with the first, 2440 with both.)
template <int WAVES>
struct PlainPart {
  static constexpr int N = 8 / WAVES, T = 4 * N;         // octets of a thread, tokens of a wavefront
  int token, octet;
  __device__ __forceinline__ explicit PlainPart(int tid) {
    const int l = tid & 63;
    token = (tid >> 6) * T + l / 2 % T;
    octet = ((l & 1) | l / (2 * T) << 1) * N;
  }
};
template <int WAVES>
__device__ __forceinline__ void put_plain(char* buf, int tid, const Staged& x, uint32_t by) {
  constexpr int N = PlainPart<WAVES>::N;
  {
    const PlainPart<WAVES> part(tid);
    char* dst = buf + part.octet * 512 + row_of(part.token) * 16;
    *reinterpret_cast<u32x4*>(dst) = x.a;
    if (N == 2) *reinterpret_cast<u32x4*>(dst + 512) = x.b;
  }
  constexpr int PAIRS = 64 / N;                          // threads of four tokens
  const int quad = tid / PAIRS, ch = tid % PAIRS * 2 * N, g = quad & 3;                    // tokens 4 quad .. = 16 i + 4 g ..
  char* dst = buf + kUnitValues + (ch >> 5) * 2048 + (g >> 1) * 1024 + (g & 1) * 512 + (quad >> 2) * 8 + ((ch & 31) >> 1) * 16;
  const uint32_t w[4][2] = {{x.c.x, x.c.y}, {x.c.z, x.c.w}, {x.d.x, x.d.y}, {x.d.z, x.d.w}};
#pragma unroll
  for (int p = 0; p < N; ++p) {                          // channels ch + 2 p, ch + 2 p + 1
    const u32x2 even = {__builtin_amdgcn_perm(w[1][p], w[0][p], 0x05040100u), __builtin_amdgcn_perm(w[3][p], w[2][p], 0x05040100u)};
    const u32x2 odd = {__builtin_amdgcn_perm(w[1][p], w[0][p], 0x07060302u), __builtin_amdgcn_perm(w[3][p], w[2][p], 0x07060302u)};
    *reinterpret_cast<u32x2*>(dst + 16 * p) = u32x2{times(even.x, by), times(even.y, by)};
    *reinterpret_cast<u32x2*>(dst + 16 * p + 256) = u32x2{times(odd.x, by), times(odd.y, by)};
  }
}

// ---- the two products and what is between them

// Largest of a lane's scores, as an exponent.
__device__ __forceinline__ float unit_top(const float16_t& s, const Scales& u) {
  float t = s[0];
#pragma unroll
  for (int i = 1; i < 16; ++i) t = fmaxf(t, s[i]);
  return __builtin_fmaf(t, u.by, u.add);
}
__device__ __forceinline__ void raise_level(State& r, float mine) {
  const float top = fmaxf(mine, other_half(mine));
  const bool up = top > r.raise;
  const float level = up ? fmaxf(r.m, __builtin_fabsf(top) > kFar ? top : top - kTop) : r.m;
  const float f = up ? __builtin_amdgcn_exp2f(r.m - level) : 1.f;                // (0 from the empty state)
  r.l *= f;
#pragma unroll
  for (int x = 0; x < 4; ++x) r.o[x] *= f;
  r.m = level;
  r.zero = level == -INFINITY ? 0.f : level;
  r.raise = threshold(level);
  r.far = __builtin_amdgcn_ballot_w64(__builtin_fabsf(r.zero) > kFar) != 0;
}
__device__ __forceinline__ void shift_level(State& r, int e) {
  r.m -= (float)e;
  r.l = __builtin_amdgcn_ldexpf(r.l, e);
  r.zero = r.m == -INFINITY ? 0.f : r.m;
  r.raise = threshold(r.m);
}
// Weights of scores 2 e, 2 e + 1.
__device__ __forceinline__ void two_weights(int e, const float16_t& s, float by, float bias, half8_t (&p)[2], float& sum) {
  const half2_t w = {(_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * e], by, bias)), (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[2 * e + 1], by, bias))};
  p[e / 4][2 * (e % 4)] = w.x;
  p[e / 4][2 * (e % 4) + 1] = w.y;
  sum = __builtin_amdgcn_fdot2(w, half2_t{(_Float16)1.0f, (_Float16)1.0f}, sum, false);
}

// Units u0 .. u1 of one kind.  fetch(u, regs, scales): a unit's bytes into registers, and its scales; put(buffer, regs, scales): into LDS; mask(u,
// scores): scores of tokens that a row does not attend to are -infinity.
template <typename Fetch, typename Put, typename Mask>
__device__ __forceinline__ void walk(int u0, int u1, char* lds, State& r, int lane, Fetch fetch, Put put, Mask mask) {
  if (u0 >= u1) return;
  auto at = [&](int u) { return lds + ((u - u0) % kUnits) * kUnitBytes; };
  auto bound = [&](int u) { return u < u1 ? u : u1 - 1; };      // (behind the last unit: that one again)
  Staged x, y;
  Scales now, next, third, sx, sy;
  // units u0 .. u0 + 2 into LDS, u0 + 3 and u0 + 4 under way
  fetch(u0, x, now);
  fetch(bound(u0 + 1), y, next);
  put(at(u0), x, now);
  fetch(bound(u0 + 2), x, third);
  put(at(u0 + 1), y, next);
  fetch(bound(u0 + 3), y, sy);
  put(at(u0 + 2), x, third);
  fetch(bound(u0 + 4), x, sx);
  __syncthreads();
  half8_t k[8];
  auto keys = [&](int u) {
#pragma unroll
    for (int e = 0; e < 8; ++e) k[e] = *reinterpret_cast<const half8_t*>(at(u) + lane * 16 + 1024 * e);
  };
  float16_t s, t;
  float top;
  keys(u0);
  s = float16_t{};
#pragma unroll
  for (int e = 0; e < 8; ++e) s = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[e], r.q[e], s, 0, 0, 0);
  keys(u0 + 1);
  mask(u0, s);
  top = unit_top(s, now);
  // s: scores of unit u; k: keys of unit u + 1; x: unit u + 3
  auto step = [&](int u, float16_t& s, float16_t& t, Staged& x, Scales& sx) {
    if (__builtin_amdgcn_ballot_w64(top > r.raise)) raise_level(r, top);
    if (r.far) {
      // (the fused form takes the level, which is rounded, from an exact product)
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        s[i] = __builtin_fmaf(s[i], now.by, now.add);
        asm volatile("" : "+v"(s[i]));
      }
      now.by = 1.f;
      now.add = 0.f;
    }
    // the scores of the next unit and the weights of this one, piece by piece; operands of the second product on their way
    half8_t p[2], v[8];
    const float bias = now.add - r.zero;
    float sum = 0.f;
    t = float16_t{};
    const char* values = at(u) + kUnitValues + lane * 16;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      t = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[e], r.q[e], t, 0, 0, 0);
      v[e] = *reinterpret_cast<const half8_t*>(values + 2048 * (e % 4) + 1024 * (e / 4));
      two_weights(e, s, now.by, bias, p, sum);
      __builtin_amdgcn_sched_barrier(0);
    }
    r.l = __builtin_fmaf(sum, now.inv, r.l);
    mask(bound(u + 1), t);
    // the second product; the keys after the next, a unit into LDS, the largest of the next scores
    keys(u + 2);
    put(at(u + 3), x, sx);
    now = next;
    next = third;
    third = sx;
    top = unit_top(t, now);
#pragma unroll
    for (int e = 0; e < 8; ++e) r.o[e % 4] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[e], p[e / 4], r.o[e % 4], 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
      __builtin_amdgcn_sched_group_barrier(0x2, 12, 0);
    }
    fetch(bound(u + 5), x, sx);
    __syncthreads();
  };
  for (int u = u0;;) {
    step(u, s, t, y, sy);
    if (++u == u1) break;
    step(u, t, s, x, sx);
    if (++u == u1) break;
  }
}

template <bool E4M3, int WAVES>
__device__ __forceinline__ void attend(const BlockAttnArgs& a, const BlockWork& w, char* lds) {
  constexpr int ROWS = 32 * WAVES;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = w.b, h = w.h, n_splits = w.n_splits;
  const long long bh = (long long)b * a.s.n_kv_heads + h;
  const BlockSeq s = block_seq(a, b);
  const int rows = s.t * a.heads_per_kv, row0 = w.row_block * ROWS;
  if (row0 >= rows) return;                              // (uniform)
  State r;
  {
    const int row = row0 + 32 * wave + (lane & 31), i = row / a.heads_per_kv;
    const __half* src = a.q.p + b * a.q.batch + (h * a.heads_per_kv + row - i * a.heads_per_kv) * a.q.head + i * a.q.token + 8 * (lane >> 5);
#pragma unroll
    for (int st = 0; st < 8; ++st) r.q[st] = row < rows ? *reinterpret_cast<const half8_t*>(src + 16 * st) : half8_t{};
  }
#pragma unroll
  for (int x = 0; x < 4; ++x) r.o[x] = float16_t{};
  r.m = r.raise = -INFINITY;
  r.l = r.zero = 0.f;
  r.far = false;

  const bool causal = a.k.p != nullptr;
  const int last_row = (row0 + ROWS < rows ? row0 + ROWS : rows) - 1;
  const int open = s.n - s.packed, plain = open + (causal ? last_row / a.heads_per_kv + 1 : 0);
  const int tiles1 = s.packed / kBlockTile, tiles = tiles1 + (plain + kBlockTile - 1) / kBlockTile;
  const int share = tiles / n_splits, more = tiles % n_splits;
  const int t0 = w.split * share + (w.split < more ? w.split : more), t1 = t0 + share + (w.split < more ? 1 : 0);

  const int u1 = t1 < tiles1 ? t1 : tiles1;
  BlockUnits<E4M3> units;
  if (t0 < u1) {
    // (eight wavefronts: half of them bring keys, half values)
    const bool keys = WAVES == 4 || wave < 4;
    const uint32_t mine_at = (uint32_t)(64 * (wave & 3) + lane) * 16;
    const int to = put_at(keys, wave & 3, lane), apart = keys ? 512 : 256;
    const uint8_t* codes = keys ? a.s.k.codes : a.s.v.codes;
    auto fetch = [&](int u, Staged& x, Scales& sc) {
      units.look(a.s, b, h, u, u1, lane);
      const long long tile = units.tile(u) * kBlockTileBytes;
      x.a = *reinterpret_cast<const u32x4*>(codes + tile + mine_at);
      if (WAVES == 4) x.b = *reinterpret_cast<const u32x4*>(a.s.v.codes + tile + mine_at);
      sc = units.scales(u);
    };
    auto put = [&](char* buf, const Staged& x, const Scales& sc) {
      put_codes<E4M3>(buf + to, apart, x.a, keys ? codes_times<E4M3>(0) : sc.values);
      if (WAVES == 4) put_codes<E4M3>(buf + put_at(false, wave, lane), 256, x.b, sc.values);
    };
    walk(t0, u1, lds, r, lane, fetch, put, [](int, float16_t&) {});
  }
  if (t1 > tiles1) {
    const long long open_at = bh * a.s.block * D;
    const __half *ko = a.s.k.open + open_at, *vo = a.s.v.open + open_at;
    const __half *kf = a.k.p + b * a.k.batch + h * a.k.head, *vf = a.v.p + b * a.v.batch + h * a.v.head;
    const int shift = plain_shift(units.largest);
    const uint32_t by = half_power(-shift) * 0x10001u;
    if (shift) shift_level(r, shift);                    // (uniform)
    // (selections, no branches: the lanes of a wavefront may differ)
    auto row_at = [&](const __half* o, const __half* f, long long pitch, int i) {
      const bool waits = i < open;
      const unsigned long long step = waits ? (unsigned long long)D : (unsigned long long)pitch;
      const unsigned at = (unsigned)(waits ? i : i - open);
      return (waits ? o : f) + at * step;
    };
    auto fetch = [&](int u, Staged& x, Scales& sc) {
      sc = kPlainScales;
      const int i0 = u * kBlockTile;
      auto token = [&](int i) { return i0 + i < plain ? i0 + i : plain - 1; };   // (behind the last one: that one again, masked)
      constexpr int N = PlainPart<WAVES>::N, PAIRS = 64 / N;                     // (as put_plain)
      const PlainPart<WAVES> part(tid);
      const __half* k = row_at(ko, kf, a.k.token, token(part.token)) + part.octet * 8;
      x.a = *reinterpret_cast<const u32x4*>(k);
      if (N == 2) x.b = *reinterpret_cast<const u32x4*>(k + 8);
      u32x2 w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const __half* v = row_at(vo, vf, a.v.token, token(4 * (WAVES == 8 ? wave : tid / PAIRS) + e)) + tid % PAIRS * 2 * N;
        if (N == 2) w[e] = *reinterpret_cast<const u32x2*>(v);
        else w[e] = u32x2{*reinterpret_cast<const uint32_t*>(v), 0u};
      }
      x.c = u32x4{w[0].x, w[0].y, w[1].x, w[1].y};
      x.d = u32x4{w[2].x, w[2].y, w[3].x, w[3].y};
    };
    const int row = row0 + 32 * wave + (lane & 31), half = lane >> 5;
    const int limit = causal ? open + (row < rows ? row : rows - 1) / a.heads_per_kv : plain - 1;      // last token that the lane's row attends to
    auto mask = [&](int u, float16_t& sc) {
      const int left = limit - u * kBlockTile;
      if (!__builtin_amdgcn_ballot_w64(left < kBlockTile - 1)) return;
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (token_of(i, half) > left) sc[i] = -INFINITY;
    };
    walk(t0 > tiles1 ? t0 - tiles1 : 0, t1 - tiles1, lds, r, lane, fetch,
         [&](char* buf, const Staged& x, const Scales&) { put_plain<WAVES>(buf, tid, x, by); }, mask);
    if (shift) shift_level(r, -shift);
  }

  // results: a lane has channels 32 x + 16 y + 8 half + 2 i + m of its row, at o[x][4 y + 8 m + i]
  const float l = r.l + other_half(r.l);
  int again = (int)threadIdx.x;
  asm("" : "+v"(again));                                 // (where its row is, is found anew: registers held over the loops would be spilled)
  const int row = row0 + 32 * (again >> 6) + (again & 31), half = again >> 5 & 1;
  if (row >= rows) return;
  const int row_token = row / a.heads_per_kv, row_head = h * a.heads_per_kv + row - row_token * a.heads_per_kv;
  if (n_splits > 1) {
    const long long slot_row = w.slot * ROWS + row - row0;
    float* dst = a.ws + a.slots * (ROWS * 2) + slot_row * D + 8 * half;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const float16_t& o = r.o[x];
        *reinterpret_cast<float4*>(dst + 32 * x + 16 * y) = float4{o[4 * y], o[4 * y + 8], o[4 * y + 1], o[4 * y + 9]};
        *reinterpret_cast<float4*>(dst + 32 * x + 16 * y + 4) = float4{o[4 * y + 2], o[4 * y + 10], o[4 * y + 3], o[4 * y + 11]};
      }
    if (half == 0) *reinterpret_cast<float2*>(a.ws + slot_row * 2) = float2{r.m, l};
    return;
  }
  const float f = l > 0.f ? 1.0f / l : 0.f;              // (no token: zero)
  const long long out = b * a.out_batch + row_head * a.out_head + row_token * a.out_token + 8 * half;
#pragma unroll
  for (int x = 0; x < 4; ++x)
#pragma unroll
    for (int y = 0; y < 2; ++y) {
      const float16_t& o = r.o[x];
      const float c[8] = {o[4 * y] * f,     o[4 * y + 8] * f,  o[4 * y + 1] * f, o[4 * y + 9] * f,
                          o[4 * y + 2] * f, o[4 * y + 10] * f, o[4 * y + 3] * f, o[4 * y + 11] * f};
      if (a.out_is_fp32) {
        float* dst = static_cast<float*>(a.out) + out + 32 * x + 16 * y;
        *reinterpret_cast<float4*>(dst) = float4{c[0], c[1], c[2], c[3]};
        *reinterpret_cast<float4*>(dst + 4) = float4{c[4], c[5], c[6], c[7]};
      } else {
        half8_t v;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = (_Float16)c[e];
        *reinterpret_cast<half8_t*>(static_cast<_Float16*>(a.out) + out + 32 * x + 16 * y) = v;
      }
    }
}

template <bool E4M3, int WAVES>
__global__ void __launch_bounds__(64 * WAVES) __attribute__((amdgpu_waves_per_eu(2, 2))) block_rows_kernel(BlockAttnArgs a) {
  __shared__ __align__(16) char lds[kUnits * kUnitBytes];
  attend<E4M3, WAVES>(a, uniform_work(a), lds);
}

// A ragged batch with sequences of many rows and of few.  With lists: the first work-groups have the former, those behind them the latter, which wait for memory
// while others compute.  Without: the same work-groups for every sequence, each in the form that its sequence's rows ask for.
template <bool E4M3>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) block_list_kernel(BlockAttnArgs a) {
  constexpr int kFew = (int)sizeof(float) * block_few::kFloats<2>, kMany = kUnits * kUnitBytes;
  __shared__ __align__(16) char lds[kFew > kMany ? kFew : kMany];
  BlockWork w;
  bool many = (int)blockIdx.x < a.list_many;
  if (!a.table) {
    w = uniform_work(a);
    many = block_seq(a, w.b).t * a.heads_per_kv > a.few_most;
  } else if (many) {
    if (!find_work<128, 4>(a, a.few_most, 0x7fffffff, (int)blockIdx.x, w)) return;          // (uniform)
  } else {
    if (!find_work<32, 4>(a, 0, a.few_most, (int)blockIdx.x - a.list_many, w)) return;
  }
  if (many) attend<E4M3, 4>(a, w, lds);
  else block_few::attend<E4M3, 2>(a, w, reinterpret_cast<float*>(lds), a.ws_few, a.few_slots, a.few_rows);
}

}  // namespace

hipError_t launch_block_rows(const BlockAttnArgs& a, bool e4m3, const BlockForm& form, hipStream_t stream) {
  const long long groups = (long long)a.s.batch * a.s.n_kv_heads * a.row_blocks * a.n_splits;
  if (groups >= (1LL << 31)) return hipErrorInvalidValue;
  if (form.rows == 128) {
    if (e4m3) block_rows_kernel<true, 4><<<(unsigned)groups, 256, 0, stream>>>(a);
    else block_rows_kernel<false, 4><<<(unsigned)groups, 256, 0, stream>>>(a);
  } else if (form.rows == 256) {
    if (e4m3) block_rows_kernel<true, 8><<<(unsigned)groups, 512, 0, stream>>>(a);
    else block_rows_kernel<false, 8><<<(unsigned)groups, 512, 0, stream>>>(a);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

hipError_t launch_block_list(const BlockAttnArgs& a, bool e4m3, hipStream_t stream) {
  const long long groups = a.table ? (long long)a.list_many + a.list_few : (long long)a.s.batch * a.s.n_kv_heads * a.row_blocks * a.n_splits;
  if (groups >= (1LL << 31)) return hipErrorInvalidValue;
  if (e4m3) block_list_kernel<true><<<(unsigned)groups, 256, 0, stream>>>(a);
  else block_list_kernel<false><<<(unsigned)groups, 256, 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace innerq
