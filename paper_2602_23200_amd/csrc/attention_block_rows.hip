// Attention over the cache in 8 bits with block scales, many rows of a kv head (chunks of a prompt, a decoder's prompt).
//
// A work-group of four wavefronts, one a SIMD, has 128 RG rows of a kv head, 32 RG of them a wavefront, and walks over the tokens in units of 32:
//   S^T = K Q^T   (32 x 32 x 16 instructions: rows are tokens, columns query rows)
//   O^T = V^T P^T (rows are channels)
// Every unit is brought to fp16 once, in LDS, in the order of the operands (a wavefront's reads are whole kilobytes), a wavefront a quarter of it.
// A lane's scores are those of 16 tokens of one query row (two: RG = 2), which, as weights rounded to fp16, are the second product's operand
// where they stand.
//
// Matrix and vector instructions are to run side by side: the scores of the next unit are formed while the weights of this one are, and what
// is left of the vector work, the next unit's level and the decoding of the one after it, stands between the matrix instructions of the
// second product.  That wants 400 registers, so there is one wavefront a SIMD.
//
// Codes are exact in fp16.  The scale of a block of keys is a factor of its scores, that of a block of values a summand of the exponent,
// so a weight carries it: w = 2^(s + log2 S_v - level), O = sum w code, and the normaliser is l = sum w / S_v of the same rounded weights.  A block
// of far smaller values than the largest ones so far would have weights that fp16 does not hold; below 1/16 of their scale it counts as one of
// 2^k S_v and its codes are multiplied by 2^-k in LDS.
#include "block.h"
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

// What is uniform over a unit: factor of the scores, summand of the exponent, 1 / S_v, 2^-k.
struct Scales { float by, add, inv, shrink; };

template <int RG>
struct State {
  half8_t q[RG][8];
  float16_t o[RG][4];
  float m[RG], l[RG];                  // level, the lane's part of the sum
  float zero[RG], raise[RG];           // the level (0: none yet), and what raises it
  bool far;                            // some row's level is
};

// ---- a unit on its way into LDS

struct Staged { u32x4 a, b, c, d; };                     // packed: keys, values; fp16: two pieces of a key row, four of values

template <bool E4M3>
__device__ __forceinline__ void put_packed(char* buf, int wave, int lane, const u32x4& k, const u32x4& v, float shrink) {
  const int g = lane >> 4, c = lane & 15;
  {
    // tokens 16 a + c, channels 32 g + 16 h + ..
    char* dst = buf + (2 * g + (wave & 1)) * 1024 + (16 * (wave >> 1) + c) * 16;
    *reinterpret_cast<half8_t*>(dst) = expand<E4M3>(k.x, k.y);
    *reinterpret_cast<half8_t*>(dst + 512) = expand<E4M3>(k.z, k.w);
  }
  const half8_t even = expand_by<E4M3>(v.x, v.y, shrink), odd = expand_by<E4M3>(v.z, v.w, shrink);
  // (the lane's g is that of value_lane: neighbours in LDS are neighbours in the wavefront)
  const int vg = (g >> 1) | (g & 1) << 1;
  char* dst = buf + kUnitValues + wave * 2048 + (vg & 1) * 512 + c * 16 + (vg >> 1) * 8;
  const u32x4 e = __builtin_bit_cast(u32x4, even), o = __builtin_bit_cast(u32x4, odd);
  *reinterpret_cast<u32x2*>(dst) = u32x2{e.x, e.y};
  *reinterpret_cast<u32x2*>(dst + 1024) = u32x2{e.z, e.w};
  *reinterpret_cast<u32x2*>(dst + 256) = u32x2{o.x, o.y};
  *reinterpret_cast<u32x2*>(dst + 1024 + 256) = u32x2{o.z, o.w};
}
// Which sixteen bytes of a kilobyte of value codes a lane takes: those of groups 0, 2, 1, 3.
__device__ __forceinline__ int value_lane(int lane) {
  const int g = lane >> 4;
  return ((g >> 1) | (g & 1) << 1) * 16 + (lane & 15);
}

// fp16 rows.  Keys: thread tid has sixteen channels of a token; values: four channels of four tokens.
__device__ __forceinline__ void put_plain(char* buf, int tid, const Staged& x) {
  {
    char* dst = buf + (tid & 7) * 1024 + (tid >> 3) * 16;
    *reinterpret_cast<u32x4*>(dst) = x.a;
    *reinterpret_cast<u32x4*>(dst + 512) = x.b;
  }
  const int quad = tid >> 5, ch = (tid & 31) * 4;        // tokens 4 quad ..
  const int g = quad & 3;
  char* dst = buf + kUnitValues + (ch >> 5) * 2048 + (quad >> 2) * 1024 + (g & 1) * 512 + (g >> 1) * 8 + ((ch & 31) >> 1) * 16;
  const uint32_t w[4][2] = {{x.c.x, x.c.y}, {x.c.z, x.c.w}, {x.d.x, x.d.y}, {x.d.z, x.d.w}};
#pragma unroll
  for (int p = 0; p < 2; ++p) {                          // channels ch + 2 p, ch + 2 p + 1
    const u32x2 even = {__builtin_amdgcn_perm(w[1][p], w[0][p], 0x05040100u), __builtin_amdgcn_perm(w[3][p], w[2][p], 0x05040100u)};
    const u32x2 odd = {__builtin_amdgcn_perm(w[1][p], w[0][p], 0x07060302u), __builtin_amdgcn_perm(w[3][p], w[2][p], 0x07060302u)};
    *reinterpret_cast<u32x2*>(dst + 16 * p) = even;
    *reinterpret_cast<u32x2*>(dst + 16 * p + 256) = odd;
  }
}

// ---- the two products and what is between them

template <int RG>
__device__ __forceinline__ void unit_scores(const char* buf, const State<RG>& r, int lane, float16_t (&s)[RG]) {
  const char* keys = buf + lane * 16;
#pragma unroll
  for (int n = 0; n < RG; ++n) s[n] = float16_t{};
#pragma unroll
  for (int st = 0; st < 8; ++st) {
    const half8_t k = *reinterpret_cast<const half8_t*>(keys + 1024 * st);
#pragma unroll
    for (int n = 0; n < RG; ++n) s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k, r.q[n][st], s[n], 0, 0, 0);
  }
}
__device__ __forceinline__ float threshold(float m) { return __builtin_fmaf(-kFarShare, __builtin_fabsf(m), m) + kRaise; }
// Largest of a lane's scores, as exponents.
template <int RG>
__device__ __forceinline__ void unit_tops(const float16_t (&s)[RG], const Scales& u, float (&top)[RG]) {
#pragma unroll
  for (int n = 0; n < RG; ++n) {
    float t = s[n][0];
#pragma unroll
    for (int i = 1; i < 16; ++i) t = fmaxf(t, s[n][i]);
    top[n] = __builtin_fmaf(t, u.by, u.add);
  }
}
template <int RG>
__device__ __forceinline__ void raise_levels(State<RG>& r, const float (&tops)[RG]) {
  bool far = false;
#pragma unroll
  for (int n = 0; n < RG; ++n) {
    const float top = fmaxf(tops[n], other_half(tops[n]));
    const bool up = top > r.raise[n];
    const float level = up ? fmaxf(r.m[n], __builtin_fabsf(top) > kFar ? top : top - kTop) : r.m[n];
    const float f = up ? __builtin_amdgcn_exp2f(r.m[n] - level) : 1.f;           // (0 from the empty state)
    r.l[n] *= f;
#pragma unroll
    for (int x = 0; x < 4; ++x) r.o[n][x] *= f;
    r.m[n] = level;
    r.zero[n] = level == -INFINITY ? 0.f : level;
    r.raise[n] = threshold(level);
    far |= __builtin_fabsf(r.zero[n]) > kFar;
  }
  r.far = __builtin_amdgcn_ballot_w64(far) != 0;
}
// Weights of scores 2 e, 2 e + 1 of every row.
template <int RG>
__device__ __forceinline__ void two_weights(int e, const float16_t (&s)[RG], float by, const float (&bias)[RG], half8_t (&p)[RG][2], float (&sum)[RG]) {
#pragma unroll
  for (int n = 0; n < RG; ++n) {
    const half2_t w = {(_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[n][2 * e], by, bias[n])), (_Float16)__builtin_amdgcn_exp2f(__builtin_fmaf(s[n][2 * e + 1], by, bias[n]))};
    p[n][e / 4][2 * (e % 4)] = w.x;
    p[n][e / 4][2 * (e % 4) + 1] = w.y;
    sum[n] = __builtin_amdgcn_fdot2(w, half2_t{(_Float16)1.0f, (_Float16)1.0f}, sum[n], false);
  }
}

// Units u0 .. u1 of one kind.  fetch(u, regs, scales): a unit's bytes into registers, and its scales; put(buffer, regs, scales): into LDS; mask(u,
// scores): scores of tokens that a row does not attend to are -infinity.
template <int RG, bool MASKED, typename Fetch, typename Put, typename Mask>
__device__ __forceinline__ void walk(int u0, int u1, char* lds, State<RG>& r, int lane, Fetch fetch, Put put, Mask mask) {
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
  float16_t s[RG], t[RG];
  float top[RG];
  keys(u0);
#pragma unroll
  for (int n = 0; n < RG; ++n) s[n] = float16_t{};
#pragma unroll
  for (int e = 0; e < 8; ++e)
#pragma unroll
    for (int n = 0; n < RG; ++n) s[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[e], r.q[n][e], s[n], 0, 0, 0);
  keys(u0 + 1);
  if (MASKED) mask(u0, s);
  unit_tops<RG>(s, now, top);
  // s: scores of unit u; k: keys of unit u + 1; x: unit u + 3
  auto step = [&](int u, float16_t (&s)[RG], float16_t (&t)[RG], Staged& x, Scales& sx) {
    bool raise = false;
#pragma unroll
    for (int n = 0; n < RG; ++n) raise |= top[n] > r.raise[n];
    if (__builtin_amdgcn_ballot_w64(raise)) raise_levels<RG>(r, top);
    if (r.far) {
      // (the fused form takes the level, which is rounded, from an exact product)
#pragma unroll
      for (int n = 0; n < RG; ++n)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[n][i] = __builtin_fmaf(s[n][i], now.by, now.add);
          asm volatile("" : "+v"(s[n][i]));
        }
      now.by = 1.f;
      now.add = 0.f;
    }
    // the scores of the next unit and the weights of this one, piece by piece; operands of the second product on their way
    half8_t p[RG][2], v[8];
    float bias[RG], sum[RG];
#pragma unroll
    for (int n = 0; n < RG; ++n) {
      bias[n] = now.add - r.zero[n];
      sum[n] = 0.f;
      t[n] = float16_t{};
    }
    const char* values = at(u) + kUnitValues + lane * 16;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int e = 0; e < 8; ++e) {
#pragma unroll
      for (int n = 0; n < RG; ++n) t[n] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[e], r.q[n][e], t[n], 0, 0, 0);
      v[e] = *reinterpret_cast<const half8_t*>(values + 2048 * (e % 4) + 1024 * (e / 4));
      two_weights<RG>(e, s, now.by, bias, p, sum);
      __builtin_amdgcn_sched_barrier(0);
    }
#pragma unroll
    for (int n = 0; n < RG; ++n) r.l[n] = __builtin_fmaf(sum[n], now.inv, r.l[n]);
    // the second product; the keys after the next, a unit into LDS, the largest of the next scores
    keys(u + 2);
    put(at(u + 3), x, sx);
    now = next;
    next = third;
    third = sx;
    if (!MASKED) unit_tops<RG>(t, now, top);
#pragma unroll
    for (int e = 0; e < 8; ++e)
#pragma unroll
      for (int n = 0; n < RG; ++n) r.o[n][e % 4] = __builtin_amdgcn_mfma_f32_32x32x16_f16(v[e], p[n][e / 4], r.o[n][e % 4], 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 8 * RG; ++e) {
      __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2 / RG, 0);
      __builtin_amdgcn_sched_group_barrier(0x2, 12 / RG, 0);
    }
    if (MASKED) {
      mask(bound(u + 1), t);
      unit_tops<RG>(t, now, top);
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

template <bool E4M3, int RG>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(RG == 2 ? 1 : 2, RG == 2 ? 1 : 2)))
block_rows_kernel(BlockAttnArgs a) {
  __shared__ __align__(16) char lds[kUnits * kUnitBytes];
  constexpr int ROWS = 128 * RG;
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  // Sequence-heads that can be shared out evenly stay on one XCD (its L2 then brings every unit from memory once); the last rows, which have the
  // most keys, go first.
  const unsigned heads = (unsigned)(a.s.batch * a.s.n_kv_heads);
  const bool pinned = heads % 8u == 0u;
  const unsigned slot = pinned ? blockIdx.x / 8u : blockIdx.x, mine_heads = pinned ? heads / 8u : heads;
  const unsigned rank = slot / (mine_heads * (unsigned)a.n_splits), rest = slot % (mine_heads * (unsigned)a.n_splits);
  const int bh = (int)(rest / (unsigned)a.n_splits + (pinned ? blockIdx.x % 8u * mine_heads : 0u)), split = (int)(rest % (unsigned)a.n_splits);
  const int row_block = a.row_blocks - 1 - (int)rank;
  const int b = bh / a.s.n_kv_heads, h = bh % a.s.n_kv_heads;
  const BlockSeq s = block_seq(a, b);
  const int rows = s.t * a.heads_per_kv, row0 = row_block * ROWS;
  if (row0 >= rows) return;                              // (uniform)
  State<RG> r;
#pragma unroll
  for (int n = 0; n < RG; ++n) {
    const int row = row0 + 32 * (RG * wave + n) + (lane & 31), i = row / a.heads_per_kv;
    const __half* src = a.q.p + b * a.q.batch + (h * a.heads_per_kv + row - i * a.heads_per_kv) * a.q.head + i * a.q.token + 8 * half;
#pragma unroll
    for (int st = 0; st < 8; ++st) r.q[n][st] = row < rows ? *reinterpret_cast<const half8_t*>(src + 16 * st) : half8_t{};
#pragma unroll
    for (int x = 0; x < 4; ++x) r.o[n][x] = float16_t{};
    r.m[n] = r.raise[n] = -INFINITY;
    r.l[n] = r.zero[n] = 0.f;
  }
  r.far = false;
  const float scale = 0.08838834764831845f * 1.4426950408889634f;

  const bool causal = a.k.p != nullptr;
  const int last_row = (row0 + ROWS < rows ? row0 + ROWS : rows) - 1;
  const int open = s.n - s.packed, plain = open + (causal ? last_row / a.heads_per_kv + 1 : 0);
  const int tiles1 = s.packed / kBlockTile, tiles = tiles1 + (plain + kBlockTile - 1) / kBlockTile;
  const int share = tiles / a.n_splits, more = tiles % a.n_splits;
  const int t0 = split * share + (split < more ? split : more), t1 = t0 + share + (split < more ? 1 : 0);

  const int u1 = t1 < tiles1 ? t1 : tiles1;
  if (t0 < u1) {
    // Where 64 units lie, and their scales: a unit a lane, two such sets (loads run four units ahead of the arithmetic).
    long long at = 0;
    float by = 0.f, add = 0.f, inv = 0.f, shrink = 1.f, largest = 0.f;
    int base = -64;
    auto look = [&](int u) {
      if (u < base + 64 && base >= 0) return;
      base = u;
      const int mine = u + lane < u1 ? u + lane : u1 - 1;
      at = block_tile(a.s, b, h, mine);
      const long long sc = block_scale(a.s, at);
      by = a.s.k.scales[sc] * scale;
      const float vs = a.s.v.scales[sc];
      float most = vs;
#pragma unroll
      for (int i = 32; i > 0; i /= 2) most = fmaxf(most, __shfl_xor(most, i));
      largest = fmaxf(largest, most);
      // S = 2^k vs, at least a sixteenth of the largest (no values but zeros: any)
      const float least = largest > 0.f ? largest * 0.0625f : 1.f;
      float eff = vs;
      shrink = 1.f;
      if (vs < least) {
        const int k = vs > 0.f ? ilogbf(least) - ilogbf(vs) + 1 : 0;
        eff = vs > 0.f ? ldexpf(vs, k) : least;
        shrink = vs > 0.f ? ldexpf(1.f, -k) : 1.f;
      }
      add = __builtin_amdgcn_logf(eff);
      inv = 1.0f / eff;
    };
    auto lane_of = [&](float x, int i) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), i)); };
    const uint32_t k_at = (uint32_t)(64 * wave + lane) * 16, v_at = (uint32_t)(64 * wave + value_lane(lane)) * 16;
    auto fetch = [&](int u, Staged& x, Scales& sc) {
      look(u);
      const int i = u - base;
      const long long tile = (long long)(((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)(at >> 32), i) << 32) |
                                         (unsigned)__builtin_amdgcn_readlane((int)at, i)) * kBlockTileBytes;
      x.a = *reinterpret_cast<const u32x4*>(a.s.k.codes + tile + k_at);
      x.b = *reinterpret_cast<const u32x4*>(a.s.v.codes + tile + v_at);
      sc = Scales{lane_of(by, i), lane_of(add, i), lane_of(inv, i), lane_of(shrink, i)};
    };
    walk<RG, false>(t0, u1, lds, r, lane, fetch, [&](char* buf, const Staged& x, const Scales& sc) { put_packed<E4M3>(buf, wave, lane, x.a, x.b, sc.shrink); },
                    [](int, float16_t (&)[RG]) {});
  }
  if (t1 > tiles1) {
    const long long open_at = (long long)bh * a.s.block * D;
    const __half *ko = a.s.k.open + open_at, *vo = a.s.v.open + open_at;
    const __half *kf = a.k.p + b * a.k.batch + h * a.k.head, *vf = a.v.p + b * a.v.batch + h * a.v.head;
    auto fetch = [&](int u, Staged& x, Scales& sc) {
      sc = Scales{scale, 0.f, 1.f, 1.f};
      const int i0 = u * kBlockTile;
      auto token = [&](int i) { return i0 + i < plain ? i0 + i : plain - 1; };   // (behind the last one: that one again, masked)
      const int i = token(tid >> 3);
      const __half* k = (i < open ? ko + i * D : kf + (i - open) * a.k.token) + 16 * (tid & 7);
      x.a = *reinterpret_cast<const u32x4*>(k);
      x.b = *reinterpret_cast<const u32x4*>(k + 8);
      u32x2 w[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = token(4 * (tid >> 5) + e);
        w[e] = *reinterpret_cast<const u32x2*>((j < open ? vo + j * D : vf + (j - open) * a.v.token) + 4 * (tid & 31));
      }
      x.c = u32x4{w[0].x, w[0].y, w[1].x, w[1].y};
      x.d = u32x4{w[2].x, w[2].y, w[3].x, w[3].y};
    };
    int limit[RG];                                       // last token that the lane's row attends to
#pragma unroll
    for (int n = 0; n < RG; ++n) {
      const int row = row0 + 32 * (RG * wave + n) + (lane & 31);
      limit[n] = causal ? open + (row < rows ? row : rows - 1) / a.heads_per_kv : plain - 1;
    }
    walk<RG, true>(t0 > tiles1 ? t0 - tiles1 : 0, t1 - tiles1, lds, r, lane, fetch, [&](char* buf, const Staged& x, const Scales&) { put_plain(buf, tid, x); },
             [&](int u, float16_t (&sc)[RG]) {
#pragma unroll
               for (int n = 0; n < RG; ++n) {
                 const int left = limit[n] - u * kBlockTile - 4 * half;
                 if (!__builtin_amdgcn_ballot_w64(left < kBlockTile - 1)) continue;
#pragma unroll
                 for (int i = 0; i < 16; ++i)
                   if (8 * (i / 4) + i % 4 > left) sc[n][i] = -INFINITY;
               }
             });
  }

  // results: a lane has channels 32 x + 16 y + 8 half + 2 i + m of its rows, at o[x][4 y + 8 m + i]
#pragma unroll
  for (int n = 0; n < RG; ++n) {
    const float l = r.l[n] + other_half(r.l[n]);
    const int in_block = 32 * (RG * wave + n) + (lane & 31), row = row0 + in_block;
    if (row >= rows) continue;
    if (a.n_splits > 1) {
      const long long slot_row = (((long long)bh * a.row_blocks + row_block) * a.n_splits + split) * ROWS + in_block;
      float* dst = a.ws + a.slots * (ROWS * 2) + slot_row * D + 8 * half;
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          const float16_t& o = r.o[n][x];
          *reinterpret_cast<float4*>(dst + 32 * x + 16 * y) = float4{o[4 * y], o[4 * y + 8], o[4 * y + 1], o[4 * y + 9]};
          *reinterpret_cast<float4*>(dst + 32 * x + 16 * y + 4) = float4{o[4 * y + 2], o[4 * y + 10], o[4 * y + 3], o[4 * y + 11]};
        }
      if (half == 0) *reinterpret_cast<float2*>(a.ws + slot_row * 2) = float2{r.m[n], l};
      continue;
    }
    const float f = l > 0.f ? 1.0f / l : 0.f;            // (no token: zero)
    const int i = row / a.heads_per_kv;
    const long long out = b * a.out_batch + (h * a.heads_per_kv + row - i * a.heads_per_kv) * a.out_head + i * a.out_token + 8 * half;
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const float16_t& o = r.o[n][x];
        const float c[8] = {o[4 * y] * f, o[4 * y + 8] * f, o[4 * y + 1] * f, o[4 * y + 9] * f, o[4 * y + 2] * f, o[4 * y + 10] * f, o[4 * y + 3] * f, o[4 * y + 11] * f};
        if (a.out_is_fp32) {
          float* dst = static_cast<float*>(a.out) + out + 32 * x + 16 * y;
          *reinterpret_cast<float4*>(dst) = float4{c[0], c[1], c[2], c[3]};
          *reinterpret_cast<float4*>(dst + 4) = float4{c[4], c[5], c[6], c[7]};
        } else {
          half8_t w;
#pragma unroll
          for (int e = 0; e < 8; ++e) w[e] = (_Float16)c[e];
          *reinterpret_cast<half8_t*>(static_cast<_Float16*>(a.out) + out + 32 * x + 16 * y) = w;
        }
      }
  }
}

}  // namespace

hipError_t launch_block_rows(const BlockAttnArgs& a, bool e4m3, int group_rows, hipStream_t stream) {
  const long long groups = (long long)a.s.batch * a.s.n_kv_heads * a.row_blocks * a.n_splits;
  if (groups >= (1LL << 31)) return hipErrorInvalidValue;
  if (group_rows == 128) {
    if (e4m3) block_rows_kernel<true, 1><<<(unsigned)groups, 256, 0, stream>>>(a);
    else block_rows_kernel<false, 1><<<(unsigned)groups, 256, 0, stream>>>(a);
  } else if (group_rows == 256) {
    if (e4m3) block_rows_kernel<true, 2><<<(unsigned)groups, 256, 0, stream>>>(a);
    else block_rows_kernel<false, 2><<<(unsigned)groups, 256, 0, stream>>>(a);
  } else {
    return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace innerq
