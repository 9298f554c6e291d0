// Rotary positions of rows where they lie, and appends of any number of new tokens a sequence with the keys rotated on their way
// into the cache.
//
// This translation unit is compiled with -ffp-contract=off: rotated values, codes and flags depend on every fp32 rounding.
//
// Both are bound by memory where there is much to do and by latency where there is little.  A rotation reads and writes a row once
// (512 bytes a token and head); an append reads the new rows once (512 bytes a token and kv head) and writes them packed (96 bytes
// at 2 bits, groups of 32), so rotating beforehand would almost double the keys' traffic.  Calls, least time by bytes at the rate of a copy
// in brackets: rotation of 40 heads x 32k tokens 150 us (139); append of 4 x 8 heads x 32k tokens at 2 bits, keys rotated, 171 to 180 us (144);
// rotation of 8 x 40 heads, one token, 3.2 us in the kernel; a step of 32 x 8 heads 5.1, and 1.7 for the counts.
#include "quantize_rows.h"
#include "rotate.h"

namespace innerq {
namespace {

// ---- rotation: a thread holds the cosines and sines of one unit of one token and takes it through a range of heads.

constexpr int kRotateHeads = 4;                          // in flight a thread
__global__ void __launch_bounds__(256) rotate_kernel(RotateArgs a) {
  const long long idx = (long long)blockIdx.x * blockDim.x + threadIdx.x;
  const int u = (int)(idx % kUnits);
  const long long bt = idx / kUnits;
  if (bt >= (long long)a.batch * a.t_new) return;
  const int b = (int)div32(bt, a.t_new), t = (int)(bt - (long long)b * a.t_new);
  if (a.t_dev && t >= a.t_dev[b]) return;
  Turn turn;
  // (a count from the device may be anything: the sum saturates, so that a place beyond 32 bits is the table's last)
  load_turn(turn, a.rot, bt, a.rot.positions ? 0 : __builtin_elementwise_add_sat(a.n_dev ? a.n_dev[b] : a.n_tokens, t), u);
  const UnitChunks ch = unit_chunks(a.rot, u);
  const __half* x = a.x.p + b * a.x.batch + t * a.x.token;
  __half* y = a.y + b * a.y_batch + t * a.y_token;
  const int h0 = (int)blockIdx.y * a.heads_per_block, h1 = h0 + a.heads_per_block < a.n_heads ? h0 + a.heads_per_block : a.n_heads;
  for (int h = h0; h < h1; h += kRotateHeads) {
    uint4 p[kRotateHeads], q[kRotateHeads];
#pragma unroll
    for (int i = 0; i < kRotateHeads; ++i) {
      const __half* row = x + (h + i < h1 ? h + i : h) * a.x.head;
      p[i] = *reinterpret_cast<const uint4*>(row + ch.a);
      q[i] = *reinterpret_cast<const uint4*>(row + ch.b);
    }
#pragma unroll
    for (int i = 0; i < kRotateHeads; ++i) {
      if (h + i >= h1) break;
      turn_unit(turn, a.rot, u, p[i], q[i]);
      __half* row = y + (h + i) * a.y_head;
      *reinterpret_cast<uint4*>(row + ch.a) = p[i];
      *reinterpret_cast<uint4*>(row + ch.b) = q[i];
    }
  }
}

// ---- appends

// A sequence's state: n cached tokens, t new ones, the store filled for a cache of `to` tokens.  Counts from the device are
// clamped into the cache; a sequence whose cached count is none takes nothing.
struct SeqState { int n, t, to; };
__device__ __forceinline__ SeqState sequence_state(const AppendArgs& a, int b) {
  const int cap = (int)a.q.capacity;
  int n = (int)a.q.n_old, t = a.t_new;
  if (a.q.n_dev) {
    const int count = a.q.n_dev[b];
    n = count < 0 ? 0 : count > cap ? cap : count;
    t = a.t_dev[b];
    t = t < 0 || n != count ? 0 : t > a.t_new ? a.t_new : t;
  }
  t = t < cap - n ? t : cap - n;
  return {n, t, n + t + a.ahead < cap ? n + t + a.ahead : cap};
}
__device__ __forceinline__ int rows_of(const AppendArgs& a, int form, int n) {
  return (int)quantised_rows(a.q.w_sink, a.q.w_recent, a.q.group, form, n);
}

__device__ __forceinline__ void scale_chunk(uint4& x, const float* inv) {
  __half* h = reinterpret_cast<__half*>(&x);
#pragma unroll
  for (int e = 0; e < 8; ++e) h[e] = scaled_half(h2f(h[e]), inv[e]);
}

// The two chunks of a unit of new token i of kv head h.
__device__ __forceinline__ void load_new_unit(const RowView& x, int b, int h, int i, const UnitChunks& ch, uint4& p, uint4& q) {
  const __half* row = x.p + b * x.batch + h * x.head + i * x.token;
  p = *reinterpret_cast<const uint4*>(row + ch.a);
  q = *reinterpret_cast<const uint4*>(row + ch.b);
}
__device__ __forceinline__ void finish_key_unit(const AppendArgs& a, const Turn& turn, int h, int u, const UnitChunks& ch, uint4& p, uint4& q) {
  if (a.rot.cos) turn_unit(turn, a.rot, u, p, q);
  if (a.q.inv_norm) {
    const float* inv = a.q.inv_norm + h * kHeadDim;
    scale_chunk(p, inv + ch.a);
    scale_chunk(q, inv + ch.b);
  }
}

// The new tokens that stay in a window: token k of the first ones (sink) or of those from ring_from on, and where it goes.
__device__ __forceinline__ void copy_unit(const AppendArgs& a, int y, int b, int h, int k, int u, const SeqState& s) {
  const QuantTensorJob& kj = a.q.job[0];
  const QuantTensorJob& vj = a.q.job[1];
  const int form = y ? vj.form : kj.form, slots = y ? vj.slots : kj.slots;
  int n_a = a.q.w_sink - s.n;
  n_a = n_a < 0 ? 0 : n_a > s.t ? s.t : n_a;
  int i_b = a.q.w_sink + rows_of(a, form, s.n + s.t) - s.n;
  i_b = i_b < n_a ? n_a : i_b > s.t ? s.t : i_b;
  const int i = k < n_a ? k : i_b + (k - n_a);
  if (i >= s.t) return;
  const int token = s.n + i;
  const long long bh = (long long)b * a.q.n_kv_heads + h;
  __half* sink = y ? vj.sink : kj.sink;
  __half* ring = y ? vj.ring : kj.ring;
  __half* dst = token < a.q.w_sink ? sink + (bh * a.q.w_sink + token) * kHeadDim : ring + (bh * slots + mod32(token, slots)) * kHeadDim;
  uint4 p, q;
  UnitChunks ch = {16 * u, 16 * u + 8};
  if (y) {
    load_new_unit(a.v, b, h, i, ch, p, q);
  } else {
    Turn turn;
    if (a.rot.cos) {
      ch = unit_chunks(a.rot, u);
      load_turn(turn, a.rot, (long long)b * a.t_new + i, token, u);
    }
    load_new_unit(a.k, b, h, i, ch, p, q);
    finish_key_unit(a, turn, h, u, ch, p, q);
  }
  *reinterpret_cast<uint4*>(dst + ch.a) = p;
  *reinterpret_cast<uint4*>(dst + ch.b) = q;
}

// per_seq: most window copies of a sequence
__device__ __forceinline__ void copy_rows(const AppendArgs& a, int y, long long idx, int per_seq) {
  const int u = (int)(idx % kUnits);
  const uint32_t row = (uint32_t)(idx / kUnits), H = (uint32_t)a.q.n_kv_heads;
  const uint32_t bk = row / H, b = bk / (uint32_t)per_seq;
  if (b >= (uint32_t)a.q.batch) return;
  copy_unit(a, y, (int)b, (int)(row % H), (int)(bk - b * (uint32_t)per_seq), u, sequence_state(a, (int)b));
}

__global__ void __launch_bounds__(256) append_copies_kernel(AppendArgs a, int per_seq) {
  copy_rows(a, (int)blockIdx.y, (long long)blockIdx.x * 256 + threadIdx.x, per_seq);
}

__global__ void __launch_bounds__(256) advance_counts_kernel(AppendArgs a, int* counts) {
  const int b = (int)(blockIdx.x * 256 + threadIdx.x);
  if (b >= a.q.batch) return;
  const int t = sequence_state(a, b).t;
  if (t > 0) counts[b] += t;
}

// A step: one new token a sequence, everything that leaves a ring was there before.  Groups spread over eight lanes (the chain of a
// group in one lane is the longest of a short launch), the copies in the same launch: a ring has a spare slot for the token that
// enters.  rows, groups: key rows and value groups that a sequence can lose.
template <int G>
__global__ void __launch_bounds__(256) append_step_kernel(AppendArgs a, int rows, int groups, unsigned quant_blocks, int per_seq) {
  const int y = (int)blockIdx.y;
  if (blockIdx.x >= quant_blocks) {
    copy_rows(a, y, (long long)(blockIdx.x - quant_blocks) * 256 + threadIdx.x, per_seq);
    return;
  }
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  const QuantTensorJob j = pick_job(a.q, y);
  const int sub = (int)(idx % 8);
  if (y == 0) {
    constexpr int GPR = kHeadDim / G;
    const long long unit = idx / 8 / GPR;
    const int g = (int)(idx / 8 % GPR);
    const uint32_t bh = div32(unit, rows), i = (uint32_t)unit - bh * (uint32_t)rows;
    if (bh >= (uint32_t)(a.q.batch * a.q.n_kv_heads)) return;
    const SeqState s = sequence_state(a, (int)(bh / (uint32_t)a.q.n_kv_heads));
    const int row = rows_of(a, kPerToken, s.n) + (int)i;
    if (row >= rows_of(a, kPerToken, s.to)) return;
    const __half* token = j.ring + ((long long)bh * j.slots + mod32(a.q.w_sink + row, j.slots)) * kHeadDim;
    if (j.bits == 2) per_token_group_lanes<G, 2>(a.q, j, bh, row, g, sub, token, false);
    else if (j.bits == 3) per_token_group_lanes<G, 3>(a.q, j, bh, row, g, sub, token, false);
    else per_token_group_lanes<G, 4>(a.q, j, bh, row, g, sub, token, false);
  } else {
    const int c = (int)(idx / 8 % kHeadDim);
    const long long unit = idx / 8 / kHeadDim;
    const uint32_t bh = div32(unit, groups), i = (uint32_t)unit - bh * (uint32_t)groups;
    if (bh >= (uint32_t)(a.q.batch * a.q.n_kv_heads)) return;
    const SeqState s = sequence_state(a, (int)(bh / (uint32_t)a.q.n_kv_heads));
    const int tg = rows_of(a, kPerChannel, s.n) / G + (int)i;
    if (tg * G >= rows_of(a, kPerChannel, s.to)) return;
    if (j.bits == 2) per_channel_group_lanes<G, 2>(a.q, j, bh, tg, c, sub, s.n);
    else if (j.bits == 3) per_channel_group_lanes<G, 3>(a.q, j, bh, tg, c, sub, s.n);
    else per_channel_group_lanes<G, 4>(a.q, j, bh, tg, c, sub, s.n);
  }
}

// Chunks and prompts, keys: a work-group takes 32 store rows of one sequence through a range of kv heads, two at a turn (groups of 64:
// four), so that every lane has a group.  A thread holds the cosines and sines of one unit of one token in registers for all heads; rotated
// rows meet in LDS, where a lane finds a whole group (a group's rotation partners are anywhere in the row): two buffers and one barrier a
// turn, or (groups of 64, whose rows would leave room for two work-groups a compute unit) one buffer and two.
constexpr int kTileRows = 32;
constexpr int kTilePitch = kHeadDim + 8;                 // halfs: rows 16 bytes apart in the banks
template <int G>
using KeyTile = __half[G == 32 ? 2 : 1][G / 16][kTileRows][kTilePitch];

template <int G, int BITS, bool FAST>
__device__ __forceinline__ void append_keys(const AppendArgs& a, const QuantTensorJob& j, KeyTile<G>& tile, int tiles, int head_blocks, int heads) {
  constexpr int HS = G / 16;                             // heads a turn
  const uint32_t bt = blockIdx.x / (uint32_t)head_blocks, hb = blockIdx.x - bt * (uint32_t)head_blocks;
  const int b = (int)(bt / (uint32_t)tiles), tl = (int)(bt - (uint32_t)b * (uint32_t)tiles);
  if (b >= a.q.batch) return;
  const SeqState s = sequence_state(a, b);
  const int r0 = rows_of(a, kPerToken, s.n) + tl * kTileRows, r1 = rows_of(a, kPerToken, s.to);
  if (r0 >= r1) return;                                  // (uniform)
  const int h0 = (int)hb * heads, h1 = h0 + heads < a.q.n_kv_heads ? h0 + heads : a.q.n_kv_heads;
  const int tid = (int)threadIdx.x, u = tid % kUnits, row = tid / kUnits;
  // (behind the last row: that one again, and nothing comes of it)
  const int i = a.q.w_sink + (r0 + row < r1 ? r0 + row : r1 - 1) - s.n;      // index among the new tokens; negative: in the ring
  Turn turn;
  UnitChunks ch = {16 * u, 16 * u + 8};
  if (a.rot.cos) {
    ch = unit_chunks(a.rot, u);
    if (i >= 0) load_turn(turn, a.rot, (long long)b * a.t_new + i, s.n + i, u);
  }
  const __half* src = i >= 0 ? a.k.p + b * a.k.batch + i * a.k.token : j.ring + ((long long)b * a.q.n_kv_heads * j.slots + mod32(s.n + i, j.slots)) * kHeadDim;
  const long long head = i >= 0 ? a.k.head : (long long)j.slots * kHeadDim;
  int buf = 0;
  for (int h = h0; h < h1; h += HS) {
    uint4 p[HS], q[HS];
#pragma unroll
    for (int x = 0; x < HS; ++x) {
      const __half* at = src + (h + x < h1 ? h + x : h1 - 1) * head;
      p[x] = *reinterpret_cast<const uint4*>(at + ch.a);
      q[x] = *reinterpret_cast<const uint4*>(at + ch.b);
    }
#pragma unroll
    for (int x = 0; x < HS; ++x) {
      if (i >= 0) finish_key_unit(a, turn, h + x < h1 ? h + x : h1 - 1, u, ch, p[x], q[x]);
      *reinterpret_cast<uint4*>(tile[buf][x][row] + ch.a) = p[x];
      *reinterpret_cast<uint4*>(tile[buf][x][row] + ch.b) = q[x];
    }
    __syncthreads();
    constexpr int GPR = kHeadDim / G;
    const int x = tid / (kTileRows * GPR), r = tid / GPR % kTileRows, g = tid % GPR;
    if (h + x < h1 && r0 + r < r1) {
      const long long bh = (long long)b * a.q.n_kv_heads + h + x;
      per_token_group<G, BITS, FAST>(a.q, j, tile[buf][x][r] + g * G, false, (uint32_t)bh, (uint32_t)g,
                                     store_row(a.q.pages, a.q.n_kv_heads, a.q.capacity, bh, r0 + r), 0u);
    }
    if (G == 32) buf ^= 1;
    else __syncthreads();
  }
}

// Values: a lane per channel and token group, heads next to each other (they are next to each other in a projection's output).
template <int G, int BITS, bool FAST>
__device__ __forceinline__ void append_values(const AppendArgs& a, const QuantTensorJob& j, int groups) {
  constexpr int W = G * BITS / 32;
  const long long idx = (long long)blockIdx.x * 256 + threadIdx.x;
  const int c = (int)(idx % kHeadDim);
  const uint32_t unit = (uint32_t)(idx / kHeadDim), H = (uint32_t)a.q.n_kv_heads;
  const uint32_t h = unit % H, bg = unit / H, b = bg / (uint32_t)groups;
  if (b >= (uint32_t)a.q.batch) return;
  const SeqState s = sequence_state(a, (int)b);
  const int tg = rows_of(a, kPerChannel, s.n) / G + (int)(bg - b * (uint32_t)groups);
  if (tg * G >= rows_of(a, kPerChannel, s.to)) return;
  const int first = a.q.w_sink + tg * G - s.n;           // index of the group's first token among the new ones
  const long long bh = (long long)b * H + h;
  const __half* fresh = a.v.p + b * a.v.batch + h * a.v.head + c;
  uint32_t x[G];                                         // a value each, in the low half
  if (first >= 0) {
    const __half* src = fresh + first * a.v.token;
#pragma unroll
    for (int i = 0; i < G; ++i) x[i] = __half_as_ushort(src[i * a.v.token]);
  } else {
    const __half* ring = j.ring + bh * j.slots * kHeadDim + c;
    uint32_t slot = mod32(a.q.w_sink + tg * G, j.slots);
#pragma unroll
    for (int i = 0; i < G; ++i) {
      x[i] = __half_as_ushort(*(first + i >= 0 ? fresh + (first + i) * a.v.token : ring + slot * kHeadDim));
      slot = slot + 1u == (uint32_t)j.slots ? 0u : slot + 1u;
    }
  }
  uint32_t mn, mx, words[W];
  pair_range(x, mn, mx);
  __half sc, z;
  quantize_group_bulk<G, BITS, FAST>([&](int i) { return HalfRef{x[i], false}; }, NoDistances{}, half_lo(mn), half_lo(mx), j.mode,
                                     a.q.sym_den_literal, words, sc, z);
  const long long go = (store_row(a.q.pages, a.q.n_kv_heads, a.q.capacity, bh, (long long)tg * G) / G) * kHeadDim + c;
  uint32_t* dst = reinterpret_cast<uint32_t*>(j.codes) + go * W;
#pragma unroll
  for (int i = 0; i < W; ++i) dst[i] = words[i];
  j.scales[go] = sc;
  if (j.zeros) j.zeros[go] = z;
}

struct ChunkPlan {
  int tiles, head_blocks, heads;       // keys: tiles a sequence, blocks of heads, heads of a block
  int groups;                          // value groups a sequence
  int per_seq;                         // most window copies of a sequence
};
// Wavefronts a SIMD that the registers are made to fit: groups of 32 get four (LDS allows no more, as the compiler warns), but the code made for
// five is the faster by 1 to 2 % (4 x 8 heads x 32k tokens, in turn in one session: 183 us, 185 with four asked for).
template <int G, bool FAST>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(G == 32 ? 5 : 3))) append_chunk_kernel(AppendArgs a, ChunkPlan plan) {
  __shared__ __align__(16) KeyTile<G> tile;
  const int y = (int)blockIdx.y;
  const QuantTensorJob j = pick_job(a.q, y & 1);
  if (y >= 2) {
    copy_rows(a, y - 2, (long long)blockIdx.x * 256 + threadIdx.x, plan.per_seq);
  } else if (y == 0) {
    if (j.bits == 2) append_keys<G, 2, FAST>(a, j, tile, plan.tiles, plan.head_blocks, plan.heads);
    else if (j.bits == 3) append_keys<G, 3, false>(a, j, tile, plan.tiles, plan.head_blocks, plan.heads);
    else append_keys<G, 4, FAST && G == 64>(a, j, tile, plan.tiles, plan.head_blocks, plan.heads);
  } else {
    if (j.bits == 2) append_values<G, 2, FAST>(a, j, plan.groups);
    else if (j.bits == 3) append_values<G, 3, false>(a, j, plan.groups);
    else append_values<G, 4, FAST && G == 64>(a, j, plan.groups);
  }
}

inline long long div_up(long long a, long long b) { return (a + b - 1) / b; }

// Most window copies of a sequence that brings t tokens.
long long copies_of(const AppendArgs& a) {
  const long long most = (long long)a.q.w_sink + a.q.w_recent + a.q.group - 1;
  return a.t_new < most ? a.t_new : most;
}

template <int G>
hipError_t launch_append(const AppendArgs& a, hipStream_t stream) {
  const long long B = a.q.batch, H = a.q.n_kv_heads, moved = (long long)a.t_new + a.ahead;
  // what a sequence can lose at most: exact where the host knows its count
  long long rows = moved, groups = div_up(moved, G);
  if (!a.q.n_dev) {
    const long long to = a.q.n_old + moved < a.q.capacity ? a.q.n_old + moved : a.q.capacity;
    auto gone = [&](int form) {
      return quantised_rows(a.q.w_sink, a.q.w_recent, G, form, to) - quantised_rows(a.q.w_sink, a.q.w_recent, G, form, a.q.n_old);
    };
    rows = gone(kPerToken);
    groups = gone(kPerChannel) / G;
  }
  const long long per_seq = copies_of(a), copy_blocks = div_up(B * H * per_seq * kUnits, 256);
  if (B * H * per_seq >= (1LL << 32) || B * H * groups >= (1LL << 32) || B * H * rows >= (1LL << 32)) return hipErrorInvalidValue;
  if (a.t_new == 1 && moved <= a.q.w_recent) {
    const long long kthreads = B * H * rows * (kHeadDim / G) * 8, vthreads = B * H * groups * kHeadDim * 8;
    const long long quant = div_up(kthreads > vthreads ? kthreads : vthreads, 256);
    if (quant + copy_blocks >= (1LL << 31)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)(quant + copy_blocks), 2);
    append_step_kernel<G><<<grid, 256, 0, stream>>>(a, (int)(rows ? rows : 1), (int)(groups ? groups : 1), (unsigned)quant, (int)per_seq);
    return hipGetLastError();
  }
  // one launch where no new token enters a ring slot that the call still reads
  auto apart = [&](int form, int slots, long long gone) {
    const long long oldest = a.q.w_sink + quantised_rows(a.q.w_sink, a.q.w_recent, G, form, a.q.n_old);
    return gone == 0 || oldest >= a.q.n_old || a.q.n_old + a.t_new - oldest <= slots;
  };
  const bool together = !a.q.n_dev && apart(kPerToken, a.q.job[0].slots, rows) && apart(kPerChannel, a.q.job[1].slots, groups);
  if (rows > 0 || groups > 0) {
    ChunkPlan p;
    p.tiles = (int)div_up(rows > 0 ? rows : 1, kTileRows);
    // as many heads a work-group as leave four work-groups a compute unit
    long long heads = B * p.tiles * H / (4LL * compute_units());
    heads = heads < 1 ? 1 : heads > H ? H : heads;
    heads = div_up(heads, G / 16) * (G / 16);             // (whole turns)
    p.heads = (int)heads;
    p.head_blocks = (int)div_up(H, heads);
    p.groups = (int)(groups ? groups : 1);
    p.per_seq = (int)per_seq;
    long long x = rows > 0 ? B * p.tiles * p.head_blocks : 0;
    const long long vx = div_up(B * H * groups * kHeadDim, 256);
    x = vx > x ? vx : x;
    if (together) x = copy_blocks > x ? copy_blocks : x;
    if (x >= (1LL << 31)) return hipErrorInvalidValue;
    const dim3 grid((unsigned)x, together ? 4 : 2);
    // the shorter error sum from 2 M groups on, as for ordinary appends
    const bool fast = B * H * rows * (kHeadDim / G) >= (1LL << 21);
    if (fast) append_chunk_kernel<G, true><<<grid, 256, 0, stream>>>(a, p);
    else append_chunk_kernel<G, false><<<grid, 256, 0, stream>>>(a, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || together) return e;
  }
  append_copies_kernel<<<dim3((unsigned)copy_blocks, 2), 256, 0, stream>>>(a, (int)per_seq);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_rotate(const RotateArgs& args, hipStream_t stream) {
  RotateArgs a = args;
  const long long blocks = div_up((long long)a.batch * a.t_new * kUnits, 256);
  // ranges of heads: enough work-groups for the chip, in whole rounds of loads
  long long heads = blocks * a.n_heads / (16LL * compute_units());
  heads = div_up(heads < 1 ? 1 : heads, kRotateHeads) * kRotateHeads;
  if (blocks < 2LL * compute_units()) heads = 1;
  a.heads_per_block = (int)(heads < a.n_heads ? heads : a.n_heads);
  const long long ranges = div_up(a.n_heads, a.heads_per_block);
  if (blocks >= (1LL << 31) || ranges > 65535) return hipErrorInvalidValue;
  rotate_kernel<<<dim3((unsigned)blocks, (unsigned)ranges), 256, 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_append_rows(const AppendArgs& a, int* counts, hipStream_t stream) {
  hipError_t e = a.q.group == 32 ? launch_append<32>(a, stream) : launch_append<64>(a, stream);
  if (e != hipSuccess || !counts) return e;
  advance_counts_kernel<<<(unsigned)div_up(a.q.batch, 256), 256, 0, stream>>>(a, counts);
  return hipGetLastError();
}

}  // namespace innerq
