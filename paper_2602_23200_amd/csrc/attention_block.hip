// Attention over the cache in 8 bits with block scales: one or a few new tokens of a sequence, and cross attention.
//
// A row is a query head of a new token; the rows of a kv head share its keys and values.  A wavefront takes tiles of 32 tokens:
//   S^T = K Q^T   (16 x 16 x 32 instructions: rows are tokens, columns query rows)
//   O^T = V^T P^T (rows are channels)
// The store holds the codes in the order of these operands, so that a wavefront's loads are whole kilobytes, go from memory to registers and
// are used where they stand: a lane's scores are those of four tokens of either half of the tile and of one query row, which
// is what the second product wants of it as an operand.  Nothing passes through LDS but the wavefronts' results.
//
// Codes become fp16 exactly (8-bit integers: put under the exponent that gives the last bit weight one, the bias subtracted; E4M3: the
// conversion instruction); scales are taken as block_math.h says.  Up to 32 rows weights enter the second product as two fp16 pieces (22 bits), so
// the result is that of fp32 arithmetic on the values the cache stands for, and the kernel still waits for memory; for 64 rows that would cost
// (8 sequences of 32k tokens, 48 rows: 133 us, with one piece 110), and weights are rounded to fp16 as they are for more rows.
//
// The softmax reference level is put 2^10 below the score that raises it and raised again only when a score passes it by 2^15.9, so outputs
// are scaled rarely; the statistics of a row are shared by its four lanes only then.
//
// What bounds it is the read of the cache: 8 sequences of 8 kv heads over 32k tokens, 538 MB, take 82 us for one token (6.5 TB/s; a copy of 2 GiB reaches 4.95
// read and written), 96 for five (5.6), and 18 us for cross attention of 32 sequences over 67 MB; one token over 500 is the launch and a chain of loads (7.4).
#include "block_few.h"

namespace innerq {
namespace {

using namespace block_few;

template <bool E4M3, int NR>
__global__ void __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(NR == 4 ? 1 : 2))) block_attention_kernel(BlockAttnArgs a) {
  __shared__ float lds[kFloats<NR>];
  BlockWork work;
  bool listed = false;
  if constexpr (NR <= 2) {                               // (lists have work-groups of 16 or 32 rows)
    listed = a.table != nullptr;
    if (listed && !find_work<16 * NR, W>(a, 0, a.few_most, (int)blockIdx.x, work)) return;      // (uniform)
  }
  if (!listed) work = uniform_work(a);
  attend<E4M3, NR>(a, work, lds, a.ws, a.slots);
}

// The splits of a row joined: half a wavefront a row, a lane four channels, eight splits under way (only those that are there: with the last one read again in
// place of the others, of a ragged batch with one to four, 15 us, now 11).  The launch is bounded, and its work-groups walk over the rows: of a padded
// batch most rows are not there, and starting work-groups for them cost more than the joining (16 sequences of 2 to 256 new tokens 183 us with a
// work-group for every eight rows, 177 with 4096 at most, 174 with 2048).  What bounds it is memory: three partial results of 9600 rows x 4 sequences
// (60 MB) 15 us; of few rows the launch (4 us).
constexpr int kMergeRows = 8;                            // of a work-group at once
constexpr int kMergeGroups = 2048;                       // of a launch where rows are many
__global__ void __launch_bounds__(256) block_merge_kernel(BlockAttnArgs a, int blocks, int group_rows) {
  const int bh = (int)(blockIdx.x / (unsigned)blocks), first = (int)(blockIdx.x % (unsigned)blocks) * kMergeRows;
  const int b = bh / a.s.n_kv_heads, h = bh % a.s.n_kv_heads, channel = 4 * ((int)threadIdx.x & 31);
  const int own = block_seq(a, b).t * a.heads_per_kv;
  if (first >= own) return;
  int n_splits = a.n_splits, step = 1;                   // slots from one split to the next
  const float* ws = a.ws;
  long long slots = a.slots, slot;                       // the first one's of the first rows
  int row_step;                                          // .. and from one block of rows to the next
  if (a.table) {
    n_splits = __builtin_amdgcn_readfirstlane(a.table[2 * b + 1]);
    if (n_splits == 1) return;                           // (written already)
    if (own <= a.few_most) {
      group_rows = a.few_rows;
      ws = a.ws_few;
      slots = a.few_slots;
    }
    step = (own + group_rows - 1) / group_rows;
    slot = a.table[2 * b] + (long long)h * step * n_splits;
    row_step = 1;
  } else {
    slot = (long long)bh * a.row_blocks * n_splits;
    row_step = n_splits;
  }
  for (int row = first + ((int)threadIdx.x >> 5); row < own; row += blocks * kMergeRows) {
    const long long at = (slot + (long long)(row / group_rows) * row_step) * group_rows + row % group_rows;
    const float *ml = ws + at * 2, *po = ws + slots * (group_rows * 2) + at * D + channel;
    const long long step_ml = (long long)step * group_rows * 2, step_o = (long long)step * group_rows * D;
    float level = -INFINITY, den = 0.f;
    float4_t o = {};
    for (int p0 = 0; p0 < n_splits; p0 += 8) {
      float2 st[8];
      float4_t v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        st[e] = float2{-INFINITY, 0.f};
        v[e] = float4_t{};
        if (p0 + e < n_splits) {                         // (uniform)
          st[e] = *reinterpret_cast<const float2*>(ml + (p0 + e) * step_ml);
          v[e] = *reinterpret_cast<const float4_t*>(po + (p0 + e) * step_o);
        }
      }
      float top = level;
#pragma unroll
      for (int e = 0; e < 8; ++e) top = fmaxf(top, st[e].x);
      const float old = level == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(level - top);
      den *= old;
      o *= old;
      level = top;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float f = st[e].x == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(st[e].x - top);
        den = __builtin_fmaf(f, st[e].y, den);
#pragma unroll
        for (int i = 0; i < 4; ++i) o[i] = __builtin_fmaf(f, v[e][i], o[i]);
      }
    }
    const float inv = den > 0.f ? 1.0f / den : 0.f;
    const int i = row / a.heads_per_kv;
    const long long out = b * a.out_batch + (h * a.heads_per_kv + row - i * a.heads_per_kv) * a.out_head + i * a.out_token + channel;
    store_four(a, out, o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
  }
}

template <bool E4M3, int NR>
hipError_t launch_form(const BlockAttnArgs& a, hipStream_t stream) {
  const long long groups = a.table ? a.list_few : (long long)a.s.batch * a.s.n_kv_heads * a.row_blocks * a.n_splits;
  if (groups >= (1LL << 31)) return hipErrorInvalidValue;
  block_attention_kernel<E4M3, NR><<<(unsigned)groups, 64 * W, 0, stream>>>(a);
  return hipGetLastError();
}
template <bool E4M3>
hipError_t launch_rows(const BlockAttnArgs& a, const BlockForm& form, hipStream_t stream) {
  switch (form.rows) {
    case 16: return launch_form<E4M3, 1>(a, stream);
    case 32: return launch_form<E4M3, 2>(a, stream);
    case 64: return a.table ? hipErrorInvalidValue : launch_form<E4M3, 4>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

hipError_t launch_block_attention(const BlockAttnArgs& a, bool e4m3, const BlockForm& form, hipStream_t stream) {
  return e4m3 ? launch_rows<true>(a, form, stream) : launch_rows<false>(a, form, stream);
}

hipError_t launch_block_merge(const BlockAttnArgs& a, const BlockForm& form, hipStream_t stream) {
  const long long heads = (long long)a.s.batch * a.s.n_kv_heads, most = ceil_div((long long)a.s.t_new * a.heads_per_kv, kMergeRows);
  const long long even = ceil_div(kMergeGroups, heads), blocks = most < even ? most : even, all = heads * blocks;
  if (all >= (1LL << 31)) return hipErrorInvalidValue;
  block_merge_kernel<<<(unsigned)all, 256, 0, stream>>>(a, (int)blocks, form.rows);
  return hipGetLastError();
}

}  // namespace innerq
