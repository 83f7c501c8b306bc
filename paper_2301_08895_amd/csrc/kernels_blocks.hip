// Rounds of the MLP whose hidden layers are residual blocks (abs_create_blocks):
//   a_1 = x W_0 + b_0,   u_l = dropout(act(group norm(a_l; gamma_l, beta_l))),
//   a_{l+1} = u_l W_l + b_l (+ a_l where the widths agree),   logits = a_L,   softmax cross-entropy.
// A round is a chain of the library's own operators over the stacked minibatches, layer by layer; within a layer one
// call per model version that the round's uploads computed at (their rows are contiguous: the descriptor lists them grouped by
// version).  Activations and gradients of activations are bf16, the matrix cores' operands; the models of the ring, the logits, the sums and the update are
// fp32, each version's matrices are narrowed to bf16 once.  The gradient of a version's matrix (coefficients of Eq. 3 in it) goes from
// the shares of its product, in fp32, into the fp32 model, oldest version first.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "kernels.h"
#include "operators.h"

namespace abs_impl {
namespace {

size_t up(size_t x, size_t m) { return (x + m - 1) / m * m; }

// The minibatch rows of all uploads, gathered; their labels.  A workgroup per row.
__global__ __launch_bounds__(128) void blocks_gather_kernel(const uint16_t* X, const int32_t* y, int d0, uint64_t shard_rows, uint64_t batch_key,
                                                            int B, RoundDesc rd, uint16_t* out, int32_t* label) {
  const int m = blockIdx.x, up = m / B, b = m - up * B;
  const WorkerDesc w = rd.w[up];
  const uint64_t row = (uint64_t)w.id * shard_rows + draw(job_key(batch_key, w.id, w.job), (uint32_t)b) % shard_rows;
  const Loose<uint16_t, 8>* const src = (const Loose<uint16_t, 8>*)(X + row * (uint64_t)d0);
  Loose<uint16_t, 8>* const dst = (Loose<uint16_t, 8>*)(out + (size_t)m * d0);
  for (int c = threadIdx.x; c < d0 / 8; c += 128) dst[c] = src[c];
  if (threadIdx.x == 0) label[m] = y[row];
}

// A wavefront per row of logits, C <= 256, which arrive in fp32 as the shares of the output layer's product: loss, and either the gradient
// c_k (p - 1_y) or whether the first largest logit is the label.  Rows m of one model version; row0: the stack's rows before them.
__global__ __launch_bounds__(256) void blocks_loss_kernel(OpShares z, const float* bias, int C, int rows, const int32_t* label, int row0, int B, RoundDesc rd,
                                                          float* rowloss, uint16_t* dz, float* correct) {
  const int lane = threadIdx.x & 63, m = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (m >= rows) return;
  const int lab = label[m];
  float v[4], top = -INFINITY;
  int best = 0;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = lane + 64 * q;
    v[q] = -INFINITY;
    if (c < C) {
      const float* const p = z.part + m * z.ld + c;
      float s = p[0];
#pragma unroll 4
      for (int k = 1; k < z.shares; ++k) s += p[k * z.stride];
      v[q] = s + bias[c];
    }
    if (v[q] > top || v[q] != v[q]) { top = v[q]; best = c; }       // (a NaN stays on top: the loss is NaN)
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {                                 // largest logit, lowest class among equals
    const float ov = __shfl_xor(top, o);
    const int ob = __shfl_xor(best, o);
    if (ov > top || ov != ov || (ov == top && ob < best)) { top = ov; best = ob; }
  }
  float sum = 0.f, at = 0.f;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = lane + 64 * q;
    if (c == lab) at = v[q] - top;
    v[q] = c < C ? expf(v[q] - top) : 0.f;
    sum += v[q];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) { sum += __shfl_xor(sum, o); at += __shfl_xor(at, o); }
  if (lane == 0) {
    rowloss[m] = logf(sum) - at;
    if (correct) correct[m] = best == lab ? 1.f : 0.f;
  }
  if (!dz) return;
  const float coef = rd.w[(row0 + m) / B].c, inv = 1.0f / sum;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int c = lane + 64 * q;
    if (c < C) dz[(size_t)m * C + c] = op_bf16(coef * (v[q] * inv - (c == lab ? 1.f : 0.f)));
  }
}

// The uploads' mean losses, rows added in order, to the mailbox.
__global__ __launch_bounds__(128) void blocks_publish_kernel(const float* rowloss, int B, int K, LossMailbox* box, uint32_t stamp) {
  const int k = threadIdx.x;
  if (k >= K) return;
  float s = 0.f;
  for (int b = 0; b < B; ++b) s += rowloss[(size_t)k * B + b];
  post_loss(box, k, s / (float)B, stamp);
}

// next = from - change
__global__ __launch_bounds__(256) void blocks_step_kernel(float* next, const float* from, const float* change, size_t n) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (size_t)gridDim.x * 256) next[i] = from[i] - change[i];
}

// ... for a matrix, whose change is a product's shares (their rows are whole quads), added in their order
__global__ __launch_bounds__(256) void blocks_matrix_step_kernel(float* next, const float* from, OpShares d, uint32_t rows, int cols) {
  typedef float f32x4_t __attribute__((ext_vector_type(4)));
  const uint32_t quads = (uint32_t)d.ld / 4, total = rows * quads;
  for (uint32_t i = blockIdx.x * 256 + threadIdx.x; i < total; i += gridDim.x * 256) {
    const uint32_t m = i / quads;
    const int n = (int)(i - m * quads) * 4;
    const float* const p = d.part + (int64_t)m * d.ld + n;
    f32x4_t s = *(const f32x4_t*)p;
#pragma unroll 4
    for (int k = 1; k < d.shares; ++k) s += *(const f32x4_t*)(p + k * d.stride);
    const int64_t at = (int64_t)m * cols + n;
    if (n + 4 <= cols) {
      Piece<float, 4> w;
      w.load(from + at);
      const float f[4] = {w.at(0) - s[0], w.at(1) - s[1], w.at(2) - s[2], w.at(3) - s[3]};
      w.set(f);
      w.store(next + at);
    } else {
      for (int e = 0; n + e < cols; ++e) next[at + e] = from[at + e] - s[e];
    }
  }
}

__global__ __launch_bounds__(256) void blocks_narrow_kernel(const float* w, size_t rows, int cols, uint16_t* out, int ld) {
  for (size_t i = (size_t)blockIdx.x * 256 + threadIdx.x; i < rows * cols; i += (size_t)gridDim.x * 256) out[i / cols * ld + i % cols] = op_bf16(w[i]);
}

dim3 spread(size_t n) { return dim3((unsigned)std::max<size_t>(1, std::min<size_t>((n + 255) / 256, 4096))); }

abs_linear linear_of(const BlocksPlan& p, int l, int64_t rows) {
  abs_linear q{};
  q.dtype = ABS_X_BF16; q.act = ABS_ACT_NONE; q.rows = rows;
  q.d_in = p.d[l]; q.d_out = p.d[l + 1];
  q.ldx = q.lddx = p.d[l];
  q.ldw = p.ldw[l];
  q.ldy = q.ldr = q.lddy = q.ldz = q.lddw = p.d[l + 1];
  return q;
}
abs_group_norm norm_of(const BlocksPlan& p, int l, int64_t rows) {
  abs_group_norm q{};
  q.dtype = ABS_X_BF16; q.act = p.opt.act; q.n = rows; q.spatial = 1;
  q.channels = p.d[l]; q.groups = p.opt.groups; q.eps = p.opt.eps;
  q.ldx = q.ldy = q.lddy = q.lddx = q.lddres = p.d[l];
  return q;
}
abs_dropout dropout_of(const BlocksPlan& p, int l, int64_t rows, uint64_t offset) {
  abs_dropout q{};
  q.dtype = ABS_X_BF16; q.drop = p.opt.drop; q.rows = rows; q.cols = p.d[l];
  q.ldx = q.ldy = q.ldr = p.d[l];
  q.seed = p.seed; q.offset = offset;
  return q;
}
bool adds(const BlocksPlan& p, int l) { return p.opt.residual && l >= 1 && l < p.L - 1 && p.d[l] == p.d[l + 1]; }

// Uploads of one model version: rows [row, row + rows) of the stack.
struct Group { uint32_t slot; int64_t row, rows; };

// What the output layer's rows become: losses, and gradients (dz, with the descriptor's coefficients) or hits (correct).
struct LossOut { const int32_t* label; const RoundDesc& rd; float* rowloss; uint16_t* dz; float* correct; int kind; };

struct Chain {
  const BlocksArgs& a;
  const BlocksPlan& p;
  hipStream_t s;
  LaunchHook* hook;
  const uint16_t* x0;                  // the first layer's rows
  int rc = ABS_OK;
  Chain(const BlocksArgs& args, hipStream_t stream, LaunchHook* h) : a(args), p(args.plan), s(stream), hook(h), x0(act(0)) {}

  template <typename T> T* at(size_t off) const { return (T*)(a.ws + off); }
  const float* model(uint32_t slot) const { return at<float>(p.off_ring) + (size_t)slot * p.slot_stride; }
  const uint16_t* narrow(uint32_t slot, int l) const { return at<uint16_t>(p.off_shadow) + (size_t)slot * p.shadow_stride + p.shadow_off[l]; }
  uint16_t* act(int l) const { return at<uint16_t>(p.off_a[l]); }        // a_l [rows][d_l]; l = 0: the gathered rows
  const uint16_t* in(int l) const { return l ? u(l) : x0; }
  uint16_t* u(int l) const { return at<uint16_t>(p.off_u[l]); }
  void did(int r) { if (rc == ABS_OK) rc = r; }
  void launched() { if (rc == ABS_OK) rc = op_hip("blocks", hipGetLastError()); }

  // a_1 .. a_{L-1} of `rows` stacked rows and what `out` wants of the logits; drop_base < 0: no dropout (evaluation)
  void forward(const Group* g, int groups, int64_t rows, int64_t drop_base, const LossOut& out) {
    for (int l = 0; l < p.L && rc == ABS_OK; ++l) {
      if (l) {
        hook->begin(KK_BLOCKS_NORM, 10.0 * rows * p.d[l], 4.0 * rows * p.d[l]);
        for (int i = 0; i < groups; ++i) {
          const abs_group_norm q = norm_of(p, l, g[i].rows);
          const size_t off = (size_t)g[i].row * p.d[l], st = (size_t)g[i].row * p.opt.groups;
          did(abs_group_norm_forward(&q, act(l) + off, model(g[i].slot) + p.gamma_off[l], model(g[i].slot) + p.gamma_off[l] + p.d[l],
                                     u(l) + off, at<float>(p.off_mean[l]) + st, at<float>(p.off_rstd[l]) + st, at<void>(p.off_ops),
                                     p.ops_bytes, s));
        }
        hook->end(KK_BLOCKS_NORM);
        if (drop_base >= 0 && p.opt.drop) {
          hook->begin(KK_BLOCKS_DROPOUT, 10.0 * rows * p.d[l], 4.0 * rows * p.d[l]);
          const abs_dropout q = dropout_of(p, l, rows, (uint64_t)drop_base + l);
          did(abs_dropout_forward(&q, u(l), nullptr, u(l), s));
          hook->end(KK_BLOCKS_DROPOUT);
        }
      }
      if (l == p.L - 1) {
        for (int i = 0; i < groups; ++i) output(g[i], out);
        continue;
      }
      hook->begin(KK_BLOCKS_LINEAR, 2.0 * rows * p.d[l] * p.d[l + 1], 2.0 * (rows * (double)(p.d[l] + p.d[l + 1]) + (double)p.d[l] * p.d[l + 1]));
      for (int i = 0; i < groups; ++i) {
        const abs_linear q = linear_of(p, l, g[i].rows);
        const size_t out = (size_t)g[i].row * p.d[l + 1];
        did(abs_linear_forward(&q, in(l) + (size_t)g[i].row * p.d[l], narrow(g[i].slot, l), model(g[i].slot) + p.b_off[l],
                               adds(p, l) ? act(l) + out : nullptr, act(l + 1) + out, nullptr, at<void>(p.off_ops), p.ops_bytes, s));
      }
      hook->end(KK_BLOCKS_LINEAR);
    }
  }

  // the logits of one version's rows stay in the product's fp32 shares until the loss has read them: rounded to bf16, two of them closer
  // than half a step would be equal, and the first one the largest
  void output(const Group& g, const LossOut& out) {
    const int l = p.L - 1, C = p.d[p.L];
    const abs_linear q = linear_of(p, l, g.rows);
    OpShares z{};
    hook->begin(KK_BLOCKS_LINEAR, 2.0 * g.rows * p.d[l] * C, 2.0 * (g.rows * (double)p.d[l] + 2.0 * g.rows * C + (double)p.d[l] * C));
    did(op_linear_forward_shares(&q, in(l) + (size_t)g.row * p.d[l], narrow(g.slot, l), at<void>(p.off_ops), p.ops_bytes, s, &z));
    hook->end(KK_BLOCKS_LINEAR);
    if (rc != ABS_OK) return;
    hook->begin(out.kind, 8.0 * g.rows * C, 4.0 * g.rows * C + (out.dz ? 2.0 * g.rows * C : 0));
    blocks_loss_kernel<<<dim3((unsigned)((g.rows + 3) / 4)), 256, 0, s>>>(z, model(g.slot) + p.b_off[l], C, (int)g.rows, out.label + g.row, (int)g.row, p.B, out.rd,
                                                                         out.rowloss + g.row, out.dz ? out.dz + (size_t)g.row * C : nullptr,
                                                                         out.correct ? out.correct + g.row : nullptr);
    launched();
    hook->end(out.kind);
  }

  // next -= the change of n parameters at `off`, or of matrix l; `fresh`: the first one, from the current model
  void step(float* next, const float* cur, size_t off, const float* change, size_t n, bool fresh) {
    if (rc != ABS_OK) return;
    blocks_step_kernel<<<spread(n), 256, 0, s>>>(next + off, (fresh ? cur : next) + off, change, n);
    launched();
  }
  void step(float* next, const float* cur, int l, const OpShares& change, bool fresh) {
    if (rc != ABS_OK) return;
    blocks_matrix_step_kernel<<<spread((size_t)p.d[l] * change.ld / 4), 256, 0, s>>>(next + p.w_off[l], (fresh ? cur : next) + p.w_off[l], change,
                                                                                   (uint32_t)p.d[l], p.d[l + 1]);
    launched();
  }

  void backward(const Group* g, int groups, int64_t rows, int64_t drop_base, uint32_t slot_cur, uint32_t slot_next) {
    float* const next = at<float>(p.off_ring) + (size_t)slot_next * p.slot_stride;
    const float* const cur = model(slot_cur);
    float* const dv = at<float>(p.off_dv);
    // the gradient of a_{l+1} is in da[l & 1] (the logits': where the loss left it)
    for (int l = p.L - 1; l >= 0 && rc == ABS_OK; --l) {
      const uint16_t* const dy = at<uint16_t>(p.off_da[(l + 1) & 1]);
      uint16_t* const du = at<uint16_t>(p.off_du);
      hook->begin(KK_BLOCKS_LINEAR, (l ? 4.0 : 2.0) * rows * p.d[l] * p.d[l + 1], 4.0 * rows * (double)(p.d[l] + p.d[l + 1]));
      for (int i = 0; i < groups; ++i) {
        const abs_linear q = linear_of(p, l, g[i].rows);
        const size_t off = (size_t)g[i].row * p.d[l];
        OpShares dw{};
        did(op_linear_backward_shares(&q, in(l) + off, narrow(g[i].slot, l), nullptr, dy + (size_t)g[i].row * p.d[l + 1], l ? du + off : nullptr,
                                      dv, at<void>(p.off_ops), p.ops_bytes, s, &dw));
        step(next, cur, l, dw, i == 0);
        step(next, cur, p.b_off[l], dv, (size_t)p.d[l + 1], i == 0);
      }
      hook->end(KK_BLOCKS_LINEAR);
      if (!l) break;
      if (p.opt.drop) {
        hook->begin(KK_BLOCKS_DROPOUT, 10.0 * rows * p.d[l], 4.0 * rows * p.d[l]);
        const abs_dropout q = dropout_of(p, l, rows, (uint64_t)drop_base + l);
        did(abs_dropout_backward(&q, du, du, s));
        hook->end(KK_BLOCKS_DROPOUT);
      }
      hook->begin(KK_BLOCKS_NORM, 20.0 * rows * p.d[l], 6.0 * rows * p.d[l]);
      uint16_t* const da = at<uint16_t>(p.off_da[l & 1]);
      for (int i = 0; i < groups; ++i) {
        const abs_group_norm q = norm_of(p, l, g[i].rows);
        const size_t off = (size_t)g[i].row * p.d[l], st = (size_t)g[i].row * p.opt.groups;
        did(abs_group_norm_backward(&q, act(l) + off, model(g[i].slot) + p.gamma_off[l], model(g[i].slot) + p.gamma_off[l] + p.d[l],
                                    at<float>(p.off_mean[l]) + st, at<float>(p.off_rstd[l]) + st, du + off, adds(p, l) ? dy + off : nullptr,
                                    da + off, dv, dv + p.d[l], at<void>(p.off_ops), p.ops_bytes, s));
        step(next, cur, p.gamma_off[l], dv, 2 * (size_t)p.d[l], i == 0);
      }
      hook->end(KK_BLOCKS_NORM);
    }
  }

  void narrow_model(uint32_t slot) {
    for (int l = 0; l < p.L; ++l) {
      blocks_narrow_kernel<<<spread((size_t)p.d[l] * p.d[l + 1]), 256, 0, s>>>(model(slot) + p.w_off[l], (size_t)p.d[l], p.d[l + 1],
                                                                                const_cast<uint16_t*>(narrow(slot, l)), p.ldw[l]);
      launched();
    }
  }
  hipError_t result() const { return rc == ABS_OK ? hipSuccess : rc == ABS_E_HIP ? hipErrorLaunchFailure : hipErrorInvalidValue; }
};

}  // namespace

bool blocks_plan(const abs_config& c, const abs_blocks& b, BlocksPlan& p, const char** why) {
  p = BlocksPlan{};
  const int L = c.n_layers;
  if (c.model != ABS_MODEL_MLP) { *why = "blocks: the model must be ABS_MODEL_MLP"; return false; }
  if (c.U > 1) { *why = "blocks: U must be 1"; return false; }
  if (b.reserved != 0) { *why = "blocks: reserved must be 0"; return false; }
  if (b.act < ABS_ACT_NONE || b.act > ABS_ACT_GELU) { *why = "blocks: act must be 0..3"; return false; }
  if (b.residual < 0 || b.residual > 1) { *why = "blocks: residual must be 0 or 1"; return false; }
  if (b.drop < 0 || b.drop > 65535) { *why = "blocks: drop must be in [0, 65535]"; return false; }
  if (!(b.eps > 0.f) || b.eps > 1e30f) { *why = "blocks: eps must be positive and finite"; return false; }
  for (int l = 1; l < L; ++l)
    if (b.groups < 1 || c.dims[l] % b.groups) { *why = "blocks: groups must divide every hidden width"; return false; }
  p.opt = b;
  p.L = L; p.B = c.B; p.N = c.N; p.R = c.tau_cap + 3; p.seed = c.seed;
  for (int l = 0; l <= L; ++l) p.d[l] = c.dims[l];
  size_t o = 0, so = 0;
  for (int l = 0; l < L; ++l) {
    if (l) { p.gamma_off[l] = o; o += 2 * (size_t)p.d[l]; }
    p.w_off[l] = o; o += (size_t)p.d[l] * p.d[l + 1];
    p.b_off[l] = o; o += (size_t)p.d[l + 1];
    p.ldw[l] = (int)up(p.d[l + 1], 8);
    p.shadow_off[l] = so; so = up(so + (size_t)p.d[l] * p.ldw[l], 128);
  }
  p.P = o;
  p.slot_stride = up(o, 64);
  p.shadow_stride = so;
  size_t t = 0;
  auto take = [&](size_t bytes) { const size_t at = t; t = up(t + bytes, 256); return at; };
  const size_t rows = (size_t)p.N * p.B;
  size_t widest = 0;
  for (int l = 1; l <= L; ++l) widest = std::max(widest, (size_t)p.d[l]);
  p.off_ring = take((size_t)p.R * p.slot_stride * 4);
  p.off_shadow = take((size_t)p.R * p.shadow_stride * 2);
  p.off_label = take(rows * 4);
  for (int l = 0; l < L; ++l) p.off_a[l] = take(rows * p.d[l] * 2);
  for (int l = 1; l < L; ++l) {
    p.off_u[l] = take(rows * p.d[l] * 2);
    p.off_mean[l] = take(rows * b.groups * 4);
    p.off_rstd[l] = take(rows * b.groups * 4);
  }
  for (int i = 0; i < 2; ++i) p.off_da[i] = take(rows * widest * 2);
  p.off_du = take(rows * widest * 2);
  p.off_dv = take(2 * widest * 4);
  p.off_rowloss = take(rows * 4);
  // the operators' own workspace: for any number of uploads of one version, and the last rows of an evaluation
  // (rows of a group start where the previous one ends: at any multiple of a row)
  auto needs = [&](int64_t n, int passes) {
    for (int back = 0; back < passes; ++back)
      for (int l = 0; l < L; ++l) {
        const abs_linear q = linear_of(p, l, n);
        p.ops_bytes = std::max(p.ops_bytes, back || l == L - 1 ? op_linear_shares_size(&q, back) : abs_linear_workspace_size(&q, back, 0));
        if (!l) continue;
        const abs_group_norm g = norm_of(p, l, n);
        p.ops_bytes = std::max(p.ops_bytes, abs_group_norm_workspace_size(&g, back));
      }
  };
  for (int k = 1; k <= p.N; ++k) needs((int64_t)k * p.B, 2);
  for (int n = 1; n < p.B; ++n) needs(n, 1);
  p.off_ops = take(p.ops_bytes);
  p.off_eval = take(eval_scratch_bytes(rows));
  p.total = t;
  return true;
}

hipError_t blocks_prepare(const BlocksArgs& a, hipStream_t s) {
  struct Quiet : LaunchHook { void begin(int, double, double) override {} void end(int) override {} } quiet;
  Chain c(a, s, &quiet);
  c.narrow_model(0);
  return c.result();
}

hipError_t launch_blocks_round(const BlocksArgs& a, const RoundDesc& rd, hipStream_t s, LaunchHook* hook) {
  Chain c(a, s, hook);
  const BlocksPlan& p = a.plan;
  const int K = rd.K;
  const int64_t rows = (int64_t)K * p.B, t = (int64_t)rd.stamp - 1;
  Group g[ABS_MAX_WORKERS];
  int groups = 0;
  for (int k = 0; k < K; ++k) {
    if (groups && g[groups - 1].slot == rd.w[k].slot) g[groups - 1].rows += p.B;
    else g[groups++] = Group{rd.w[k].slot, (int64_t)k * p.B, p.B};
  }
  // masks of their own for every round and layer
  const int64_t drop_base = t * 8;
  hook->begin(KK_BLOCKS_LOSS, 0, 4.0 * rows * p.d[0]);
  blocks_gather_kernel<<<dim3((unsigned)rows), 128, 0, s>>>(a.X, a.y, p.d[0], a.shard_rows, a.batch_key, p.B, rd, c.act(0), c.at<int32_t>(p.off_label));
  c.launched();
  hook->end(KK_BLOCKS_LOSS);
  c.forward(g, groups, rows, drop_base, LossOut{c.at<int32_t>(p.off_label), rd, c.at<float>(p.off_rowloss), c.at<uint16_t>(p.off_da[p.L & 1]), nullptr, KK_BLOCKS_LOSS});
  hook->begin(KK_BLOCKS_LOSS, (double)rows, 4.0 * rows);
  blocks_publish_kernel<<<dim3(1), 128, 0, s>>>(c.at<float>(p.off_rowloss), p.B, K, a.mailbox, rd.stamp);
  c.launched();
  hook->end(KK_BLOCKS_LOSS);
  c.backward(g, groups, rows, drop_base, rd.slot_cur, rd.slot_next);
  hook->begin(KK_BLOCKS_UPDATE, (double)p.P, 6.0 * p.P);
  c.narrow_model(rd.slot_next);
  hook->end(KK_BLOCKS_UPDATE);
  return c.result();
}

hipError_t launch_blocks_eval(const BlocksArgs& a, uint32_t slot, const EvalArgs& e, hipStream_t s, LaunchHook* hook) {
  Chain c(a, s, hook);
  const BlocksPlan& p = a.plan;
  const int64_t cap = (int64_t)p.N * p.B;
  if (e.cap < cap) return hipErrorInvalidValue;
  hipError_t err = launch_eval_clear(e, s);
  int n = 0;
  for (int64_t row0 = 0; row0 < e.n_rows && err == hipSuccess; row0 += n) {
    // whole minibatches, and what is left at the end (the row counts that the operators' workspace is sized for)
    const int64_t left = e.n_rows - row0;
    n = (int)(left >= cap ? cap : left >= p.B ? left / p.B * p.B : left);
    const Group g{slot, 0, n};
    c.x0 = (const uint16_t*)e.X + (size_t)row0 * p.d[0];
    const RoundDesc none{};
    c.forward(&g, 1, n, -1, LossOut{(const int32_t*)e.y + row0, none, e.rowloss, nullptr, e.correct, KK_EVAL});
    err = c.result();
    if (err == hipSuccess) err = launch_eval_reduce(e, n, s, hook);
  }
  return err;
}

}  // namespace abs_impl
