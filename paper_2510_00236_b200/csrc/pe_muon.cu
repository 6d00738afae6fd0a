// Entry points of the orthogonalised update: argument checks, workspace, and the launches of an iteration.
#include <algorithm>
#include <cmath>

#include "pe_host.cuh"
#include "pe_muon.cuh"

namespace pe {

constexpr int NS_MAX_STEPS = 100;
constexpr int NS_MAX_PARTIALS = 512;
constexpr int NS_PAIRS = 74;            // pairs of SMs that launches and the workspace are laid out for

// How a product is cut: the tile's width, and slices of the contraction index where tiles are few.
struct NsPlan {
  int nt, splits;
  long long units;      // tiles of a matrix
  double us;            // estimate
};
static long long ns_units(int rows, int cols, int nt, bool symmetric) {
  const long long tiles_m = (rows + 255) / 256, tiles_n = (cols + nt - 1) / nt;
  if (!symmetric) return tiles_m * tiles_n;
  long long units = 0;
  for (long long i = 0; i < tiles_m; ++i) units += tiles_n - i * (256 / nt);
  return units;
}
// Times in microseconds, fitted to whole launches of some shapes (a stage of 256 x 128 among many takes 0.61): a stage of 64 (12 instructions of 256 x NT x 16), what a
// tile costs beside its stages (set-up, the first stage's way from memory, write-out), and what joining slices costs.
static NsPlan plan_product(int rows, int cols, int k, int count, bool symmetric) {
  const int stages = (k + NS_BK - 1) / NS_BK;
  NsPlan best = {128, 1, 0, 0.0};
  double best_us = 1e300;
  for (int nt : {64, 128, 256}) {
    const long long units = ns_units(rows, cols, nt, symmetric), tiles = units * count;
    const double stage_us = nt == 64 ? 0.30 : nt == 128 ? 0.50 : 0.92, fixed_us = nt == 64 ? 5.0 : nt == 128 ? 6.5 : 9.0;
    for (int splits = 1; splits <= stages / 2 || splits == 1; ++splits) {
      if (splits > 1 && tiles * splits > NS_PAIRS) break;
      const long long waves = (tiles * splits + NS_PAIRS - 1) / NS_PAIRS;
      const double us = waves * (((stages + splits - 1) / splits) * stage_us + fixed_us) + (splits > 1 ? 2.5 + 0.4 * splits : 0.0);
      if (us < best_us) { best_us = us; best = {nt, splits, units, us}; }
    }
  }
  return best;
}

struct NsLayout {
  NsPlan gram, poly, apply;        // A = X X^T, A A, Q X
  bool pairs;                      // two steps at a time
  int n, m, ld_m, ld_n, tall;
  int partials;                    // partial sums of a matrix's norm
  int counters;                    // of split products, two words a tile; a word for products that gave up is behind them
  size_t norms, x[2], a, q, t, partial, counters_at, total; // byte offsets into the workspace
};
static bool ns_size_ok(int count, int rows, int cols) {
  return count >= 0 && rows >= 1 && cols >= 1 && rows <= (1 << 30) && cols <= (1 << 30) && (count == 0 || (long long)rows * cols <= ((1ll << 36) - 1) / count) && count <= 65535;
}
static NsLayout ns_layout(int count, int rows, int cols) {
  NsLayout l = {};
  l.tall = rows > cols;
  l.n = std::min(rows, cols);
  l.m = std::max(rows, cols);
  l.ld_m = (int)align_up(l.m, 8);      // TMA wants row pitches of 16 bytes
  l.ld_n = (int)align_up(l.n, 8);
  const long long elems = (long long)rows * cols;
  l.partials = (int)std::min<long long>(NS_MAX_PARTIALS, (elems + 2047) / 2048);
  size_t at = 0;
  auto part = [&](size_t bytes) { const size_t here = at; at += align_up(bytes, 256); return here; };
  l.norms = part((size_t)count * l.partials * sizeof(double));
  for (int k = 0; k < 2; ++k) l.x[k] = part(4ull * count * l.n * l.ld_m);      // two planes of halves
  l.a = part(4ull * count * l.n * l.ld_n);
  l.q = part(4ull * count * l.n * l.ld_n);
  l.gram = plan_product(l.n, l.n, l.m, count, true);
  l.poly = plan_product(l.n, l.n, l.n, count, true);
  l.apply = plan_product(l.n, l.m, l.n, count, false);
  // Two steps at a time where X is much longer than A: with Q = a I + b A + c A A, the next step's A is Q A Q and its polynomial another of A, so that X itself
  // is multiplied once, by Q' Q, and not twice, and X X^T formed once: five products of n^3 for two more passes over X.  Not more steps than two: what rounding leaves in
  // the directions of small singular values is multiplied by the square of the slope, up to 12 a step, in A, and by the slope, up to 3.4, in X; after two steps
  // the errors of either way are those of fp32 products (2 to 7e-6 and 2 to 5e-6 for the same matrices), after three A is no longer positive and the iteration diverges.
  // 8192 x 2048: 1057 us a call against 1526; 6 x 2048 x 512: 283 and 345; 512 x 32768: 496 and 706.  (Below 256 rows the launches are what counts, and there are more.)
  l.pairs = l.n >= 256 && 3.0 * l.poly.us < 0.95 * (l.gram.us + l.apply.us);
  l.t = part(l.pairs ? 4ull * count * l.n * l.ld_n : 0);
  size_t partial = 0;
  for (const NsPlan* p : {&l.gram, &l.poly, &l.apply})
    if (p->splits > 1) {
      partial = std::max(partial, (size_t)(p->splits * p->units * count * 256 * p->nt) * sizeof(float));
      l.counters = std::max(l.counters, (int)(2 * p->units * count));
    }
  l.partial = part(partial);
  l.counters_at = part(((size_t)l.counters + 1) * sizeof(unsigned int));
  l.total = at;
  return l;
}

// Planes [2 * count][rows][ld] of halves, `cols` columns of them data; one box = 64 columns (128 bytes, swizzled) x box_rows rows, or
// a piece of 32 columns (64 bytes).
static pe_status_t ns_map(CUtensorMap* map, const void* base, int planes, int rows, int cols, int ld, int box_rows, bool piece = false) {
  EncodeTiledFn enc = encode_fn();
  if (!enc) return PE_ERR_CUDA;
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)planes};
  cuuint64_t strides[2] = {(cuuint64_t)ld * 2, (cuuint64_t)rows * ld * 2};
  cuuint32_t box[3] = {piece ? 32u : 64u, (cuuint32_t)box_rows, 1u}, estr[3] = {1u, 1u, 1u};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3, const_cast<void*>(base), dims, strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE,
             piece ? CU_TENSOR_MAP_SWIZZLE_64B : CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? PE_OK : PE_ERR_CUDA;
}

// Lets `kernel` use `smem` bytes of shared memory on the current device; ready: the devices where it may already.
template <typename Kernel>
static pe_status_t allow_smem(Kernel kernel, std::atomic<unsigned long long> (&ready)[MAX_DEVICES / 64], int smem) {
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev >= MAX_DEVICES) { cudaGetLastError(); return PE_ERR_CUDA; }
  const unsigned long long bit = 1ull << (dev & 63);
  if (ready[dev >> 6].load(std::memory_order_acquire) & bit) return PE_OK;
  if (cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess) { cudaGetLastError(); return PE_ERR_CUDA; }
  ready[dev >> 6].fetch_or(bit, std::memory_order_release);
  return PE_OK;
}
static bool ns_is_small(const NsLayout& l) { return l.n <= NS_SMALL_N && l.m <= NS_SMALL_M; }

template <int NT, bool B_MN, int EPI>
static pe_status_t launch_product(const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& out, const CUtensorMap& add, NsProduct p, cudaStream_t st) {
  static std::atomic<unsigned long long> ready[MAX_DEVICES / 64];
  auto kernel = ns_product_kernel<NT, B_MN, EPI>;
  const pe_status_t rc = allow_smem(kernel, ready, NsTile<NT>::SMEM_BYTES);
  if (rc != PE_OK) return rc;
  p.tiles_n = (p.cols + NT - 1) / NT;
  return launch_dependent(kernel, dim3((unsigned)(2ll * p.units * p.count * p.splits)), NS_THREADS, NsTile<NT>::SMEM_BYTES, st, a, b, out, add, p);
}
template <bool B_MN, int EPI>
static pe_status_t launch_planned(const NsPlan& plan, const CUtensorMap& a, const CUtensorMap& b, const CUtensorMap& out, const CUtensorMap& add, NsProduct p, cudaStream_t st) {
  p.units = (int)plan.units;
  p.splits = plan.splits;
  if (plan.nt == 64) return launch_product<64, B_MN, EPI>(a, b, out, add, p, st);
  return plan.nt == 256 ? launch_product<256, B_MN, EPI>(a, b, out, add, p, st) : launch_product<128, B_MN, EPI>(a, b, out, add, p, st);
}

// The iteration on what `s` describes; `out` holds the last product's output side.
static pe_status_t newton_schulz(DeviceInfo* di, const NsSource& s, int count, int rows, int cols, int steps, const NsProduct& out, char* ws, cudaStream_t st) {
  const NsLayout l = ns_layout(count, rows, cols);
  if (ns_is_small(l)) {
    static std::atomic<unsigned long long> ready[MAX_DEVICES / 64];
    const int most = (NS_SMALL_N * ns_small_ld(NS_SMALL_M) + 2 * NS_SMALL_N * NS_SMALL_LD) * (int)sizeof(float);
    const pe_status_t rc = allow_smem(ns_small_kernel, ready, most);
    if (rc != PE_OK) return rc;
    const int smem = (NS_SMALL_N * ns_small_ld(l.m) + 2 * NS_SMALL_N * NS_SMALL_LD) * (int)sizeof(float);
    return launch_dependent(ns_small_kernel, dim3(count), NS_SMALL_THREADS, smem, st, s, out.to, l.n, l.m, l.tall, steps);
  }
  double* norms = reinterpret_cast<double*>(ws + l.norms);
  __half* x[2] = {reinterpret_cast<__half*>(ws + l.x[0]), reinterpret_cast<__half*>(ws + l.x[1])};
  __half *const a = reinterpret_cast<__half*>(ws + l.a), *const q = reinterpret_cast<__half*>(ws + l.q);
  const bool wide = (long long)rows * cols % 4 == 0 && (!s.given || (!s.bf16 && aligned(s.given, 16)));
  pe_status_t rc = launch_dependent(wide ? ns_norms_kernel<true> : ns_norms_kernel<false>, dim3(l.partials, count), NS_NORM_THREADS, 0, st, s, (long long)rows * cols, norms,
                                    reinterpret_cast<unsigned int*>(ws + l.counters_at), l.counters + 1);
  if (rc != PE_OK) return rc;
  const int tiles_m = (l.m + NS_INIT_TILE - 1) / NS_INIT_TILE, tiles_n = (l.n + NS_INIT_TILE - 1) / NS_INIT_TILE;
  rc = launch_dependent(ns_init_kernel, dim3((unsigned)(tiles_m * tiles_n), count), 256, 0, st, s, l.n, l.m, l.ld_m, l.tall, tiles_m, (const double*)norms,
                        l.partials, x[0], count);
  if (rc != PE_OK) return rc;
  __half* const t = reinterpret_cast<__half*>(ws + l.t);
  CUtensorMap xa[2], xb_rows[2], xb_cols[2], xo[2];      // as A operand, as B operand row by row, as B operand with the contraction index slow, as output
  for (int k = 0; k < 2; ++k)
    if (ns_map(&xa[k], x[k], 2 * count, l.n, l.m, l.ld_m, 128) != PE_OK || ns_map(&xb_rows[k], x[k], 2 * count, l.n, l.m, l.ld_m, l.gram.nt / 2) != PE_OK ||
        ns_map(&xb_cols[k], x[k], 2 * count, l.n, l.m, l.ld_m, NS_BK, l.apply.nt == 64) != PE_OK || ns_map(&xo[k], x[k], 2 * count, l.n, l.m, l.ld_m, 32, true) != PE_OK)
      return PE_ERR_CUDA;
  struct Square { CUtensorMap a, b, out; } A, Q, T;      // [n, n]
  auto square = [&](Square& m, const __half* base) {
    return ns_map(&m.a, base, 2 * count, l.n, l.n, l.ld_n, 128) == PE_OK && ns_map(&m.b, base, 2 * count, l.n, l.n, l.ld_n, l.poly.nt / 2) == PE_OK &&
           ns_map(&m.out, base, 2 * count, l.n, l.n, l.ld_n, 32, true) == PE_OK;
  };
  if (!square(A, a) || !square(Q, q) || (l.pairs && !square(T, t))) return PE_ERR_CUDA;
  NsProduct p = out;
  p.count = count;
  p.dev_status = di->status_ptr;
  p.partial = reinterpret_cast<float*>(ws + l.partial);
  p.counters = reinterpret_cast<unsigned int*>(ws + l.counters_at);
  p.gave_up = p.counters + l.counters;
  p.rows = l.n;
  auto gram = [&](int from) { p.cols = l.n; p.k = l.m; p.add = 0; return launch_planned<false, NS_SYMMETRIC>(l.gram, xa[from], xb_rows[from], A.out, A.out, p, st); };
  // products of symmetric matrices that commute are symmetric; add: a I + b u + c u u
  auto squares = [&](const Square& u, const Square& v, const Square& to, int add) {
    p.cols = p.k = l.n; p.add = add;
    return launch_planned<false, NS_SYMMETRIC>(l.poly, u.a, v.b, to.out, u.out, p, st);
  };
  auto apply = [&](const Square& u, int from, bool last) {
    p.cols = l.m; p.k = l.n; p.add = 0;
    return last ? launch_planned<true, NS_FINAL>(l.apply, u.a, xb_cols[from], xo[from ^ 1], A.out, p, st)
                : launch_planned<true, NS_PLANES>(l.apply, u.a, xb_cols[from], xo[from ^ 1], A.out, p, st);
  };
  for (int left = steps, from = 0; left > 0; from ^= 1) {
    if ((rc = gram(from)) != PE_OK || (rc = squares(A, A, Q, 1)) != PE_OK) return rc;
    if (l.pairs && left >= 2) {
      if ((rc = squares(Q, A, T, 0)) != PE_OK || (rc = squares(T, Q, A, 0)) != PE_OK ||      // A <- Q A Q
          (rc = squares(A, A, T, 1)) != PE_OK || (rc = squares(T, Q, A, 0)) != PE_OK)        // T <- its polynomial, A <- T Q
        return rc;
      left -= 2;
      if ((rc = apply(A, from, left == 0)) != PE_OK) return rc;
    } else {
      --left;
      if ((rc = apply(Q, from, left == 0)) != PE_OK) return rc;
    }
  }
  return PE_OK;
}

static pe_status_t ns_check(int count, int rows, int cols, int steps, const void* workspace, size_t workspace_bytes) {
  if (!ns_size_ok(count, rows, cols) || steps < 1 || steps > NS_MAX_STEPS) return PE_ERR_DIM;
  if (count == 0) return PE_OK;
  const NsLayout l = ns_layout(count, rows, cols);
  for (const NsPlan* p : {&l.gram, &l.poly, &l.apply})      // blocks of a launch
    if (2 * p->units * count >= (1ll << 31)) return PE_ERR_DIM;
  if (!workspace || workspace_bytes < l.total) return PE_ERR_WORKSPACE;
  return aligned(workspace, 256) ? PE_OK : PE_ERR_ALIGN;
}

static pe_status_t orthogonalize_impl(const void* G, int bf16, int count, int rows, int cols, int steps, void* out, void* workspace,
                                      size_t workspace_bytes, cudaStream_t st) {
  if ((!G || !out) && count > 0) return PE_ERR_NULL;
  if (!aligned(G, bf16 ? 16 : 4) || !aligned(out, bf16 ? 16 : 4)) return PE_ERR_ALIGN;
  pe_status_t rc = ns_check(count, rows, cols, steps, workspace, workspace_bytes);
  if (rc != PE_OK) return rc;
  DeviceInfo* di = nullptr;
  rc = device_info(&di);
  if (rc != PE_OK || count == 0) return rc;
  NsSource s = {};
  s.given = G; s.bf16 = bf16;
  NsProduct p = {};
  p.to.result = out; p.to.out_bf16 = bf16; p.transposed = rows > cols;
  return newton_schulz(di, s, count, rows, cols, steps, p, static_cast<char*>(workspace), st);
}

pe_status_t ns_plan_query(int product, int count, int rows, int cols, long long* plan) {
  if (product < 0 || product > 2 || !ns_size_ok(count, rows, cols)) return PE_ERR_DIM;
  const NsLayout l = ns_layout(count, rows, cols);
  const bool small = ns_is_small(l);
  const NsPlan& p = product == 0 ? l.gram : product == 1 ? l.poly : l.apply;
  plan[0] = small ? 0 : p.nt; plan[1] = small ? 0 : p.splits; plan[2] = small ? 0 : p.units; plan[3] = !small && l.pairs ? 2 : 1;
  return PE_OK;
}

pe_status_t ns_set_wait_limit(long long cycles) {
  if (cudaMemcpyToSymbol(sm100::g_wait_cycle_limit, &cycles, sizeof cycles) != cudaSuccess) { cudaGetLastError(); return PE_ERR_CUDA; }
  return PE_OK;
}

}  // namespace pe

using namespace pe;

extern "C" {

size_t pe_orthogonalize_workspace_bytes(int count, int rows, int cols) {
  return ns_size_ok(count, rows, cols) && count > 0 ? ns_layout(count, rows, cols).total : 0;
}
pe_status_t pe_orthogonalize(const void* G, int count, int rows, int cols, int steps, void* out, void* workspace, size_t workspace_bytes,
                             pe_stream_t stream) {
  return orthogonalize_impl(G, 1, count, rows, cols, steps, out, workspace, workspace_bytes, reinterpret_cast<cudaStream_t>(stream));
}
pe_status_t pe_orthogonalize_f32(const float* G, int count, int rows, int cols, int steps, float* out, void* workspace, size_t workspace_bytes,
                                 pe_stream_t stream) {
  return orthogonalize_impl(G, 0, count, rows, cols, steps, out, workspace, workspace_bytes, reinterpret_cast<cudaStream_t>(stream));
}
pe_status_t muon_step(float* theta, void* theta_lp, float* m, const float* sum_g, int count, int rows, int cols, int B, float grad_scale, float lr, float beta,
                      int nesterov, int steps, float update_scale, float weight_decay, void* workspace, size_t workspace_bytes, pe_stream_t stream) {
  if ((!theta || !m || !sum_g) && count > 0) return PE_ERR_NULL;
  if (B < 1) return PE_ERR_DIM;
  if (!aligned(theta, 16) || !aligned(m, 16) || !aligned(sum_g, 16) || !aligned(theta_lp, 16)) return PE_ERR_ALIGN;
  pe_status_t rc = ns_check(count, rows, cols, steps, workspace, workspace_bytes);
  if (rc != PE_OK) return rc;
  DeviceInfo* di = nullptr;
  rc = device_info(&di);
  if (rc != PE_OK || count == 0) return rc;
  NsSource s = {};
  s.m = m; s.sum_g = sum_g; s.grad_scale = (float)((double)grad_scale / (double)B); s.beta = beta; s.nesterov = nesterov != 0;
  NsProduct p = {};
  p.to.theta = theta; p.to.theta_lp = static_cast<__nv_bfloat16*>(theta_lp); p.to.step = lr * update_scale; p.to.wd = weight_decay; p.transposed = rows > cols;
  return newton_schulz(di, s, count, rows, cols, steps, p, static_cast<char*>(workspace), reinterpret_cast<cudaStream_t>(stream));
}

}  // extern "C"
