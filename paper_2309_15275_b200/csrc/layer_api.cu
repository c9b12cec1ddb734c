// C-ABI entry points of what a layer does around its product: checks, workspace layout
// and the launches.
#include <cmath>
#include <initializer_list>

#include "layer_math.cuh"

namespace lbp {
namespace layer {

static size_t align_up(size_t v, size_t a) { return (v + a - 1) / a * a; }
static int elem_size(int dtype) { return dtype == LBP_BF16 ? 2 : 4; }
static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
static const lbp_epilogue kNoEpilogue{};
static const lbp_pitches kDense{};

// The numbers of a call's elements are below 2^62, so that no sum in a kernel overflows.
constexpr int64_t kMostElements = int64_t{1} << 62;
// How many elements (places or numbers) there are from the first to the last of `count` steps along each of three strides,
// C of them behind the last.  (Up to 2^91.)
struct Steps3 {
  long long count[3];
  int64_t stride[3];
};
static __int128 extent(const Steps3& s, int C) {
  __int128 n = C;
  for (int i = 0; i < 3; ++i)
    if (s.count[i] > 0) n += static_cast<__int128>(s.count[i] - 1) * s.stride[i];
  return n;
}
static int check_numbers(int64_t first, const Steps3& s, int C) {
  return first + extent(s, C) > kMostElements ? LBP_ERR_SHAPE : LBP_OK;
}
// Bytes of a tensor's places fit 64 bits with room to spare: nothing that exists is larger.
constexpr __int128 kMostPlaces = static_cast<__int128>(1) << 58;
static Steps3 along_rows(long long rows, int64_t pitch) { return Steps3{{rows, 0, 0}, {pitch, 0, 0}}; }
static Steps3 along_grid(int B, int H, int W, const lbp_view& v) { return Steps3{{B, H, W}, {v.image, v.row, v.token}}; }

static int check_rows(long long rows, int C, int dtype) {
  if (dtype != LBP_F32 && dtype != LBP_BF16) return LBP_ERR_DTYPE;
  if (rows < 0 || rows > (1ll << 40) || C <= 0 || C > (1 << 30)) return LBP_ERR_SHAPE;
  if ((static_cast<long long>(C) * elem_size(dtype)) % 16 != 0) return LBP_ERR_ALIGN;
  return extent(along_rows(rows, C), C) > kMostPlaces ? LBP_ERR_SHAPE : LBP_OK;
}
static int check_pitch(long long rows, int64_t pitch, int C, int dtype) {
  if (pitch == 0) return LBP_OK;
  if (pitch < C || pitch >= (int64_t{1} << 40) / elem_size(dtype)) return LBP_ERR_SHAPE;   // (a tensor map's stride: 2^40 bytes)
  if (extent(along_rows(rows, pitch), C) > kMostPlaces) return LBP_ERR_SHAPE;
  return (pitch * elem_size(dtype)) % 16 != 0 ? LBP_ERR_ALIGN : LBP_OK;
}
static bool in_quads(int64_t v, int dtype) { return v % (dtype == LBP_BF16 ? 8 : 4) == 0; }

static int check_epilogue(const lbp_epilogue& e, int dtype) {
  if (e.act < LBP_ACT_NONE || e.act > LBP_ACT_SILU || !(e.p >= 0.f && e.p <= 1.f)) return LBP_ERR_SHAPE;
  if (e.first < 0 || e.first >= kMostElements) return LBP_ERR_SHAPE;
  for (int64_t v : {e.number.image, e.number.row, e.number.token})
    if (v < 0 || v >= (int64_t{1} << 50)) return LBP_ERR_SHAPE;
  if (e.number.token == 0 && (e.number.image != 0 || e.number.row != 0)) return LBP_ERR_SHAPE;   // (would read as dense)
  for (int64_t v : {e.first, e.number.image, e.number.row, e.number.token})
    if (!in_quads(v, dtype)) return LBP_ERR_ALIGN;
  if (((reinterpret_cast<uintptr_t>(e.seed_dev) | reinterpret_cast<uintptr_t>(e.offset_dev) |
        reinterpret_cast<uintptr_t>(e.used)) & 7u) != 0)
    return LBP_ERR_ALIGN;
  // (one thread writes it while others still read)
  for (const uint64_t* q : {e.seed_dev, e.offset_dev})
    if (e.used != nullptr && (q == e.used || q == e.used + 1)) return LBP_ERR_OVERLAP;
  return LBP_OK;
}

static Drop drop_of(const lbp_epilogue& e) {
  // t = p 2^16, to the nearest
  const long t = std::lround(static_cast<double>(e.p) * 65536.0);
  Drop d{};
  d.seed = e.seed;
  d.offset = e.offset;
  d.seed_dev = e.seed_dev;
  d.offset_dev = e.offset_dev;
  d.used = e.used;
  d.on = t > 0;
  d.above = static_cast<uint32_t>(static_cast<uint64_t>(t > 0 ? t : 1) * 65536u - 1u);
  // (t = 2^16: a bound that no half reaches)
  d.low15 = t < 65536 ? static_cast<uint32_t>(t & 0x7fff) * 0x10001u : 0x80008000u;
  d.low_half = t < 32768 ? 0x80008000u : 0u;
  d.scale = t < 65536 ? static_cast<float>(65536.0 / static_cast<double>(65536 - t)) : 0.f;
  return d;
}

// The bytes of `rows` rows at p: runs of `width`, `pitch` apart, from lo to hi.
struct Range {
  uintptr_t lo, hi, width, pitch;
};
static Range range(const void* p, long long rows, int64_t pitch, int C, int dtype) {
  const uintptr_t lo = reinterpret_cast<uintptr_t>(p), es = elem_size(dtype);
  if (p == nullptr || rows == 0) return Range{};
  return Range{lo, lo + (static_cast<uintptr_t>(rows - 1) * pitch + C) * es, C * es, static_cast<uintptr_t>(pitch) * es};
}
static bool overlap(const Range& a, const Range& b) {
  if (a.lo >= b.hi || b.lo >= a.hi) return false;
  if (a.pitch != b.pitch || a.pitch == 0) return true;
  // columns of one wide matrix: how far b's runs start behind a's
  const uintptr_t behind = b.lo >= a.lo ? (b.lo - a.lo) % a.pitch : (a.pitch - (a.lo - b.lo) % a.pitch) % a.pitch;
  return behind < a.width || behind + b.width > a.pitch;
}

static lbp_view rows_at(int64_t pitch) { return lbp_view{pitch, 0, 0}; }

// drop(a) act'(z) (+ residual) on rows, after its checks.
static int run_rows(const void* a, const void* z, const void* residual, void* out, long long rows, int C, int dtype,
                    int64_t pa, int64_t pz, int64_t pr, int64_t po, const lbp_epilogue& e, cudaStream_t st) {
  PointCall c{};
  c.a = a;
  c.z = z;
  c.residual = residual;
  c.out = out;
  c.rows = rows;
  c.C = C;
  c.HW = c.W = 1;
  c.dtype = dtype;
  c.act = e.act;
  c.va = rows_at(pa ? pa : C);
  c.vz = rows_at(pz ? pz : C);
  c.vr = rows_at(pr ? pr : C);
  c.vo = rows_at(po ? po : C);
  c.number = rows_at(e.number.token ? e.number.token : C);
  c.first = e.first;
  c.drop = drop_of(e);
  return launch_pointwise(c, st);
}

// Whether g_y and z of a call on rows are as they should be.
static int check_pointwise(const void* a, const void* b, bool need_b, const void* out, long long rows, int C, int dtype,
                           const lbp_pitches& p, int64_t pa, int64_t pb, int64_t po, const lbp_epilogue& e) {
  if (int s = check_rows(rows, C, dtype)) return s;
  if (int s = check_epilogue(e, dtype)) return s;
  if (int s = check_numbers(e.first, along_rows(rows, e.number.token ? e.number.token : C), C)) return s;
  for (int64_t v : {p.x, p.residual, p.y, p.z})
    if (int s = check_pitch(rows, v, C, dtype)) return s;
  if (rows == 0) return LBP_OK;
  if (a == nullptr || out == nullptr || (need_b && b == nullptr)) return LBP_ERR_NULL;
  if (!aligned16(a) || !aligned16(b) || !aligned16(out)) return LBP_ERR_ALIGN;
  // in place, or apart
  const Range ro = range(out, rows, po ? po : C, C, dtype);
  const auto bad = [&](const void* q, int64_t pq) {
    return overlap(ro, range(q, rows, pq ? pq : C, C, dtype)) && (q != out || (pq ? pq : C) != (po ? po : C));
  };
  return bad(a, pa) || bad(b, pb) ? LBP_ERR_OVERLAP : LBP_OK;
}

// Whether a token's place in its image has 31 bits.
static bool fits_grid(int H, int W) { return static_cast<long long>(H) * W < (1ll << 31); }
static int check_shape(int B, int H, int W, int C, int k, int dtype) {
  if (int s = check_order(k)) return s;
  if (B <= 0 || H <= 0 || W <= 0) return LBP_ERR_SHAPE;
  if (!fits_grid(H, W)) return LBP_ERR_SHAPE;
  return check_rows(static_cast<long long>(B) * H * W, C, dtype);
}
static int check_grid_view(const lbp_view& v, int B, int H, int W, int C, int dtype) {
  if (v.image == 0 && v.row == 0 && v.token == 0) return LBP_OK;
  if (v.image <= 0 || v.row <= 0 || v.token < C) return LBP_ERR_SHAPE;
  for (int64_t s : {v.image, v.row, v.token}) {
    if (s >= (int64_t{1} << 40) / elem_size(dtype)) return LBP_ERR_SHAPE;
    if ((s * elem_size(dtype)) % 16 != 0) return LBP_ERR_ALIGN;
  }
  return extent(along_grid(B, H, W, v), C) > kMostPlaces ? LBP_ERR_SHAPE : LBP_OK;
}

// g_z = drop(g_y) act'(z) of a token grid into a dense tensor.
static int run_grid(const void* g_y, const void* z, void* g_z, int B, int H, int W, int C, int dtype,
                    const lbp_view* view, const lbp_epilogue& e, cudaStream_t st) {
  PointCall c{};
  c.a = g_y;
  c.z = z;
  c.out = g_z;
  c.rows = static_cast<long long>(B) * H * W;
  c.C = C;
  c.HW = H * W;
  c.W = W;
  c.dtype = dtype;
  c.act = e.act;
  c.va = c.vz = resolve_view(view, H, W, C);
  c.vo = resolve_view(nullptr, H, W, C);
  c.number = resolve_view(&e.number, H, W, C);
  c.first = e.first;
  c.drop = drop_of(e);
  return launch_pointwise(c, st);
}

static GradOf grad_of(const void* z, int H, int W, int C, const lbp_epilogue& e) {
  return GradOf{e.act != LBP_ACT_NONE ? z : nullptr, e.act, e.first, resolve_view(&e.number, H, W, C), drop_of(e)};
}

// Whether g_z is g_y.
static bool does_nothing(const lbp_epilogue& e) { return e.act == LBP_ACT_NONE && !drop_of(e).on && e.used == nullptr; }

static size_t grid_bytes(long long tokens, int C, int dtype) {
  return align_up(static_cast<size_t>(tokens) * C * elem_size(dtype), 1024);
}

// What lbp_backward_act hands on: the extras of the call on g_z, which lies dense.
static lbp_extras with_dense_gradient(const lbp_extras* ex) {
  lbp_extras d = ex != nullptr ? *ex : lbp_extras{};
  d.gy_view = lbp_view{0, 0, 0};
  d.gy_extra_pitch = 0;
  return d;
}
// Whether the projection of lbp_backward_act may form the gradient of the grid's tokens itself.  (The sum for a bias
// then has to come from the coefficients: only with the basis (0, 0) among them.)
static bool may_form(const lbp_layer& L, int r, bool x_hat) {
  return project_forms_gradient(L.dtype, L.B, L.H, L.W, L.k, r) && (x_hat || r < L.k * L.k);
}
// Workspace of the call on g_z, dense or with g_y's strides.
static size_t inner_bytes(const lbp_layer* layer, int r, const lbp_extras* ex, bool x_hat) {
  const auto of = x_hat ? lbp_workspace_bytes_projected : lbp_workspace_bytes_ex;
  const lbp_extras d = with_dense_gradient(ex);
  const size_t as_given = of(layer, r, ex), dense = of(layer, r, &d);
  return as_given == 0 || dense == 0 ? 0 : align_up(as_given > dense ? as_given : dense, 1024);
}

}  // namespace layer
}  // namespace lbp

using namespace lbp;
using namespace lbp::layer;

extern "C" {

size_t lbp_linear_workspace_bytes(long long rows, int Cin, int Cout, int dtype) {
  if (check_rows(rows, Cin, dtype) != LBP_OK || check_rows(rows, Cout, dtype) != LBP_OK) return 0;
  return kStatusBytes + linear_scratch_bytes(rows, Cin, Cout, dtype);
}

int lbp_linear(const void* x, const void* W, const void* bias, const void* residual, void* y, void* z,
               long long rows, int Cin, int Cout, int dtype, const lbp_pitches* pitch,
               const lbp_epilogue* epilogue, void* ws, size_t ws_bytes, void* stream) {
  const lbp_epilogue& e = epilogue != nullptr ? *epilogue : kNoEpilogue;
  const lbp_pitches& p = pitch != nullptr ? *pitch : kDense;
  if (int s = check_rows(rows, Cin, dtype)) return s;
  if (int s = check_rows(rows, Cout, dtype)) return s;
  if (int s = check_epilogue(e, dtype)) return s;
  if (int s = check_numbers(e.first, along_rows(rows, e.number.token ? e.number.token : Cout), Cout)) return s;
  if (int s = check_pitch(rows, p.x, Cin, dtype)) return s;
  for (int64_t v : {p.residual, p.y, p.z})
    if (int s = check_pitch(rows, v, Cout, dtype)) return s;
  if (rows == 0) return LBP_OK;
  if (x == nullptr || W == nullptr || y == nullptr) return LBP_ERR_NULL;
  for (const void* q : {x, W, bias, residual, static_cast<const void*>(y), static_cast<const void*>(z),
                        static_cast<const void*>(ws)})
    if (!aligned16(q)) return LBP_ERR_ALIGN;
  LinearCall c{};
  c.px = p.x ? p.x : Cin;
  c.pr = p.residual ? p.residual : Cout;
  c.py = p.y ? p.y : Cout;
  c.pz = p.z ? p.z : Cout;
  const Range out[2] = {range(y, rows, c.py, Cout, dtype), range(z, rows, c.pz, Cout, dtype)};
  const Range in[4] = {range(x, rows, c.px, Cin, dtype), range(W, Cout, Cin, Cin, dtype), range(bias, 1, Cout, Cout, dtype),
                       range(residual, rows, c.pr, Cout, dtype)};
  const bool in_place = residual == y && c.pr == c.py;
  for (int o = 0; o < 2; ++o)
    for (int i = 0; i < 4; ++i)
      if (overlap(out[o], in[i]) && !(o == 0 && i == 3 && in_place)) return LBP_ERR_OVERLAP;
  if (overlap(out[0], out[1])) return LBP_ERR_OVERLAP;
  const size_t need = lbp_linear_workspace_bytes(rows, Cin, Cout, dtype);
  if (ws == nullptr || ws_bytes < need) return LBP_ERR_WORKSPACE;
  const Range scratch{reinterpret_cast<uintptr_t>(ws), reinterpret_cast<uintptr_t>(ws) + need, need, 0};
  for (const Range& q : {out[0], out[1], in[0], in[1], in[2], in[3]})
    if (overlap(scratch, q)) return LBP_ERR_OVERLAP;
  if (int s = check_device_arch()) return s;
  c.x = x;
  c.W = W;
  c.bias = bias;
  c.residual = residual;
  c.y = y;
  c.z = z;
  c.rows = rows;
  c.Cin = Cin;
  c.Cout = Cout;
  c.dtype = dtype;
  c.act = e.act;
  c.first = e.first;
  c.step = e.number.token ? e.number.token : Cout;
  c.drop = drop_of(e);
  c.status = static_cast<uint32_t*>(ws);
  c.scratch = static_cast<uint8_t*>(ws) + kStatusBytes;
  c.scratch_bytes = ws_bytes - kStatusBytes;
  return launch_linear(c, static_cast<cudaStream_t>(stream));
}

int lbp_linear_grad(const void* g_y, const void* z, void* g_z, long long rows, int C, int dtype,
                    const lbp_pitches* pitch, const lbp_epilogue* epilogue, void* stream) {
  const lbp_epilogue& e = epilogue != nullptr ? *epilogue : kNoEpilogue;
  const lbp_pitches& p = pitch != nullptr ? *pitch : kDense;
  if (int s = check_pointwise(g_y, z, e.act != LBP_ACT_NONE, g_z, rows, C, dtype, p, p.y, p.z, p.x, e)) return s;
  if (rows == 0) return LBP_OK;
  if (int s = check_device_arch()) return s;
  return run_rows(g_y, z, nullptr, g_z, rows, C, dtype, p.y, p.z, 0, p.x, e, static_cast<cudaStream_t>(stream));
}

int lbp_dropout(const void* x, const void* residual, void* y, long long rows, int C, int dtype,
                const lbp_pitches* pitch, const lbp_epilogue* epilogue, void* stream) {
  const lbp_epilogue& e = epilogue != nullptr ? *epilogue : kNoEpilogue;
  const lbp_pitches& p = pitch != nullptr ? *pitch : kDense;
  if (e.act != LBP_ACT_NONE) return LBP_ERR_SHAPE;
  if (int s = check_pointwise(x, residual, false, y, rows, C, dtype, p, p.x, p.residual, p.y, e)) return s;
  if (rows == 0) return LBP_OK;
  if (int s = check_device_arch()) return s;
  return run_rows(x, nullptr, residual, y, rows, C, dtype, p.x, 0, p.residual, p.y, e, static_cast<cudaStream_t>(stream));
}

size_t lbp_project_grad_workspace_bytes(int B, int H, int W, int C, int k, int r, int dtype) {
  if (check_shape(B, H, W, C, k, dtype) != LBP_OK || r < 1 || r > k * k) return 0;
  // where the projection does not form it, the gradient lies behind the status block
  return project_forms_gradient(dtype, B, H, W, k, r) ? kStatusBytes
                                                      : 1024 + grid_bytes(static_cast<long long>(B) * H * W, C, dtype);
}

int lbp_project_grad(const void* g_y, const void* z, void* t_hat, int B, int H, int W, int C, int k,
                     const lbp_basis* set, int r, int dtype, const lbp_view* view,
                     const lbp_epilogue* epilogue, void* ws, size_t ws_bytes, void* stream) {
  const lbp_epilogue& e = epilogue != nullptr ? *epilogue : kNoEpilogue;
  if (g_y == nullptr || t_hat == nullptr || (z == nullptr && e.act != LBP_ACT_NONE)) return LBP_ERR_NULL;
  if (int s = check_shape(B, H, W, C, k, dtype)) return s;
  if (int s = check_epilogue(e, dtype)) return s;
  if (int s = check_numbers(e.first, along_grid(B, H, W, resolve_view(&e.number, H, W, C)), C)) return s;
  if (view != nullptr)
    if (int s = check_grid_view(*view, B, H, W, C, dtype)) return s;
  BasisPlan plan;
  if (int s = make_basis_plan(k, set, r, &plan)) return s;
  if (!aligned16(g_y) || !aligned16(z) || !aligned16(t_hat) || !aligned16(ws)) return LBP_ERR_ALIGN;
  if (ws == nullptr || ws_bytes < lbp_project_grad_workspace_bytes(B, H, W, C, k, r, dtype)) return LBP_ERR_WORKSPACE;
  if (int s = check_device_arch()) return s;
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  const GradOf of = grad_of(z, H, W, C, e);
  const bool as_it_is = does_nothing(e);
  if (as_it_is || project_forms_gradient(dtype, B, H, W, k, r)) {
    if (!as_it_is) set_projection_gradient(&of);
    const int s = launch_project(g_y, t_hat, dtype, B, H, W, C, plan, static_cast<uint32_t*>(ws), st, 0.f, view);
    set_projection_gradient(nullptr);
    return s;
  }
  void* const g_z = static_cast<uint8_t*>(ws) + 1024;
  if (int s = run_grid(g_y, z, g_z, B, H, W, C, dtype, view, e, st)) return s;
  return launch_project(g_z, t_hat, dtype, B, H, W, C, plan, static_cast<uint32_t*>(ws), st);
}

size_t lbp_workspace_bytes_act(const lbp_layer* layer, int r, const lbp_extras* ex, int x_hat) {
  const lbp_extras d = with_dense_gradient(ex);
  const size_t inner = inner_bytes(layer, r, ex, x_hat != 0);
  if (inner == 0 || !fits_grid(layer->H, layer->W)) return 0;
  return inner + grid_bytes(d.n_extra, layer->Cout, layer->dtype) +
         (may_form(*layer, r, x_hat != 0) && d.g_bias == nullptr
              ? 0
              : grid_bytes(static_cast<long long>(layer->B) * layer->H * layer->W, layer->Cout, layer->dtype));
}

int lbp_backward_act(const void* x, const void* x_hat, const void* g_y, const void* W, void* g_x, void* g_W,
                     const lbp_layer* layer, const lbp_basis* set, int r, const lbp_extras* ex,
                     const lbp_layer_grad* grad, void* ws, size_t ws_bytes, void* stream) {
  if (grad == nullptr || layer == nullptr || g_y == nullptr) return LBP_ERR_NULL;
  const lbp_epilogue& e = grad->epilogue;
  const bool has_act = e.act != LBP_ACT_NONE;
  if (int s = check_epilogue(e, layer->dtype)) return s;
  const int n_extra = ex != nullptr ? ex->n_extra : 0, dtype = layer->dtype, C = layer->Cout;
  if (has_act && (grad->z == nullptr || (n_extra > 0 && grad->z_extra == nullptr))) return LBP_ERR_NULL;
  if (!aligned16(grad->z) || !aligned16(grad->z_extra)) return LBP_ERR_ALIGN;
  if (grad->first_extra < 0 || grad->first_extra >= kMostElements || grad->number_extra < 0 ||
      grad->number_extra >= (int64_t{1} << 50))
    return LBP_ERR_SHAPE;
  if (!in_quads(grad->first_extra, dtype) || !in_quads(grad->number_extra, dtype)) return LBP_ERR_ALIGN;
  if (n_extra > 0)
    if (int s = check_pitch(n_extra, ex->gy_extra_pitch, C, dtype)) return s;
  // the call as it is, for what is wrong with it apart from the epilogue
  if (int s = backward_ex_call(x, x_hat, g_y, W, g_x, g_W, layer, set, r, ex, ws, ws_bytes, stream, true)) return s;
  const size_t need = lbp_workspace_bytes_act(layer, r, ex, x_hat != nullptr);
  if (!fits_grid(layer->H, layer->W)) return LBP_ERR_SHAPE;
  if (int s = check_numbers(e.first, along_grid(layer->B, layer->H, layer->W, resolve_view(&e.number, layer->H, layer->W, C)), C))
    return s;
  if (int s = check_numbers(grad->first_extra, along_rows(n_extra, grad->number_extra ? grad->number_extra : C), C)) return s;
  if (need == 0 || ws_bytes < need) return LBP_ERR_WORKSPACE;
  if (int s = check_device_arch()) return s;
  if (does_nothing(e)) return backward_ex_call(x, x_hat, g_y, W, g_x, g_W, layer, set, r, ex, ws, ws_bytes, stream, false);
  cudaStream_t st = static_cast<cudaStream_t>(stream);
  lbp_extras d = with_dense_gradient(ex);
  const size_t inner = inner_bytes(layer, r, ex, x_hat != nullptr);
  uint8_t* const g_ze = static_cast<uint8_t*>(ws) + inner;
  if (n_extra > 0) {
    lbp_epilogue ee = e;
    ee.first = grad->first_extra;
    ee.number = lbp_view{0, 0, grad->number_extra};
    ee.used = nullptr;
    if (int s = run_rows(ex->gy_extra, grad->z_extra, nullptr, g_ze, n_extra, C, dtype, ex->gy_extra_pitch,
                         ex->gy_extra_pitch, 0, 0, ee, st))
      return s;
    d.gy_extra = g_ze;
  }
  bool dc = false;
  for (int q = 0; q < r; ++q) dc |= set[q].i == 0 && set[q].j == 0;
  if (may_form(*layer, r, x_hat != nullptr) && (dc || d.g_bias == nullptr)) {
    d.gy_view = ex != nullptr ? ex->gy_view : lbp_view{0, 0, 0};
    const GradOf of = grad_of(grad->z, layer->H, layer->W, C, e);
    set_projection_gradient(&of);
    const int s = backward_ex_call(x, x_hat, g_y, W, g_x, g_W, layer, set, r, &d, ws, inner, stream, false);
    set_projection_gradient(nullptr);
    return s;
  }
  uint8_t* const g_z = g_ze + grid_bytes(n_extra, C, dtype);
  if (int s = run_grid(g_y, grad->z, g_z, layer->B, layer->H, layer->W, C, dtype, ex != nullptr ? &ex->gy_view : nullptr, e, st))
    return s;
  return backward_ex_call(x, x_hat, g_z, W, g_x, g_W, layer, set, r, &d, ws, inner, stream, false);
}

}  // extern "C"
