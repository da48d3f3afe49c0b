// The host-only half of the C ABI (see include/jenga.h): configuration checks, plan tables without a
// device, table export, status strings.  No HIP in this file, so that it can be built and run under
// the host sanitizers together with jenga_plan.cpp.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>

#include "jenga_internal.h"

namespace jenga {

bool config_ok(const jenga_config& c, int* why) {
  *why = JENGA_EINVAL;
  if (c.T < 1 || c.H < 1 || c.W < 1 || c.n_text < 0 || c.batch < 1 || c.heads < 1) return false;
  if (!(c.topk_ratio > 0.0 && c.topk_ratio <= 1.0)) return false;
  if (!(c.cum_prob >= 0.0 && c.cum_prob < 1.0)) return false;
  if (!std::isfinite(c.text_bias)) return false;   // NaN and +-inf: exp2(-inf + inf) would poison a row
  if (c.flags & ~15u) return false;
  *why = JENGA_EUNSUPPORTED;
  if (c.head_dim != 64 && c.head_dim != 128) return false;
  if (c.block != 32 && c.block != 64 && c.block != 128) return false;
  // at most 2^24 vision tokens; multiply step by step so that no product can overflow
  const long long lim = 1ll << 24;
  if (c.T > lim || c.H > lim || c.W > lim || (long long)c.T * c.H > lim) return false;
  const long long nv = (long long)c.T * c.H * c.W;
  if (nv > lim || c.n_text > (1 << 20)) return false;
  const long long M = (nv + c.block - 1) / c.block + (c.n_text + c.block - 1) / c.block;
  if (M > 2048) return false;   // select keeps a row of M block probabilities in one wavefront
  if ((long long)c.batch * c.heads > 65535) return false;
  return true;
}

// The largest group of output rows whose input rows fit the LDS tile.
StageTiles stage_switch_tiles(long long channels, int T_in, int H_in, int W_in, int T_out, int H_out, int W_out, bool on_16) {
  constexpr long long TILE_FLOATS = 12288;   // 48 KB of LDS for the staged clean-latent estimate
  auto window_len_max = [](long long n_in, long long n_out) { return (n_in + n_out - 1) / n_out + 1; };
  const unsigned quads_per_row = ((unsigned)W_out + 3u) / 4u;
  const long long nt_max = window_len_max(T_in, T_out);
  StageTiles s;
  s.rows_per_wg = quads_per_row >= 256u ? 1u : 256u / quads_per_row;
  if (s.rows_per_wg > (unsigned)H_out) s.rows_per_wg = (unsigned)H_out;
  auto tile_floats = [&](unsigned rows) {
    // input rows touched by `rows` consecutive output rows: at most floor((rows-1)*H_in/H_out) + window + 1
    const long long nh = ((long long)(rows - 1) * H_in) / H_out + window_len_max(H_in, H_out) + 1;
    const long long plane = (nh < H_in ? nh : H_in) * W_in;
    // rows off the 16-byte grid are read from the boundary below them
    return nt_max * (W_in % 4 == 0 ? plane : (plane + 6) & ~3ll);
  };
  while (s.rows_per_wg > 1 && tile_floats(s.rows_per_wg) > TILE_FLOATS) --s.rows_per_wg;
  s.floats = tile_floats(s.rows_per_wg);
  // Rows off the 16-byte grid: with the chip full a workgroup costs 1 to 1.8 ns however little it has to read and write,
  // and small planes are done sooner directly, above all where every window is a single cell.  Direct -> tiled, by the
  // larger of a quarter of the cells it reads and of those it writes:
  //   windows of one cell: 26214 x 8 x 2 x 5 -> 2 x 5 (2)     13 -> 214 us      1134 x 8 x 11 x 21 -> 11 x 21 (57)  10.7 -> 16.0 us
  //                        748 x 8 x 14 x 25 -> 14 x 25 (87)  10.8 -> 12.2 us   497 x 8 x 17 x 31 -> 17 x 31 (131)  10.4 -> 10.8 us
  //   others:              2880 x 8 x 7 x 13 -> 10 x 18 (45)  24.4 -> 27.6 us   8 x 33 x 3 -> 66 x 5 (82)            7 % slower
  //                        1134 x 8 x 11 x 21 -> 15 x 29 (109)  26 -> 16 us     227 x 8 x 18 x 33 -> 25 x 46 (252)  18.2 -> 9.8 us
  //                        16 x 33 x 45 x 79 -> 67 x 117 (614)  30 -> 13.6 us
  // No shape tried (W 1 to 1001, up, down and equal) was slower tiled from 192 and 96 on.
  const long long rows_in = std::min<long long>(H_in, ((long long)s.rows_per_wg * H_in + H_out - 1) / H_out);
  const long long read = std::max(1, T_in / T_out) * rows_in * W_in / 4, written = (long long)s.rows_per_wg * W_out / 4;
  const bool one_cell = T_out % T_in == 0 && H_out % H_in == 0 && W_out % W_in == 0;
  const bool worth_it = W_in % 4 == 0 || std::max(read, written) >= (one_cell ? 192 : 96);
  // a workgroup of 256 threads for every (channel, t) plane: below 2^32 threads in x, which a grid has to stay under
  s.tiled = on_16 && worth_it && s.floats <= TILE_FLOATS && channels * T_out < 1ll << 24;
  return s;
}

// Figures in us, with weights that no cache holds but where 256 x 256 is compared.
MatmulTiles matmul_tiles(int64_t m, int64_t n, bool float32) {
  auto tiles = [&](int bm, int bn) { return (m + bm - 1) / bm * ((n + bn - 1) / bn); };
  auto rounds = [](int64_t t, int at_once) { return (t + at_once - 1) / at_once; };
  // Up to 16 rows without tiles, up to 32 where their second reading by each 16 columns is short.  Rows -> 64 x 128: 16 x 5120 x 5120
  // 12.9 -> 20.8; 16 x 15360 24.0 -> 23.3; 20 x 1536 x 1536 6.8 -> 8.0; 20 x 5120 x 5120 16.4 -> 21.1; 32 19.1 -> 22.4; 32 x 9216 x 1536
  // 11.7 -> 9.5; 48 x 5120 x 5120 (three times 16) 24.8 -> 23.7.
  if (m <= 16) return {16, 0, 0, 0, 0};
  if (m <= 32 && n <= 6144) return {32, 0, 0, 0, 0};
  // Tiles of 256 x 256 read each row of either operand half as often as those of 128 x 128; a round of them (one a compute unit) takes 1.5 to
  // 1.65 times as long as a round of the others (two a unit).  256 -> 128, by rounds of either: 1 and 1, 1500 x 5120 x 5120 55.5 -> 40.7; 1 and 2, 2048
  // 57.5 -> 71.1, 3000 63.8 -> 78.2; 2 and 3, 4096 117.9 -> 112.0, 4864 121.5 -> 121.0, 4096 x 5120 x 1536 43.3 -> 38.6, 4500 x 4700 x 2048 62.8 ->
  // 57.2; 3 and 5, 9000 x 4000 x 4096 150.2 -> 150.9, 7000 x 5000 x 5120 187.2 -> 191.6; 2 and 4, 5120 x 5120 x 5120 119.6 -> 146.7; 31 and 61,
  // 33272 x 15360 2144 -> 2603.  (4 and 7, 11264 x 4608 x 1536 loses by it, 93.0 -> 89.6: a short k favours 128.)
  if (!float32 && 1.55 * rounds(tiles(256, 256), 256) <= rounds(tiles(128, 128), 512)) return {0, 256, 256, 2, 1};
  // No more tiles than units: one a unit, four LDS tiles deep, which is what hides the memory's latency then (two -> three -> four -> five ->
  // six deep: 64 x 5120 x 5120 40.2 -> 29.5 -> 25.4 -> 25.9 -> 26.2).  64 x 128, or 128 x 128 where the former are more than units.  64 x 128
  // two deep, two a unit -> four deep -> 128 x 128 four deep: 256 x 5120 x 5120 (160 and 80) 36.9 -> 23.5 -> 31.4; 400 (280 and 160) 36.9 ->
  // 37.6 -> 29.1; 900 x 4096 x 4096 (480 and 256) 31.4 -> 32.0 -> 24.1; float32 200 x 5120 x 5120 41.9 -> 31.2 -> 41.6, 900 x 4096 x 4096
  // 41.7 -> 50.9 -> 40.2.
  if (tiles(64, 128) <= 256) return {0, 64, 128, 4, 1};
  if (tiles(128, 128) <= 256) return {0, 128, 128, 4, 1};
  return {0, 128, 128, 2, 2};
}

// The same for 4-bit operands, whose products take half the time, so that a tile's start and end weigh more: a round of tiles of 256 x 256 takes
// 1.6 times as long as one of 128 x 128 at k of 8192, 1.7 to 1.77 at 4096 and 5120, 2 to 2.2 at 1536, 2.5 at 512.  256 -> 128, us, by rounds of either: 31 and 62, 33272 x
// 15360 x 5120 1403 -> 1740; 1 and 2, 2048 x 5120 x 5120 40.2 -> 45.6; 3 and 5, 9000 x 4000 x 4096 108 -> 102, 7000 x 5000 x 5120 132 -> 124; 4 and 7, 11264 x 4608 x
// 1536 75.0 -> 59.8; 2 and 4, 25000 x 1024 x 512 24.7 -> 19.9; 1 and 2, 600 x 16000 x 1024 17.9 -> 13.4.  Float32 results, twice the stores: 9 and 18, 31712 x 4608 x
// 1536 215 -> 195; 31 and 62, 33272 x 15360 x 5120 1612 -> 1992.
MatmulTiles matmul_mx_tiles(int64_t m, int64_t n, int64_t k, bool float32) {
  auto rounds = [&](int size, int at_once) {
    const int64_t tiles = (m + size - 1) / size * ((n + size - 1) / size);
    return (double)((tiles + at_once - 1) / at_once);
  };
  const MatmulTiles small = matmul_tiles(m, n, true);
  if (small.rows || small.stages == 4) return small;
  const double longer = float32 ? 1.8 + 500.0 / (double)k : 1.7 + 400.0 / (double)k;
  return longer * rounds(256, 256) <= rounds(128, 512) ? MatmulTiles{0, 256, 256, 2, 1} : small;
}

// ---- arguments of the calls around the attention

namespace {

constexpr int64_t MOST_COLS = 1 << 17, MOST_ROWS = 1ll << 40, MOST_STRIDE = 1ll << 40;

int type_size(int type) { return type == JENGA_F32 ? 4 : type == JENGA_E4M3 ? 1 : 2; }
bool float_type(int type) { return type == JENGA_BF16 || type == JENGA_F16 || type == JENGA_F32; }
bool aligned(const void* p, size_t to) { return (uintptr_t)p % to == 0; }

// `rows` rows of `width` bytes, `pitch` bytes apart.
struct Span {
  const void* at;
  int64_t rows, pitch, width;
  __int128 end() const { return (__int128)(uintptr_t)at + (__int128)(rows - 1) * pitch + width; }
};

// Whether two spans share a byte.  Rows of the same pitch may lie between each other's (columns of one matrix).
bool overlap(const Span& a, const Span& b) {
  if (!a.at || !b.at || a.rows < 1 || b.rows < 1) return false;
  if ((__int128)(uintptr_t)a.at >= b.end() || (__int128)(uintptr_t)b.at >= a.end()) return false;
  if (a.pitch == b.pitch && a.pitch > 0 && a.rows > 1 && b.rows > 1) {
    const int64_t p = a.pitch;
    const int64_t d = (int64_t)((((__int128)(uintptr_t)b.at - (__int128)(uintptr_t)a.at) % p + p) % p);   // b's columns behind a's
    if (d >= a.width && d + b.width <= p) return false;
  }
  return true;
}

int64_t groups_of(const jenga_norm_config& c) { return (c.rows + c.group_rows - 1) / c.group_rows; }

int norm_config_ok(const jenga_norm_config& c) {
  if (c.rows < 0 || c.group_rows < 1 || c.cols < 1) return JENGA_EINVAL;
  if (!float_type(c.x_type) || !(float_type(c.y_type) || c.y_type == JENGA_E4M3) || !float_type(c.param_type)) return JENGA_EINVAL;
  if (!std::isfinite(c.eps) || c.eps < 0.0f || !std::isfinite(c.weight_offset)) return JENGA_EINVAL;
  if (c.x_stride < c.cols || c.y_stride < c.cols || c.param_stride < c.cols) return JENGA_EINVAL;
  if (c.cols > MOST_COLS || c.rows > MOST_ROWS || c.group_rows > MOST_ROWS) return JENGA_EUNSUPPORTED;
  if (c.x_stride > MOST_STRIDE || c.y_stride > MOST_STRIDE || c.param_stride > MOST_STRIDE) return JENGA_EUNSUPPORTED;
  const __int128 lim = (__int128)1 << 60;   // bytes: offsets stay in 64 bits
  if ((__int128)c.rows * c.x_stride > lim || (__int128)c.rows * c.y_stride > lim || (__int128)c.rows * c.param_stride > lim)
    return JENGA_EUNSUPPORTED;
  if (c.y_type != c.x_type && c.y_type != JENGA_E4M3) return JENGA_EUNSUPPORTED;
  if (c.param_type != c.x_type && c.param_type != JENGA_F32) return JENGA_EUNSUPPORTED;
  return JENGA_OK;
}

}  // namespace

int norm_args_ok(const jenga_norm_config* c, const void* x, const void* weight, const void* bias, const void* y, const uint8_t* y_scale,
                 const float* mean, const float* rstd) {
  if (!c || !x || !y) return JENGA_EINVAL;
  const int why = norm_config_ok(*c);
  if (why != JENGA_OK) return why;
  const bool e4m3 = c->y_type == JENGA_E4M3;
  const int64_t padded = ((int64_t)c->cols + 127) / 128 * 128, scales = ((int64_t)c->cols + 511) / 512 * 4;
  if (e4m3 != (y_scale != nullptr) || (e4m3 && (c->y_stride != padded || !aligned(y, 16) || !aligned(y_scale, 4)))) return JENGA_EINVAL;
  const int xs = type_size(c->x_type), ys = type_size(c->y_type), ps = type_size(c->param_type);
  if (!aligned(x, xs) || !aligned(y, ys) || !aligned(weight, ps) || !aligned(bias, ps) || !aligned(mean, 4) || !aligned(rstd, 4))
    return JENGA_EINVAL;
  if (c->rows == 0) return JENGA_OK;
  const Span in[3] = {{x, c->rows, c->x_stride * xs, (int64_t)c->cols * xs},
                      {weight, groups_of(*c), c->param_stride * ps, (int64_t)c->cols * ps},
                      {bias, groups_of(*c), c->param_stride * ps, (int64_t)c->cols * ps}};
  const Span out[4] = {{y, c->rows, c->y_stride * ys, e4m3 ? padded : (int64_t)c->cols * ys}, {y_scale, c->rows, scales, scales},
                       {mean, 1, c->rows * 4, c->rows * 4}, {rstd, 1, c->rows * 4, c->rows * 4}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 3; ++j)
      if (overlap(out[i], in[j]) && !(i == 0 && j == 0 && x == y && !e4m3 && c->x_stride == c->y_stride)) return JENGA_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return JENGA_EINVAL;
  }
  return JENGA_OK;
}

int norm_grad_args_ok(const jenga_norm_config* c, const void* x, const void* dy, const void* weight, const float* mean,
                      const float* rstd, const void* dx, const float* dweight, const float* dbias, const void* workspace,
                      size_t workspace_bytes) {
  if (!c || !x || !dy || !mean || !rstd || !dx) return JENGA_EINVAL;
  const int why = norm_config_ok(*c);
  if (why != JENGA_OK) return why;
  if (c->y_type != c->x_type) return JENGA_EUNSUPPORTED;
  const int xs = type_size(c->x_type), ps = type_size(c->param_type);
  if (!aligned(x, xs) || !aligned(dy, xs) || !aligned(dx, xs) || !aligned(weight, ps) || !aligned(mean, 4) || !aligned(rstd, 4) ||
      !aligned(dweight, 4) || !aligned(dbias, 4))
    return JENGA_EINVAL;
  if (c->rows == 0) return JENGA_OK;
  const int64_t groups = groups_of(*c);
  if (groups > 1 << 20) return JENGA_EUNSUPPORTED;
  uint64_t need = 0;
  if (dweight || dbias) {
    if (!workspace || !aligned(workspace, 256)) return JENGA_EINVAL;
    need = (uint64_t)(1024 + groups) * c->cols * 8;
  }
  const int64_t width = (int64_t)c->cols * xs, sums = groups * c->cols * 4;
  const Span in[5] = {{x, c->rows, c->x_stride * xs, width}, {dy, c->rows, c->y_stride * xs, width},
                      {weight, groups, c->param_stride * ps, (int64_t)c->cols * ps}, {mean, 1, c->rows * 4, c->rows * 4},
                      {rstd, 1, c->rows * 4, c->rows * 4}};
  const Span out[4] = {{dx, c->rows, c->x_stride * xs, width}, {dweight, 1, sums, sums}, {dbias, 1, sums, sums},
                       {need ? workspace : nullptr, 1, (int64_t)need, (int64_t)need}};
  for (int i = 0; i < 4; ++i) {
    for (int j = 0; j < 5; ++j)
      if (overlap(out[i], in[j])) return JENGA_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i], out[j])) return JENGA_EINVAL;
  }
  return workspace_bytes < need ? JENGA_EWORKSPACE : JENGA_OK;
}

int quantize_args_ok(const void* x, int64_t x_stride, int32_t x_type, int64_t rows, int32_t cols, int32_t block_rows, const void* q,
                     const uint8_t* scale) {
  if (!x || !q || !scale || rows < 0 || cols < 1 || x_stride < cols || (block_rows != 1 && block_rows != 128)) return JENGA_EINVAL;
  if (!float_type(x_type) || !aligned(x, type_size(x_type)) || !aligned(q, 16) || !aligned(scale, 4)) return JENGA_EINVAL;
  if (cols > MOST_COLS || rows > 1ll << 30 || x_stride > 1ll << 28) return JENGA_EUNSUPPORTED;
  if (rows == 0) return JENGA_OK;
  const int64_t size = type_size(x_type), padded = ((int64_t)cols + 127) / 128 * 128, scales = ((int64_t)cols + 511) / 512 * 4;
  const Span from = {x, rows, x_stride * size, cols * size}, to = {q, rows, padded, padded},
             bytes = {scale, block_rows == 1 ? rows : (rows + 127) / 128, scales, scales};
  return overlap(from, to) || overlap(from, bytes) || overlap(to, bytes) ? JENGA_EINVAL : JENGA_OK;
}

int matmul_args_ok(const jenga_matmul_config* c, const void* a, const uint8_t* a_scale, const void* b, const uint8_t* b_scale,
                   const float* bias, const void* out) {
  if (!c || !a || !a_scale || !b || !b_scale || !out) return JENGA_EINVAL;
  if (c->m < 0 || c->n < 1 || c->k < 1 || c->k % 128 != 0 || c->out_stride < c->n || c->reserved != 0) return JENGA_EINVAL;
  if (!float_type(c->out_type)) return JENGA_EINVAL;
  const int64_t size = type_size(c->out_type);
  if (!aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 4) || !aligned(b_scale, 4) || !aligned(bias, 4) || !aligned(out, size))
    return JENGA_EINVAL;
  if (c->k > MOST_COLS || c->m > 1ll << 30 || c->n > 1 << 22 || c->out_stride > 1ll << 31) return JENGA_EUNSUPPORTED;
  if ((c->m + 127) / 128 * (((int64_t)c->n + 127) / 128) > 1ll << 23) return JENGA_EUNSUPPORTED;
  if (c->m == 0) return JENGA_OK;
  const int64_t scales = ((int64_t)c->k + 511) / 512 * 4;
  const Span to = {out, c->m, c->out_stride * size, c->n * size};
  const Span in[5] = {{a, c->m, c->k, c->k}, {a_scale, c->m, scales, scales}, {b, c->n, c->k, c->k},
                      {b_scale, ((int64_t)c->n + 127) / 128, scales, scales}, {bias, 1, (int64_t)c->n * 4, (int64_t)c->n * 4}};
  for (const Span& s : in)
    if (overlap(to, s)) return JENGA_EINVAL;
  return JENGA_OK;
}

int rotary_config_ok(const jenga_rotary_config* c) {
  if (!c) return JENGA_EINVAL;
  if (c->T < 1 || c->H < 1 || c->W < 1 || c->head_dim < 1 || !float_type(c->type) || c->reserved != 0) return JENGA_EINVAL;
  if (c->flags & ~(uint32_t)(JENGA_ROTARY_HALVES | JENGA_ROTARY_INVERSE)) return JENGA_EINVAL;
  if (!std::isfinite(c->theta) || c->theta <= 0.0) return JENGA_EINVAL;
  int64_t dims = 0;
  for (int i = 0; i < 3; ++i) {
    if (!std::isfinite(c->origin[i]) || !std::isfinite(c->step[i])) return JENGA_EINVAL;
    if (c->dim[i] < 0 || c->dim[i] % 2 != 0) return JENGA_EINVAL;
    dims += c->dim[i];
  }
  if (dims < 1 || dims > c->head_dim) return JENGA_EINVAL;
  const int64_t lim = 1ll << 24;
  if (c->head_dim % 2 != 0 || c->head_dim > 1024) return JENGA_EUNSUPPORTED;
  if (c->T > lim || c->H > lim || c->W > lim || (int64_t)c->T * c->H > lim || (int64_t)c->T * c->H * c->W > lim) return JENGA_EUNSUPPORTED;
  // the kernels' places in the table are 32-bit numbers: all its pairs, and up to 1023 that no axis has behind them
  if (((int64_t)c->T * c->dim[0] + (int64_t)c->H * c->dim[1] + (int64_t)c->W * c->dim[2]) / 2 > (1ll << 31) - 1024) return JENGA_EUNSUPPORTED;
  return JENGA_OK;
}

namespace {

// A tensor [batch][tokens][heads][head_dim] of one rotary call.
struct Layout4 {
  const void* at;
  int64_t batch, token, head;   // strides
  int64_t n[3];                 // batch, tokens, heads
  int64_t width, size;          // head_dim, bytes of an element
  int64_t end() const { return (n[0] - 1) * batch + (n[1] - 1) * token + (n[2] - 1) * head + width; }

  // The same bytes as rows of a common pitch, where the heads of a token lie within one token stride.
  Span rows() const {
    const int64_t row = (n[2] - 1) * head + width;
    if (n[1] > 1 && row <= token && (n[0] == 1 || (batch % token == 0 && batch >= n[1] * token)))
      return {at, n[0] == 1 ? n[1] : (n[0] - 1) * (batch / token) + n[1], token * size, row * size};
    return {at, 1, end() * size, end() * size};
  }
};

// The steps of two tensors along one axis.
struct Axis {
  int64_t stride, a, b;       // entries of either tensor
  int64_t reach_a, reach_b;   // elements from the first to behind the last one of all axes behind this one
};
constexpr int MOST_STEPS = 16;

// Whether steps along the axes bring rows of `width` elements over each other that start `apart` elements from each other.  Steps of an outer
// axis leave few distances that the inner ones can bridge, two at most where strides are nested; more than MOST_STEPS are not looked
// through, which refuses a call rather than take a wrong one.
bool meet(const Axis* axis, int axes, __int128 apart, int64_t width) {
  if (axes == 0) return apart < width && -apart < width;
  const __int128 s = axis->stride, from = apart - axis->reach_a, to = apart + axis->reach_b;   // wanted: t with from < s t < to
  auto floor_div = [](__int128 x, __int128 y) { return x / y - (x % y != 0 && x < 0); };
  const __int128 first = std::max<__int128>(floor_div(from, s) + 1, 1 - (__int128)axis->b);
  const __int128 last = std::min<__int128>(-floor_div(-to, s) - 1, (__int128)axis->a - 1);
  if (last - first >= MOST_STEPS) return true;
  for (__int128 t = first; t <= last; ++t)
    if (meet(axis + 1, axes - 1, apart - s * t, width)) return true;
  return false;
}

// The axes of two tensors, the outermost first, without those along which there is nothing to step; -1: their strides differ.
int common_axes(const Layout4& a, const Layout4& b, Axis axis[3]) {
  const int64_t of_a[3] = {a.batch, a.token, a.head}, of_b[3] = {b.batch, b.token, b.head};
  int axes = 0;
  for (int i = 0; i < 3; ++i) {
    const int64_t na = of_a[i] == 0 ? 1 : a.n[i], nb = of_b[i] == 0 ? 1 : b.n[i];   // stride 0: all in one place
    if (na == 1 && nb == 1) continue;
    if (na > 1 && nb > 1 && of_a[i] != of_b[i]) return -1;
    axis[axes++] = {na > 1 ? of_a[i] : of_b[i], na, nb, 0, 0};
  }
  std::sort(axis, axis + axes, [](const Axis& x, const Axis& y) { return x.stride > y.stride; });
  int64_t reach_a = a.width, reach_b = b.width;
  for (int i = axes - 1; i >= 0; --i) {
    axis[i].reach_a = reach_a;
    axis[i].reach_b = reach_b;
    reach_a += (axis[i].a - 1) * axis[i].stride;
    reach_b += (axis[i].b - 1) * axis[i].stride;
  }
  return axes;
}

// Whether two tensors may share an element: not where they are rows of a common pitch that lie between each other's, nor where they have
// the same strides and no steps of them lead from the one to the other.
bool share(const Layout4& a, const Layout4& b) {
  if (!overlap(a.rows(), b.rows())) return false;
  Axis axis[3];
  const int axes = common_axes(a, b, axis);
  return axes < 0 || meet(axis, axes, ((__int128)(uintptr_t)b.at - (__int128)(uintptr_t)a.at) / a.size, a.width);
}

// No two elements of a tensor in one place: no steps along an axis that those along the smaller strides undo.
bool distinct(const Layout4& a) {
  for (int i = 0; i < 3; ++i)
    if (a.n[i] > 1 && (i == 0 ? a.batch : i == 1 ? a.token : a.head) == 0) return false;
  Axis axis[3];
  const int axes = common_axes(a, a, axis);
  for (int i = 0; i < axes; ++i) {
    const int64_t most = std::min(axis[i].a - 1, (axis[i].reach_a - 1) / axis[i].stride);   // further ones are behind all of them
    if (most > MOST_STEPS) return false;
    for (int64_t t = 1; t <= most; ++t)
      if (meet(axis + i + 1, axes - i - 1, (__int128)t * axis[i].stride, a.width)) return false;
  }
  return true;
}

}  // namespace

int rotary_args_ok(const jenga_rotary_config* c, const jenga_plan* plan, const int32_t* cells, const float* table,
                   const jenga_rotary_tensor* tensors, int32_t count, int64_t batch, int64_t tokens) {
  const int why = rotary_config_ok(c);
  if (why != JENGA_OK) return why;
  if (!table || !tensors || count < 1 || count > 2 || batch < 0 || tokens < 0 || (plan && cells)) return JENGA_EINVAL;
  if (!aligned(table, 8) || !aligned(cells, 4)) return JENGA_EINVAL;
  if (plan && (plan->cfg.T != c->T || plan->cfg.H != c->H || plan->cfg.W != c->W || plan->info.N_pad != tokens)) return JENGA_EINVAL;
  if (batch > 1ll << 31 || tokens > 1ll << 31) return JENGA_EUNSUPPORTED;
  if (batch > 0 && tokens > 0 && (__int128)batch * tokens * (c->head_dim / 2) > (__int128)0xFFFFFF00u) return JENGA_EUNSUPPORTED;
  const int64_t size = type_size(c->type);
  Layout4 src[2], dst[2];
  for (int i = 0; i < count; ++i) {
    const jenga_rotary_tensor& t = tensors[i];
    if (!t.src || !t.dst || t.heads < 1 || t.reserved != 0 || !aligned(t.src, size) || !aligned(t.dst, size)) return JENGA_EINVAL;
    const int64_t strides[6] = {t.src_batch, t.src_token, t.src_head, t.dst_batch, t.dst_token, t.dst_head};
    for (const int64_t s : strides) {
      if (s < 0) return JENGA_EINVAL;
      if (s > MOST_STRIDE) return JENGA_EUNSUPPORTED;
    }
    if (t.heads > 65535 * 8) return JENGA_EUNSUPPORTED;
    if (batch == 0 || tokens == 0) continue;
    const __int128 lim = (__int128)1 << 60;
    if ((__int128)t.src_batch * batch + (__int128)t.src_token * tokens + (__int128)t.src_head * t.heads > lim ||
        (__int128)t.dst_batch * batch + (__int128)t.dst_token * tokens + (__int128)t.dst_head * t.heads > lim)
      return JENGA_EUNSUPPORTED;
    src[i] = {t.src, t.src_batch, t.src_token, t.src_head, {batch, tokens, t.heads}, c->head_dim, size};
    dst[i] = {t.dst, t.dst_batch, t.dst_token, t.dst_head, {batch, tokens, t.heads}, c->head_dim, size};
    if (!distinct(dst[i])) return JENGA_EINVAL;
  }
  if (batch == 0 || tokens == 0) return JENGA_OK;
  const int64_t n_table = (int64_t)c->T * c->dim[0] + (int64_t)c->H * c->dim[1] + (int64_t)c->W * c->dim[2];
  const Span angles = {table, 1, n_table * 4, n_table * 4}, where = {cells, 1, batch * tokens * 12, batch * tokens * 12};
  for (int i = 0; i < count; ++i) {
    const Span to = dst[i].rows();
    if ((n_table > 0 && overlap(to, angles)) || overlap(to, where)) return JENGA_EINVAL;
    for (int j = 0; j < count; ++j) {
      const bool in_place = i == j && src[i].at == dst[i].at && (batch == 1 || src[i].batch == dst[i].batch) &&
                            (tokens == 1 || src[i].token == dst[i].token) && (tensors[i].heads == 1 || src[i].head == dst[i].head);
      if (!in_place && share(dst[i], src[j])) return JENGA_EINVAL;
      if (j < i && share(dst[i], dst[j])) return JENGA_EINVAL;
    }
  }
  return JENGA_OK;
}

// ---- the norm without a mean, 4-bit products, dense attention

namespace {

constexpr int RMS_PARTS = 1024;   // workgroups that leave sums of the weight's gradient, at most

// Rows and heads of a tensor as one of the calls sees them; null where there is none.
Layout4 rows_and_heads(const void* at, int64_t row, int64_t head, int64_t rows, int64_t heads, int64_t width, int64_t size) {
  return {at, 0, row, head, {1, rows, heads}, width, size};
}
bool same_place(const Layout4& a, const Layout4& b) {
  return a.at == b.at && (a.n[1] == 1 || a.token == b.token) && (a.n[2] == 1 || a.head == b.head);
}
bool touch(const Layout4& a, const Layout4& b) { return a.at && b.at && share(a, b); }
bool touch(const Layout4& a, const Span& b) { return a.at && overlap(a.rows(), b); }

int rms_strides_ok(int64_t row, int64_t head, const jenga_rms_config& c) {
  if (row < 0 || head < 0) return JENGA_EINVAL;
  if (row > MOST_STRIDE || head > MOST_STRIDE) return JENGA_EUNSUPPORTED;
  const __int128 lim = (__int128)1 << 60;
  return (__int128)c.rows * row + (__int128)c.heads * head > lim ? JENGA_EUNSUPPORTED : JENGA_OK;
}

int rms_config_ok(const jenga_rms_config& c) {
  if (c.rows < 0 || c.heads < 1 || c.cols < 1 || c.reserved != 0) return JENGA_EINVAL;
  if (!float_type(c.x_type) || !float_type(c.param_type)) return JENGA_EINVAL;
  if (!float_type(c.y_type) && c.y_type != JENGA_E4M3 && c.y_type != JENGA_E2M1) return JENGA_EINVAL;
  if (!std::isfinite(c.eps) || c.eps < 0.0f || !std::isfinite(c.weight_offset)) return JENGA_EINVAL;
  if (c.cols > MOST_COLS || c.rows > MOST_ROWS || c.heads > 1 << 20) return JENGA_EUNSUPPORTED;
  if (c.heads > 1 && c.rows * c.heads >= 1ll << 31) return JENGA_EUNSUPPORTED;
  if (float_type(c.y_type) ? c.y_type != c.x_type : c.heads != 1) return JENGA_EUNSUPPORTED;
  if (c.param_type != c.x_type && c.param_type != JENGA_F32) return JENGA_EUNSUPPORTED;
  return JENGA_OK;
}

}  // namespace

int rms_args_ok(const jenga_rms_config* c, const void* x, const void* residual, const void* weight, const void* total, const void* y,
                const uint8_t* y_scale, const float* rstd) {
  if (!c || !x || !y) return JENGA_EINVAL;
  int why = rms_config_ok(*c);
  if (why != JENGA_OK) return why;
  const int64_t xs = type_size(c->x_type), ps = type_size(c->param_type), blocks = ((int64_t)c->cols + 127) / 128;
  const bool packed = !float_type(c->y_type);
  const int64_t y_bytes = c->y_type == JENGA_E4M3 ? blocks * 128 : blocks * 64;
  const int64_t scales = c->y_type == JENGA_E4M3 ? (blocks + 3) / 4 * 4 : blocks * 4;
  if (packed != (y_scale != nullptr) || (packed && (!aligned(y, 16) || !aligned(y_scale, 4)))) return JENGA_EINVAL;
  if (!aligned(x, xs) || !aligned(residual, xs) || !aligned(total, xs) || (!packed && !aligned(y, xs)) || !aligned(weight, ps) ||
      !aligned(rstd, 4))
    return JENGA_EINVAL;
  if ((why = rms_strides_ok(c->x_row, c->x_head, *c)) != JENGA_OK) return why;
  if (residual && (why = rms_strides_ok(c->add_row, c->add_head, *c)) != JENGA_OK) return why;
  if (total && (why = rms_strides_ok(c->sum_row, c->sum_head, *c)) != JENGA_OK) return why;
  if (!packed && (why = rms_strides_ok(c->y_row, c->y_head, *c)) != JENGA_OK) return why;
  if (c->rows == 0) return JENGA_OK;
  const Layout4 from = rows_and_heads(x, c->x_row, c->x_head, c->rows, c->heads, c->cols, xs),
                add = rows_and_heads(residual, c->add_row, c->add_head, c->rows, c->heads, c->cols, xs),
                sum = rows_and_heads(total, c->sum_row, c->sum_head, c->rows, c->heads, c->cols, xs),
                to = rows_and_heads(packed ? nullptr : y, c->y_row, c->y_head, c->rows, c->heads, c->cols, xs);
  const int64_t stats = c->rows * c->heads * 4;
  const Span read[1] = {{weight, 1, c->cols * ps, c->cols * ps}};
  const Span written[3] = {{rstd, 1, stats, stats}, {packed ? y : nullptr, c->rows, y_bytes, y_bytes}, {y_scale, c->rows, scales, scales}};
  if ((!packed && !distinct(to)) || (total && !distinct(sum))) return JENGA_EINVAL;
  for (const Layout4* out : {&to, &sum}) {
    for (const Layout4* in : {&from, &add})
      if (touch(*out, *in) && !same_place(*out, *in)) return JENGA_EINVAL;
    if (touch(*out, read[0])) return JENGA_EINVAL;
  }
  if (touch(to, sum)) return JENGA_EINVAL;
  for (int i = 0; i < 3; ++i) {
    for (const Layout4* t : {&from, &add, &sum, &to})
      if (touch(*t, written[i])) return JENGA_EINVAL;
    if (overlap(written[i], read[0])) return JENGA_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlap(written[i], written[j])) return JENGA_EINVAL;
  }
  return JENGA_OK;
}

int rms_grad_args_ok(const jenga_rms_config* c, const void* x, const void* dy, const void* weight, const float* rstd, const void* dtotal,
                     const void* dx, const float* dweight, const void* workspace, size_t workspace_bytes) {
  if (!c || !x || !dy || !rstd || !dx) return JENGA_EINVAL;
  int why = rms_config_ok(*c);
  if (why != JENGA_OK) return why;
  if (c->y_type != c->x_type) return JENGA_EUNSUPPORTED;
  const int64_t xs = type_size(c->x_type), ps = type_size(c->param_type);
  if (!aligned(x, xs) || !aligned(dy, xs) || !aligned(dtotal, xs) || !aligned(dx, xs) || !aligned(weight, ps) || !aligned(rstd, 4) ||
      !aligned(dweight, 4))
    return JENGA_EINVAL;
  if ((why = rms_strides_ok(c->x_row, c->x_head, *c)) != JENGA_OK) return why;
  if (dtotal && (why = rms_strides_ok(c->add_row, c->add_head, *c)) != JENGA_OK) return why;
  if ((why = rms_strides_ok(c->sum_row, c->sum_head, *c)) != JENGA_OK) return why;
  if ((why = rms_strides_ok(c->y_row, c->y_head, *c)) != JENGA_OK) return why;
  if (c->rows == 0) return JENGA_OK;
  uint64_t need = 0;
  if (dweight) {
    if (!workspace || !aligned(workspace, 256)) return JENGA_EINVAL;
    need = (uint64_t)RMS_PARTS * c->cols * 4;
  }
  const Layout4 from = rows_and_heads(x, c->x_row, c->x_head, c->rows, c->heads, c->cols, xs),
                up = rows_and_heads(dy, c->y_row, c->y_head, c->rows, c->heads, c->cols, xs),
                add = rows_and_heads(dtotal, c->add_row, c->add_head, c->rows, c->heads, c->cols, xs),
                to = rows_and_heads(dx, c->sum_row, c->sum_head, c->rows, c->heads, c->cols, xs);
  const int64_t stats = c->rows * c->heads * 4;
  const Span params = {weight, 1, c->cols * ps, c->cols * ps}, r = {rstd, 1, stats, stats},
             sums = {dweight, 1, (int64_t)c->cols * 4, (int64_t)c->cols * 4},
             room = {need ? workspace : nullptr, 1, (int64_t)need, (int64_t)need};
  if (!distinct(to) || touch(to, from) || touch(to, up) || (touch(to, add) && !same_place(to, add))) return JENGA_EINVAL;
  for (const Layout4* t : {&from, &up, &add, &to})
    if (touch(*t, sums) || touch(*t, room)) return JENGA_EINVAL;
  if (touch(to, params) || touch(to, r)) return JENGA_EINVAL;
  for (const Span* s : {&params, &r})
    if (overlap(sums, *s) || overlap(room, *s)) return JENGA_EINVAL;
  if (overlap(sums, room)) return JENGA_EINVAL;
  return workspace_bytes < need ? JENGA_EWORKSPACE : JENGA_OK;
}

int quantize_mx_args_ok(const void* x, int64_t x_stride, int32_t x_type, int64_t rows, int32_t cols, const void* q, const uint8_t* scale) {
  if (!x || !q || !scale || rows < 0 || cols < 1 || x_stride < cols) return JENGA_EINVAL;
  if (!float_type(x_type) || !aligned(x, type_size(x_type)) || !aligned(q, 16) || !aligned(scale, 4)) return JENGA_EINVAL;
  if (cols > MOST_COLS || rows > 1ll << 30 || x_stride > 1ll << 28) return JENGA_EUNSUPPORTED;
  if (rows == 0) return JENGA_OK;
  const int64_t size = type_size(x_type), blocks = ((int64_t)cols + 127) / 128;
  const Span from = {x, rows, x_stride * size, cols * size}, to = {q, rows, blocks * 64, blocks * 64}, bytes = {scale, rows, blocks * 4, blocks * 4};
  return overlap(from, to) || overlap(from, bytes) || overlap(to, bytes) ? JENGA_EINVAL : JENGA_OK;
}

int matmul_mx_args_ok(const jenga_matmul_config* c, const void* a, const uint8_t* a_scale, const void* b, const uint8_t* b_scale,
                      const float* bias, const void* out) {
  if (!c || !a || !a_scale || !b || !b_scale || !out) return JENGA_EINVAL;
  if (c->m < 0 || c->n < 1 || c->k < 1 || c->k % 128 != 0 || c->out_stride < c->n || c->reserved != 0) return JENGA_EINVAL;
  if (!float_type(c->out_type)) return JENGA_EINVAL;
  const int64_t size = type_size(c->out_type);
  if (!aligned(a, 16) || !aligned(b, 16) || !aligned(a_scale, 4) || !aligned(b_scale, 4) || !aligned(bias, 4) || !aligned(out, size))
    return JENGA_EINVAL;
  if (c->k > MOST_COLS || c->m > 1ll << 30 || c->n > 1 << 22 || c->out_stride > 1ll << 31) return JENGA_EUNSUPPORTED;
  if ((c->m + 127) / 128 * (((int64_t)c->n + 127) / 128) > 1ll << 23) return JENGA_EUNSUPPORTED;
  if (c->m == 0) return JENGA_OK;
  const int64_t values = c->k / 2, scales = c->k / 32;
  const Span to = {out, c->m, c->out_stride * size, c->n * size};
  const Span in[5] = {{a, c->m, values, values}, {a_scale, c->m, scales, scales}, {b, c->n, values, values}, {b_scale, c->n, scales, scales},
                      {bias, 1, (int64_t)c->n * 4, (int64_t)c->n * 4}};
  for (const Span& s : in)
    if (overlap(to, s)) return JENGA_EINVAL;
  return JENGA_OK;
}

constexpr int64_t DENSE_WORKGROUPS = 1 << 23;   // of a launch, at most

int dense_config_ok(const jenga_dense_config* c) {
  if (!c || c->q_rows < 0 || c->kv_rows < 0 || c->sequences < 0 || c->heads < 1 || c->kv_heads < 1 || c->heads % c->kv_heads != 0 ||
      c->reserved != 0)
    return JENGA_EINVAL;
  if ((c->type != JENGA_BF16 && c->type != JENGA_F16) || (c->flags & ~(uint32_t)JENGA_DENSE_CAUSAL) || !std::isnormal(c->scale * 1.4426950408889634f) || c->scale < 0.0f)
    return JENGA_EINVAL;
  if (c->head_dim < 1) return JENGA_EINVAL;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->sequences > 1 << 16 || c->heads > 1 << 12) return JENGA_EUNSUPPORTED;
  const int64_t most = (1ll << 31) - 1;
  if (c->q_rows > most || c->kv_rows > most || c->q_rows * (c->heads / c->kv_heads) > most) return JENGA_EUNSUPPORTED;
  if (dense_shape(*c).items * c->kv_heads > DENSE_WORKGROUPS) return JENGA_EUNSUPPORTED;
  return JENGA_OK;
}

int dense_args_ok(const jenga_dense_config* c, const void* q, const void* k, const void* v, const int32_t* q_start,
                  const int32_t* kv_start, const int32_t* kv_len, const void* out, const void* workspace, size_t workspace_bytes) {
  const int why = dense_config_ok(c);
  if (why != JENGA_OK) return why;
  if (!q || !k || !v || !q_start || !kv_start || !out || !workspace) return JENGA_EINVAL;
  if (!aligned(q, 2) || !aligned(k, 2) || !aligned(v, 2) || !aligned(out, 2) || !aligned(q_start, 4) || !aligned(kv_start, 4) ||
      !aligned(kv_len, 4) || !aligned(workspace, 256))
    return JENGA_EINVAL;
  const struct { int64_t row, head, heads; } strides[4] = {{c->q_row, c->q_head, c->heads},
                                                                 {c->k_row, c->k_head, c->kv_heads},
                                                                 {c->v_row, c->v_head, c->kv_heads},
                                                                 {c->out_row, c->out_head, c->heads}};
  for (const auto& s : strides) {
    if (s.row < 0 || s.head < 0) return JENGA_EINVAL;
    if (s.row > 1 << 23 || s.head > MOST_STRIDE || (__int128)s.head * s.heads > (__int128)1 << 60) return JENGA_EUNSUPPORTED;
  }
  const uint64_t need = dense_shape(*c).workspace;
  if (c->q_rows > 0) {
    const Layout4 to = rows_and_heads(out, c->out_row, c->out_head, c->q_rows, c->heads, c->head_dim, 2),
                  from = rows_and_heads(q, c->q_row, c->q_head, c->q_rows, c->heads, c->head_dim, 2);
    const Layout4 keys = rows_and_heads(c->kv_rows ? k : nullptr, c->k_row, c->k_head, c->kv_rows, c->kv_heads, c->head_dim, 2),
                  values = rows_and_heads(c->kv_rows ? v : nullptr, c->v_row, c->v_head, c->kv_rows, c->kv_heads, c->head_dim, 2);
    if (!distinct(to) || (touch(to, from) && !same_place(to, from)) || touch(to, keys) || touch(to, values)) return JENGA_EINVAL;
    const int64_t starts = ((int64_t)c->sequences + 1) * 4, lengths = (int64_t)c->sequences * 4;
    const Span room = {workspace, 1, (int64_t)need, (int64_t)need};
    for (const Span& s : {Span{q_start, 1, starts, starts}, Span{kv_start, 1, starts, starts}, Span{lengths ? kv_len : nullptr, 1, lengths, lengths}})
      if (touch(to, s) || overlap(s, room)) return JENGA_EINVAL;
    if (touch(to, room) || touch(from, room) || touch(keys, room) || touch(values, room)) return JENGA_EINVAL;
  }
  return workspace_bytes < need ? JENGA_EWORKSPACE : JENGA_OK;
}

namespace {

// What a call of `rows` packed rows and so many sequences needs, in tiles of `tile` rows.  Everything here grows with rows and sequences as long as may_split and
// listed stay as they are, and is largest where tiles may be cut and there is no list.
DenseShape dense_shape_of(const jenga_dense_config& c, int64_t rows, int64_t sequences, int tile, bool may_split, bool listed) {
  DenseShape s;
  s.rows = tile;
  s.may_split = may_split;
  s.listed = listed;
  s.workgroups = tile == 16 ? 512 : c.head_dim == 128 ? 768 : 1024;   // that the chip holds, or that keep its memory busy
  // each sequence ends with a tile that may not be full
  s.tiles = rows == 0 ? 0 : rows / tile + sequences;
  // A tile of n steps makes ceil(n / chunk) parts, and a chunk is half of a workgroup's share of the steps at least.  Without a list the tiles of a
  // sequence have as many places as the longest has parts, and their steps are taken as half of that at least; sums are float32 there.
  const int64_t split = (2 * s.workgroups + c.kv_heads - 1) / c.kv_heads, chunks = listed ? split : 2 * split + 16;
  s.split_tiles = may_split ? std::min<int64_t>(s.tiles, split) : 0;
  s.slots = may_split ? s.split_tiles + chunks : 0;
  s.items = std::max<int64_t>(s.tiles, s.slots);
  auto up = [](uint64_t bytes) { return (bytes + 255) / 256 * 256; };
  s.bins_at = 256;
  s.items_at = s.bins_at + up(((uint64_t)sequences + 1) * 4);
  s.merge_at = s.items_at + up((uint64_t)s.items * sizeof(DenseItem));
  s.stat_at = s.merge_at + up((uint64_t)s.split_tiles * sizeof(DenseMerge));
  const uint64_t results = (uint64_t)s.slots * c.kv_heads * tile;
  s.part_at = s.stat_at + up(results * 8);
  s.workspace = s.part_at + up(results * c.head_dim * 4);
  return s;
}

}  // namespace

DenseShape dense_shape(const jenga_dense_config& c) {
  const int64_t group = c.heads / c.kv_heads, rows = c.q_rows * group;
  // Tiles of 16 rows for a few tokens each: 16 sequences of 3 tokens over 4000 keys x 8 heads 56 us, in tiles of 128 76; 64 x 4 tokens, four heads on one of
  // keys, 59 and 58; 64 x 20 tokens 130 and 101.  Few tokens on average may be a long prompt and many single tokens: 8000 and 300 x 1, 16 heads, 1353 and 685.
  const int tile = c.q_rows <= 4 * (int64_t)c.sequences && rows <= 32 * (int64_t)c.sequences ? 16 : 128;
  const int64_t workgroups = dense_shape_of(c, rows, c.sequences, tile, false, false).workgroups;
  // full tiles that there are at least
  const int64_t least = rows / tile;
  return dense_shape_of(c, rows, c.sequences, tile, least * c.kv_heads < 2 * workgroups, c.sequences > 64);
}

// The most workgroups and bytes that a call with no more rows, keys and sequences has.  Neither is the larger call's own: it may have tiles enough that none is cut,
// and fewer sequences may leave tiles of 128 rows where it has 16.
void dense_most(const jenga_dense_config& c, int64_t* workgroups, uint64_t* workspace) {
  const int64_t group = c.heads / c.kv_heads, rows = c.q_rows * group, few = std::min(std::min<int64_t>(rows, 4 * group * c.sequences), (int64_t)32 * c.sequences);
  const DenseShape s[2] = {dense_shape_of(c, few, c.sequences, 16, true, false), dense_shape_of(c, rows, c.sequences, 128, true, false)};
  *workgroups = std::max(s[0].items, s[1].items) * c.kv_heads;
  *workspace = std::max(s[0].workspace, s[1].workspace);
}

}  // namespace jenga

extern "C" {

int jenga_rms_norm_grad_workspace(const jenga_rms_config* c, uint64_t* bytes) {
  if (!c || !bytes) return JENGA_EINVAL;
  const int why = jenga::rms_config_ok(*c);
  if (why != JENGA_OK) return why;
  *bytes = (uint64_t)jenga::RMS_PARTS * c->cols * 4;
  return JENGA_OK;
}

int jenga_dense_attn_workspace(const jenga_dense_config* c, uint64_t* bytes) {
  if (!bytes) return JENGA_EINVAL;
  const int why = jenga::dense_config_ok(c);
  if (why != JENGA_OK) return why;
  *bytes = jenga::dense_shape(*c).workspace;
  return JENGA_OK;
}

int jenga_dense_attn_workspace_up_to(const jenga_dense_config* c, uint64_t* bytes) {
  if (!bytes) return JENGA_EINVAL;
  const int why = jenga::dense_config_ok(c);
  if (why != JENGA_OK) return why;
  int64_t workgroups;
  jenga::dense_most(*c, &workgroups, bytes);
  return workgroups > jenga::DENSE_WORKGROUPS ? JENGA_EUNSUPPORTED : JENGA_OK;
}

int jenga_layer_norm_grad_workspace(const jenga_norm_config* c, uint64_t* bytes) {
  if (!c || !bytes) return JENGA_EINVAL;
  const int why = jenga::norm_config_ok(*c);
  if (why != JENGA_OK) return why;
  if (jenga::groups_of(*c) > 1 << 20) return JENGA_EUNSUPPORTED;
  *bytes = (uint64_t)(1024 + jenga::groups_of(*c)) * c->cols * 8;
  return JENGA_OK;
}

int jenga_rotary_table(const jenga_rotary_config* c, float* table) {
  const int why = jenga::rotary_config_ok(c);
  if (why != JENGA_OK) return why;
  if (!table) return JENGA_EINVAL;
  const int cells[3] = {c->T, c->H, c->W};
  for (int a = 0; a < 3; ++a)
    for (int n = 0; n < cells[a]; ++n)
      for (int i = 0; i < c->dim[a] / 2; ++i) {
        const double angle = (c->origin[a] + c->step[a] * n) * std::pow(c->theta, -2.0 * i / c->dim[a]);
        if (!std::isfinite(angle)) return JENGA_EINVAL;
        *table++ = (float)std::cos(angle);
        *table++ = (float)std::sin(angle);
      }
  return JENGA_OK;
}

int jenga_plan_info(const jenga_plan* p, jenga_plan_info_t* info) {
  if (!p || !info) return JENGA_EINVAL;
  *info = p->info;
  return JENGA_OK;
}

int jenga_plan_export(const jenga_plan* p, int32_t* perm, int32_t* inv_perm, uint8_t* adja) {
  if (!p) return JENGA_EINVAL;
  const size_t nv = (size_t)p->info.N_v;
  if (perm) std::memcpy(perm, p->perm.data(), nv * sizeof(int32_t));
  if (inv_perm) std::memcpy(inv_perm, p->inv_perm.data(), nv * sizeof(int32_t));
  if (adja) {
    const int mv = p->info.M_v;
    const bool on = (p->cfg.flags & JENGA_FLAG_ADJACENCY) != 0;
    for (int i = 0; i < mv; ++i)
      for (int j = 0; j < mv; ++j)
        adja[(size_t)i * mv + j] =
            on ? (uint8_t)((p->fixed_bits[(size_t)i * p->nt64 + (j >> 6)] >> (j & 63)) & 1ull) : 0;
  }
  return JENGA_OK;
}

int jenga_plan_tables(const jenga_config* cfg, jenga_plan_info_t* info, int32_t* perm, int32_t* inv_perm,
                      uint8_t* adja) {
  if (!cfg || !info) return JENGA_EINVAL;
  int why;
  if (!jenga::config_ok(*cfg, &why)) return why;
  jenga_plan* p = new (std::nothrow) jenga_plan();
  if (!p) return JENGA_ENOMEM;
  p->cfg = *cfg;
  p->d_src_of_pos = nullptr;
  p->d_blk_valid = nullptr;
  p->d_fixed_bits = nullptr;
  int rc = JENGA_OK;
  try {
    rc = jenga::build_host_tables(p);
  } catch (const std::bad_alloc&) {
    rc = JENGA_ENOMEM;
  }
  if (rc == JENGA_OK) {
    *info = p->info;
    rc = jenga_plan_export(p, perm, inv_perm, adja);
  }
  delete p;
  return rc;
}

const char* jenga_strerror(int status) {
  switch (status) {
    case JENGA_OK: return "ok";
    case JENGA_EINVAL: return "invalid argument";
    case JENGA_EUNSUPPORTED: return "configuration not supported by this build";
    case JENGA_EWORKSPACE: return "workspace too small";
    case JENGA_EHIP: return "HIP runtime or kernel launch failure";
    case JENGA_ENOMEM: return "out of memory";
    default: return "unknown status";
  }
}

}  // extern "C"
