// C ABI of the operators on rows: 4-bit linear layers and log probabilities of classes.  Argument checks only; the kernels are in
// linear_q4.cu and log_probs.cu.
#include <cuda_runtime.h>

#include <string>

#include "gi_internal.h"
#include "kernels.h"

using namespace gi;

namespace {

int elem_of(int dtype) { return dtype == GI_F32 ? 4 : 2; }
bool known_dtype(int dtype) { return dtype == GI_F16 || dtype == GI_BF16 || dtype == GI_F32; }
bool aligned_to(const void* p, int bytes) { return reinterpret_cast<uintptr_t>(p) % static_cast<unsigned>(bytes) == 0; }

gi_status check_layer(const char* who, const gi_linear_q4* l) {
  const std::string w(who);
  if (!l) return fail(GI_E_INVALID, w + ": null layer");
  if (l->cin <= 0 || l->cout <= 0) return fail(GI_E_INVALID, w + ": cin and cout must be positive");
  if (l->cin > (1 << 20) || l->cout > (1 << 20)) return fail(GI_E_UNSUPPORTED, w + ": cin or cout above 2^20");
  if (l->group <= 0) return fail(GI_E_INVALID, w + ": group must be positive");
  if (l->group % 32 != 0) return fail(GI_E_UNSUPPORTED, w + ": group must be a multiple of 32");
  if (!known_dtype(l->scale_dtype)) return fail(GI_E_INVALID, w + ": scale_dtype must be GI_F16, GI_BF16 or GI_F32");
  if (!known_dtype(l->dtype)) return fail(GI_E_INVALID, w + ": dtype must be GI_F16, GI_BF16 or GI_F32");
  if (l->has_zeros != 0 && l->has_zeros != 1) return fail(GI_E_INVALID, w + ": has_zeros must be 0 or 1");
  if (l->act != GI_ACT_NONE && l->act != GI_ACT_RELU && l->act != GI_ACT_RELU6) return fail(GI_E_INVALID, w + ": unknown activation");
  return GI_OK;
}

// Whether an element of x is one of y: [rows][cin] and [rows][cout], rows ldx and ldy elements apart.  Rows at one and the same distance
// may lie between one another (columns of one tensor); of rows at other distances the whole ranges count.
bool overlap(const void* x, int64_t ldx, int64_t cin, const void* y, int64_t ldy, int64_t cout, int64_t rows, int elem) {
  const uint64_t a = reinterpret_cast<uintptr_t>(x), b = reinterpret_cast<uintptr_t>(y);
  const uint64_t na = (static_cast<uint64_t>(rows - 1) * ldx + cin) * elem, nb = (static_cast<uint64_t>(rows - 1) * ldy + cout) * elem;
  if (a >= b + nb || b >= a + na) return false;
  if (ldx != ldy) return true;
  const uint64_t pitch = static_cast<uint64_t>(ldx) * elem;
  const uint64_t behind = b >= a ? (b - a) % pitch : (pitch - (a - b) % pitch) % pitch;  // y's row behind the start of a row of x
  return behind < static_cast<uint64_t>(cin) * elem || behind + static_cast<uint64_t>(cout) * elem > pitch;
}

constexpr int64_t kMaxPitch = int64_t{1} << 30;  // elements between rows: with 2^31 rows and 4 bytes, below 2^63 bytes

}  // namespace

extern "C" {

gi_status gi_linear_q4_blob_bytes(const gi_linear_q4* layer, uint64_t* bytes) {
  const gi_status st = check_layer("gi_linear_q4_blob_bytes", layer);
  if (st != GI_OK) return st;
  if (!bytes) return fail(GI_E_INVALID, "gi_linear_q4_blob_bytes: null argument");
  *bytes = linear_q4_layout(layer->cin, layer->cout, layer->group, layer->scale_dtype, layer->has_zeros != 0, layer->dtype).bytes;
  return GI_OK;
}

gi_status gi_linear_q4_pack(const gi_linear_q4* layer, const uint8_t* q, const void* scales, const uint8_t* zeros, const float* bias,
                            void* host_blob, uint64_t blob_bytes) {
  const gi_status st = check_layer("gi_linear_q4_pack", layer);
  if (st != GI_OK) return st;
  if (!q || !scales || !host_blob) return fail(GI_E_INVALID, "gi_linear_q4_pack: null argument");
  if ((zeros != nullptr) != (layer->has_zeros != 0)) return fail(GI_E_INVALID, "gi_linear_q4_pack: zeros must be given exactly where has_zeros is 1");
  const LinearQ4Layout l = linear_q4_layout(layer->cin, layer->cout, layer->group, layer->scale_dtype, zeros != nullptr, layer->dtype);
  if (blob_bytes < l.bytes) return fail(GI_E_INVALID, "gi_linear_q4_pack: host_blob too small");
  if (zeros) {
    const size_t n = static_cast<size_t>(layer->cout) * ((static_cast<int64_t>(layer->cin) + layer->group - 1) / layer->group);
    for (size_t i = 0; i < n; ++i)
      if (zeros[i] > 15) return fail(GI_E_INVALID, "gi_linear_q4_pack: zero point above 15");
  }
  linear_q4_pack(LinearQ4Weights{q, scales, zeros, layer->cin, layer->cout, layer->group, layer->scale_dtype, layer->dtype}, bias, static_cast<uint8_t*>(host_blob));
  return GI_OK;
}

gi_status gi_linear_q4_pack_device(const gi_linear_q4* layer, const uint8_t* dev_q, const void* dev_scales, const uint8_t* dev_zeros,
                                   const float* dev_bias, void* dev_blob, uint64_t blob_bytes, void* stream) {
  const gi_status st = check_layer("gi_linear_q4_pack_device", layer);
  if (st != GI_OK) return st;
  if (!dev_q || !dev_scales || !dev_blob) return fail(GI_E_INVALID, "gi_linear_q4_pack_device: null argument");
  if ((dev_zeros != nullptr) != (layer->has_zeros != 0))
    return fail(GI_E_INVALID, "gi_linear_q4_pack_device: zeros must be given exactly where has_zeros is 1");
  if (!aligned_to(dev_blob, 256)) return fail(GI_E_INVALID, "gi_linear_q4_pack_device: the blob must be 256-byte aligned");
  if (!aligned_to(dev_scales, elem_of(layer->scale_dtype)) || !aligned_to(dev_bias, 4))
    return fail(GI_E_INVALID, "gi_linear_q4_pack_device: scales or bias not aligned to their elements");
  if (blob_bytes < linear_q4_layout(layer->cin, layer->cout, layer->group, layer->scale_dtype, dev_zeros != nullptr, layer->dtype).bytes)
    return fail(GI_E_INVALID, "gi_linear_q4_pack_device: dev_blob too small");
  const int err = launch_linear_q4_pack(LinearQ4Weights{dev_q, dev_scales, dev_zeros, layer->cin, layer->cout, layer->group, layer->scale_dtype, layer->dtype},
                                        dev_bias, dev_blob, stream);
  if (err != 0) return fail(GI_E_CUDA, std::string("gi_linear_q4_pack_device: ") + cudaGetErrorString(static_cast<cudaError_t>(err)));
  return GI_OK;
}

gi_status gi_linear_q4_run(const gi_linear_q4* layer, const void* dev_blob, const void* dev_x, int64_t ldx, void* dev_y, int64_t ldy,
                           int32_t rows, void* stream) {
  const gi_status st = check_layer("gi_linear_q4_run", layer);
  if (st != GI_OK) return st;
  if (rows < 0) return fail(GI_E_INVALID, "gi_linear_q4_run: negative number of rows");
  if (rows > (1 << 30)) return fail(GI_E_UNSUPPORTED, "gi_linear_q4_run: more than 2^30 rows");
  if (rows == 0) return GI_OK;
  if (!dev_blob || !dev_x || !dev_y) return fail(GI_E_INVALID, "gi_linear_q4_run: null argument");
  const int elem = elem_of(layer->dtype);
  if (!aligned_to(dev_blob, 256)) return fail(GI_E_INVALID, "gi_linear_q4_run: the blob must be 256-byte aligned");
  if (!aligned_to(dev_x, elem) || !aligned_to(dev_y, elem)) return fail(GI_E_INVALID, "gi_linear_q4_run: x or y not aligned to its elements");
  if (rows == 1) {
    ldx = layer->cin;
    ldy = layer->cout;
  }
  if (ldx < layer->cin || ldy < layer->cout) return fail(GI_E_INVALID, "gi_linear_q4_run: rows overlap (ldx < cin or ldy < cout)");
  if (ldx > kMaxPitch || ldy > kMaxPitch) return fail(GI_E_INVALID, "gi_linear_q4_run: ldx or ldy too large");
  if (overlap(dev_x, ldx, layer->cin, dev_y, ldy, layer->cout, rows, elem))
    return fail(GI_E_INVALID, "gi_linear_q4_run: x and y overlap");
  LinearQ4Call c;
  c.blob = dev_blob;
  c.x = dev_x;
  c.y = dev_y;
  c.x_row = ldx;
  c.y_row = ldy;
  c.rows = rows;
  c.cin = layer->cin;
  c.cout = layer->cout;
  c.group = layer->group;
  c.scale_dtype = layer->scale_dtype;
  c.dtype = layer->dtype;
  c.zeros = layer->has_zeros != 0;
  c.ep.act_pre = layer->act;
  const int err = launch_linear_q4(c, stream);
  if (err != 0) return fail(GI_E_CUDA, std::string("gi_linear_q4_run: ") + cudaGetErrorString(static_cast<cudaError_t>(err)));
  return GI_OK;
}

gi_status gi_log_probs(const gi_log_probs_desc* d, const void* dev_logits, const int32_t* dev_given, float* dev_given_log_probs,
                       float* dev_entropy, int32_t* dev_top_ids, float* dev_top_log_probs, void* stream) {
  if (!d) return fail(GI_E_INVALID, "gi_log_probs: null descriptor");
  if (d->rows < 0 || d->classes <= 0) return fail(GI_E_INVALID, "gi_log_probs: negative number of rows, or no classes");
  if (d->rows > (1 << 28) || d->classes > (1 << 24)) return fail(GI_E_UNSUPPORTED, "gi_log_probs: more than 2^28 rows or 2^24 classes");
  if (!known_dtype(d->dtype)) return fail(GI_E_INVALID, "gi_log_probs: dtype must be GI_F16, GI_BF16 or GI_F32");
  if (!(d->temperature >= 1e-4f && d->temperature <= 1e4f)) return fail(GI_E_INVALID, "gi_log_probs: temperature must be 1e-4 .. 1e4");
  if (d->n_given < 0 || d->n_given > 65536) return fail(GI_E_INVALID, "gi_log_probs: n_given must be 0 .. 65536");
  if (d->top < 0 || d->top > GI_MAX_TOP || d->top > d->classes) return fail(GI_E_INVALID, "gi_log_probs: top must be 0 .. GI_MAX_TOP and at most classes");
  if (d->rows == 0) return GI_OK;
  if (!dev_logits || (d->n_given && (!dev_given || !dev_given_log_probs)) || (d->top && (!dev_top_ids || !dev_top_log_probs)))
    return fail(GI_E_INVALID, "gi_log_probs: null argument");
  if (!d->n_given && !d->top && !dev_entropy) return fail(GI_E_INVALID, "gi_log_probs: nothing asked for");
  const int64_t ld = d->rows == 1 ? d->classes : d->ld;
  if (ld < d->classes || ld > kMaxPitch) return fail(GI_E_INVALID, "gi_log_probs: ld below classes or too large");
  if (!aligned_to(dev_logits, elem_of(d->dtype)) || !aligned_to(dev_given, 4) || !aligned_to(dev_given_log_probs, 4) || !aligned_to(dev_entropy, 4) ||
      !aligned_to(dev_top_ids, 4) || !aligned_to(dev_top_log_probs, 4))
    return fail(GI_E_INVALID, "gi_log_probs: a pointer not aligned to its elements");
  LogProbsCall c;
  c.x = dev_logits;
  c.given = dev_given;
  c.given_lp = dev_given_log_probs;
  c.entropy = dev_entropy;
  c.top_ids = dev_top_ids;
  c.top_lp = dev_top_log_probs;
  c.ld = ld;
  c.rows = d->rows;
  c.classes = d->classes;
  c.n_given = d->n_given;
  c.top = d->top;
  c.dtype = d->dtype;
  c.temperature = d->temperature;
  const int err = launch_log_probs(c, stream);
  if (err != 0) return fail(GI_E_CUDA, std::string("gi_log_probs: ") + cudaGetErrorString(static_cast<cudaError_t>(err)));
  return GI_OK;
}

}  // extern "C"
