// C ABI entry points: host-side argument checks, workspace carving, launches.
#include <math.h>
#include <stdarg.h>
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <mutex>
#include <string>

#include "../../include/octnet_hip.h"
#include "oc_attention.h"
#include "oc_internal.h"

namespace {

// Scratch of oc_build_noalloc: the per-tree leaf counts and the scan's chunk
// sums for up to kNoAllocMaxTrees trees, in a file-scope device array (each
// device the library runs on holds its own copy until the process ends).
// In host code `scratch` only names the symbol; its device address comes
// from hipGetSymbolAddress, once per device, and only that address is used.
constexpr int64_t kNoAllocMaxTrees = 1LL << 22;
constexpr size_t kNoAllocBytes = ((4 * (size_t)kNoAllocMaxTrees + 255) & ~(size_t)255) +
                                 ((8 * ((size_t)kNoAllocMaxTrees / 256 + 2) + 255) & ~(size_t)255) + 1024;
static __device__ __align__(256) unsigned char scratch[kNoAllocBytes];

constexpr int kMaxScratchDevices = 64;

struct ScratchSlot {
  std::once_flag once;
  hipError_t err = hipSuccess;
  void* ptr = nullptr;
};

ScratchSlot g_scratch[kMaxScratchDevices];

// The current device's address of `scratch` (looked up on the first call on
// each device, with that device current).
hipError_t scratch_address(void** out) {
  int dev = 0;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return e;
  if (dev < 0 || dev >= kMaxScratchDevices) return hipErrorInvalidDevice;
  ScratchSlot& sl = g_scratch[dev];
  std::call_once(sl.once, [&sl]() {
    void* p = nullptr;
    sl.err = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    sl.ptr = p;
  });
  if (sl.err != hipSuccess) return sl.err;
  *out = sl.ptr;
  return hipSuccess;
}

thread_local std::string g_last_error;

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  g_last_error = buf;
  return code;
}

int hip_fail(hipError_t e, const char* where) {
  return fail(OC_EHIP, "%s: %s", where, hipGetErrorString(e));
}

#define OC_CHECK_HIP(expr, where)                 \
  do {                                            \
    hipError_t _e = (expr);                       \
    if (_e != hipSuccess) return hip_fail(_e, where); \
  } while (0)

inline hipStream_t as_stream(void* s) { return reinterpret_cast<hipStream_t>(s); }

bool dims_ok(int n, int gd, int gh, int gw) { return n > 0 && gd > 0 && gh > 0 && gw > 0; }

// Voxel and tree counts must fit the int64 index arithmetic of the kernels,
// and a launch grid (blocks of 256 threads over voxels) must fit 2^31 blocks.
bool sizes_ok(int n, int gd, int gh, int gw) {
  const double vox = 512.0 * n * gd * gh * gw;
  return vox < 4.0e12;
}

int64_t n_trees_of(int n, int gd, int gh, int gw) { return (int64_t)n * gd * gh * gw; }

// Scan counts (already in ws) into prefix and read the total back.
int finish_prefix(int64_t nt, int64_t* prefix, int64_t* n_leaves, void* ws, hipStream_t s,
                  const char* where) {
  OC_CHECK_HIP(oci::scan_counts(oci::scan_counts_buffer(ws), nt, prefix, ws, s), where);
  int64_t total = 0;
  OC_CHECK_HIP(hipMemcpyAsync(&total, prefix + nt, sizeof(int64_t), hipMemcpyDeviceToHost, s), where);
  OC_CHECK_HIP(hipStreamSynchronize(s), where);
  *n_leaves = total;
  return OC_OK;
}

}  // namespace

extern "C" {

const char* oc_error_string(int code) {
  switch (code) {
    case OC_OK: return "ok";
    case OC_EINVAL: return "invalid argument";
    case OC_ESTRUCT: return "invalid octree structure";
    case OC_EWORKSPACE: return "workspace too small";
    case OC_EHIP: return "HIP runtime error";
    case OC_EOVERFLOW: return "size overflow";
    default: return "unknown error";
  }
}

const char* oc_last_error(void) { return g_last_error.c_str(); }

int oc_version(void) { return 100; }

size_t oc_structure_workspace(int64_t n_trees) {
  if (n_trees < 0) return 0;
  return oci::scan_workspace(n_trees) + 256;
}

int oc_build(const uint8_t* occ, int n, int gd, int gh, int gw, int rule, uint32_t* trees,
             int64_t* prefix, int64_t* n_leaves, void* ws, size_t ws_bytes, void* stream) {
  g_last_error.clear();
  if (!occ || !trees || !prefix || !n_leaves || !ws) return fail(OC_EINVAL, "oc_build: null pointer");
  if (!dims_ok(n, gd, gh, gw)) return fail(OC_EINVAL, "oc_build: non-positive dims");
  if (!sizes_ok(n, gd, gh, gw)) return fail(OC_EOVERFLOW, "oc_build: grid too large");
  if (rule != OC_SPLIT_MIXED && rule != OC_SPLIT_ANY) return fail(OC_EINVAL, "oc_build: bad rule %d", rule);
  const int64_t nt = n_trees_of(n, gd, gh, gw);
  if (ws_bytes < oc_structure_workspace(nt)) return fail(OC_EWORKSPACE, "oc_build: workspace too small");
  hipStream_t s = as_stream(stream);
  OC_CHECK_HIP(oci::launch_build(occ, n, gd, gh, gw, rule, trees, oci::scan_counts_buffer(ws), s),
               "oc_build");
  return finish_prefix(nt, prefix, n_leaves, ws, s, "oc_build");
}

int oc_build_noalloc(const uint8_t* occ, int n, int gd, int gh, int gw, int rule, uint32_t* trees,
                     int64_t* prefix, int64_t* n_leaves, void* stream) {
  g_last_error.clear();
  if (!occ || !trees || !prefix || !n_leaves) return fail(OC_EINVAL, "oc_build_noalloc: null pointer");
  if (!dims_ok(n, gd, gh, gw)) return fail(OC_EINVAL, "oc_build_noalloc: non-positive dims");
  if (!sizes_ok(n, gd, gh, gw)) return fail(OC_EOVERFLOW, "oc_build_noalloc: grid too large");
  if (rule != OC_SPLIT_MIXED && rule != OC_SPLIT_ANY)
    return fail(OC_EINVAL, "oc_build_noalloc: bad rule %d", rule);
  const int64_t nt = n_trees_of(n, gd, gh, gw);
  if (nt > kNoAllocMaxTrees || oci::scan_workspace(nt) > kNoAllocBytes)
    return fail(OC_EOVERFLOW, "oc_build_noalloc: %lld trees exceed the static scratch (at most %lld trees)",
                (long long)nt, (long long)kNoAllocMaxTrees);
  void* ws = nullptr;
  OC_CHECK_HIP(scratch_address(&ws), "oc_build_noalloc");
  hipStream_t s = as_stream(stream);
  OC_CHECK_HIP(oci::launch_build(occ, n, gd, gh, gw, rule, trees, oci::scan_counts_buffer(ws), s),
               "oc_build_noalloc");
  return finish_prefix(nt, prefix, n_leaves, ws, s, "oc_build_noalloc");
}

int oc_prefix(const uint32_t* trees, int64_t n_trees, int64_t* prefix, int64_t* n_leaves, void* ws,
              size_t ws_bytes, void* stream) {
  g_last_error.clear();
  if (!trees || !prefix || !n_leaves || !ws) return fail(OC_EINVAL, "oc_prefix: null pointer");
  if (n_trees <= 0) return fail(OC_EINVAL, "oc_prefix: n_trees <= 0");
  if (ws_bytes < oc_structure_workspace(n_trees)) return fail(OC_EWORKSPACE, "oc_prefix: workspace too small");
  hipStream_t s = as_stream(stream);
  // Trees made outside the library enter here: count the non-canonical ones
  // (the counter sits in the workspace's last 256 bytes) with the leaves.
  int32_t* counter = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + oc_structure_workspace(n_trees) - 256);
  OC_CHECK_HIP(hipMemsetAsync(counter, 0, sizeof(int32_t), s), "oc_prefix");
  OC_CHECK_HIP(oci::launch_validate(trees, n_trees, counter, s), "oc_prefix");
  OC_CHECK_HIP(oci::launch_count(trees, n_trees, oci::scan_counts_buffer(ws), s), "oc_prefix");
  int rc = finish_prefix(n_trees, prefix, n_leaves, ws, s, "oc_prefix");
  if (rc != OC_OK) return rc;
  int32_t bad = 0;
  OC_CHECK_HIP(hipMemcpyAsync(&bad, counter, sizeof(int32_t), hipMemcpyDeviceToHost, s), "oc_prefix");
  OC_CHECK_HIP(hipStreamSynchronize(s), "oc_prefix");
  if (bad) return fail(OC_ESTRUCT, "oc_prefix: %d non-canonical trees", bad);
  return OC_OK;
}

int oc_validate(const uint32_t* trees, int64_t n_trees, int64_t* n_bad, void* ws, size_t ws_bytes,
                void* stream) {
  g_last_error.clear();
  if (!trees || !n_bad || !ws) return fail(OC_EINVAL, "oc_validate: null pointer");
  if (n_trees <= 0) return fail(OC_EINVAL, "oc_validate: n_trees <= 0");
  if (ws_bytes < oc_structure_workspace(n_trees)) return fail(OC_EWORKSPACE, "oc_validate: workspace too small");
  hipStream_t s = as_stream(stream);
  int32_t* counter = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + oc_structure_workspace(n_trees) - 256);
  OC_CHECK_HIP(hipMemsetAsync(counter, 0, sizeof(int32_t), s), "oc_validate");
  OC_CHECK_HIP(oci::launch_validate(trees, n_trees, counter, s), "oc_validate");
  int32_t total = 0;
  OC_CHECK_HIP(hipMemcpyAsync(&total, counter, sizeof(int32_t), hipMemcpyDeviceToHost, s), "oc_validate");
  OC_CHECK_HIP(hipStreamSynchronize(s), "oc_validate");
  *n_bad = total;
  return OC_OK;
}

int oc_leaf_index(const uint32_t* trees, const int64_t* prefix, int64_t n_trees, uint64_t* leaf_info,
                  void* stream) {
  g_last_error.clear();
  if (!trees || !prefix || !leaf_info) return fail(OC_EINVAL, "oc_leaf_index: null pointer");
  if (n_trees <= 0) return fail(OC_EINVAL, "oc_leaf_index: n_trees <= 0");
  if (n_trees >= (1LL << 54)) return fail(OC_EOVERFLOW, "oc_leaf_index: too many trees");
  OC_CHECK_HIP(oci::launch_leaf_index(trees, prefix, n_trees, leaf_info, as_stream(stream)),
               "oc_leaf_index");
  return OC_OK;
}

int oc_rowmap(const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh, int gw,
              int64_t* rowmap, void* stream) {
  g_last_error.clear();
  if (!trees || !prefix || !rowmap) return fail(OC_EINVAL, "oc_rowmap: null pointer");
  if (!dims_ok(n, gd, gh, gw)) return fail(OC_EINVAL, "oc_rowmap: non-positive dims");
  if (!sizes_ok(n, gd, gh, gw)) return fail(OC_EOVERFLOW, "oc_rowmap: grid too large");
  OC_CHECK_HIP(oci::launch_rowmap(trees, prefix, n, gd, gh, gw, rowmap, as_stream(stream)),
               "oc_rowmap");
  return OC_OK;
}

int oc_oc2ten(const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh, int gw,
              const float* data, int c, float* dense, void* stream) {
  g_last_error.clear();
  if (!trees || !prefix || !data || !dense) return fail(OC_EINVAL, "oc_oc2ten: null pointer");
  if (!dims_ok(n, gd, gh, gw) || c <= 0) return fail(OC_EINVAL, "oc_oc2ten: non-positive dims");
  if (!sizes_ok(n, gd, gh, gw)) return fail(OC_EOVERFLOW, "oc_oc2ten: grid too large");
  OC_CHECK_HIP(oci::launch_oc2ten(trees, prefix, n, gd, gh, gw, data, c, dense, as_stream(stream)),
               "oc_oc2ten");
  return OC_OK;
}

int oc_ten2oc(const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh, int gw,
              const float* dense, int c, int pool, float* data, void* stream) {
  g_last_error.clear();
  if (!trees || !prefix || !data || !dense) return fail(OC_EINVAL, "oc_ten2oc: null pointer");
  if (!dims_ok(n, gd, gh, gw) || c <= 0) return fail(OC_EINVAL, "oc_ten2oc: non-positive dims");
  if (pool != OC_POOL_AVG && pool != OC_POOL_MAX) return fail(OC_EINVAL, "oc_ten2oc: bad pool %d", pool);
  if (!sizes_ok(n, gd, gh, gw)) return fail(OC_EOVERFLOW, "oc_ten2oc: grid too large");
  OC_CHECK_HIP(oci::launch_ten2oc(trees, prefix, n, gd, gh, gw, dense, c, pool, data,
                                  as_stream(stream)),
               "oc_ten2oc");
  return OC_OK;
}

int oc_conv3x3x3_workspace(int64_t n_trees, int64_t n_leaves, int cin, int cout, size_t* bytes) {
  g_last_error.clear();
  if (!bytes) return fail(OC_EINVAL, "oc_conv3x3x3_workspace: null pointer");
  if (n_trees <= 0 || n_leaves <= 0 || cin <= 0 || cout <= 0)
    return fail(OC_EINVAL, "oc_conv3x3x3_workspace: non-positive size");
  *bytes = oci::conv_workspace(n_trees, n_leaves, cin, cout);
  return OC_OK;
}

int oc_conv3x3x3_workspace_exact(const uint32_t* trees, int n, int gd, int gh, int gw, int64_t n_leaves,
                                 int cin, int cout, size_t* bytes, void* scratch, void* stream) {
  g_last_error.clear();
  if (!trees || !bytes || !scratch) return fail(OC_EINVAL, "oc_conv3x3x3_workspace_exact: null pointer");
  if (!dims_ok(n, gd, gh, gw) || n_leaves <= 0 || cin <= 0 || cout <= 0)
    return fail(OC_EINVAL, "oc_conv3x3x3_workspace_exact: non-positive size");
  const int64_t nt = n_trees_of(n, gd, gh, gw);
  hipStream_t s = as_stream(stream);
  unsigned long long* count = static_cast<unsigned long long*>(scratch);
  OC_CHECK_HIP(oci::launch_count_slots(trees, nt, count, s), "oc_conv3x3x3_workspace_exact");
  unsigned long long slots = 0;
  OC_CHECK_HIP(hipMemcpyAsync(&slots, count, sizeof(slots), hipMemcpyDeviceToHost, s),
               "oc_conv3x3x3_workspace_exact");
  OC_CHECK_HIP(hipStreamSynchronize(s), "oc_conv3x3x3_workspace_exact");
  *bytes = oci::conv_workspace_slots(nt, n_leaves, cin, cout, (int64_t)slots);
  return OC_OK;
}

int oc_conv3x3x3_workspace_slots(int64_t n_trees, int64_t n_leaves, int cin, int cout, int64_t slots,
                                 size_t* bytes) {
  g_last_error.clear();
  if (!bytes) return fail(OC_EINVAL, "oc_conv3x3x3_workspace_slots: null pointer");
  if (n_trees <= 0 || n_leaves <= 0 || cin <= 0 || cout <= 0)
    return fail(OC_EINVAL, "oc_conv3x3x3_workspace_slots: non-positive size");
  *bytes = oci::conv_workspace_slots(n_trees, n_leaves, cin, cout, slots);
  return OC_OK;
}

int oc_conv3x3x3_workspace_capacity(int64_t n_trees, int64_t n_leaves, int cin, int cout, size_t ws_bytes,
                                    int64_t* slots) {
  g_last_error.clear();
  if (!slots) return fail(OC_EINVAL, "oc_conv3x3x3_workspace_capacity: null pointer");
  if (n_trees <= 0 || n_leaves <= 0 || cin <= 0 || cout <= 0)
    return fail(OC_EINVAL, "oc_conv3x3x3_workspace_capacity: non-positive size");
  const int64_t cap = oci::conv_slot_capacity(n_trees, n_leaves, cin, cout, ws_bytes);
  if (cap < 0) return fail(OC_EWORKSPACE, "oc_conv3x3x3_workspace_capacity: below the one-slot size");
  *slots = cap;
  return OC_OK;
}

int oc_conv3x3x3_mfma_supported(int cin, int cout) { return oci::conv_mfma_supported(cin, cout) ? 1 : 0; }

namespace {

// Shared argument checks of the convolution entry points; fills `a`.
int conv_args(const char* who, const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh,
              int gw, int64_t n_leaves, int cin, int cout, size_t ws_bytes, const void* ws,
              oci::ConvArgs* a) {
  if (!trees || !prefix || !ws) return fail(OC_EINVAL, "%s: null pointer", who);
  if (!dims_ok(n, gd, gh, gw)) return fail(OC_EINVAL, "%s: non-positive dims", who);
  if (cin <= 0 || cout <= 0 || cin > 256 || cout > 4096)
    return fail(OC_EINVAL, "%s: channels (%d, %d) outside [1,256] x [1,4096]", who, cin, cout);
  if (n_leaves <= 0) return fail(OC_EINVAL, "%s: n_leaves <= 0", who);
  if (n_leaves >= (1LL << 31)) return fail(OC_EOVERFLOW, "%s: n_leaves >= 2^31", who);
  const int64_t nt = n_trees_of(n, gd, gh, gw);
  if (n_leaves > 512 * nt) return fail(OC_EINVAL, "%s: n_leaves > 512 * n_trees", who);
  const int64_t cap = oci::conv_slot_capacity(nt, n_leaves, cin, cout, ws_bytes);
  if (cap < 0)
    return fail(OC_EWORKSPACE, "%s: workspace %zu < %zu", who, ws_bytes,
                oci::conv_workspace_slots(nt, n_leaves, cin, cout, 1));
  *a = oci::ConvArgs();
  a->slot_cap = cap;
  a->trees = trees; a->prefix = prefix;
  a->n = n; a->gd = gd; a->gh = gh; a->gw = gw;
  a->n_trees = nt; a->n_leaves = n_leaves;
  a->cin = cin; a->cout = cout;
  return OC_OK;
}

int conv_impl(const char* who, int impl, int64_t n_leaves, int cin, int cout, int* use) {
  if (impl != OC_CONV_AUTO && impl != OC_CONV_GENERIC && impl != OC_CONV_MFMA && impl != OC_CONV_GEMM &&
      impl != OC_CONV_TRUNCATED)
    return fail(OC_EINVAL, "%s: bad impl %d", who, impl);
  const bool mfma_ok = oci::conv_mfma_supported(cin, cout);
  if (impl == OC_CONV_MFMA && !mfma_ok)
    return fail(OC_EINVAL, "%s: no MFMA kernel for (%d, %d)", who, cin, cout);
  *use = impl == OC_CONV_AUTO ? oci::conv_auto_impl(n_leaves, cin, cout) : impl;
  return OC_OK;
}

}  // namespace

int oc_conv3x3x3_prepare(const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh, int gw,
                         int64_t n_leaves, const float* weight, int cin, int cout, void* ws,
                         size_t ws_bytes, void* stream) {
  g_last_error.clear();
  oci::ConvArgs a;
  int rc = conv_args("oc_conv3x3x3_prepare", trees, prefix, n, gd, gh, gw, n_leaves, cin, cout,
                     ws_bytes, ws, &a);
  if (rc != OC_OK) return rc;
  if (!weight) return fail(OC_EINVAL, "oc_conv3x3x3_prepare: null weight");
  a.weight = weight;
  OC_CHECK_HIP(oci::launch_conv_prepare(a, ws, as_stream(stream)), "oc_conv3x3x3_prepare");
  return OC_OK;
}

int oc_conv3x3x3_execute(const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh, int gw,
                         int64_t n_leaves, const float* in, int cin, const float* bias, int cout,
                         int relu, float* out, void* ws, size_t ws_bytes, int impl,
                         void* stream) {
  g_last_error.clear();
  oci::ConvArgs a;
  int rc = conv_args("oc_conv3x3x3_execute", trees, prefix, n, gd, gh, gw, n_leaves, cin, cout,
                     ws_bytes, ws, &a);
  if (rc != OC_OK) return rc;
  if (!in || !out) return fail(OC_EINVAL, "oc_conv3x3x3_execute: null pointer");
  int use = 0;
  rc = conv_impl("oc_conv3x3x3_execute", impl, n_leaves, cin, cout, &use);
  if (rc != OC_OK) return rc;
  if (use == OC_CONV_TRUNCATED)
    return fail(OC_EINVAL, "oc_conv3x3x3_execute: OC_CONV_TRUNCATED runs through oc_conv3x3x3_ex");
  a.in = in; a.bias = bias; a.relu = relu ? 1 : 0; a.out = out;
  OC_CHECK_HIP(oci::launch_conv_execute(a, ws, use, as_stream(stream)), "oc_conv3x3x3_execute");
  return OC_OK;
}

int oc_conv3x3x3_ex(const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh, int gw,
                    int64_t n_leaves, const float* in, int cin, const float* weight,
                    const float* bias, int cout, int relu, float* out, void* ws, size_t ws_bytes,
                    int impl, void* stream) {
  g_last_error.clear();
  oci::ConvArgs a;
  int rc = conv_args("oc_conv3x3x3", trees, prefix, n, gd, gh, gw, n_leaves, cin, cout, ws_bytes, ws,
                     &a);
  if (rc != OC_OK) return rc;
  if (!in || !weight || !out) return fail(OC_EINVAL, "oc_conv3x3x3: null pointer");
  int use = 0;
  rc = conv_impl("oc_conv3x3x3", impl, n_leaves, cin, cout, &use);
  if (rc != OC_OK) return rc;
  a.in = in; a.weight = weight; a.bias = bias; a.relu = relu ? 1 : 0; a.out = out;
  hipStream_t s = as_stream(stream);
  if (use == OC_CONV_TRUNCATED) {
    // Needs only the leaf index, at the start of the workspace.
    OC_CHECK_HIP(oci::launch_conv_truncated(a, static_cast<uint64_t*>(ws), s), "oc_conv3x3x3");
    return OC_OK;
  }
  OC_CHECK_HIP(oci::launch_conv_prepare(a, ws, s), "oc_conv3x3x3");
  OC_CHECK_HIP(oci::launch_conv_execute(a, ws, use, s), "oc_conv3x3x3");
  return OC_OK;
}

int oc_conv3x3x3(const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh, int gw,
                 int64_t n_leaves, const float* in, int cin, const float* weight, const float* bias,
                 int cout, int relu, float* out, void* ws, size_t ws_bytes, void* stream) {
  return oc_conv3x3x3_ex(trees, prefix, n, gd, gh, gw, n_leaves, in, cin, weight, bias, cout, relu,
                         out, ws, ws_bytes, OC_CONV_AUTO, stream);
}

int oc_pool2_structure(const uint32_t* in_trees, int n, int gd, int gh, int gw, uint32_t* out_trees,
                       int64_t* out_prefix, int64_t* out_n_leaves, void* ws, size_t ws_bytes,
                       void* stream) {
  g_last_error.clear();
  if (!in_trees || !out_trees || !out_prefix || !out_n_leaves || !ws)
    return fail(OC_EINVAL, "oc_pool2_structure: null pointer");
  if (!dims_ok(n, gd, gh, gw)) return fail(OC_EINVAL, "oc_pool2_structure: non-positive dims");
  if ((gd | gh | gw) & 1) return fail(OC_EINVAL, "oc_pool2_structure: odd tree grid %dx%dx%d", gd, gh, gw);
  const int64_t no = (int64_t)n * (gd / 2) * (gh / 2) * (gw / 2);
  if (ws_bytes < oc_structure_workspace(no)) return fail(OC_EWORKSPACE, "oc_pool2_structure: workspace too small");
  hipStream_t s = as_stream(stream);
  OC_CHECK_HIP(oci::launch_pool_structure(in_trees, n, gd, gh, gw, out_trees,
                                          oci::scan_counts_buffer(ws), s),
               "oc_pool2_structure");
  return finish_prefix(no, out_prefix, out_n_leaves, ws, s, "oc_pool2_structure");
}

int oc_pool2_max(const uint32_t* in_trees, const int64_t* in_prefix, int n, int gd, int gh, int gw,
                 const float* in, int c, const uint32_t* out_trees, const int64_t* out_prefix,
                 float* out, void* stream) {
  g_last_error.clear();
  if (!in_trees || !in_prefix || !in || !out_trees || !out_prefix || !out)
    return fail(OC_EINVAL, "oc_pool2_max: null pointer");
  if (!dims_ok(n, gd, gh, gw) || c <= 0) return fail(OC_EINVAL, "oc_pool2_max: non-positive dims");
  if ((gd | gh | gw) & 1) return fail(OC_EINVAL, "oc_pool2_max: odd tree grid");
  OC_CHECK_HIP(oci::launch_pool_max(in_trees, in_prefix, n, gd, gh, gw, in, c, out_trees, out_prefix,
                                    out, as_stream(stream)),
               "oc_pool2_max");
  return OC_OK;
}

int oc_unpool2_structure(const uint32_t* in_trees, int n, int gd, int gh, int gw,
                         const uint32_t* guide_trees, uint32_t* out_trees, int64_t* out_prefix,
                         int64_t* out_n_leaves, void* ws, size_t ws_bytes, void* stream) {
  g_last_error.clear();
  if (!in_trees || !out_trees || !out_prefix || !out_n_leaves || !ws)
    return fail(OC_EINVAL, "oc_unpool2_structure: null pointer");
  if (!dims_ok(n, gd, gh, gw)) return fail(OC_EINVAL, "oc_unpool2_structure: non-positive dims");
  if (!sizes_ok(n, 2 * gd, 2 * gh, 2 * gw)) return fail(OC_EOVERFLOW, "oc_unpool2_structure: grid too large");
  const int64_t no = 8LL * n * gd * gh * gw;
  if (ws_bytes < oc_structure_workspace(no)) return fail(OC_EWORKSPACE, "oc_unpool2_structure: workspace too small");
  hipStream_t s = as_stream(stream);
  // The mismatch flag of the guided check sits in the last 256 bytes.
  int32_t* mismatch = reinterpret_cast<int32_t*>(static_cast<char*>(ws) + oc_structure_workspace(no) - 256);
  if (guide_trees) OC_CHECK_HIP(hipMemsetAsync(mismatch, 0, sizeof(int32_t), s), "oc_unpool2_structure");
  OC_CHECK_HIP(oci::launch_unpool_structure(in_trees, guide_trees, n, gd, gh, gw, out_trees,
                                            oci::scan_counts_buffer(ws), mismatch, s),
               "oc_unpool2_structure");
  int rc = finish_prefix(no, out_prefix, out_n_leaves, ws, s, "oc_unpool2_structure");
  if (rc != OC_OK) return rc;
  if (guide_trees) {
    int32_t bad = 0;
    OC_CHECK_HIP(hipMemcpyAsync(&bad, mismatch, sizeof(int32_t), hipMemcpyDeviceToHost, s),
                 "oc_unpool2_structure");
    OC_CHECK_HIP(hipStreamSynchronize(s), "oc_unpool2_structure");
    if (bad) return fail(OC_ESTRUCT, "oc_unpool2_structure: guide does not pool to the input (%d trees)", bad);
  }
  return OC_OK;
}

int oc_unpool2(const uint32_t* in_trees, const int64_t* in_prefix, int n, int gd, int gh, int gw,
               const float* in, int c, const uint32_t* out_trees, const int64_t* out_prefix,
               float* out, void* stream) {
  g_last_error.clear();
  if (!in_trees || !in_prefix || !in || !out_trees || !out_prefix || !out)
    return fail(OC_EINVAL, "oc_unpool2: null pointer");
  if (!dims_ok(n, gd, gh, gw) || c <= 0) return fail(OC_EINVAL, "oc_unpool2: non-positive dims");
  OC_CHECK_HIP(oci::launch_unpool(in_trees, in_prefix, n, gd, gh, gw, in, c, out_trees, out_prefix,
                                  out, as_stream(stream)),
               "oc_unpool2");
  return OC_OK;
}

int oc_relu(float* data, int64_t count, void* stream) {
  g_last_error.clear();
  if (!data) return fail(OC_EINVAL, "oc_relu: null pointer");
  if (count < 0) return fail(OC_EINVAL, "oc_relu: negative count");
  OC_CHECK_HIP(oci::launch_relu(data, count, as_stream(stream)), "oc_relu");
  return OC_OK;
}

int oc_conv3x3x3_backward_workspace(int64_t n_trees, int64_t n_leaves, int cin, int cout,
                                    size_t* bytes) {
  g_last_error.clear();
  if (!bytes) return fail(OC_EINVAL, "oc_conv3x3x3_backward_workspace: null pointer");
  if (n_trees <= 0 || n_leaves <= 0 || cin <= 0 || cout <= 0)
    return fail(OC_EINVAL, "oc_conv3x3x3_backward_workspace: non-positive size");
  *bytes = oci::conv_backward_workspace(n_trees, n_leaves, cin, cout);
  return OC_OK;
}

int oc_conv3x3x3_backward(const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh,
                          int gw, int64_t n_leaves, const float* in, int cin, const float* weight,
                          int cout, const float* dout, float* din, float* dweight, float* dbias,
                          void* ws, size_t ws_bytes, void* stream) {
  g_last_error.clear();
  const char* who = "oc_conv3x3x3_backward";
  if (!trees || !prefix || !ws || !dout) return fail(OC_EINVAL, "%s: null pointer", who);
  if (din && !weight) return fail(OC_EINVAL, "%s: din needs weight", who);
  if (dweight && !in) return fail(OC_EINVAL, "%s: dweight needs in", who);
  if (!dims_ok(n, gd, gh, gw)) return fail(OC_EINVAL, "%s: non-positive dims", who);
  if (cin <= 0 || cout <= 0 || cin > 256 || cout > 256)
    return fail(OC_EINVAL, "%s: channels (%d, %d) outside [1,256] x [1,256]", who, cin, cout);
  if (n_leaves <= 0) return fail(OC_EINVAL, "%s: n_leaves <= 0", who);
  if (n_leaves >= (1LL << 31)) return fail(OC_EOVERFLOW, "%s: n_leaves >= 2^31", who);
  const int64_t nt = n_trees_of(n, gd, gh, gw);
  if (n_leaves > 512 * nt) return fail(OC_EINVAL, "%s: n_leaves > 512 * n_trees", who);
  const size_t need = oci::conv_backward_workspace(nt, n_leaves, cin, cout);
  if (ws_bytes < need) return fail(OC_EWORKSPACE, "%s: workspace %zu < %zu", who, ws_bytes, need);
  if (dweight && !oci::conv_backward_supported(cin, cout))
    return fail(OC_EINVAL, "%s: no weight-gradient kernel for (%d, %d)", who, cin, cout);
  oci::ConvBwdArgs a;
  a.trees = trees; a.prefix = prefix;
  a.n = n; a.gd = gd; a.gh = gh; a.gw = gw;
  a.n_trees = nt; a.n_leaves = n_leaves;
  a.in = in; a.cin = cin; a.weight = weight; a.cout = cout;
  a.dy = dout; a.dx = din; a.dweight = dweight; a.dbias = dbias;
  OC_CHECK_HIP(oci::launch_conv_backward(a, ws, as_stream(stream)), who);
  return OC_OK;
}

int oc_pool2_max_backward(const uint32_t* in_trees, const int64_t* in_prefix, int n, int gd, int gh,
                          int gw, const float* in, int c, const uint32_t* out_trees,
                          const int64_t* out_prefix, const float* dout, float* din, void* stream) {
  g_last_error.clear();
  if (!in_trees || !in_prefix || !in || !out_trees || !out_prefix || !dout || !din)
    return fail(OC_EINVAL, "oc_pool2_max_backward: null pointer");
  if (!dims_ok(n, gd, gh, gw) || c <= 0)
    return fail(OC_EINVAL, "oc_pool2_max_backward: non-positive dims");
  if ((gd | gh | gw) & 1) return fail(OC_EINVAL, "oc_pool2_max_backward: odd tree grid");
  OC_CHECK_HIP(oci::launch_pool_max_bwd(in_trees, in_prefix, n, gd, gh, gw, in, c, out_trees,
                                        out_prefix, dout, din, as_stream(stream)),
               "oc_pool2_max_backward");
  return OC_OK;
}

int oc_unpool2_backward(const uint32_t* in_trees, const int64_t* in_prefix, int n, int gd, int gh,
                        int gw, int64_t in_n_leaves, int c, const uint32_t* out_trees,
                        const int64_t* out_prefix, const float* dout, float* din, void* stream) {
  g_last_error.clear();
  if (!in_trees || !in_prefix || !out_trees || !out_prefix || !dout || !din)
    return fail(OC_EINVAL, "oc_unpool2_backward: null pointer");
  if (!dims_ok(n, gd, gh, gw) || c <= 0 || in_n_leaves <= 0)
    return fail(OC_EINVAL, "oc_unpool2_backward: non-positive dims");
  if (in_n_leaves > 512 * n_trees_of(n, gd, gh, gw))
    return fail(OC_EINVAL, "oc_unpool2_backward: in_n_leaves > 512 * n_trees");
  if (!sizes_ok(n, 2 * gd, 2 * gh, 2 * gw)) return fail(OC_EOVERFLOW, "oc_unpool2_backward: grid too large");
  OC_CHECK_HIP(oci::launch_unpool_bwd(in_trees, in_prefix, n, gd, gh, gw, in_n_leaves, c, out_trees,
                                      out_prefix, dout, din, as_stream(stream)),
               "oc_unpool2_backward");
  return OC_OK;
}

int oc_relu_backward(const float* out, const float* dout, float* din, int64_t count, void* stream) {
  g_last_error.clear();
  if (count < 0) return fail(OC_EINVAL, "oc_relu_backward: negative count");
  if (count == 0) return OC_OK;
  if (!out || !dout || !din) return fail(OC_EINVAL, "oc_relu_backward: null pointer");
  OC_CHECK_HIP(oci::launch_relu_bwd(out, dout, din, count, as_stream(stream)), "oc_relu_backward");
  return OC_OK;
}

int oc_concat(const float* a, int ca, const float* b, int cb, int64_t n_rows, float* out, void* stream) {
  g_last_error.clear();
  if (ca <= 0 || cb <= 0 || n_rows < 0) return fail(OC_EINVAL, "oc_concat: non-positive size");
  if (n_rows == 0) return OC_OK;
  if (!a || !b || !out) return fail(OC_EINVAL, "oc_concat: null pointer");
  if ((double)n_rows * (ca + cb) >= 9.0e18) return fail(OC_EOVERFLOW, "oc_concat: too large");
  OC_CHECK_HIP(oci::launch_concat(a, ca, b, cb, n_rows, out, as_stream(stream)), "oc_concat");
  return OC_OK;
}

int oc_concat_backward(const float* dout, int ca, int cb, int64_t n_rows, float* da, float* db,
                       void* stream) {
  g_last_error.clear();
  if (ca <= 0 || cb <= 0 || n_rows < 0) return fail(OC_EINVAL, "oc_concat_backward: non-positive size");
  if (n_rows == 0 || (!da && !db)) return OC_OK;
  if (!dout) return fail(OC_EINVAL, "oc_concat_backward: null pointer");
  OC_CHECK_HIP(oci::launch_split(dout, ca, cb, n_rows, da, db, as_stream(stream)), "oc_concat_backward");
  return OC_OK;
}

int oc_add(const float* a, const float* b, float* out, int64_t count, void* stream) {
  g_last_error.clear();
  if (count < 0) return fail(OC_EINVAL, "oc_add: negative count");
  if (count == 0) return OC_OK;
  if (!a || !b || !out) return fail(OC_EINVAL, "oc_add: null pointer");
  OC_CHECK_HIP(oci::launch_add(a, b, out, count, as_stream(stream)), "oc_add");
  return OC_OK;
}

int oc_points_voxelize(const float* pts, const int32_t* batch, int64_t n_pts, int n, int gd, int gh,
                       int gw, uint8_t* occ, void* stream) {
  g_last_error.clear();
  if (!occ || (n_pts > 0 && !pts)) return fail(OC_EINVAL, "oc_points_voxelize: null pointer");
  if (!dims_ok(n, gd, gh, gw) || n_pts < 0) return fail(OC_EINVAL, "oc_points_voxelize: non-positive dims");
  if (!sizes_ok(n, gd, gh, gw)) return fail(OC_EOVERFLOW, "oc_points_voxelize: grid too large");
  OC_CHECK_HIP(oci::launch_voxelize(pts, batch, n_pts, n, gd, gh, gw, occ, as_stream(stream)),
               "oc_points_voxelize");
  return OC_OK;
}

int oc_points_leaf_rows(const uint32_t* trees, const int64_t* prefix, int n, int gd, int gh, int gw,
                        const float* pts, const int32_t* batch, int64_t n_pts, int32_t* rows,
                        void* stream) {
  g_last_error.clear();
  if (n_pts < 0 || !dims_ok(n, gd, gh, gw)) return fail(OC_EINVAL, "oc_points_leaf_rows: bad size");
  if (n_pts == 0) return OC_OK;
  if (!trees || !prefix || !pts || !rows) return fail(OC_EINVAL, "oc_points_leaf_rows: null pointer");
  if (!sizes_ok(n, gd, gh, gw)) return fail(OC_EOVERFLOW, "oc_points_leaf_rows: grid too large");
  OC_CHECK_HIP(oci::launch_point_rows(trees, prefix, n, gd, gh, gw, pts, batch, n_pts, rows,
                                      as_stream(stream)),
               "oc_points_leaf_rows");
  return OC_OK;
}

size_t oc_points_workspace(int64_t n_leaves, int n_labels) {
  const int64_t per = n_labels > 1 ? n_labels : 1;
  return (size_t)(n_leaves > 0 ? n_leaves : 0) * (size_t)per * sizeof(uint32_t) + 256;
}

int oc_points_average(const int32_t* rows, int64_t n_pts, const float* feat, int c, int64_t n_leaves,
                      float* out, void* ws, size_t ws_bytes, void* stream) {
  g_last_error.clear();
  if (n_pts < 0 || c < 0 || n_leaves <= 0) return fail(OC_EINVAL, "oc_points_average: bad size");
  if (!out || !ws || (n_pts > 0 && (!rows || (c > 0 && !feat))))
    return fail(OC_EINVAL, "oc_points_average: null pointer");
  if (ws_bytes < oc_points_workspace(n_leaves, 1))
    return fail(OC_EWORKSPACE, "oc_points_average: workspace too small");
  OC_CHECK_HIP(oci::launch_point_means(rows, n_pts, feat, c, n_leaves, out, static_cast<uint32_t*>(ws),
                                       as_stream(stream)),
               "oc_points_average");
  return OC_OK;
}

int oc_points_vote(const int32_t* rows, int64_t n_pts, const int32_t* labels, int n_labels,
                   int64_t n_leaves, int32_t* out, void* ws, size_t ws_bytes, void* stream) {
  g_last_error.clear();
  if (n_pts < 0 || n_labels <= 0 || n_leaves <= 0) return fail(OC_EINVAL, "oc_points_vote: bad size");
  if (!out || !ws || (n_pts > 0 && (!rows || !labels))) return fail(OC_EINVAL, "oc_points_vote: null pointer");
  if (ws_bytes < oc_points_workspace(n_leaves, n_labels))
    return fail(OC_EWORKSPACE, "oc_points_vote: workspace too small");
  OC_CHECK_HIP(oci::launch_label_vote(rows, n_pts, labels, n_labels, n_leaves, out,
                                      static_cast<uint32_t*>(ws), as_stream(stream)),
               "oc_points_vote");
  return OC_OK;
}

namespace {

int type_bytes(int dtype) { return dtype == OC_F32 ? 4 : 2; }

bool type_ok(int dtype) { return dtype == OC_F32 || dtype == OC_F16 || dtype == OC_BF16; }

bool aligned16(const void* p) { return ((uintptr_t)p & 15) == 0; }

// Sizes that the attention kernels' 32-bit row numbers and grids hold.
int attention_sizes(const char* who, int64_t n_q, int64_t n_k, int n_seq, int heads, int kv_heads, int dim) {
  if (n_q < 0 || n_k < 0 || n_seq <= 0) return fail(OC_EINVAL, "%s: negative size, or no sequence", who);
  if (heads <= 0 || kv_heads <= 0 || heads % kv_heads)
    return fail(OC_EINVAL, "%s: %d heads for %d key heads", who, heads, kv_heads);
  if (dim < 8 || dim > 128 || dim % 8) return fail(OC_EINVAL, "%s: head size %d is no multiple of 8 in [8, 128]", who, dim);
  const int64_t most = (1LL << 31) - 256;
  if (n_q > most / heads || n_k > most / kv_heads) return fail(OC_EOVERFLOW, "%s: more than 2^31 rows", who);
  const int64_t rows = n_q * (heads / kv_heads) > n_k ? n_q * (heads / kv_heads) : n_k;
  if ((rows / 32 + n_seq) > most / kv_heads / 128) return fail(OC_EOVERFLOW, "%s: too many row tiles", who);
  return OC_OK;
}

int attention_args(const char* who, const void* q, int64_t q_row, int64_t q_head, const void* k, int64_t k_row,
                   int64_t k_head, const void* v, int64_t v_row, int64_t v_head, const int64_t* q_off,
                   const int64_t* k_off, int n_seq, int64_t n_q, int64_t n_k, int heads, int kv_heads, int dim,
                   int dtype, float scale, int causal, oci::AttnArgs* a) {
  const int rc = attention_sizes(who, n_q, n_k, n_seq, heads, kv_heads, dim);
  if (rc != OC_OK) return rc;
  if (!type_ok(dtype)) return fail(OC_EINVAL, "%s: bad type %d", who, dtype);
  if ((n_q > 0 && !q) || (n_k > 0 && (!k || !v))) return fail(OC_EINVAL, "%s: null pointer", who);
  if (n_seq > 1 && (!q_off || !k_off)) return fail(OC_EINVAL, "%s: %d sequences without offsets", who, n_seq);
  if (!(scale > 0.f) || !isfinite(scale)) return fail(OC_EINVAL, "%s: scale %g is not positive", who, scale);
  const int64_t strides[] = {q_row, q_head, k_row, k_head, v_row, v_head};
  for (int64_t x : strides)
    if (x < 0 || x >= (1LL << 40) || x * type_bytes(dtype) % 16)
      return fail(OC_EINVAL, "%s: stride %lld is negative, too large or no multiple of 16 bytes", who, (long long)x);
  // The gradient forms a query's place from 32-bit factors.
  if (q_row >= (1LL << 32) || q_head >= (1LL << 32)) return fail(OC_EOVERFLOW, "%s: query strides >= 2^32", who);
  if (!aligned16(q) || !aligned16(k) || !aligned16(v)) return fail(OC_EINVAL, "%s: pointer not aligned to 16 bytes", who);
  *a = oci::AttnArgs();
  a->q = q; a->k = k; a->v = v;
  a->q_row = q_row; a->q_head = q_head; a->k_row = k_row; a->k_head = k_head; a->v_row = v_row; a->v_head = v_head;
  a->q_off = q_off; a->k_off = k_off;
  a->n_seq = n_seq; a->n_q = n_q; a->n_k = n_k;
  a->heads = heads; a->kv_heads = kv_heads; a->dim = dim;
  a->scale = scale; a->causal = causal ? 1 : 0;
  a->n_split = 1;
  oci::attention_set_group(a);
  return OC_OK;
}

}  // namespace

int oc_attention_workspace(int64_t n_q, int64_t n_k, int n_seq, int heads, int kv_heads, int dim, int dtype,
                           size_t* bytes) {
  g_last_error.clear();
  if (!bytes) return fail(OC_EINVAL, "oc_attention_workspace: null pointer");
  const int rc = attention_sizes("oc_attention_workspace", n_q, n_k, n_seq, heads, kv_heads, dim);
  if (rc != OC_OK) return rc;
  if (!type_ok(dtype)) return fail(OC_EINVAL, "oc_attention_workspace: bad type %d", dtype);
  // Causal calls take as many parts as others, or more.
  const int n = oci::attention_splits(n_q, n_k, n_seq, heads, kv_heads, dtype, true);
  const size_t rows = (size_t)n_q * heads;
  *bytes = n > 1 ? oci::align256(4 * n * rows * dim) + oci::align256(4 * n * rows) : 0;
  return OC_OK;
}

int oc_attention(const void* q, int64_t q_row, int64_t q_head, const void* k, int64_t k_row, int64_t k_head,
                 const void* v, int64_t v_row, int64_t v_head, const int64_t* q_off, const int64_t* k_off,
                 const int64_t* k_len, int n_seq, int64_t n_q, int64_t n_k, int heads, int kv_heads, int dim,
                 int dtype, float scale, int causal, void* out, float* lse, void* ws, size_t ws_bytes,
                 void* stream) {
  g_last_error.clear();
  oci::AttnArgs a;
  const int rc = attention_args("oc_attention", q, q_row, q_head, k, k_row, k_head, v, v_row, v_head, q_off, k_off,
                                n_seq, n_q, n_k, heads, kv_heads, dim, dtype, scale, causal, &a);
  if (rc != OC_OK) return rc;
  if (n_q == 0) return OC_OK;
  if (!out || !lse) return fail(OC_EINVAL, "oc_attention: null pointer");
  if (!aligned16(out)) return fail(OC_EINVAL, "oc_attention: pointer not aligned to 16 bytes");
  a.k_len = k_len;
  a.out = out;
  a.lse = lse;
  a.n_split = oci::attention_splits(n_q, n_k, n_seq, heads, kv_heads, dtype, causal != 0);
  if (a.n_split > 1) {
    const size_t rows = (size_t)n_q * heads, part = oci::align256(4 * a.n_split * rows * dim);
    if (!ws || ws_bytes < part + oci::align256(4 * a.n_split * rows))
      return fail(OC_EWORKSPACE, "oc_attention: workspace too small");
    if (!aligned16(ws)) return fail(OC_EINVAL, "oc_attention: workspace not aligned to 16 bytes");
    a.part = static_cast<float*>(ws);
    a.part_lse = reinterpret_cast<float*>(static_cast<char*>(ws) + part);
  }
  OC_CHECK_HIP(oci::launch_attention(a, dtype, as_stream(stream)), "oc_attention");
  return OC_OK;
}

int oc_attention_backward_workspace(int64_t n_q, int64_t n_k, int n_seq, int heads, int kv_heads, int dim,
                                    int dtype, size_t* bytes) {
  g_last_error.clear();
  if (!bytes) return fail(OC_EINVAL, "oc_attention_backward_workspace: null pointer");
  const int rc = attention_sizes("oc_attention_backward_workspace", n_q, n_k, n_seq, heads, kv_heads, dim);
  if (rc != OC_OK) return rc;
  if (!type_ok(dtype)) return fail(OC_EINVAL, "oc_attention_backward_workspace: bad type %d", dtype);
  *bytes = 2 * oci::align256(4 * (size_t)n_q * heads) +
           oci::attention_back_parts(n_q, n_k, n_seq, heads, kv_heads, dim, dtype, true).bytes;
  return OC_OK;
}

int oc_attention_backward(const void* q, int64_t q_row, int64_t q_head, const void* k, int64_t k_row,
                          int64_t k_head, const void* v, int64_t v_row, int64_t v_head, const void* out,
                          const float* lse, const void* dout, const int64_t* q_off, const int64_t* k_off,
                          int n_seq, int64_t n_q, int64_t n_k, int heads, int kv_heads, int dim, int dtype,
                          float scale, int causal, void* dq, void* dk, void* dv, void* ws, size_t ws_bytes,
                          void* stream) {
  g_last_error.clear();
  oci::AttnArgs a;
  const int rc = attention_args("oc_attention_backward", q, q_row, q_head, k, k_row, k_head, v, v_row, v_head, q_off,
                                k_off, n_seq, n_q, n_k, heads, kv_heads, dim, dtype, scale, causal, &a);
  if (rc != OC_OK) return rc;
  if ((n_q > 0 && (!out || !lse || !dout || !dq)) || (n_k > 0 && (!dk || !dv)))
    return fail(OC_EINVAL, "oc_attention_backward: null pointer");
  if (!aligned16(out) || !aligned16(dout) || !aligned16(dq) || !aligned16(dk) || !aligned16(dv))
    return fail(OC_EINVAL, "oc_attention_backward: pointer not aligned to 16 bytes");
  const size_t part = oci::align256(4 * (size_t)n_q * heads);
  const size_t need = 2 * part +
                      oci::attention_back_parts(n_q, n_k, n_seq, heads, kv_heads, dim, dtype, causal != 0).bytes;
  if (need && (!ws || ws_bytes < need)) return fail(OC_EWORKSPACE, "oc_attention_backward: workspace too small");
  if (!aligned16(ws)) return fail(OC_EINVAL, "oc_attention_backward: workspace not aligned to 16 bytes");
  a.out = const_cast<void*>(out);
  a.lse = const_cast<float*>(lse);
  a.dout = dout;
  a.dq = dq; a.dk = dk; a.dv = dv;
  a.delta = static_cast<float*>(ws);
  a.lse2 = reinterpret_cast<float*>(static_cast<char*>(ws) + part);
  a.part = reinterpret_cast<float*>(static_cast<char*>(ws) + 2 * part);
  OC_CHECK_HIP(oci::launch_attention_backward(a, dtype, as_stream(stream)), "oc_attention_backward");
  return OC_OK;
}

namespace {

int norm_sizes(const char* who, int64_t rows, int c) {
  if (rows < 0 || c <= 0 || c > oci::kNormMaxWidth)
    return fail(OC_EINVAL, "%s: %lld rows of width %d (1 to %d)", who, (long long)rows, c, oci::kNormMaxWidth);
  if (rows > (1LL << 62) / c / 8) return fail(OC_EOVERFLOW, "%s: too many rows", who);
  return OC_OK;
}

}  // namespace

int oc_rms_norm(const void* x, int x_type, const void* residual, int sum_type, const float* weight, int64_t rows,
                int c, float eps, void* sum, void* y, int y_type, float* scale, void* stream) {
  g_last_error.clear();
  const int rc = norm_sizes("oc_rms_norm", rows, c);
  if (rc != OC_OK) return rc;
  if (!type_ok(x_type) || (sum_type != x_type && sum_type != OC_F32))
    return fail(OC_EINVAL, "oc_rms_norm: bad types %d, %d", x_type, sum_type);
  if (y_type != x_type && y_type != OC_F8 && !(x_type == OC_F32 && type_ok(y_type)))
    return fail(OC_EINVAL, "oc_rms_norm: output type %d for input type %d", y_type, x_type);
  if (!(eps >= 0.f)) return fail(OC_EINVAL, "oc_rms_norm: eps %g is negative", eps);
  if (rows == 0) return OC_OK;
  if (!x || !weight || !y || (y_type == OC_F8 && !scale)) return fail(OC_EINVAL, "oc_rms_norm: null pointer");
  oci::NormArgs a = oci::NormArgs();
  a.x = x; a.residual = residual; a.weight = weight;
  a.rows = rows; a.c = c; a.eps = eps;
  a.sum = sum; a.y = y; a.scale = scale;
  OC_CHECK_HIP(oci::launch_rms_norm(a, x_type, sum_type, y_type, as_stream(stream)), "oc_rms_norm");
  return OC_OK;
}

int oc_rms_norm_backward_workspace(int64_t rows, int c, size_t* bytes) {
  g_last_error.clear();
  if (!bytes) return fail(OC_EINVAL, "oc_rms_norm_backward_workspace: null pointer");
  const int rc = norm_sizes("oc_rms_norm_backward_workspace", rows, c);
  if (rc != OC_OK) return rc;
  *bytes = oci::align256(4 * (size_t)oci::norm_back_groups(rows, c) * c);
  return OC_OK;
}

int oc_rms_norm_backward(const void* sum, int sum_type, const float* weight, const void* dy, int y_type,
                         const void* dsum, int64_t rows, int c, float eps, void* dx, float* dweight, void* ws,
                         size_t ws_bytes, void* stream) {
  g_last_error.clear();
  const int rc = norm_sizes("oc_rms_norm_backward", rows, c);
  if (rc != OC_OK) return rc;
  if (!type_ok(sum_type) || !type_ok(y_type) || (sum_type != y_type && sum_type != OC_F32))
    return fail(OC_EINVAL, "oc_rms_norm_backward: bad types %d, %d", sum_type, y_type);
  if (!(eps >= 0.f)) return fail(OC_EINVAL, "oc_rms_norm_backward: eps %g is negative", eps);
  if (!weight || (rows > 0 && (!sum || !dy || !dx))) return fail(OC_EINVAL, "oc_rms_norm_backward: null pointer");
  if (rows == 0 && !dweight) return OC_OK;
  const size_t need = 4 * (size_t)oci::norm_back_groups(rows, c) * c;
  if (dweight && need && (!ws || ws_bytes < need)) return fail(OC_EWORKSPACE, "oc_rms_norm_backward: workspace too small");
  oci::NormArgs a = oci::NormArgs();
  a.weight = weight;
  a.rows = rows; a.c = c; a.eps = eps;
  a.sum = const_cast<void*>(sum); a.dy = dy; a.dsum = dsum; a.dx = dx;
  a.part = dweight ? static_cast<float*>(ws) : nullptr;
  OC_CHECK_HIP(oci::launch_rms_norm_back(a, sum_type, y_type, dweight, as_stream(stream)), "oc_rms_norm_backward");
  return OC_OK;
}

namespace {

int label_sizes(const char* who, int64_t rows, int classes, int top) {
  if (rows < 0 || classes <= 0) return fail(OC_EINVAL, "%s: %lld rows of %d classes", who, (long long)rows, classes);
  if (top < 0 || top > oci::kMostTop || top > classes)
    return fail(OC_EINVAL, "%s: top %d of %d classes (at most %d)", who, top, classes, oci::kMostTop);
  if (rows >= (1LL << 31)) return fail(OC_EOVERFLOW, "%s: rows >= 2^31", who);
  if (classes > (1 << 29)) return fail(OC_EOVERFLOW, "%s: classes > 2^29", who);
  return OC_OK;
}

// Offsets of the parts of long rows in the workspace: statistics, values,
// indices, end.
void label_parts_at(int64_t rows, int classes, int top, size_t at[4]) {
  const int parts = oci::label_parts(rows, classes);
  const size_t n = parts > 1 ? (size_t)rows * parts : 0;
  at[0] = 0;
  at[1] = oci::align256(12 * n);
  at[2] = at[1] + oci::align256(4 * n * top);
  at[3] = at[2] + oci::align256(4 * n * top);
}

}  // namespace

int oc_label_logprobs_workspace(int64_t rows, int classes, int top, size_t* bytes) {
  g_last_error.clear();
  if (!bytes) return fail(OC_EINVAL, "oc_label_logprobs_workspace: null pointer");
  const int rc = label_sizes("oc_label_logprobs_workspace", rows, classes, top);
  if (rc != OC_OK) return rc;
  size_t at[4];
  label_parts_at(rows, classes, top, at);
  *bytes = at[3];
  return OC_OK;
}

int oc_label_logprobs(const void* logits, int dtype, const int32_t* labels, int64_t rows, int classes, int top,
                      float* logprob, float* lse, float* entropy, float* top_logprob, int32_t* top_label, void* ws,
                      size_t ws_bytes, void* stream) {
  g_last_error.clear();
  const int rc = label_sizes("oc_label_logprobs", rows, classes, top);
  if (rc != OC_OK) return rc;
  if (!type_ok(dtype)) return fail(OC_EINVAL, "oc_label_logprobs: bad type %d", dtype);
  if (rows == 0) return OC_OK;
  if (!logits || !labels || !logprob || !lse || (top && (!top_logprob || !top_label)))
    return fail(OC_EINVAL, "oc_label_logprobs: null pointer");
  size_t at[4];
  label_parts_at(rows, classes, top, at);
  if (at[3] && (!ws || ws_bytes < at[3])) return fail(OC_EWORKSPACE, "oc_label_logprobs: workspace too small");
  if (!aligned16(ws)) return fail(OC_EINVAL, "oc_label_logprobs: workspace not aligned to 16 bytes");
  oci::LabelArgs a = oci::LabelArgs();
  a.logits = logits; a.labels = labels;
  a.rows = rows; a.classes = classes; a.top = top;
  a.logprob = logprob; a.lse = lse; a.entropy = entropy;
  a.top_logprob = top_logprob; a.top_label = top_label;
  a.part_stat = static_cast<float*>(ws);
  a.part_val = reinterpret_cast<float*>(static_cast<char*>(ws) + at[1]);
  a.part_idx = reinterpret_cast<int*>(static_cast<char*>(ws) + at[2]);
  OC_CHECK_HIP(oci::launch_labels(a, dtype, as_stream(stream)), "oc_label_logprobs");
  return OC_OK;
}

int oc_label_logprobs_backward(const void* logits, int dtype, const int32_t* labels, int64_t rows, int classes,
                               const float* lse, const float* dlogprob, const float* entropy,
                               const float* dentropy, void* dlogits, void* stream) {
  g_last_error.clear();
  const int rc = label_sizes("oc_label_logprobs_backward", rows, classes, 0);
  if (rc != OC_OK) return rc;
  if (!type_ok(dtype)) return fail(OC_EINVAL, "oc_label_logprobs_backward: bad type %d", dtype);
  if (rows == 0) return OC_OK;
  if (!logits || !labels || !lse || !dlogits || (dentropy && !entropy))
    return fail(OC_EINVAL, "oc_label_logprobs_backward: null pointer");
  oci::LabelArgs a = oci::LabelArgs();
  a.logits = logits; a.labels = labels;
  a.rows = rows; a.classes = classes;
  a.lse = const_cast<float*>(lse); a.entropy = const_cast<float*>(entropy);
  a.dlogprob = dlogprob; a.dentropy = dentropy; a.dlogits = dlogits;
  OC_CHECK_HIP(oci::launch_labels_back(a, dtype, as_stream(stream)), "oc_label_logprobs_backward");
  return OC_OK;
}

}  // extern "C"

namespace {

int64_t clip_chunks(int64_t count) { return (count + oci::kClipChunk - 1) / oci::kClipChunk; }

// Walks the tensors in batches of one launch: f(batch, workgroups, first partial sum).
template <class F>
int each_clip_batch(const void* const* grads, void* const* out, const int64_t* counts, const int* dtypes, int n, F f) {
  int64_t parts = 0;
  for (int i = 0; i < n;) {
    oci::ClipBatch b;
    b.n = 0;
    b.first[0] = 0;
    int64_t chunks = 0;
    for (; i < n && b.n < oci::kClipBatch; ++i) {
      if (counts[i] == 0) continue;
      const int64_t more = clip_chunks(counts[i]);
      if (chunks + more > 0x7fffffff) break;
      b.in[b.n] = grads ? grads[i] : nullptr;
      b.out[b.n] = out ? out[i] : nullptr;
      b.count[b.n] = counts[i];
      b.type[b.n] = dtypes ? (uint8_t)dtypes[i] : 0;
      chunks += more;
      b.first[++b.n] = (uint32_t)chunks;
    }
    const int groups = (int)(chunks < oci::kClipParts ? chunks : oci::kClipParts);
    const int rc = f(b, groups, parts);
    if (rc != OC_OK) return rc;
    parts += groups;
  }
  return OC_OK;
}

int clip_counts(const char* who, const int64_t* counts, int n) {
  if (n < 0 || (n > 0 && !counts)) return fail(OC_EINVAL, "%s: null pointer or negative count of tensors", who);
  for (int i = 0; i < n; ++i) {
    if (counts[i] < 0) return fail(OC_EINVAL, "%s: tensor %d has %lld elements", who, i, (long long)counts[i]);
    if (clip_chunks(counts[i]) > 0x7fffffff) return fail(OC_EOVERFLOW, "%s: tensor %d too large", who, i);
  }
  return OC_OK;
}

}  // namespace

extern "C" {

int oc_clip_grad_norm_workspace(const int64_t* counts, int n, size_t* bytes) {
  g_last_error.clear();
  if (!bytes) return fail(OC_EINVAL, "oc_clip_grad_norm_workspace: null pointer");
  const int rc = clip_counts("oc_clip_grad_norm_workspace", counts, n);
  if (rc != OC_OK) return rc;
  int64_t parts = 0;
  each_clip_batch(nullptr, nullptr, counts, nullptr, n, [&](const oci::ClipBatch&, int groups, int64_t) {
    parts += groups;
    return OC_OK;
  });
  *bytes = oci::align256(8 * (size_t)parts + 8);
  return OC_OK;
}

int oc_clip_grad_norm(const void* const* grads, void* const* out, const int64_t* counts, const int* dtypes, int n,
                      float max_norm, float* norm, void* ws, size_t ws_bytes, void* stream) {
  g_last_error.clear();
  const int rc = clip_counts("oc_clip_grad_norm", counts, n);
  if (rc != OC_OK) return rc;
  if (!norm || (n > 0 && (!grads || !out || !dtypes))) return fail(OC_EINVAL, "oc_clip_grad_norm: null pointer");
  if (!(max_norm >= 0.f)) return fail(OC_EINVAL, "oc_clip_grad_norm: max_norm %g is negative", max_norm);
  for (int i = 0; i < n; ++i) {
    if (!type_ok(dtypes[i])) return fail(OC_EINVAL, "oc_clip_grad_norm: tensor %d has a bad type %d", i, dtypes[i]);
    if (counts[i] > 0 && (!grads[i] || !out[i])) return fail(OC_EINVAL, "oc_clip_grad_norm: tensor %d is null", i);
    const uintptr_t step = (uintptr_t)type_bytes(dtypes[i]) - 1;
    if (((uintptr_t)grads[i] | (uintptr_t)out[i]) & step)
      return fail(OC_EINVAL, "oc_clip_grad_norm: tensor %d is not aligned to its elements", i);
  }
  size_t need = 0;
  oc_clip_grad_norm_workspace(counts, n, &need);
  if (!ws || ws_bytes < need) return fail(OC_EWORKSPACE, "oc_clip_grad_norm: workspace too small");
  if ((uintptr_t)ws & 7) return fail(OC_EINVAL, "oc_clip_grad_norm: workspace not aligned to 8 bytes");
  hipStream_t s = as_stream(stream);
  double* parts = static_cast<double*>(ws);
  int64_t total = 0;
  int done = each_clip_batch(grads, out, counts, dtypes, n, [&](const oci::ClipBatch& b, int groups, int64_t at) {
    total = at + groups;
    if (groups == 0) return OC_OK;
    OC_CHECK_HIP(oci::launch_square_sums(b, parts + at, groups, s), "oc_clip_grad_norm");
    return OC_OK;
  });
  if (done != OC_OK) return done;
  bool any = false;
  done = each_clip_batch(grads, out, counts, dtypes, n, [&](const oci::ClipBatch& b, int groups, int64_t) {
    if (groups == 0) return OC_OK;
    any = true;
    OC_CHECK_HIP(oci::launch_clip(b, parts, (int)total, max_norm, norm, groups, s), "oc_clip_grad_norm");
    return OC_OK;
  });
  if (done != OC_OK || any) return done;
  // No element at all: the norm of nothing.
  oci::ClipBatch none;
  none.n = 0;
  none.first[0] = 0;
  OC_CHECK_HIP(oci::launch_clip(none, parts, 0, max_norm, norm, 1, s), "oc_clip_grad_norm");
  return OC_OK;
}

}  // extern "C"
