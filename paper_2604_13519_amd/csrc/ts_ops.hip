// Host side shared by the device-tensor operators (include/toolspec_ops.h), and their door to the caches of toolspec.h.
#include "ts_ops.h"

ts_status ops_device(const char* call, std::initializer_list<const void*> pointers, ts_stream stream, int* device) {
  int dev = -1;
  // A lookup is 0.2 us of a call's 4 to 6 in the library.  Small tensors of a program mostly lie in a few allocations: what lies in one
  // that this call has met needs none (append of 15 pointers 12.0 -> 11.4 us a call, through the binding).  An allocation's bounds cost about as
  // much as half a lookup, so calls of few pointers do without (product with 4-bit weights, three allocations: 6.2 us, with bounds 6.4).
  struct { uintptr_t from, to; } met[4];
  int n_met = 0;
  const bool bounds = pointers.size() > 8;
  for (const void* p : pointers) {
    if (!p) continue;
    bool inside = false;
    for (int i = 0; i < n_met; ++i) inside = inside || ((uintptr_t)p >= met[i].from && (uintptr_t)p < met[i].to);
    if (inside) continue;
    hipPointerAttribute_t a;
    const hipError_t e = hipPointerGetAttributes(&a, p);
    if (e != hipSuccess || (a.type != hipMemoryTypeDevice && a.type != hipMemoryTypeManaged)) {
      (void)hipGetLastError();                                   // a pointer HIP does not know is no lasting error
      return ts_fail(TS_ERR_INVALID_ARG, "%s: %p is not device memory", call, p);
    }
    if (dev >= 0 && a.device != dev) return ts_fail(TS_ERR_INVALID_ARG, "%s: pointers of GPUs %d and %d", call, dev, a.device);
    dev = a.device;
    hipDeviceptr_t base = nullptr;
    size_t size = 0;
    if (bounds && n_met < 4) {
      if (hipMemGetAddressRange(&base, &size, (hipDeviceptr_t)p) == hipSuccess) met[n_met++] = {(uintptr_t)base, (uintptr_t)base + size};
      else (void)hipGetLastError();
    }
  }
  if (dev < 0) return ts_fail(TS_ERR_INVALID_ARG, "%s: null argument", call);
  if (stream) {
    hipDevice_t d = -1;
    const hipError_t e = hipStreamGetDevice((hipStream_t)stream, &d);
    if (e != hipSuccess) { (void)hipGetLastError(); return ts_fail(TS_ERR_INVALID_ARG, "%s: not a stream: %s", call, hipGetErrorString(e)); }
    if (d != dev) return ts_fail(TS_ERR_INVALID_ARG, "%s: pointers of GPU %d on a stream of GPU %d", call, dev, (int)d);
  }
  *device = dev;
  return TS_OK;
}

// ---------------------------------------------------------------------------------
// one layer of a cache, its page table, its length
// ---------------------------------------------------------------------------------
extern "C" ts_status ts_kv_layer_pages(const ts_kv* kv, int32_t layer, ts_kv_pages* pages) {
  if (!kv || !pages) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_layer_pages: null argument");
  const ts_model* m = kv->model;
  if (layer < 0 || layer >= m->cfg.n_layers) return ts_fail(TS_ERR_INVALID_ARG, "layer %d outside [0,%d)", layer, m->cfg.n_layers);
  const size_t off = kv->layer_stride_elems * layer * m->esz;
  pages->k = (char*)kv->k_pool + off;
  pages->v = (char*)kv->v_pool + off;
  pages->n_pages = kv->pool_pages;
  pages->n_kv_heads = m->cfg.n_kv_heads;
  pages->head_dim = m->cfg.head_dim;
  pages->dtype = m->cfg.dtype;
  return TS_OK;
}

extern "C" ts_status ts_kv_page_table(const ts_kv* kv, int32_t* host_pages, int32_t n_pages) {
  if (!kv || !host_pages) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_page_table: null argument");
  if (n_pages != kv->n_pages) return ts_fail(TS_ERR_INVALID_ARG, "n_pages must be %d", kv->n_pages);
  for (int i = 0; i < n_pages; ++i) host_pages[i] = kv->page_table_host[i];
  return TS_OK;
}

extern "C" ts_status ts_kv_extend(ts_kv* kv, int32_t n_pos, ts_stream stream) {
  if (!kv) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_extend: null cache");
  if (n_pos < 0) return ts_fail(TS_ERR_INVALID_ARG, "ts_kv_extend: %d positions", n_pos);
  if (n_pos > kv->capacity - kv->P) return ts_fail(TS_ERR_KV_CAPACITY, "committed %d + %d positions exceed the capacity %d", kv->P, n_pos, kv->capacity);
  int dev;
  if (ts_status st = ops_device("ts_kv_extend", {kv->k_pool}, stream, &dev)) return st;      // a stream of another GPU wrote nothing here
  DeviceGuard on(dev);
  TS_HIP(hipStreamSynchronize((hipStream_t)stream));
  kv->P += n_pos;
  kv->have_result = false;
  return TS_OK;
}
