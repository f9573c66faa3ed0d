// C ABI of the prefix-cache operators (rosa_kv.h) except rosa_generate_kv:
// argument checks, the handle's plan and the launches.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdio>
#include <cstring>
#include <string>
#include <vector>

#include "../../include/rosa_kv.h"
#include "rosa_internal.h"
#include "rosa_plan.h"

using namespace rosa;

struct rosa_kv {
  rosa_model_config cfg{};
  rosa_capacity cap{};
  Dims dims{};
  bool bf16 = true;
  int device = 0;
  hipStream_t stream = nullptr;
  bool poisoned = false;
  std::string last_error;

  // The plan in force.
  bool planned = false;
  bool fp4 = false, has_mass = false;
  int n = 0;
  struct Set {
    int items = 0, item_base = 0;                        // fp32: the set's items
    int list_at = 0, blocks = 0;                         // bf16: its launch list
    int groups = 0, group_base = 0;
  } sets[2];
  int n_mass = 0, mass_keys = 0;
  size_t rows = 0;                   // of the planned set

  // device plan region, two pinned staging copies
  uint8_t *d_plan = nullptr;
  void *h_plan[2] = {nullptr, nullptr};
  hipEvent_t copied[2] = {nullptr, nullptr};
  bool pending[2] = {false, false};
  int flip = 0;
  size_t plan_bytes = 0, off_items = 0, off_groups = 0, off_lists = 0, off_mass = 0;
  size_t max_items = 0, max_groups = 0, max_lists = 0, max_mass = 0;
  float *part_o = nullptr, *part_ml = nullptr;
};

namespace {

thread_local std::string g_kv_error;

rosa_status fail(rosa_kv *h, rosa_status st, const std::string &msg) {
  (h ? h->last_error : g_kv_error) = msg;
  return st;
}

rosa_status device_fail(rosa_kv *h, hipError_t e, const char *what) {
  if (h) h->poisoned = true;
  return fail(h, ROSA_E_DEVICE, std::string(what) + ": " + hipGetErrorString(e));
}

// Makes `device` current and gives the caller's device back at the end.
class DeviceGuard {
 public:
  explicit DeviceGuard(int device) {
    err_ = hipGetDevice(&old_);
    if (err_ == hipSuccess && old_ != device) { err_ = hipSetDevice(device); changed_ = err_ == hipSuccess; }
  }
  ~DeviceGuard() { if (changed_) (void)hipSetDevice(old_); }
  hipError_t error() const { return err_; }

 private:
  int old_ = 0;
  bool changed_ = false;
  hipError_t err_;
};

// The device of a stream; the null stream is the current device's.
hipError_t stream_device(hipStream_t s, int *dev) { return s ? hipStreamGetDevice(s, dev) : hipGetDevice(dev); }

bool aligned(const void *p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

size_t model_bytes(const rosa_model_config *c, int64_t P) {
  return (size_t)c->n_layers * (size_t)P * c->n_kv_heads * c->head_dim * (c->dtype == ROSA_BF16 ? 2 : 4);
}
size_t fp4_bytes(const rosa_model_config *c, int64_t P) {
  return kv4_bytes((size_t)c->n_layers, (size_t)P, (size_t)c->n_kv_heads, (size_t)c->head_dim);
}

rosa_status check_cfg(const rosa_model_config *cfg) {
  if (!cfg) return fail(nullptr, ROSA_E_INVALID, "cfg is NULL");
  const rosa_status st = check_config(cfg);
  return st == ROSA_OK ? st : fail(nullptr, st, "model configuration not supported");
}

rosa_status convert(const rosa_model_config *cfg, const rosa_kv_job *jobs, int32_t n, void *hip_stream, bool pack) {
  try {
    g_kv_error.clear();
    rosa_status st = check_cfg(cfg);
    if (st != ROSA_OK) return st;
    if (n < 0 || (n > 0 && !jobs)) return fail(nullptr, ROSA_E_INVALID, "n < 0 or jobs is NULL");
    std::vector<Range> ranges;
    std::vector<KvJob> work;
    for (int i = 0; i < n; ++i) {
      const rosa_kv_job &j = jobs[i];
      if (j.prefix_len < 0 || j.reserved != 0) return fail(nullptr, ROSA_E_INVALID, "prefix_len < 0 or reserved not 0");
      if (j.prefix_len == 0) continue;
      const void *p[4] = {j.src_k, j.src_v, j.dst_k, j.dst_v};
      for (const void *q : p)
        if (!q || !aligned(q, 16)) return fail(nullptr, ROSA_E_INVALID, "a cache is NULL or not 16-byte aligned");
      const size_t m = model_bytes(cfg, j.prefix_len), f = fp4_bytes(cfg, j.prefix_len);
      add_range(ranges, j.src_k, pack ? m : f, false);
      add_range(ranges, j.src_v, pack ? m : f, false);
      add_range(ranges, j.dst_k, pack ? f : m, true);
      add_range(ranges, j.dst_v, pack ? f : m, true);
      work.push_back({j.src_k, j.src_v, j.dst_k, j.dst_v, j.prefix_len, 0});
    }
    if (clash(ranges)) return fail(nullptr, ROSA_E_INVALID, "a destination overlaps another array of the call");
    int dev = 0;
    const hipStream_t s = (hipStream_t)hip_stream;
    hipError_t e = work.empty() ? hipSuccess : stream_device(s, &dev);
    if (e != hipSuccess) return device_fail(nullptr, e, "device of the stream");
    if (work.empty()) return ROSA_OK;
    DeviceGuard guard(dev);
    e = guard.error();
    for (size_t at = 0; at < work.size() && e == hipSuccess; at += kKvJobs) {
      KvJobs part{};
      const int k = (int)std::min<size_t>(kKvJobs, work.size() - at);
      std::copy(work.begin() + at, work.begin() + at + k, part.j);
      const bool bf16 = cfg->dtype == ROSA_BF16;
      e = pack ? launch_kv_quantize(part, k, cfg->n_layers, cfg->n_kv_heads, cfg->head_dim, bf16, s)
               : launch_kv_expand(part, k, cfg->n_layers, cfg->n_kv_heads, cfg->head_dim, bf16, s);
    }
    return e == hipSuccess ? ROSA_OK : device_fail(nullptr, e, "cache conversion");
  } catch (const std::bad_alloc &) {
    return fail(nullptr, ROSA_E_NOMEM, "host allocation failed");
  } catch (...) {
    return fail(nullptr, ROSA_E_DEVICE, "unexpected exception");
  }
}

void free_all(rosa_kv *h) {
  if (h->d_plan) hipFree(h->d_plan);
  if (h->part_o) hipFree(h->part_o);
  if (h->part_ml) hipFree(h->part_ml);
  for (int i = 0; i < 2; ++i) {
    if (h->h_plan[i]) hipHostFree(h->h_plan[i]);
    if (h->copied[i]) hipEventDestroy(h->copied[i]);
  }
}

}  // namespace

extern "C" {

const char *rosa_kv_last_error(const rosa_kv *h) { return h ? h->last_error.c_str() : g_kv_error.c_str(); }

int64_t rosa_kv_bytes(const rosa_model_config *cfg, int32_t format, int32_t prefix_len) {
  if (!cfg || check_config(cfg) != ROSA_OK || prefix_len < 0) return -1;
  if (format == ROSA_KV_MODEL) return (int64_t)model_bytes(cfg, prefix_len);
  if (format == ROSA_KV_FP4) return (int64_t)fp4_bytes(cfg, prefix_len);
  return -1;
}

rosa_status rosa_kv_quantize(const rosa_model_config *cfg, const rosa_kv_job *jobs, int32_t n, void *hip_stream) {
  return convert(cfg, jobs, n, hip_stream, true);
}

rosa_status rosa_kv_expand(const rosa_model_config *cfg, const rosa_kv_job *jobs, int32_t n, void *hip_stream) {
  return convert(cfg, jobs, n, hip_stream, false);
}

rosa_status rosa_kv_evict(const rosa_model_config *cfg, int32_t format, const rosa_kv_evict_job *jobs, int32_t n,
                          void *hip_stream) {
  try {
    g_kv_error.clear();
    rosa_status st = check_cfg(cfg);
    if (st != ROSA_OK) return st;
    if (format != ROSA_KV_MODEL && format != ROSA_KV_FP4) return fail(nullptr, ROSA_E_INVALID, "unknown cache format");
    if (n < 0 || (n > 0 && !jobs)) return fail(nullptr, ROSA_E_INVALID, "n < 0 or jobs is NULL");
    const size_t rows = (size_t)cfg->n_layers * cfg->n_kv_heads;
    std::vector<Range> ranges;
    std::vector<KvEvictJob> work;
    for (int i = 0; i < n; ++i) {
      const rosa_kv_evict_job &j = jobs[i];
      if (j.prefix_len < 0 || j.first < 0 || j.last < 0 || j.keep < 0 || j.keep > j.prefix_len ||
          (int64_t)j.first + j.last > j.keep) {
        char buf[160];
        snprintf(buf, sizeof buf, "job %d: P=%d keep=%d first=%d last=%d (0 <= first + last <= keep <= P)", i,
                 j.prefix_len, j.keep, j.first, j.last);
        return fail(nullptr, ROSA_E_INVALID, buf);
      }
      if (j.keep == 0) continue;
      const void *p[4] = {j.src_k, j.src_v, j.dst_k, j.dst_v};
      for (const void *q : p)
        if (!q || !aligned(q, 16)) return fail(nullptr, ROSA_E_INVALID, "a cache is NULL or not 16-byte aligned");
      if (!j.mass || !j.kept || !aligned(j.mass, 4) || !aligned(j.kept, 4) || !aligned(j.kept_mass, 4))
        return fail(nullptr, ROSA_E_INVALID, "mass or kept is NULL, or an array is not 4-byte aligned");
      const bool four = format == ROSA_KV_FP4;
      const size_t sb = four ? fp4_bytes(cfg, j.prefix_len) : model_bytes(cfg, j.prefix_len);
      const size_t db = four ? fp4_bytes(cfg, j.keep) : model_bytes(cfg, j.keep);
      add_range(ranges, j.src_k, sb, false);
      add_range(ranges, j.src_v, sb, false);
      add_range(ranges, j.mass, rows * j.prefix_len * 4, false);
      add_range(ranges, j.dst_k, db, true);
      add_range(ranges, j.dst_v, db, true);
      add_range(ranges, j.kept, rows * j.keep * 4, true);
      add_range(ranges, j.kept_mass, rows * j.keep * 4, true);
      work.push_back({j.src_k, j.src_v, j.dst_k, j.dst_v, j.mass, j.kept, j.kept_mass, j.prefix_len, j.keep, j.first, j.last});
    }
    if (clash(ranges)) return fail(nullptr, ROSA_E_INVALID, "an output overlaps another array of the call");
    if (work.empty()) return ROSA_OK;
    int dev = 0;
    const hipStream_t s = (hipStream_t)hip_stream;
    hipError_t e = stream_device(s, &dev);
    if (e != hipSuccess) return device_fail(nullptr, e, "device of the stream");
    DeviceGuard guard(dev);
    e = guard.error();
    for (size_t at = 0; at < work.size() && e == hipSuccess; at += kKvEvictJobs) {
      KvEvictJobs part{};
      const int k = (int)std::min<size_t>(kKvEvictJobs, work.size() - at);
      std::copy(work.begin() + at, work.begin() + at + k, part.j);
      e = launch_kv_evict(part, k, cfg->n_layers, cfg->n_kv_heads, cfg->head_dim, cfg->dtype == ROSA_BF16 ? 2 : 4,
                          format == ROSA_KV_FP4, s);
    }
    return e == hipSuccess ? ROSA_OK : device_fail(nullptr, e, "eviction");
  } catch (const std::bad_alloc &) {
    return fail(nullptr, ROSA_E_NOMEM, "host allocation failed");
  } catch (...) {
    return fail(nullptr, ROSA_E_DEVICE, "unexpected exception");
  }
}

// ---------------------------------------------------------------- planned attention

rosa_status rosa_kv_create(const rosa_model_config *cfg, const rosa_capacity *cap, void *hip_stream, rosa_kv **out) {
  rosa_kv *h = nullptr;
  try {
    g_kv_error.clear();
    if (!out) return fail(nullptr, ROSA_E_INVALID, "out is NULL");
    *out = nullptr;
    rosa_status st = check_cfg(cfg);
    if (st != ROSA_OK) return st;
    if (!cap) return fail(nullptr, ROSA_E_INVALID, "cap is NULL");
    st = check_capacity(cap);
    if (st != ROSA_OK) return fail(nullptr, st, "bad capacity");
    const int G = cfg->n_q_heads / cfg->n_kv_heads;
    if ((int64_t)cap->max_horizon * G > (int64_t(1) << 30))
      return fail(nullptr, ROSA_E_UNSUPPORTED, "max_horizon x query heads per KV head above 2^30");
    h = new rosa_kv();
    h->cfg = *cfg;
    h->cap = *cap;
    h->dims = make_dims(cfg);
    h->bf16 = cfg->dtype == ROSA_BF16;
    h->stream = (hipStream_t)hip_stream;
    const Dims &D = h->dims;
    hipError_t e = stream_device(h->stream, &h->device);
    if (e != hipSuccess) { delete h; return device_fail(nullptr, e, "device of the stream"); }
    DeviceGuard guard(h->device);
    e = guard.error();

    const int n_sets = cfg->attention_layout == ROSA_ATTN_ALTERNATING ? 2 : 1;
    const int64_t blocks = (int64_t)D.nkv * (((int64_t)cap->max_action_tokens * G + 127) / 128 + 2 * (int64_t)cap->max_requests);
    h->max_groups = (size_t)n_sets * kAttnMaxSlots;
    h->max_items = (size_t)n_sets * (kAttnMaxSlots + (size_t)blocks);
    h->max_lists = 2 * h->max_items + 8 * (size_t)n_sets;
    h->max_mass = (size_t)D.nkv * ((size_t)(cap->max_prefix_tokens / kMassSmall) + (size_t)cap->max_requests);
    auto align = [](size_t v) { return (v + 255) / 256 * 256; };
    h->off_items = 0;
    h->off_groups = align(h->off_items + (h->bf16 ? 0 : h->max_items) * sizeof(AttnItem));
    h->off_lists = align(h->off_groups + h->max_groups * sizeof(AttnGroup));
    h->off_mass = align(h->off_lists + (h->bf16 ? h->max_lists : 0) * sizeof(AttnItem));
    h->plan_bytes = align(h->off_mass + h->max_mass * sizeof(MassItem));
    if (e == hipSuccess) e = hipMalloc((void **)&h->d_plan, h->plan_bytes);
    if (h->bf16) {
      if (e == hipSuccess) e = hipMalloc((void **)&h->part_o, h->max_groups * kAttnQB * D.hd * sizeof(float));
      if (e == hipSuccess) e = hipMalloc((void **)&h->part_ml, h->max_groups * kAttnQB * 2 * sizeof(float));
    }
    for (int i = 0; i < 2 && e == hipSuccess; ++i) {
      e = hipHostMalloc(&h->h_plan[i], h->plan_bytes, hipHostMallocDefault);
      if (e == hipSuccess) e = hipEventCreateWithFlags(&h->copied[i], hipEventDisableTiming);
    }
    if (e != hipSuccess) {
      free_all(h);
      delete h;
      return e == hipErrorOutOfMemory ? fail(nullptr, ROSA_E_NOMEM, "allocation failed") : device_fail(nullptr, e, "allocation");
    }
    *out = h;
    return ROSA_OK;
  } catch (const std::bad_alloc &) {
    if (h) { free_all(h); delete h; }
    return fail(nullptr, ROSA_E_NOMEM, "host allocation failed");
  } catch (...) {
    if (h) { free_all(h); delete h; }
    return fail(nullptr, ROSA_E_DEVICE, "unexpected exception");
  }
}

rosa_status rosa_kv_plan(rosa_kv *h, const rosa_request *reqs, int32_t n, int32_t format, float *const *mass) {
  if (!h) return ROSA_E_INVALID;
  try {
    h->last_error.clear();
    if (h->poisoned) return fail(h, ROSA_E_DEVICE, "handle is poisoned by an earlier device error");
    if (format != ROSA_KV_MODEL && format != ROSA_KV_FP4) return fail(h, ROSA_E_INVALID, "unknown cache format");
    if (n < 0 || (n > 0 && !reqs)) return fail(h, ROSA_E_INVALID, "n < 0 or reqs is NULL");
    if (n > h->cap.max_requests) return fail(h, ROSA_E_CAPACITY, "more requests than max_requests");
    // The plan's checks of the fields that attention does not read pass with these.
    std::vector<rosa_request> rq(reqs, reqs + n);
    static const float kUnread = 0.f;
    for (rosa_request &r : rq) {
      r.noise = &kUnread;
      r.actions = const_cast<float *>(&kUnread);
      r.num_steps = 1;
      r.start_step = 0;
    }
    Plan p;
    std::string err;
    const rosa_status st = build_plan(&h->cfg, &h->cap, rq.data(), n, false, h->bf16, 1, p, err);
    if (st != ROSA_OK) return fail(h, st, err);
    for (int i = 0; i < n; ++i) {
      if (!aligned(rq[i].prefix_k, 16) || !aligned(rq[i].prefix_v, 16))
        return fail(h, ROSA_E_INVALID, "a prefix cache is not 16-byte aligned");
    }
    if (mass)
      if (const char *why = masses_unusable(rq.data(), n, mass, (size_t)h->dims.L * h->dims.nkv, [&](const rosa_request &r) {
            return (size_t)rosa_kv_bytes(&h->cfg, format, r.prefix_len);
          }))
        return fail(h, ROSA_E_INVALID, why);
    const Plan::AttnSet &S0 = p.sets[0], &S1 = p.sets[1];
    const size_t n_items = S0.items.size() + S1.items.size(), n_groups = S0.groups.size() + S1.groups.size();
    std::vector<MassItem> mi;
    int64_t large = 0;
    for (int i = 0; i < n; ++i) large += (int64_t)h->dims.nkv * ((rq[i].prefix_len + kMassLarge - 1) / kMassLarge);
    const int keys = kv_mass_keys(h->bf16, large);
    if (mass)
      for (int i = 0; i < n; ++i)
        for (int kvh = 0; kvh < h->dims.nkv; ++kvh)
          for (int k0 = 0; k0 < rq[i].prefix_len; k0 += keys)
            mi.push_back({rq[i].prefix_k, mass[i], rq[i].prefix_len, rq[i].horizon, p.tok_off[i], kvh, k0,
                          std::min(keys, rq[i].prefix_len - k0), {0, 0}});
    if (n_items > h->max_items || n_groups > h->max_groups || p.attn_lists.size() > h->max_lists || mi.size() > h->max_mass)
      return fail(h, ROSA_E_CAPACITY, "internal: plan above the handle's size");

    DeviceGuard guard(h->device);
    hipError_t e = guard.error();
    hipStreamCaptureStatus cs = hipStreamCaptureStatusNone;
    if (e == hipSuccess && (hipStreamIsCapturing(h->stream, &cs) != hipSuccess || cs != hipStreamCaptureStatusNone)) {
      (void)hipGetLastError();
      return fail(h, ROSA_E_INVALID, "a plan cannot be made while its stream is captured");
    }
    const int slot = h->flip;
    h->flip ^= 1;
    if (e == hipSuccess && h->pending[slot]) e = hipEventSynchronize(h->copied[slot]);
    if (e != hipSuccess) return device_fail(h, e, "plan upload");
    uint8_t *hp = (uint8_t *)h->h_plan[slot];
    std::vector<AttnItem> all(S0.items);
    all.insert(all.end(), S1.items.begin(), S1.items.end());
    if (h->bf16)
      attn_order_items(all, p.attn_lists.data(), p.attn_next.data(), p.attn_lists.size(), (AttnItem *)(hp + h->off_lists));
    else if (!all.empty())
      std::memcpy(hp + h->off_items, all.data(), all.size() * sizeof(AttnItem));
    if (!S0.groups.empty()) std::memcpy(hp + h->off_groups, S0.groups.data(), S0.groups.size() * sizeof(AttnGroup));
    if (!S1.groups.empty())
      std::memcpy(hp + h->off_groups + S0.groups.size() * sizeof(AttnGroup), S1.groups.data(), S1.groups.size() * sizeof(AttnGroup));
    if (!mi.empty()) std::memcpy(hp + h->off_mass, mi.data(), mi.size() * sizeof(MassItem));
    // only the parts in use are copied
    struct Part { size_t off, bytes; } parts[4] = {
        {h->off_items, h->bf16 ? 0 : all.size() * sizeof(AttnItem)}, {h->off_groups, n_groups * sizeof(AttnGroup)},
        {h->off_lists, h->bf16 ? p.attn_lists.size() * sizeof(AttnItem) : 0}, {h->off_mass, mi.size() * sizeof(MassItem)}};
    for (const Part &q : parts)
      if (e == hipSuccess && q.bytes)
        e = hipMemcpyAsync(h->d_plan + q.off, hp + q.off, q.bytes, hipMemcpyHostToDevice, h->stream);
    if (e == hipSuccess) e = hipEventRecord(h->copied[slot], h->stream);
    if (e != hipSuccess) return device_fail(h, e, "plan upload");
    h->pending[slot] = true;
    for (int v = 0; v < 2; ++v) {
      const Plan::AttnSet &S = p.sets[v];
      rosa_kv::Set &d = h->sets[v];
      d = {};
      if (v >= p.n_sets || n == 0) continue;
      d.items = (int)S.items.size(); d.item_base = S.item_base;
      d.groups = (int)S.groups.size(); d.group_base = S.group_base;
      d.list_at = p.lanes[0].list_at[v][0];
      d.blocks = p.lanes[0].list_blocks[v][0];
    }
    h->n = n;
    h->n_mass = (int)mi.size();
    h->mass_keys = keys;
    h->rows = (size_t)p.M0;
    h->has_mass = mass != nullptr;
    h->fp4 = format == ROSA_KV_FP4;
    h->planned = true;
    return ROSA_OK;
  } catch (const std::bad_alloc &) {
    return fail(h, ROSA_E_NOMEM, "host allocation failed");
  } catch (...) {
    return fail(h, ROSA_E_DEVICE, "unexpected exception");
  }
}

rosa_status rosa_kv_attention(rosa_kv *h, int32_t layer, const void *qkv, void *o, float *lse) {
  if (!h) return ROSA_E_INVALID;
  try {
    h->last_error.clear();
    if (h->poisoned) return fail(h, ROSA_E_DEVICE, "handle is poisoned by an earlier device error");
    if (!h->planned) return fail(h, ROSA_E_INVALID, "no plan");
    const Dims &D = h->dims;
    if (layer < 0 || layer >= D.L) return fail(h, ROSA_E_INVALID, "layer out of range");
    if (h->n == 0) return ROSA_OK;
    if (!qkv || !o || !aligned(qkv, 16) || !aligned(o, 16) || !aligned(lse, 4))
      return fail(h, ROSA_E_INVALID, "qkv or o is NULL, or an array is misaligned");
    const size_t es = h->bf16 ? 2 : 4;
    std::vector<Range> ranges;
    add_range(ranges, qkv, h->rows * D.qkv_dim * es, false);
    add_range(ranges, o, h->rows * D.o_dim * es, true);
    add_range(ranges, lse, h->rows * D.nq * 4, true);
    if (clash(ranges)) return fail(h, ROSA_E_INVALID, "o or lse overlaps another array of the call");
    DeviceGuard guard(h->device);
    hipError_t e = guard.error();
    const rosa_kv::Set &S = h->sets[attn_set_of(&h->cfg, layer)];
    KvAttnArgs ka{};
    AttnArgs &a = ka.a;
    a.ordered = (const AttnItem *)(h->d_plan + h->off_lists) + S.list_at;
    a.n_blocks = S.blocks;
    a.items = h->bf16 ? a.ordered : (const AttnItem *)(h->d_plan + h->off_items) + S.item_base;
    a.n_items = S.items;
    a.layer = layer;
    a.qkv = qkv; a.ldqkv = D.qkv_dim; a.o = o; a.ldo = D.o_dim;
    a.nq = D.nq; a.nkv = D.nkv; a.hd = D.hd;
    a.part_o = h->part_o; a.part_ml = h->part_ml;
    a.lse = lse;
    ka.L = D.L; ka.fp4 = h->fp4;
    if (e == hipSuccess)
      e = launch_kv_attention(ka, (const AttnGroup *)(h->d_plan + h->off_groups) + S.group_base, S.groups, h->bf16, h->stream);
    return e == hipSuccess ? ROSA_OK : device_fail(h, e, "attention");
  } catch (...) {
    return fail(h, ROSA_E_DEVICE, "unexpected exception");
  }
}

rosa_status rosa_kv_mass(rosa_kv *h, int32_t layer, const void *qkv, const float *lse, int32_t accumulate) {
  if (!h) return ROSA_E_INVALID;
  try {
    h->last_error.clear();
    if (h->poisoned) return fail(h, ROSA_E_DEVICE, "handle is poisoned by an earlier device error");
    if (!h->planned || !h->has_mass) return fail(h, ROSA_E_INVALID, "no plan, or one without masses");
    const Dims &D = h->dims;
    if (layer < 0 || layer >= D.L) return fail(h, ROSA_E_INVALID, "layer out of range");
    if (attn_set_of(&h->cfg, layer) == 1) return fail(h, ROSA_E_INVALID, "the layer does not attend to the prefix");
    if (h->n == 0) return ROSA_OK;
    if (!qkv || !lse || !aligned(qkv, 16) || !aligned(lse, 4))
      return fail(h, ROSA_E_INVALID, "qkv or lse is NULL or misaligned");
    DeviceGuard guard(h->device);
    hipError_t e = guard.error();
    KvMassArgs a{};
    a.items = (const MassItem *)(h->d_plan + h->off_mass);
    a.n_items = h->n_mass;
    a.keys = h->mass_keys;
    a.layer = layer; a.L = D.L;
    a.qkv = qkv; a.ldqkv = D.qkv_dim; a.lse = lse;
    a.nq = D.nq; a.nkv = D.nkv; a.hd = D.hd;
    a.fp4 = h->fp4; a.accumulate = accumulate != 0;
    if (e == hipSuccess) e = launch_kv_mass(a, h->bf16, h->stream);
    return e == hipSuccess ? ROSA_OK : device_fail(h, e, "mass");
  } catch (...) {
    return fail(h, ROSA_E_DEVICE, "unexpected exception");
  }
}

void rosa_kv_destroy(rosa_kv *h) {
  if (!h) return;
  try {
    DeviceGuard guard(h->device);
    hipStreamSynchronize(h->stream);
    free_all(h);
  } catch (...) {
  }
  delete h;
}

}  // extern "C"
